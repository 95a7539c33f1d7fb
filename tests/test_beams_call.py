"""The native marshalling of the calls of beams and of the residual norm: plain
arguments give what the ctypes path gives, anything else goes there (GPU); host
tensors are refused (CPU)."""
import pytest
import torch

from paper_2609_39056_amd import _build
from paper_2609_39056_amd import binding as B

R, W, V, K, P = 6, 3, 300, 256, 16


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os

    if not (os.path.exists(B.LIB_PATH) and os.path.exists(B.CALL_PATH)):
        _build.build()
    B.lib()
    assert not isinstance(B._call, B._NoCall)


def inputs(dev):
    g = torch.Generator(device=dev)
    g.manual_seed(3)

    def rand(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=dev).to(dtype)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    act = B.ActParams(tok2stream=ints([0, 1, 0, 1, 1, 0]), gamma=rand(2, 2).abs() + 0.5, step=1, dinv=rand(K).abs() + 0.5)
    kv = B.KVCache(rand(20, 1, P, 64, dtype=torch.float16), rand(20, 1, P, 64, dtype=torch.float16))
    return dict(ints=ints, x=rand(R, K + 8, dtype=torch.bfloat16)[:, :K], res=rand(R, K), w=rand(K), act=act, kv=kv,
                logits=rand(R, V + 4)[:, :V], scores=rand(R), done=ints([0, 0, 1, 0, 0, 0]),
                table=ints([[0, 1], [0, 2], [0, 3], [4, 5], [4, 6], [4, 7]]), kv_len=ints([20, 21, 22, 25, 25, 25]),
                free=ints(list(range(20))), head=ints([8]), q=rand(R, 2, 64, dtype=torch.float16), start=ints([0, 3, 6]), shared=ints([16, 16]))


def step(s, stream, **kw):
    """All five calls; keyword arguments replace what a call is given."""
    dev, ints = s["res"].device, s["ints"]
    total, y = torch.zeros((R, K), device=dev), torch.zeros((R, K), dtype=torch.float16, device=dev)
    qx, r = torch.zeros((R, K), dtype=torch.int8, device=dev), torch.zeros(R, device=dev)
    B.sq_add_rmsnorm(kw.get("x", s["x"]), s["res"], s["w"], kw.get("eps", 1e-6), total, y, kw.get("out", B.SQ_OUT_F16),
                     kw.get("act", s["act"]), qx, r, stream)
    parent, token, done = (ints([[0] * W] * 2) for _ in range(3))
    score = torch.zeros((2, W), device=dev)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    B.sq_beam_select(s["logits"], W, s["scores"], s["done"], kw.get("end", 5), parent, token, score, done, kw.get("ws", ws), stream)
    table, free = torch.full_like(s["table"], -1), s["free"].clone()
    n, src, dst, rows = (ints([0] * R) for _ in range(4))
    head = ints([0])
    kv = B.KVCache(s["kv"].k.clone(), s["kv"].v.clone())
    B.sq_kv_reorder(parent.view(-1), s["kv_len"], kw.get("page", P), 20, free, s["head"], s["table"], table, n, src, dst, rows, head,
                    ws, stream)
    B.sq_kv_copy_pages(kw.get("caches", [kv]), src, dst, rows, stream)
    out, lse = torch.zeros((R, 2, 64), device=dev), torch.zeros((R, 2), device=dev)
    B.sq_attn_shared(kw.get("q", s["q"]), kv, table, n, s["start"], s["shared"], 16, kw.get("own", 32), kw.get("scale", 0.125), out,
                     B.SQ_OUT_F32, lse, ws, stream)
    if y.is_cuda:
        torch.cuda.synchronize()
    return [total, y, qx, r, parent, token, score, done, table, free, n, src, dst, rows, head, kv.k, kv.v, out, lse]


def test_host_tensors_go_to_ctypes():
    s = inputs("cpu")
    with pytest.raises(ValueError, match="device tensors"):
        step(s, None)
    a, z, t = B.lib().sq_address, s["kv_len"], s["table"]
    assert B._call.norm(a["sq_add_rmsnorm"], s["x"], s["res"], s["w"], 1e-6, None, s["res"], 0, None, None, None, None) is NotImplemented
    assert B._call.beams(a["sq_beam_select"], s["logits"], W, s["scores"], None, 0, t, t, s["res"], None, z, None) is NotImplemented
    assert B._call.reorder(a["sq_kv_reorder"], z, z, P, 20, z, None, t, t, z, z, z, z, z, z, None) is NotImplemented
    assert B._call.copy(a["sq_kv_copy_pages"], [s["kv"]], z, z, z, None) is NotImplemented
    assert B._call.copy(a["sq_kv_copy_pages"], 7, z, z, z, None) is NotImplemented
    assert B._call.attn_shared(a["sq_attn_shared"], s["q"], s["kv"], t, z, s["start"], s["shared"], 16, 32, 1.0, s["res"], 0, None, z,
                               None) is NotImplemented
    for name in ("norm", "beams", "reorder", "copy", "attn_shared"):
        assert getattr(B._call, name)(1, 2, 3) is NotImplemented
        assert getattr(B._call, name)() is NotImplemented


@pytest.mark.gpu
def test_native_equals_ctypes(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    s = inputs("cuda")
    made, real = [], B._call

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                st = getattr(real, name)(*args)
                made.append((name, st is not NotImplemented))
                return st

            return call

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    monkeypatch.setattr(B, "_call", Recorder())
    native = [step(s, None), step(s, torch.cuda.current_stream().cuda_stream)]
    with torch.cuda.stream(side):
        native += [step(s, None), step(s, side)]
    assert made == [(n, True) for n in ("norm", "beams", "reorder", "copy", "attn_shared")] * 4
    monkeypatch.setattr(B, "_call", B._NoCall())
    want = step(s, None)
    assert all(torch.isfinite(t.float()).all() for t in want[:-2])
    for got in native:
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    # errors are the same from both, and what is not plain gives what plain arguments give
    for call in (real, B._NoCall()):
        monkeypatch.setattr(B, "_call", call)
        for kw, status in ((dict(eps=-1.0), -4), (dict(end=V), -2), (dict(page=24), -4), (dict(own=-1), -2), (dict(scale=float("nan")), -4),
                           (dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda")), -5)):
            with pytest.raises(B.SqError) as e:
                step(s, None, **kw)
            assert e.value.status == status, kw
        with pytest.raises(ValueError, match="sizes or types"):
            step(s, None, out=B.SQ_OUT_BF16)
        with pytest.raises(ValueError, match="contiguous"):
            step(s, None, x=s["res"].t().contiguous().t())
        with pytest.raises(ValueError, match="stream id"):
            step(s, None, act=B.ActParams(tok2stream=s["act"].tok2stream[:5].clone(), gamma=s["act"].gamma, step=1))
        with pytest.raises(ValueError, match="heads are contiguous"):
            step(s, None, q=s["q"].transpose(0, 1).contiguous().transpose(0, 1).transpose(1, 2).contiguous().transpose(1, 2))
        kv = B.KVCache(s["kv"].k.clone(), s["kv"].v.clone())
        for a, b in zip(step(s, None, caches=(kv,))[:15], want[:15]):
            assert torch.equal(a, b)
        assert torch.equal(kv.k, want[15]) and torch.equal(kv.v, want[16])
