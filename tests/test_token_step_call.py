"""The native marshalling of the token step's calls: plain arguments give what
the ctypes path gives, anything else goes there (GPU); host tensors are refused
(CPU)."""
import math

import pytest
import torch

from paper_2609_39056_amd import _build
from paper_2609_39056_amd import binding as B

R, Hq, Hk, D, P = 5, 8, 2, 64, 16


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os

    if not (os.path.exists(B.LIB_PATH) and os.path.exists(B.CALL_PATH)):
        _build.build()
    B.lib()
    assert not isinstance(B._call, B._NoCall)


def inputs(dev):
    g = torch.Generator(device=dev)
    g.manual_seed(7)

    def rand(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=dev).to(dtype)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    kv = B.KVCache(rand(12, Hk, P, D, dtype=torch.bfloat16), rand(12, Hk, P, D, dtype=torch.bfloat16))
    rope = B.RopeParams(rand(D), rand(D), 1e-5, rand(100, D // 2), rand(100, D // 2), True)
    w = B.Weight(torch.randint(0, 256, (64, Hq * D // 2), generator=g, device=dev, dtype=torch.uint8),
                 rand(Hq * D // 128, 64).half(), 128, rand(64, dtype=torch.bfloat16))
    return dict(qkv=rand(R, (Hq + 2 * Hk) * D, dtype=torch.bfloat16), kv=kv, rope=rope, w=w, dinv=rand(Hq * D),
                cached=ints([0, 5, 16, 31, 15]), new=ints([1] * R), free=ints([0, 2, 4, 6, 8]), head=ints([1]),
                table=ints([[-1, -1, -1], [9, -1, -1], [10, -1, -1], [1, 3, -1], [5, -1, -1]]), ints=ints)


def heads(qkv):
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D], dim=1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hk, D)), v.unflatten(1, (Hk, D))


def step(s, stream, ws=None, **kw):
    """All four calls; keyword arguments replace what a call is given."""
    kv = B.KVCache(s["kv"].k.clone(), s["kv"].v.clone())
    table, z = s["table"].clone(), s["ints"]([0] * R)
    slot, pos, kv_len, start, head = z.clone(), z.clone(), z.clone(), s["ints"]([0] * (R + 1)), s["ints"]([0])
    B.sq_kv_plan(s["cached"], s["new"], kw.get("page", P), s["free"], kw.get("head", s["head"]), table, slot, pos,
                 start, kv_len, head, stream)
    q, k, v = kw.get("heads", heads(s["qkv"]))
    q_out, k_out = torch.zeros_like(q.contiguous()), torch.zeros_like(k.contiguous())
    B.sq_qk_norm_rope(q, k, v, kw.get("rope", s["rope"]), pos, slot, q_out, k_out, kv, stream)
    out = torch.zeros((R, Hq, D), dtype=torch.bfloat16, device=z.device)
    lse = torch.zeros((R, Hq), device=z.device)
    ws = B.alloc_attn_workspace(R, Hq, kv, 48) if ws is None else ws
    B.sq_attn_paged(q_out, kv, table, kv_len, 48, kw.get("window", 0), kw.get("scale", 1 / math.sqrt(D)), out,
                    B.SQ_OUT_BF16, lse, ws, stream)
    y = torch.zeros((R, 64), device=z.device)
    B.sq_linear_w4a16(out.view(R, -1), s["dinv"], s["w"], y, kw.get("out", B.SQ_OUT_F32), stream)
    if y.is_cuda:
        torch.cuda.synchronize()
    return [slot, pos, start, kv_len, head, table, q_out, k_out, kv.k, kv.v, out, lse, y]


def test_host_tensors_go_to_ctypes():
    s = inputs("cpu")
    with pytest.raises(ValueError, match="device tensors"):
        step(s, None)
    q, k, v = heads(s["qkv"])
    z = s["ints"]([0] * R)
    a = B.lib().sq_address
    assert B._call.rope(a["sq_qk_norm_rope"], q, k, v, s["rope"], z, z, q, None, s["kv"], None) is NotImplemented
    assert B._call.attn(a["sq_attn_paged"], q, s["kv"], s["table"], z, 48, 0, 1.0, q, 1, None, z, None) is NotImplemented
    assert B._call.linear16(a["sq_linear_w4a16"], s["qkv"], None, s["w"], s["qkv"], 1, None) is NotImplemented
    assert B._call.kv_plan(a["sq_kv_plan"], z, z, P, z, None, s["table"], z, z, z, z, z, None) is NotImplemented
    for name in ("kv_plan", "rope", "attn", "linear16"):
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
    assert made == [(n, True) for n in ("kv_plan", "rope", "attn", "linear16")] * 4
    monkeypatch.setattr(B, "_call", B._NoCall())
    want = step(s, None)
    assert all(torch.isfinite(t.float()).all() for t in want)
    for got in native:
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    # errors are the same from both, and what is not plain gives what plain arguments give
    for call in (real, B._NoCall()):
        monkeypatch.setattr(B, "_call", call)
        for kw, status in ((dict(page=24), -4), (dict(window=-1), -2), (dict(scale=float("nan")), -4)):
            with pytest.raises(B.SqError) as e:
                step(s, None, **kw)
            assert e.value.status == status
        with pytest.raises(B.SqError) as e:
            step(s, None, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
        assert e.value.status == -5
        with pytest.raises(ValueError, match="sizes or types"):
            step(s, None, out=B.SQ_OUT_BF16)
        q, k, v = heads(s["qkv"])
        with pytest.raises(ValueError, match="heads are contiguous"):
            step(s, None, heads=(q.transpose(1, 2).contiguous().transpose(1, 2), k, v))
        with pytest.raises(ValueError, match="sizes"):
            step(s, None, heads=(q, k, q))
        rope = B.RopeParams(s["rope"].q_weight, s["rope"].k_weight, 1e-5, s["rope"].cos, s["rope"].sin, 1)  # not a bool
        for a, b in zip(step(s, None, rope=rope), want):
            assert torch.equal(a, b)
