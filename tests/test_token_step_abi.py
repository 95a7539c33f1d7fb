"""Refusals of the token step's entry points on the host: every call below
fails its checks (or has nothing to do), so no kernel is enqueued and no GPU is
needed.  The plain 64-bit forms are held by hand-worked cases."""
import ctypes
import math

import pytest
import torch

import token_ref as T
from paper_2609_39056_amd import binding as B
from test_abi import A, ALIGN, NULL, OK, SHAPE, UNSUP, WS, L, wt  # noqa: F401

NAN, INF = float("nan"), float("inf")


def cache(**kw):
    d = dict(k=A, v=A + 4096, num_pages=10, num_heads=2, page_size=16, head_dim=128, dtype=B.SQ_OUT_BF16)
    d.update(kw)
    return B.sq_kv_cache(**d)


CACHE_CASES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(dtype=B.SQ_OUT_F32), UNSUP), (dict(dtype=7), UNSUP),
               (dict(page_size=24), UNSUP), (dict(page_size=4), UNSUP), (dict(page_size=2048), UNSUP),
               (dict(page_size=0), UNSUP), (dict(page_size=-16), UNSUP), (dict(head_dim=80), UNSUP),
               (dict(head_dim=512), UNSUP), (dict(head_dim=0), UNSUP), (dict(num_heads=0), SHAPE),
               (dict(num_heads=257), SHAPE), (dict(num_pages=0), SHAPE), (dict(num_pages=1 << 27), SHAPE),
               (dict(k=A + 8), ALIGN), (dict(v=A + 2), ALIGN)]


def plan(L, **kw):  # noqa: F811
    d = dict(cached=A, new=A + 64, R=4, page=16, free=A, nfree=3, head=A, table=A, max_pages=4, max_tokens=8, slot=A,
             pos=A, start=A, kv_len=A + 128, head_out=A + 256)
    d.update(kw)
    return L.sq_kv_plan(d["cached"], d["new"], d["R"], d["page"], d["free"], d["nfree"], d["head"], d["table"],
                        d["max_pages"], d["max_tokens"], d["slot"], d["pos"], d["start"], d["kv_len"], d["head_out"],
                        None)


@pytest.mark.parametrize("kw,code", [
    (dict(cached=None), NULL), (dict(new=None), NULL), (dict(table=None), NULL), (dict(start=None), NULL),
    (dict(kv_len=None), NULL), (dict(head_out=None), NULL), (dict(free=None), NULL), (dict(slot=None), NULL),
    (dict(pos=None), NULL), (dict(page=24), UNSUP), (dict(page=4), UNSUP), (dict(page=0), UNSUP), (dict(R=0), SHAPE),
    (dict(R=8193), SHAPE), (dict(nfree=-1), SHAPE), (dict(max_tokens=-1), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=1 << 27), SHAPE), (dict(R=8192, page=8, max_pages=1 << 18), SHAPE), (dict(cached=A + 2), ALIGN),
    (dict(new=A + 1), ALIGN), (dict(free=A + 2), ALIGN), (dict(head=A + 2), ALIGN), (dict(table=A + 2), ALIGN),
    (dict(slot=A + 3), ALIGN), (dict(pos=A + 2), ALIGN), (dict(start=A + 2), ALIGN), (dict(kv_len=A + 130), ALIGN),
    (dict(head_out=A + 257), ALIGN), (dict(kv_len=A), UNSUP), (dict(kv_len=A + 64), UNSUP), (dict(head_out=A), UNSUP),
])
def test_plan_rejects(L, kw, code):  # noqa: F811
    assert plan(L, **kw) == code


def rope(L, p=None, kv=None, no_cache=False, **kw):  # noqa: F811
    pp = dict(q_weight=A, k_weight=A, cos=A, sin=A, eps=1e-6, num_pos=100, rot_dim=128, interleaved=0)
    pp.update(p or {})
    d = dict(q=A, qs=6144, k=A, ks=6144, v=A, vs=6144, T=5, Hq=16, Hk=2, D=128, dtype=B.SQ_OUT_BF16, pos=A, slot=A,
             q_out=A, k_out=None)
    d.update(kw)
    c = None if no_cache else ctypes.byref(cache(**(kv or {})))
    return L.sq_qk_norm_rope(d["q"], d["qs"], d["k"], d["ks"], d["v"], d["vs"], d["T"], d["Hq"], d["Hk"], d["D"],
                             d["dtype"], None if p is False else ctypes.byref(B.sq_rope_params(**pp)), d["pos"],
                             d["slot"], d["q_out"], d["k_out"], c, None)


@pytest.mark.parametrize("kw,code", [
    (dict(p=False), NULL), (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(q_out=None), NULL),
    (dict(slot=None), NULL), (dict(pos=None), NULL), (dict(p=dict(cos=None)), NULL), (dict(p=dict(sin=None)), NULL),
    (dict(no_cache=True), NULL), (dict(dtype=B.SQ_OUT_F32), UNSUP), (dict(dtype=B.SQ_OUT_F16), UNSUP),
    (dict(D=80), UNSUP), (dict(p=dict(eps=-1.0)), UNSUP), (dict(p=dict(eps=NAN)), UNSUP), (dict(p=dict(eps=INF)), UNSUP),
    (dict(T=-1), SHAPE), (dict(T=(1 << 24) + 1), SHAPE), (dict(Hq=0), SHAPE), (dict(Hq=1025), SHAPE),
    (dict(Hk=0), SHAPE), (dict(Hk=3), SHAPE), (dict(D=64), SHAPE), (dict(p=dict(rot_dim=-16)), SHAPE),
    (dict(p=dict(rot_dim=24)), SHAPE), (dict(p=dict(rot_dim=144)), SHAPE), (dict(p=dict(num_pos=0)), SHAPE),
    (dict(qs=2040), SHAPE), (dict(qs=2052), SHAPE), (dict(ks=248), SHAPE), (dict(vs=-6144), SHAPE),
    (dict(q=A + 8), ALIGN), (dict(k=A + 2), ALIGN), (dict(v=A + 4), ALIGN), (dict(q_out=A + 8), ALIGN),
    (dict(k_out=A + 8), ALIGN), (dict(pos=A + 2), ALIGN), (dict(slot=A + 2), ALIGN), (dict(p=dict(cos=A + 4)), ALIGN),
    (dict(p=dict(sin=A + 8)), ALIGN), (dict(p=dict(q_weight=A + 4)), ALIGN), (dict(p=dict(k_weight=A + 8)), ALIGN),
    (dict(T=0), OK), (dict(T=0, q=None, k=None, v=None, q_out=None, slot=None, pos=None), OK),
] + [(dict(kv=kv), code) for kv, code in CACHE_CASES])
def test_rope_rejects(L, kw, code):  # noqa: F811
    assert rope(L, **kw) == code


def attn(L, kv=None, no_cache=False, **kw):  # noqa: F811
    d = dict(q=A, qs=2048, R=3, Hq=16, table=A, max_pages=8, kv_len=A, n=128, window=0, scale=0.1, out=A,
             out_dtype=B.SQ_OUT_BF16, lse=None, ws=A, nbytes=1 << 30)
    d.update(kw)
    c = None if no_cache else ctypes.byref(cache(**(kv or {})))
    return L.sq_attn_paged(d["q"], d["qs"], d["R"], d["Hq"], c, d["table"], d["max_pages"], d["kv_len"], d["n"],
                           d["window"], d["scale"], d["out"], d["out_dtype"], d["lse"], d["ws"], d["nbytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(no_cache=True), NULL), (dict(q=None), NULL), (dict(table=None), NULL), (dict(kv_len=None), NULL),
    (dict(out=None), NULL), (dict(ws=None), NULL), (dict(out_dtype=3), UNSUP), (dict(scale=NAN), UNSUP),
    (dict(scale=INF), UNSUP), (dict(R=-1), SHAPE), (dict(R=65536), SHAPE), (dict(Hq=0), SHAPE), (dict(Hq=15), SHAPE),
    (dict(Hq=1026), SHAPE), (dict(n=-1), SHAPE), (dict(n=129), SHAPE), (dict(window=-1), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 27), SHAPE), (dict(qs=2040), SHAPE), (dict(qs=2049), SHAPE),
    (dict(q=A + 8), ALIGN), (dict(out=A + 8), ALIGN), (dict(ws=A + 8), ALIGN), (dict(table=A + 2), ALIGN),
    (dict(kv_len=A + 2), ALIGN), (dict(lse=A + 2), ALIGN), (dict(nbytes=255), WS), (dict(R=0), OK),
] + [(dict(kv=kv), code) for kv, code in CACHE_CASES])
def test_attn_rejects(L, kw, code):  # noqa: F811
    assert attn(L, **kw) == code


def test_attn_workspace(L):  # noqa: F811
    def n(R, Hq, length, **kw):
        return L.sq_attn_workspace_bytes(R, Hq, ctypes.byref(cache(**kw)), length)

    for args in ((1, 16, 0), (1, 16, 1), (64, 16, 8192), (2, 32, 131072), (65535, 2, 2 ** 31 - 1)):
        assert n(*args) >= 256 and n(*args) % 256 == 0
    assert n(1, 15, 100) == 0 and n(-1, 16, 100) == 0 and n(1, 16, -1) == 0 and n(1, 16, 100, page_size=3) == 0
    assert L.sq_attn_workspace_bytes(1, 16, None, 100) == 0


def lin(L, x=A, M=3, dinv=None, w=None, y=A, out=0):  # noqa: F811
    return L.sq_linear_w4a16(x, M, dinv, ctypes.byref(wt() if w is None else w) if w is not False else None, y, out, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(w=False), NULL), (dict(M=0), SHAPE), (dict(M=-1), SHAPE),
    (dict(M=65), UNSUP), (dict(out=3), UNSUP), (dict(x=A + 8), ALIGN), (dict(y=A + 4), ALIGN), (dict(dinv=A + 4), ALIGN),
    (dict(w=wt(N=100)), SHAPE), (dict(w=wt(K=200)), SHAPE), (dict(w=wt(w_group=64)), UNSUP), (dict(w=wt(qw=None)), NULL),
    (dict(w=wt(w_scale=A + 2)), ALIGN), (dict(w=wt(qw=A + 4)), ALIGN), (dict(w=wt(bias=A + 1)), ALIGN),
])
def test_linear_rejects(L, kw, code):  # noqa: F811
    assert lin(L, **kw) == code


def test_binding_refuses_host_tensors_sizes_and_types(L):  # noqa: F811
    bf, i = torch.bfloat16, torch.int32
    k = torch.zeros((2, 1, 8, 64), dtype=bf)
    q = torch.zeros((3, 2, 64), dtype=bf)
    with pytest.raises(ValueError, match="device tensors"):
        B.alloc_attn_workspace(1, 2, B.KVCache(k, k), 8)
    with pytest.raises(ValueError, match="one shape"):
        B.KVCache(k, k.half()).struct()
    with pytest.raises(ValueError, match="one shape"):
        B.KVCache(k.float(), k.float()).struct()
    with pytest.raises(ValueError, match="device tensors"):
        B.sq_qk_norm_rope(q, q, None, B.RopeParams(), None, None, q, q, None)
    with pytest.raises(ValueError, match="two tables"):
        B.RopeParams(cos=torch.zeros(3, 32)).struct(64)
    with pytest.raises(ValueError, match="head_dim"):
        B.RopeParams(q_weight=torch.zeros(32)).struct(64)
    with pytest.raises(ValueError, match="float32"):
        B.RopeParams(q_weight=torch.zeros(64).half()).struct(64)
    t = torch.zeros(4, dtype=i)
    with pytest.raises(ValueError, match="int32"):
        B.sq_kv_plan(t.long(), t, 16, t, None, t.view(4, 1), t, t, t, t, t)
    with pytest.raises(ValueError, match="sizes"):
        B.sq_kv_plan(t, t, 16, t, None, t.view(4, 1), t, t, t, t, t)  # token_start holds 4 values, not 5
    w = B.Weight(torch.zeros((64, 64), dtype=torch.uint8), torch.zeros((1, 64)).half(), 128)
    x = torch.zeros((2, 128), dtype=bf)
    with pytest.raises(ValueError, match="sizes or types"):
        B.sq_linear_w4a16(x, None, w, torch.zeros((2, 64)), B.SQ_OUT_BF16)
    with pytest.raises(ValueError, match="device tensors"):
        B.sq_linear_w4a16(x, None, w, torch.zeros((2, 64)), B.SQ_OUT_F32)


# ------------------------------------------------------------------ the plain forms, by hand
def test_plain_plan_by_hand():
    # pages of 8: request 0 fills its page and takes one, 1 is new and takes two, 2 has room, 3 is idle
    table, slot, pos, start, kv_len, head = T.plan([8, 0, 3, 5], [1, 9, 2, 0], 8, [70, 71, 72, 73], 1,
                                                   [[5, -1], [-1, -1], [6, -1], [9, -1]], 14)
    assert table == [[5, 71], [72, 73], [6, -1], [9, -1]]
    assert slot == [568] + list(range(576, 584)) + [584, 51, 52, -1, -1]
    assert pos == [8] + list(range(9)) + [3, 4, -1, -1]
    assert (start, kv_len, head) == ([0, 1, 10, 12, 12], [9, 9, 5, 5], 4)


def test_plain_rotation_by_hand():
    x = torch.tensor([[[3.0, 4.0, 0.0, 0.0]]])
    cos, sin = torch.tensor([[0.0, 1.0]]), torch.tensor([[1.0, 0.0]])
    pos = torch.tensor([0])
    # a quarter turn of the first pair, none of the second
    y, _ = T.norm_rope(x, None, 0.0, cos, sin, pos, True)
    assert y.tolist() == [[[-4.0, 3.0, 0.0, 0.0]]]
    y, _ = T.norm_rope(x, None, 0.0, cos, sin, pos, False)
    assert y.tolist() == [[[0.0, 4.0, 3.0, 0.0]]]
    y, _ = T.norm_rope(x, torch.tensor([1.0, 2.0, 1.0, 1.0]), 0.0, None, None, None, False)
    assert torch.allclose(y, torch.tensor([[[1.2, 3.2, 0.0, 0.0]]], dtype=torch.float64))  # root mean square 2.5


def test_plain_attention_by_hand():
    # two tokens with scores 0 and log 3: weights 1/4 and 3/4; a third is masked by the window or the length
    k = torch.zeros((1, 1, 8, 2))
    k[0, 0, :, 0] = torch.tensor([9.0, 0.0, math.log(3.0), NAN, NAN, NAN, NAN, NAN])
    v = torch.zeros((1, 1, 8, 2))
    v[0, 0, :3, 0], v[0, 0, :3, 1] = torch.tensor([100.0, 4.0, 8.0]), torch.tensor([100.0, 0.0, 4.0])
    q = torch.tensor([[[1.0, 0.0]]])
    out, lse, _, _ = T.attn(q, k, v, torch.tensor([[0]]), [3], 2, 1.0, 8, torch.float32)
    assert torch.allclose(out, torch.tensor([[[7.0, 3.0]]], dtype=torch.float64)) and abs(lse.item() - math.log(4)) < 1e-6
    out, lse, _, _ = T.attn(q, k, v, torch.tensor([[-1]]), [3], 0, 1.0, 8, torch.float32)
    assert out.abs().sum() == 0 and lse.item() == -INF


def test_plain_linear_by_hand():
    # 8 codes a group of bytes: byte b holds code b low and code b + 4 high
    qw = torch.zeros((1, 4), dtype=torch.uint8)
    qw[0] = torch.tensor([0x71, 0xF2, 0x83, 0x04], dtype=torch.uint8)
    assert T.unpack(qw.numpy()).tolist() == [[1, 2, 3, 4, 7, -1, -8, 0]]
    x = torch.arange(1, 9).view(1, 8).to(torch.bfloat16)
    step = torch.tensor([[0.5], [2.0]]).half()
    y, _ = T.linear(x, torch.full((8,), 2.0), qw.numpy(), step, 4, torch.tensor([10.0]).to(torch.bfloat16), torch.float32)
    assert y.item() == 2 * (0.5 * (1 + 4 + 9 + 16) + 2.0 * (35 - 6 - 56)) + 10
