"""Refusals of the operators of beams and of the residual norm on the host: every
call below fails its checks (or has nothing to do), so no kernel is enqueued and
no GPU is needed.  The plain forms are held by hand-worked cases."""
import ctypes
import math

import pytest
import torch

import beam_ref as R
from paper_2609_39056_amd import binding as B
from test_abi import A, ALIGN, NULL, OK, SHAPE, UNSUP, WS, L, act  # noqa: F401
from test_token_step_abi import CACHE_CASES, cache

NAN, INF = float("nan"), float("inf")


def norm(L, a=False, **kw):  # noqa: F811
    d = dict(x=A, xs=256, xd=1, res=A, rs=256, rd=1, w=A, eps=1e-6, M=5, K=256, sum=A, ss=256, y=A, yd=1, qx=A, r=A)
    d.update(kw)
    p = None if a is False else ctypes.byref(act(**a))
    return L.sq_add_rmsnorm(d["x"], d["xs"], d["xd"], d["res"], d["rs"], d["rd"], d["w"], d["eps"], d["M"], d["K"], d["sum"],
                            d["ss"], d["y"], d["yd"], p, d["qx"], d["r"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(res=None), NULL), (dict(sum=None, y=None), NULL), (dict(a={}, qx=None), NULL),
    (dict(a={}, r=None), NULL), (dict(a=dict(gamma=None)), NULL), (dict(a=dict(tok2stream=None)), NULL), (dict(xd=3), UNSUP),
    (dict(rd=-1), UNSUP), (dict(yd=7), UNSUP), (dict(eps=-1.0), UNSUP), (dict(eps=NAN), UNSUP), (dict(eps=INF), UNSUP),
    (dict(a=dict(act_bits=4)), UNSUP), (dict(a=dict(range_mode=2)), UNSUP), (dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE),
    (dict(K=0), SHAPE), (dict(K=12), SHAPE), (dict(K=32776, xs=32776), SHAPE), (dict(a={}, K=264), SHAPE), (dict(xs=248), SHAPE),
    (dict(xs=260), SHAPE), (dict(rs=-256), SHAPE), (dict(ss=128), SHAPE), (dict(a=dict(step=9)), SHAPE), (dict(x=A + 8), ALIGN),
    (dict(res=A + 2), ALIGN), (dict(w=A + 4), ALIGN), (dict(sum=A + 8), ALIGN), (dict(y=A + 8), ALIGN), (dict(a={}, qx=A + 8), ALIGN),
    (dict(a={}, r=A + 2), ALIGN), (dict(a=dict(dinv=A + 4)), ALIGN), (dict(M=0), OK), (dict(M=0, x=None, y=None, sum=None), OK),
    (dict(rs=512), UNSUP), (dict(ss=512), UNSUP), (dict(y=None, x=A + 64, ss=264), UNSUP), (dict(sum=None, xs=512), UNSUP),
    (dict(sum=None, res=A + 64, yd=0), UNSUP), (dict(res=A + 64, rd=0, y=None), UNSUP), (dict(sum=None, x=A + 64, yd=2), UNSUP),
])
def test_norm_rejects(L, kw, code):  # noqa: F811
    assert norm(L, **kw) == code


def select(L, **kw):  # noqa: F811
    d = dict(x=A, stride=104, dt=0, rows=8, beams=4, vocab=100, scores=A, done=None, end=0, width=4, parent=A + 64, token=A + 64,
             score=A + 64, done_out=None, ws=A, nbytes=1 << 20)
    d.update(kw)
    return L.sq_beam_select(d["x"], d["stride"], d["dt"], d["rows"], d["beams"], d["vocab"], d["scores"], d["done"], d["end"],
                            d["width"], d["parent"], d["token"], d["score"], d["done_out"], d["ws"], d["nbytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(scores=None), NULL), (dict(parent=None), NULL), (dict(token=None), NULL), (dict(score=None), NULL),
    (dict(ws=None), NULL), (dict(dt=3), UNSUP), (dict(rows=-4), SHAPE), (dict(rows=10), SHAPE), (dict(rows=65536), SHAPE),
    (dict(beams=0), SHAPE), (dict(beams=65, rows=65), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=(1 << 20) + 1), SHAPE),
    (dict(width=0), SHAPE), (dict(width=65), SHAPE), (dict(stride=96), SHAPE), (dict(stride=100), SHAPE), (dict(stride=-104), SHAPE),
    (dict(done=A, end=-1), SHAPE), (dict(done_out=A, end=100), SHAPE), (dict(x=A + 8), ALIGN), (dict(ws=A + 8), ALIGN),
    (dict(scores=A + 2), ALIGN), (dict(done=A + 1), ALIGN), (dict(parent=A + 2), ALIGN), (dict(token=A + 2), ALIGN),
    (dict(score=A + 2), ALIGN), (dict(done_out=A + 2), ALIGN), (dict(width=5, score=A), UNSUP),
    (dict(width=2, done=A, done_out=A), UNSUP), (dict(nbytes=255), WS), (dict(rows=0), OK), (dict(rows=0, x=None, ws=None), OK),
])
def test_select_rejects(L, kw, code):  # noqa: F811
    assert select(L, **kw) == code


def test_select_workspace(L):  # noqa: F811
    n = L.sq_beam_workspace_bytes
    assert n(0, 4, 100, 4) == 256 and n(8, 4, 100, 4) >= 256 and n(128, 8, 131071, 8) % 256 == 0
    assert n(65535, 1, 1 << 20, 64) >= 65535 * 256 * 64 * 8
    assert n(8, 3, 100, 4) == 0 and n(8, 4, 0, 4) == 0 and n(8, 4, 100, 65) == 0 and n(-4, 4, 100, 4) == 0
    # one for the largest serves every smaller one
    assert all(n(r, 4, v, w) <= n(64, 8, 5000, 8) for r in (4, 64) for v in (1, 4096, 5000) for w in (1, 8))


def reorder(L, **kw):  # noqa: F811
    d = dict(parent=A, kv_len=A + 64, R=4, page=16, pages=100, free=A, nfree=3, head=A, table=A, max_pages=4, table_out=A + 128,
             len_out=A + 256, src=A, dst=A, rows=A, head_out=A + 512, ws=A, nbytes=1 << 20)
    d.update(kw)
    return L.sq_kv_reorder(d["parent"], d["kv_len"], d["R"], d["page"], d["pages"], d["free"], d["nfree"], d["head"], d["table"],
                           d["max_pages"], d["table_out"], d["len_out"], d["src"], d["dst"], d["rows"], d["head_out"], d["ws"],
                           d["nbytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(parent=None), NULL), (dict(kv_len=None), NULL), (dict(free=None), NULL), (dict(table=None), NULL),
    (dict(table_out=None), NULL), (dict(len_out=None), NULL), (dict(src=None), NULL), (dict(dst=None), NULL), (dict(rows=None), NULL),
    (dict(head_out=None), NULL), (dict(ws=None), NULL), (dict(page=24), UNSUP), (dict(page=4), UNSUP), (dict(R=0), SHAPE),
    (dict(R=8193), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 27), SHAPE), (dict(nfree=-1), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=1 << 27), SHAPE), (dict(R=8192, page=8, max_pages=1 << 18), SHAPE), (dict(ws=A + 8), ALIGN),
    (dict(parent=A + 2), ALIGN), (dict(kv_len=A + 65), ALIGN), (dict(free=A + 2), ALIGN), (dict(head=A + 2), ALIGN),
    (dict(table=A + 2), ALIGN), (dict(table_out=A + 130), ALIGN), (dict(len_out=A + 258), ALIGN), (dict(src=A + 2), ALIGN),
    (dict(dst=A + 2), ALIGN), (dict(rows=A + 2), ALIGN), (dict(head_out=A + 514), ALIGN), (dict(table_out=A), UNSUP),
    (dict(len_out=A + 64), UNSUP), (dict(len_out=A), UNSUP), (dict(head_out=A), UNSUP), (dict(nbytes=100), WS),
])
def test_reorder_rejects(L, kw, code):  # noqa: F811
    assert reorder(L, **kw) == code


def test_reorder_workspace(L):  # noqa: F811
    n = L.sq_kv_reorder_workspace_bytes
    assert n(1, 1) == 256 and n(8192, 1 << 20) >= 4 << 20 and n(0, 5) == 0 and n(8193, 5) == 0 and n(4, 0) == 0


def shared(L, kv=None, no_cache=False, **kw):  # noqa: F811
    d = dict(q=A, qs=2048, R=3, Hq=16, table=A, max_pages=8, kv_len=A, start=A, shared=A, groups=1, most=128, own=128, scale=0.1, out=A,
             out_dtype=B.SQ_OUT_BF16, lse=None, ws=A, nbytes=1 << 30)
    d.update(kw)
    c = None if no_cache else ctypes.byref(cache(**(kv or {})))
    return L.sq_attn_shared(d["q"], d["qs"], d["R"], d["Hq"], c, d["table"], d["max_pages"], d["kv_len"], d["start"], d["shared"],
                            d["groups"], d["most"], d["own"], d["scale"], d["out"], d["out_dtype"], d["lse"], d["ws"], d["nbytes"],
                            None)


@pytest.mark.parametrize("kw,code", [
    (dict(no_cache=True), NULL), (dict(q=None), NULL), (dict(table=None), NULL), (dict(kv_len=None), NULL),
    (dict(start=None), NULL), (dict(shared=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL), (dict(out_dtype=3), UNSUP),
    (dict(scale=NAN), UNSUP), (dict(scale=INF), UNSUP), (dict(R=-1), SHAPE), (dict(R=65536), SHAPE), (dict(Hq=0), SHAPE),
    (dict(Hq=15), SHAPE), (dict(Hq=1026), SHAPE), (dict(groups=-1), SHAPE), (dict(groups=65536), SHAPE), (dict(most=-1), SHAPE),
    (dict(most=129), SHAPE), (dict(own=-1), SHAPE), (dict(own=129), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=1 << 27), SHAPE), (dict(qs=2040), SHAPE), (dict(qs=2049), SHAPE), (dict(q=A + 8), ALIGN), (dict(out=A + 8), ALIGN),
    (dict(ws=A + 8), ALIGN), (dict(table=A + 2), ALIGN), (dict(kv_len=A + 2), ALIGN), (dict(start=A + 2), ALIGN),
    (dict(shared=A + 2), ALIGN), (dict(lse=A + 2), ALIGN), (dict(nbytes=255), WS), (dict(R=0), OK), (dict(R=0, q=None, ws=None), OK),
] + [(dict(kv=kv), code) for kv, code in CACHE_CASES])
def test_shared_rejects(L, kw, code):  # noqa: F811
    assert shared(L, **kw) == code


def test_shared_workspace(L):  # noqa: F811
    def n(R, groups, Hq, most, own, **kw):
        return L.sq_attn_shared_workspace_bytes(R, groups, Hq, ctypes.byref(cache(**kw)), most, own)

    for args in ((0, 0, 16, 0, 0), (1, 1, 16, 0, 1), (64, 1, 16, 8192, 500), (2, 65535, 32, 131072, 131072)):
        assert n(*args) >= 256 and n(*args) % 256 == 0
    assert n(1, 1, 15, 100, 100) == 0 and n(-1, 1, 16, 100, 100) == 0 and n(1, -1, 16, 1, 1) == 0 and n(1, 1, 16, -1, 1) == 0
    assert n(1, 1, 16, 1, -1) == 0 and n(1, 1, 16, 1, 1, page_size=3) == 0
    assert L.sq_attn_shared_workspace_bytes(1, 1, 16, None, 100, 100) == 0


def copy(L, caches=None, n_caches=None, null=False, **kw):  # noqa: F811
    d = dict(src=A, dst=A + 64, rows=None, n=3)
    d.update(kw)
    caches = [{}] if caches is None else caches
    c = (B.sq_kv_cache * max(1, len(caches)))(*[cache(**k) for k in caches])
    return L.sq_kv_copy_pages(None if null else c, len(caches) if n_caches is None else n_caches, d["src"], d["dst"], d["rows"],
                              d["n"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(null=True), NULL), (dict(src=None), NULL), (dict(dst=None), NULL), (dict(n_caches=-1), SHAPE), (dict(n_caches=1025), SHAPE),
    (dict(n=-1), SHAPE), (dict(n=65536), SHAPE), (dict(src=A + 2), ALIGN), (dict(dst=A + 2), ALIGN), (dict(rows=A + 2), ALIGN),
    (dict(caches=[{}, dict(num_pages=11)]), SHAPE), (dict(caches=[{}, dict(num_heads=1)]), SHAPE),
    (dict(caches=[{}, dict(page_size=32)]), SHAPE), (dict(caches=[{}, {}, dict(head_dim=64)]), SHAPE),
    (dict(caches=[{}, dict(dtype=B.SQ_OUT_F16)]), UNSUP), (dict(n=0), OK), (dict(n=0, src=None, dst=None), OK),
    (dict(n_caches=0, src=None), OK), (dict(n_caches=0, null=True), OK),
] + [(dict(caches=[{}, kv]), code) for kv, code in CACHE_CASES])
def test_copy_rejects(L, kw, code):  # noqa: F811
    assert copy(L, **kw) == code


def test_binding_refuses_host_tensors_sizes_and_types(L):  # noqa: F811
    x, w = torch.zeros((2, 128)), torch.zeros(128)
    with pytest.raises(ValueError, match="device tensors"):
        B.sq_add_rmsnorm(x, None, w, 1e-6, None, x, B.SQ_OUT_F32, None, None, None)
    with pytest.raises(ValueError, match="device tensors"):
        B.sq_beam_select(x, 2, torch.zeros(2), None, 0, torch.zeros((1, 2)).int(), torch.zeros((1, 2)).int(), torch.zeros((1, 2)),
                         None, torch.zeros(256, dtype=torch.uint8))
    i = torch.zeros(2, dtype=torch.int32)
    t = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="int32"):
        B.sq_kv_reorder(i.long(), i, 16, 9, i, None, t, t, i, i, i, i, i, i)
    with pytest.raises(ValueError, match="sizes"):
        B.sq_kv_reorder(i, i, 16, 9, i, None, t, t[:1], i, i, i, i, i, i)
    with pytest.raises(ValueError, match="device tensors"):
        B.sq_kv_reorder(i, i, 16, 9, i, None, t, t, i, i, i, i, i, i)
    k = torch.zeros((2, 1, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        B.alloc_attn_shared_workspace(1, 1, 2, B.KVCache(k, k), 8, 8)
    with pytest.raises(ValueError, match="sizes"):
        B.sq_kv_copy_pages([], i, i[:1], None)
    with pytest.raises(ValueError, match="device tensors"):
        B.sq_kv_copy_pages([B.KVCache(k, k)], i, i, None)
    with pytest.raises(ValueError, match="invalid sizes"):
        B.alloc_beam_workspace(5, 2, 100, 2, device="cpu")
    with pytest.raises(ValueError, match="invalid sizes"):
        B.alloc_reorder_workspace(0, 2, device="cpu")


# ------------------------------------------------------------------ the plain forms, by hand
def test_plain_norm_by_hand():
    h, u, _, _ = R.add_rmsnorm(torch.tensor([[1.0, 3.0]]), torch.tensor([[2.0, 1.0]]), torch.tensor([10.0, 1.0]), 0.0)
    assert h.tolist() == [[3.0, 4.0]]
    assert torch.allclose(u, torch.tensor([[30.0, 4.0]], dtype=torch.float64) / math.sqrt(12.5))
    q, r = R.codes(torch.tensor([[1.0, -4.0, 0.25]]), torch.tensor([2.0, 0.5, 4.0]), torch.tensor([0.5]), None)
    assert q.tolist() == [[64, -64, 32]] and math.isclose(r.item(), 2 / 127 / 0.5, rel_tol=1e-6)  # 63.5 goes to even


def test_plain_choice_by_hand():
    logits = torch.log(torch.tensor([[0.5, 0.25, 0.25], [0.125, 0.125, 0.75], [1.0, 1.0, 2.0], [0.25, 0.3, 0.45]]))
    scores = torch.log(torch.tensor([0.5, 0.5, 0.5, 0.5]))
    best = R.beam_select(R.beam_totals(logits, scores, None, 0), logits, None, 2, 3)
    assert [[b[:2] for b in g] for g in best] == [[(1, 2), (0, 0), (0, 1)], [(2, 2), (3, 2), (3, 1)]]
    assert math.isclose(math.exp(best[0][0][2]), 0.375, rel_tol=1e-6)
    done = torch.tensor([1, 0, 0, 1])
    best = R.beam_select(R.beam_totals(logits, scores, done, 1), logits, done, 2, 2)
    assert [[b[:2] for b in g] for g in best] == [[(0, 1), (1, 2)], [(3, 1), (2, 2)]]


def test_plain_reorder_by_hand():
    # pages of 8; rows 0 and 1 share page 5, row 1 is dropped, row 0 goes on twice, row 2 is full, row 3 moves
    table = [[5, 6, -1], [5, 7, -1], [8, 9, -1], [3, -1, -1]]
    out, n, src, dst, rows, free, head = R.reorder([0, 0, 2, 2], [11, 13, 16, 2], 8, 10, [1, 1, 0, 2], 2, table, [[-9] * 3] * 4)
    # pages 7 and 3 come free: 7 is row 1's copy of page 6, 3 goes back to the list
    assert out == [[5, 6, -9], [5, 7, -9], [8, 9, -9], [8, 9, -9]]
    assert (n, src, dst, rows) == ([11, 11, 16, 16], [-1, 6, -1, -1], [-1, 7, -1, -1], [0, 3, 0, 0])
    assert (free, head) == ([1, 3, 0, 2], 1)
