"""The token step's operators on the GPU (page plan, head norm with rotation
and cache write, paged attention, bf16 linear on int4 weights) against plain
64-bit forms, at the sizes, masks, strides and contents where they can go
wrong."""
import math

import numpy as np
import pytest
import torch

import token_ref as T
from paper_2609_39056_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
OUT = {"bf16": B.SQ_OUT_BF16, "f16": B.SQ_OUT_F16, "f32": B.SQ_OUT_F32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ plan
def run_plan(cached, new, page, free, head, table, max_tokens, use_head=True):
    R = len(cached)
    d = dict(table=i32(table), slot=torch.full((max_tokens,), 77, dtype=torch.int32, device="cuda"),
             pos=torch.full((max_tokens,), 77, dtype=torch.int32, device="cuda"),
             start=torch.full((R + 1,), 77, dtype=torch.int32, device="cuda"),
             kv_len=torch.full((R,), 77, dtype=torch.int32, device="cuda"), head=i32([77]))
    B.sq_kv_plan(i32(cached), i32(new), page, i32(free), i32([head]) if use_head else None, d["table"], d["slot"],
                 d["pos"], d["start"], d["kv_len"], d["head"])
    return d


def check_plan(cached, new, page, free, head, table, max_tokens, use_head=True):
    d = run_plan(cached, new, page, free, head, table, max_tokens, use_head)
    want = T.plan(cached, new, page, free, head if use_head else 0, table, max_tokens)
    for name, w in zip(("table", "slot", "pos", "start", "kv_len"), want):
        assert d[name].tolist() == w, name
    assert d["head"].item() == want[5]


def random_plan(R, page, seed, longest, most_new, spare=0, max_tokens=None):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, longest + 1, R)
    new = rng.integers(0, most_new + 1, R)
    max_pages = -(-(longest + most_new) // page)
    ids = rng.permutation(R * max_pages + 16).astype(np.int64)
    have = -(-cached // page)
    table = np.full((R, max_pages), -1)
    at = 0
    for r in range(R):
        table[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
    wanted = int((-(-(cached + new) // page) - have).sum())
    free = ids[at:at + max(0, wanted + spare)]
    total = int(new.sum())
    return (cached.tolist(), new.tolist(), page, free.tolist(), 0, table.tolist(),
            total if max_tokens is None else max_tokens)


@pytest.mark.parametrize("R,page,longest,most_new", [(1, 8, 0, 1), (1, 16, 40, 0), (3, 16, 16, 1), (64, 16, 300, 1),
                                                     (65, 1024, 5000, 1500), (100, 8, 9, 33), (1023, 32, 70, 40),
                                                     (1025, 64, 200, 3), (5000, 16, 60, 5), (8192, 8, 20, 2)])
def test_plan(R, page, longest, most_new):
    check_plan(*random_plan(R, page, [1, R, page], longest, most_new))
    # entries past the tokens, and a head inside the free list
    cached, new, page, free, _, table, n = random_plan(R, page, [2, R, page], longest, most_new, spare=5)
    check_plan(cached, new, page, [9999] * 3 + free, 3, table, n + 70)
    check_plan(cached, new, page, free, 55, table, n, use_head=False)


def test_plan_requests_that_do_not_fit():
    # the pool ends in the middle: whoever needs a page from then on is left as it was, the others go on
    cached, new, page, free, _, table, n = random_plan(40, 16, 5, 100, 30, spare=-23)
    check_plan(cached, new, page, free, 0, table, n)
    check_plan(cached, new, page, [], 0, table, n)
    check_plan(cached, new, page, free, len(free) + 4, table, n)  # a head past the list counts as its end
    check_plan(cached, new, page, free, -3, table, n)
    # too few token entries, none at all
    check_plan(cached, new, page, free, 0, table, n // 2)
    check_plan(cached, new, page, free, 0, table, 0)
    # rows too short for some requests, lengths below zero, everything idle
    short = [row[:4] for row in table]
    check_plan(cached, new, page, free, 0, short, n)
    check_plan([-5, 3, -1], [2, -7, 0], 8, [4, 5], 0, [[1, 2], [3, 9], [7, 7]], 9)
    check_plan([0, 0, 17], [0, 0, 0], 16, [1], 0, [[1, 2]] * 3, 2)


def test_plan_sums_past_31_bits():
    big = 2 ** 31 - 1
    check_plan([5, 0, 3, 9], [1, big, big, 1], 8, [3, 4], 0, [[0, 7], [-1, -1], [2, -1], [5, 6]], 6)
    check_plan([big, big], [big, 1], 1024, [3], 0, [[1], [2]], 3)


# ------------------------------------------------------------------ norm and rotation
def rope_case(tokens, Hq, Hk, D, rot, dtype, seed, page=16, num_pos=50, norm=True):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn((tokens, (Hq + 2 * Hk) * D), generator=g) * 1.5).to(DT[dtype])
    pages = tokens // page + 3
    slot = torch.randperm(pages * page, generator=g)[:tokens].to(torch.int32)
    pos = torch.randint(0, num_pos, (tokens,), generator=g, dtype=torch.int32)
    ang = torch.rand((num_pos, rot // 2), generator=g) * 6.28
    w = [torch.randn((D,), generator=g) * 0.3 + 1 if norm else None for _ in range(2)]
    cos, sin = (ang.cos(), ang.sin()) if rot else (None, None)
    return dict(qkv=qkv, slot=slot, pos=pos, cos=cos, sin=sin, qw=w[0], kw=w[1],
                shape=(pages, Hk, page, D))


def split(qkv, Hq, Hk, D):
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D], dim=1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hk, D)), v.unflatten(1, (Hk, D))


def dev(t):
    return None if t is None else t.cuda()


def check_rope(c, tokens, Hq, Hk, D, dtype, inter, eps=1e-5, use_cache=True, use_k_out=False, skip_pos=(), skip_slot=()):
    dt = DT[dtype]
    pos, slot = c["pos"].clone(), c["slot"].clone()
    for i, p in skip_pos:
        pos[i] = p
    for i, s in skip_slot:
        slot[i] = s
    ck, cv = (torch.full(c["shape"], float("nan"), dtype=dt, device="cuda") for _ in range(2))
    q_out = torch.full((tokens, Hq, D), float("nan"), dtype=dt, device="cuda")
    k_out = torch.full((tokens, Hk, D), float("nan"), dtype=dt, device="cuda") if use_k_out else None
    q, k, v = split(c["qkv"].cuda(), Hq, Hk, D)
    rope = B.RopeParams(dev(c["qw"]), dev(c["kw"]), eps, dev(c["cos"]), dev(c["sin"]), inter)
    B.sq_qk_norm_rope(q, k, v if use_cache else None, rope, pos.cuda() if c["cos"] is not None else None,
                      slot.cuda() if use_cache else None, q_out, k_out, B.KVCache(ck, cv) if use_cache else None)
    q, k, v = split(c["qkv"], Hq, Hk, D)
    num_pos = 0 if c["cos"] is None else c["cos"].shape[0]
    done = torch.ones(tokens, dtype=torch.bool) if num_pos == 0 else (pos >= 0) & (pos < num_pos)
    safe = pos.clamp(0, max(num_pos - 1, 0))
    yq, bq = T.norm_rope(q, c["qw"], eps, c["cos"], c["sin"], safe, inter)
    yk, bk = T.norm_rope(k, c["kw"], eps, c["cos"], c["sin"], safe, inter)
    T.check(q_out.cpu()[done], yq[done], bq[done], dt, "q")
    assert torch.isnan(q_out.cpu()[~done]).all()
    if use_k_out:
        T.check(k_out.cpu()[done], yk[done], bk[done], dt, "k_out")
        assert torch.isnan(k_out.cpu()[~done]).all()
    if use_cache:
        pages, _, P, _ = c["shape"]
        kept = done & (slot >= 0) & (slot < pages * P)
        s = slot[kept].long()
        T.check(ck.cpu()[s // P, :, s % P], yk[kept], bk[kept], dt, "k")
        assert torch.equal(cv.cpu()[s // P, :, s % P], v[kept])
        other = torch.ones(pages * P, dtype=torch.bool)
        other[s] = False
        o = other.nonzero()[:, 0]
        assert torch.isnan(ck.cpu()[o // P, :, o % P]).all() and torch.isnan(cv.cpu()[o // P, :, o % P]).all()


@pytest.mark.parametrize("Hq,Hk,D,rots", [(16, 16, 128, (128, 64, 0, 16)), (40, 8, 128, (128,)), (14, 2, 64, (64, 32)),
                                          (25, 5, 64, (64, 48)), (5, 5, 96, (96, 48)), (8, 1, 256, (256, 128)),
                                          (12, 12, 192, (192, 96)), (1, 1, 64, (64, 16)), (33, 11, 128, (112,))])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rope(Hq, Hk, D, rots, dtype):
    for rot in rots:
        for tokens, inter, norm in ((1, False, True), (7, True, True), (67, False, True), (20, False, False),
                                    (33, True, False)):
            c = rope_case(tokens, Hq, Hk, D, rot, dtype, 11 * tokens + rot, norm=norm)
            check_rope(c, tokens, Hq, Hk, D, dtype, inter, use_k_out=inter)


def test_rope_skipped_tokens_and_slots():
    c = rope_case(40, 8, 2, 128, 128, "bf16", 3, page=8, num_pos=9)
    n = c["shape"][0] * 8
    check_rope(c, 40, 8, 2, 128, "bf16", False, use_k_out=True, skip_pos=((0, -1), (5, 9), (39, 2 ** 31 - 1)),
               skip_slot=((1, -1), (5, -1), (7, n), (8, 2 ** 31 - 1), (9, -2 ** 31)))
    check_rope(c, 40, 8, 2, 128, "bf16", True, skip_pos=[(i, -1) for i in range(40)])


def test_rope_without_a_cache():
    for dtype in ("bf16", "f16"):
        c = rope_case(129, 16, 16, 128, 128, dtype, 4)
        check_rope(c, 129, 16, 16, 128, dtype, False, use_cache=False, use_k_out=True)


def test_rope_small_and_zero_rows():
    """Rows of zeros stay zero; rows far below eps keep their size."""
    c = rope_case(6, 4, 2, 64, 64, "f16", 6)
    c["qkv"][1] = 0
    c["qkv"][3] *= 2.0 ** -12
    check_rope(c, 6, 4, 2, 64, "f16", False, eps=1e-6)
    c = rope_case(6, 4, 2, 64, 64, "bf16", 7)
    c["qkv"][0] *= 2.0 ** 40
    check_rope(c, 6, 4, 2, 64, "bf16", True, eps=0.0)


def test_rope_no_tokens():
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    B.sq_qk_norm_rope(q, q, None, B.RopeParams(), None, None, q, q, None)


# ------------------------------------------------------------------ attention
def attn_case(R, L, Hq, Hk, D, page, dtype, seed, lens=None, spare=3):
    g = torch.Generator().manual_seed(seed)
    if lens is None:
        lens = torch.randint(0, L + 1, (R,), generator=g).tolist()
        lens[-1] = L
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare
    ids = torch.randperm(total, generator=g).to(torch.int32)
    max_pages = max(1, -(-L // page))
    table = torch.full((R, max_pages), -7, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    dt = DT[dtype]
    k, v = (torch.randn((total, Hk, page, D), generator=g).to(dt) for _ in range(2))
    # what is not attended holds NaN and infinities
    live = torch.zeros((total, page), dtype=torch.bool)
    for r, n in enumerate(lens):
        for j in range(need[r]):
            live[table[r, j].long(), :min(page, n - j * page)] = True
    dead = ~live[:, None, :, None].expand_as(k)
    k[dead], v[dead] = float("nan"), float("nan")
    k[dead & (torch.rand(k.shape, generator=g) < 0.3)] = float("inf")
    v[dead & (torch.rand(k.shape, generator=g) < 0.3)] = float("-inf")
    q = torch.randn((R, Hq, D), generator=g).to(dt)
    return dict(q=q, k=k, v=v, table=table, kv_len=torch.tensor(lens, dtype=torch.int32), L=L)


def run_attn(c, out_dtype, window=0, scale=None, max_kv_len=None, lse=True, ws=None):
    R, Hq, D = c["q"].shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    n = c["L"] if max_kv_len is None else max_kv_len
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    out = torch.full((R, Hq, D), float("nan"), dtype=DT[out_dtype], device="cuda")
    ls = torch.full((R, Hq), float("nan"), device="cuda") if lse else None
    if ws is None:
        ws = B.alloc_attn_workspace(R, Hq, kv, n)
        ws.fill_(255)  # NaN patterns
    B.sq_attn_paged(c["q"].cuda(), kv, c["table"].cuda(), c["kv_len"].cuda(), n, window, scale, out, OUT[out_dtype], ls, ws)
    return out, ls


def check_attn(c, out_dtype, window=0, scale=None, max_kv_len=None):
    out, ls = run_attn(c, out_dtype, window, scale, max_kv_len)
    D = c["q"].shape[2]
    y, lse, b, bl = T.attn(c["q"], c["k"], c["v"], c["table"], c["kv_len"], window,
                           1 / math.sqrt(D) if scale is None else scale, c["L"] if max_kv_len is None else max_kv_len,
                           DT[out_dtype])
    T.check(out, y, b, DT[out_dtype], "out")
    ls = ls.cpu().double()
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(ls) & (ls < 0), empty)
    T.check(ls[~empty], lse[~empty], bl[~empty], torch.float32, "lse")


@pytest.mark.parametrize("Hq,Hk,D", [(4, 4, 128), (16, 2, 128), (10, 2, 64), (7, 1, 64), (3, 3, 96), (16, 1, 256),
                                     (4, 2, 192), (32, 1, 128), (17, 1, 64), (40, 1, 96)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attn_heads(Hq, Hk, D, dtype):
    for page, L, out in ((8, 75, dtype), (16, 300, "f32"), (64, 1200, dtype)):
        check_attn(attn_case(4, L, Hq, Hk, D, page, dtype, Hq + D + L), out)


@pytest.mark.parametrize("Hq,Hk,D,page,dtype,out", [
    (32, 1, 128, 16, "bf16", "f32"), (17, 1, 64, 8, "f16", "f16"), (40, 1, 96, 64, "bf16", "bf16"),
    (72, 2, 128, 32, "f16", "f32")])
def test_attn_many_heads_of_one(Hq, Hk, D, page, dtype, out):
    """Enough requests of long and short histories that a workgroup takes 32 query heads, whole and split."""
    for R, L in ((130, 410), (12, 1700)):
        lens = ([L, 0, 1, 33, L - 1, 300, 31, 32] + [(37 * r) % 90 for r in range(R)])[:R]
        c = attn_case(R, L, Hq, Hk, D, page, dtype, Hq + L, lens=lens)
        check_attn(c, out)
        check_attn(c, out, window=390)


def test_attn_short_lengths():
    """Every length around the tile's and the page's ends, in one batch."""
    lens = list(range(0, 70)) + [127, 128, 129, 255, 256, 257]
    for page in (8, 16, 32, 128):
        for Hq, Hk, D, dtype, out in ((2, 1, 128, "bf16", "f32"), (4, 4, 64, "f16", "f16")):
            check_attn(attn_case(len(lens), 257, Hq, Hk, D, page, dtype, page, lens=lens), out)


@pytest.mark.parametrize("window", [1, 15, 31, 32, 33, 100, 512, 10 ** 9])
def test_attn_window(window):
    lens = [0, 1, 14, 15, 16, 31, 32, 33, 64, 99, 100, 101, 500, 1111]
    check_attn(attn_case(len(lens), 1111, 4, 2, 128, 16, "bf16", 9, lens=lens), "f32", window=window)
    check_attn(attn_case(len(lens), 1111, 3, 3, 64, 32, "f16", 9, lens=lens), "f16", window=window)


@pytest.mark.parametrize("R,L,Hq,Hk,D,page,dtype,out", [
    (1, 20011, 8, 1, 128, 16, "bf16", "f32"), (2, 9001, 16, 16, 64, 8, "f16", "f16"),
    (1, 40000, 4, 1, 256, 1024, "bf16", "bf16"), (3, 12345, 10, 2, 96, 64, "bf16", "f32"),
    (1, 66000, 5, 1, 64, 128, "f16", "f32")])
def test_attn_long(R, L, Hq, Hk, D, page, dtype, out):
    """Histories split over workgroups, beside short ones and an empty one."""
    lens = [L, 0, 37][:R]
    c = attn_case(R, L, Hq, Hk, D, page, dtype, L, lens=lens)
    check_attn(c, out)
    check_attn(c, out, window=L // 2 + 5)
    a, la = run_attn(c, out)
    b, lb = run_attn(c, out)
    assert torch.equal(a, b) and torch.equal(la, lb)  # the same bits again


def test_attn_capacity_above_the_lengths():
    """max_kv_len is a bound: larger gives the same rows, smaller cuts the lengths."""
    c = attn_case(5, 900, 8, 2, 128, 16, "bf16", 21)
    c["table"] = torch.cat([c["table"], torch.full((5, 4000), 10 ** 6, dtype=torch.int32)], 1)
    check_attn(c, "f32", max_kv_len=900 + 40000)
    check_attn(c, "f32", max_kv_len=333)
    check_attn(c, "f32", max_kv_len=0)
    c["kv_len"] = torch.tensor([-4, 10 ** 9, 900, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)
    c["k"].nan_to_num_(0.5, 0.5, 0.5)
    c["v"].nan_to_num_(0.5, 0.5, 0.5)
    check_attn(c, "f32", max_kv_len=900)


def test_attn_absent_pages():
    """Tokens of pages outside the cache are not attended, whichever they are."""
    c = attn_case(4, 700, 8, 2, 128, 16, "bf16", 31, lens=[700, 700, 40, 16])
    pages = c["k"].shape[0]
    c["table"][0, 3], c["table"][0, 17], c["table"][0, 43] = -1, pages, 2 ** 31 - 1
    c["table"][1, :] = -2 ** 31
    c["table"][2, 0] = pages + 5
    check_attn(c, "f32")
    check_attn(c, "bf16", window=33)


def test_attn_large_scores():
    """Scores far apart and far from zero: the running maximum moves often."""
    c = attn_case(3, 2000, 4, 2, 64, 16, "bf16", 41)
    ramp = torch.linspace(-1, 1, c["k"].shape[0]).view(-1, 1, 1, 1)
    c["k"] = (c["k"].float() + 6 * ramp).to(torch.bfloat16)
    check_attn(c, "f32", scale=3.0)
    check_attn(c, "f32", scale=-2.0)
    check_attn(c, "f32", scale=0.0)


def test_attn_strided_queries_and_another_stream():
    R, Hq, Hk, D = 6, 8, 2, 128
    c = attn_case(R, 500, Hq, Hk, D, 16, "bf16", 51)
    want, _ = run_attn(c, "f32")
    torch.cuda.synchronize()
    qkv = torch.full((R, (Hq + 2 * Hk) * D), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = qkv[:, :Hq * D].unflatten(1, (Hq, D))
    q.copy_(c["q"])
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    out = torch.zeros((R, Hq, D), device="cuda")
    table, kv_len, ws = c["table"].cuda(), c["kv_len"].cuda(), B.alloc_attn_workspace(R, Hq, kv, 500)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.sq_attn_paged(q, kv, table, kv_len, 500, 0, 1 / math.sqrt(D), out, B.SQ_OUT_F32, None, ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


def test_attn_cache_past_32_bits():
    """Pages beyond 2^32 elements of the cache."""
    Hk, P, D = 8, 64, 128
    pages = 2 ** 32 // (Hk * P * D) + 40
    k, v = (torch.empty((pages, Hk, P, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = attn_case(2, 600, 16, Hk, D, P, "bf16", 61)
    n = small["k"].shape[0]
    k[pages - n:], v[pages - n:] = small["k"].cuda(), small["v"].cuda()
    want, _ = run_attn(small, "f32")
    out = torch.zeros((2, 16, D), device="cuda")
    kv = B.KVCache(k, v)
    table = torch.where(small["table"] >= 0, small["table"] + (pages - n), -1).cuda()
    B.sq_attn_paged(small["q"].cuda(), kv, table, small["kv_len"].cuda(), 600, 0, 1 / math.sqrt(D), out, B.SQ_OUT_F32,
                    None, B.alloc_attn_workspace(2, 16, kv, 600))
    assert torch.equal(out, want)
    # the cache write of the last slots
    c = rope_case(5, 16, Hk, D, 128, "bf16", 62)
    slot = i32([pages * P - 1 - 7 * i for i in range(5)])
    q, kk, vv = split(c["qkv"].cuda(), 16, Hk, D)
    k_out = torch.zeros((5, Hk, D), dtype=torch.bfloat16, device="cuda")
    rope = B.RopeParams(dev(c["qw"]), dev(c["kw"]), 1e-5, dev(c["cos"]), dev(c["sin"]))
    B.sq_qk_norm_rope(q, kk, vv, rope, c["pos"].cuda(), slot, torch.zeros_like(q.contiguous()), k_out, kv)
    s = slot.long()
    assert torch.equal(k[s // P, :, s % P], k_out) and torch.equal(v[s // P, :, s % P], vv)


def test_attn_no_requests():
    c = attn_case(1, 40, 4, 2, 64, 16, "bf16", 71)
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    B.sq_attn_paged(q, kv, i32([[0]])[:0], i32([]), 16, 0, 1.0, q, B.SQ_OUT_BF16, None,
                    torch.empty(256, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------ linear
def linear_case(M, K, N, group, use_d, use_b, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((N, K), generator=g) * 0.05
    chan = torch.where(torch.rand((K,), generator=g) < 0.03, 20.0, 1.0)
    x = (torch.randn((M, K), generator=g) * chan).to(torch.bfloat16)
    dinv = (torch.rand((K,), generator=g) + 0.5) / chan if use_d else None
    bias = torch.randn((N,), generator=g).to(torch.bfloat16) if use_b else None
    W = B.prepare_weight(w.cuda(), None if dinv is None else (1 / dinv).cuda(), group, dev(bias))
    return x, dinv, W, bias


@pytest.mark.parametrize("M,K,N,group", [(1, 128, 64, 128), (1, 2048, 2048, 128), (2, 256, 64, 256), (3, 384, 192, 128),
                                         (5, 1152, 320, 384), (1, 5120, 1728, 5120), (8, 640, 576, 128),
                                         (15, 2048, 64, 2048), (16, 1280, 128, 256), (17, 1024, 704, 128),
                                         (32, 13824, 64, 128), (33, 896, 256, 896), (48, 4224, 192, 128),
                                         (64, 2048, 1024, 128), (1, 32768, 64, 128), (64, 32768, 64, 32768),
                                         (2, 8192, 2560, 128), (7, 128, 13824, 128)])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_linear(M, K, N, group, out):
    for use_d, use_b in ((True, True), (False, False)) if out != "f16" else ((True, False), (False, True)):
        x, dinv, W, bias = linear_case(M, K, N, group, use_d, use_b, M + K + N)
        y = torch.full((M + 1, N), float("nan"), dtype=DT[out], device="cuda")
        B.sq_linear_w4a16(x.cuda(), dev(dinv), W, y[:M], OUT[out])
        assert torch.isnan(y[M]).all()
        want, bound = T.linear(x, dinv, W.qw.cpu().numpy(), W.w_scale.cpu(), group, bias, DT[out])
        T.check(y[:M], want, bound, DT[out], "y")


@pytest.mark.parametrize("M,K,N,group", [(13, 1152, 5120, 128), (30, 1408, 2112, 128), (29, 384, 4736, 384),
                                         (47, 1152, 5120, 1152), (64, 128, 6144, 128), (37, 1152, 8256, 128),
                                         (64, 640, 9024, 640), (33, 128, 13824, 128)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_linear_tiles(M, K, N, group, out):
    """Wide strips and two row tiles, with CUs to spare and without, ragged rows and blocks."""
    for use_d in (True, False):
        x, dinv, W, bias = linear_case(M, K, N, group, use_d, True, M + K + N)
        y = torch.full((M + 1, N), float("nan"), dtype=DT[out], device="cuda")
        B.sq_linear_w4a16(x.cuda(), dev(dinv), W, y[:M], OUT[out])
        assert torch.isnan(y[M]).all()
        want, bound = T.linear(x, dinv, W.qw.cpu().numpy(), W.w_scale.cpu(), group, bias, DT[out])
        T.check(y[:M], want, bound, DT[out], "y")


def test_linear_all_codes():
    """Every nibble, -8 included (the packer writes -7 .. 7, the product takes
    what a nibble holds), on integers: exact."""
    M, K, N = 4, 256, 64
    g = torch.Generator().manual_seed(5)
    qw = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    x = torch.randint(-9, 10, (M, K), generator=g).to(torch.bfloat16)
    step = torch.exp2(torch.randint(-4, 3, (K // 128, N), generator=g).float()).half()
    W = B.Weight(qw.cuda(), step.cuda(), 128)
    want = x.double() @ (T.unpack(qw.numpy()).double() * step.double().t().repeat_interleave(128, 1)).t()
    for dinv in (None, torch.full((K,), 0.25)):
        y = torch.empty((M, N), device="cuda")
        B.sq_linear_w4a16(x.cuda(), dev(dinv), W, y, B.SQ_OUT_F32)
        assert torch.equal(y.cpu().double(), want * (1.0 if dinv is None else 0.25))


def test_linear_rows_do_not_mix():
    """A row's outputs do not depend on the rows beside it, infinite ones included."""
    x, dinv, W, bias = linear_case(21, 1024, 256, 128, True, True, 9)
    y = torch.empty((21, 256), device="cuda")
    B.sq_linear_w4a16(x.cuda(), dev(dinv), W, y, B.SQ_OUT_F32)
    x2 = x.clone()
    x2[4], x2[18] = float("inf"), float("nan")
    y2 = torch.empty((21, 256), device="cuda")
    B.sq_linear_w4a16(x2.cuda(), dev(dinv), W, y2, B.SQ_OUT_F32)
    keep = [i for i in range(21) if i not in (4, 18)]
    assert torch.equal(y[keep], y2[keep])


# ------------------------------------------------------------------ graphs
def test_step_in_a_graph():
    """Plan, rotation, attention and linear captured once and replayed with
    other lengths: every replay gives what the eager calls give."""
    R, Hq, Hk, D, P, cap = 5, 8, 2, 128, 16, 512
    g = torch.Generator().manual_seed(81)
    kv = B.KVCache(*(torch.randn((R * cap // P, Hk, P, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2)))
    c = rope_case(R, Hq, Hk, D, 128, "bf16", 82, num_pos=cap)
    qkv = c["qkv"].cuda()
    q, k, v = split(qkv, Hq, Hk, D)
    rope = B.RopeParams(dev(c["qw"]), dev(c["kw"]), 1e-5, dev(c["cos"]), dev(c["sin"]))
    _, dinv, W, _ = linear_case(1, Hq * D, 256, 128, True, True, 83)
    dinv = dinv.cuda()
    ids = torch.randperm(R * cap // P, generator=g).to(torch.int32).cuda()
    table0 = ids.view(R, -1).clone()
    free, new = ids.flip(0).contiguous(), i32([1] * R)
    cached = i32([0] * R)
    bufs = dict(slot=i32([0] * R), pos=i32([0] * R), start=i32([0] * (R + 1)), kv_len=i32([0] * R), head=i32([0]))
    table = table0.clone()
    q_out, attn = torch.empty_like(q.contiguous()), torch.empty((R, Hq, D), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((R, 256), device="cuda")
    ws = B.alloc_attn_workspace(R, Hq, kv, cap)

    def step():
        B.sq_kv_plan(cached, new, P, free, None, table, bufs["slot"], bufs["pos"], bufs["start"], bufs["kv_len"],
                     bufs["head"])
        B.sq_qk_norm_rope(q, k, v, rope, bufs["pos"], bufs["slot"], q_out, None, kv)
        B.sq_attn_paged(q_out, kv, table, bufs["kv_len"], cap, 0, 0.09, attn, B.SQ_OUT_BF16, None, ws)
        B.sq_linear_w4a16(attn.view(R, Hq * D), dinv, W, y, B.SQ_OUT_F32)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, lens in enumerate([[0, 1, 2, 3, 4], [17, 300, 0, 511, 64], [15, 16, 31, 100, 7], [500, 400, 300, 200, 100]]):
        cached.copy_(i32(lens))
        table.copy_(table0)
        qkv.copy_((torch.randn(qkv.shape, generator=g) * 1.5).to(torch.bfloat16))
        k0, v0 = kv.k.clone(), kv.v.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*bufs.values(), table, q_out, attn, y, kv.k, kv.v)]
        table.copy_(table0)
        kv.k.copy_(k0)
        kv.v.copy_(v0)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (*bufs.values(), table, q_out, attn, y, kv.k, kv.v)):
            assert torch.equal(a, b), i
