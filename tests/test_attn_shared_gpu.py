"""Attention over shared prefixes on the GPU against the 64-bit form of attention
over each request's whole history."""
import math

import pytest
import torch

import token_ref as T
from paper_2609_39056_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
OUT = {"bf16": B.SQ_OUT_BF16, "f16": B.SQ_OUT_F16, "f32": B.SQ_OUT_F32}
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def case(sizes, shared, kv_len, Hq, Hk, D, page, dt, seed=0, spare_pages=3, outside=(0, 0)):
    """Groups of `sizes` requests with shared[g] tokens in common (outside: requests before and behind the groups);
    tables whose rows have the group's pages as far as they are full, and each its own copy of the shared tokens
    of a partly filled one; every other row of the cache is NaN."""
    g = torch.Generator().manual_seed(seed)
    R = sum(sizes) + sum(outside)
    start = [outside[0]]
    for n in sizes:
        start.append(start[-1] + n)
    most = max([-(-n // page) for n in list(kv_len) + list(shared)] + [1])
    need = sum(-(-n // page) for n in kv_len) + sum(s // page for s in shared)
    num_pages = need + spare_pages
    ids = iter(torch.randperm(num_pages, generator=g).tolist())
    k = torch.full((num_pages, Hk, page, D), NAN)
    v = torch.full((num_pages, Hk, page, D), NAN)
    table = torch.full((R, most), -1, dtype=torch.int32)

    def fill(p, a, b):
        k[p, :, a:b] = torch.randn((Hk, b - a, D), generator=g)
        v[p, :, a:b] = torch.randn((Hk, b - a, D), generator=g)

    for gi in range(-1, len(sizes)):
        members = [r for r in range(R) if not start[0] <= r < start[-1]] if gi < 0 else range(start[gi], start[gi + 1])
        s = 0 if gi < 0 else shared[gi]
        common = []
        if gi >= 0 and max([kv_len[r] for r in members] + [0]) >= page:
            common = [next(ids) for _ in range(min(s, max(kv_len[r] for r in members)) // page)]
        for p in common:
            fill(p, 0, page)
        tail = None
        for r in members:
            for j in range(-(-kv_len[r] // page)):
                if j < len(common):
                    table[r, j] = common[j]
                    continue
                p = next(ids)
                table[r, j] = p
                fill(p, 0, min(page, kv_len[r] - j * page))
                if j == s // page and s % page:  # the shared tokens of a partly filled page
                    n = min(s % page, kv_len[r] - j * page)
                    if tail is None or tail[0].shape[1] < n:
                        old = 0 if tail is None else tail[0].shape[1]
                        t = torch.randn((2, Hk, s % page, D), generator=g)
                        if tail is not None:
                            t[0, :, :old], t[1, :, :old] = tail
                        tail = t[0], t[1]
                    k[p, :, :n], v[p, :, :n] = tail[0][:, :n], tail[1][:, :n]
    q = torch.randn((R, Hq, D), generator=g)
    c = dict(q=q.to(DT[dt]), k=k.to(DT[dt]), v=v.to(DT[dt]), table=table, kv_len=list(kv_len), start=start, shared=list(shared),
             scale=1 / math.sqrt(D), page=page)
    return c


def run(c, out, max_shared=None, max_own=None, lse=True, q=None, ws=None, stream=None):
    R, Hq, D = c["q"].shape
    shared = max(c["shared"] + [0])
    own = max([n for n in c["kv_len"]] + [0])
    max_shared = shared if max_shared is None else max_shared
    max_own = own if max_own is None else max_own
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    o = torch.full((R, Hq, D), 7.0, dtype=DT[out], device="cuda")
    ls = torch.full((R, Hq), 7.0, device="cuda") if lse else None
    if ws is None:
        n = B.sq_attn_shared_workspace_bytes(R, len(c["shared"]), Hq, kv, max_shared, max_own)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN everywhere
    B.sq_attn_shared(c["q"].cuda() if q is None else q, kv, c["table"].cuda(), i32(c["kv_len"]), i32(c["start"]),
                     i32(c["shared"]) if c["shared"] else i32([0])[:0], max_shared, max_own, c["scale"], o, OUT[out], ls, ws, stream)
    return o, ls


def reference(c, out, max_shared=None, max_own=None):
    """Each request's whole history: the shared tokens in the pages of the group's first request that has the most."""
    R = c["q"].shape[0]
    P = c["page"]
    table, n = c["table"].clone(), list(c["kv_len"])
    cap = table.shape[1] * P
    member = [-1] * R
    for g in range(len(c["shared"])):
        for r in range(c["start"][g], c["start"][g + 1]):
            member[r] = g
    k, v, extra = c["k"], c["v"], []
    rows = []
    for r in range(R):
        g = member[r]
        p = 0 if g < 0 else min(max(c["shared"][g], 0), cap)
        if g >= 0 and max_shared is not None:
            p = min(p, max_shared)
        length = min(max(n[r], 0), cap)
        if max_own is not None:
            length = min(length, p + max_own)
        rows.append((g, p, length))
    # a request's tokens, gathered into pages of its own
    out_k, out_v, new = [], [], torch.full((R, max(1, max([-(-x[2] // P) for x in rows]))), -1, dtype=torch.int32)
    at = 0
    for r, (g, p, length) in enumerate(rows):
        reader = r
        if g >= 0:
            most = [min(min(max(n[m], 0), cap), p) for m in range(c["start"][g], c["start"][g + 1])]
            reader = c["start"][g] + most.index(max(most))
        pages = -(-length // P)
        if pages == 0:
            continue
        j = torch.arange(pages * P)
        rowtab = torch.where(j < p, table[reader].long()[(j // P).clamp(max=table.shape[1] - 1)], table[r].long()[j // P])
        ok = (rowtab >= 0) & (rowtab < k.shape[0]) & (j < length)
        kk, vv = k[rowtab.clamp(0, k.shape[0] - 1), :, j % P], v[rowtab.clamp(0, k.shape[0] - 1), :, j % P]
        extra.append((r, ok))
        out_k.append(kk.view(pages, P, *kk.shape[1:]).transpose(1, 2))
        out_v.append(vv.view(pages, P, *vv.shape[1:]).transpose(1, 2))
        new[r, :pages] = torch.arange(at, at + pages)
        at += pages
    # tokens of pages that are none are left out: move the others together
    for i, (r, ok) in enumerate(extra):
        if not ok[:rows[r][2]].all():
            keep = ok.nonzero()[:, 0]
            for o in (out_k, out_v):
                flat = o[i].transpose(1, 2).reshape(-1, *o[i].shape[1:2], o[i].shape[3])
                moved = torch.zeros_like(flat)
                moved[:len(keep)] = flat[keep]
                o[i] = moved.view(o[i].shape[0], P, *o[i].shape[1:2], o[i].shape[3]).transpose(1, 2)
            rows[r] = (rows[r][0], rows[r][1], len(keep))
    if not out_k:
        out_k, out_v = [k[:1]], [v[:1]]
    return T.attn(c["q"], torch.cat(out_k), torch.cat(out_v), new, [x[2] for x in rows], 0, c["scale"], 1 << 30, DT[out])


def check(c, out, **kw):
    o, lse = run(c, out, **kw)
    want, wl, bo, bl = reference(c, out, kw.get("max_shared"), kw.get("max_own"))
    T.check(o, want, bo, DT[out], "out")
    live = torch.isfinite(wl)
    assert torch.equal(lse.cpu() == -INF, ~live)
    T.check(torch.where(live, lse.cpu(), 0.0), torch.where(live, wl, 0.0), torch.where(live, bl, 0.0), torch.float32, "lse")
    return o


HEADS = [(4, 4, 64), (8, 2, 96), (10, 2, 128), (5, 1, 192), (4, 2, 256), (16, 1, 128), (40, 2, 64)]


@pytest.mark.parametrize("Hq,Hk,D", HEADS)
@pytest.mark.parametrize("dt,out", [("bf16", "bf16"), ("f16", "f32"), ("f16", "f16"), ("bf16", "f32")])
def test_groups(Hq, Hk, D, dt, out):
    # a group of every size that a tile of rows ends in, prefixes that end inside pages and tiles, single requests
    shared = [100, 0, 1, 64, 33, 200, 16]
    sizes = [3, 2, 1, 9, 17, 4, 0]
    g = torch.Generator().manual_seed(D + Hq)
    kv_len = []
    for n, s in zip(sizes, shared):
        kv_len += [s + int(torch.randint(0, 70, (1,), generator=g)) for _ in range(n)]
    check(case(sizes, shared, kv_len, Hq, Hk, D, 16, dt), out)


@pytest.mark.parametrize("page,Hq,Hk,D", [(8, 4, 2, 64), (128, 8, 1, 128), (1024, 2, 2, 96), (8, 6, 1, 128), (8, 3, 1, 96), (8, 4, 1, 192),
                                          (8, 4, 1, 256), (16, 6, 1, 96), (64, 10, 2, 256), (32, 5, 1, 192), (16, 12, 1, 64)])
def test_one_long_prefix(page, Hq, Hk, D):
    # many chunks, one group, requests whose own part is empty, one token, more than a chunk
    s = 5000 if page < 1024 else 4096
    kv_len = [s, s + 1, s + 31, s + 400, s + 1700, s + 2, s + 33]
    check(case([7], [s], kv_len, Hq, Hk, D, page, "bf16"), "f32")
    check(case([2], [s], kv_len[1:3], Hq, Hk, D, page, "f16"), "f16")
    check(case([1], [s], kv_len[4:5], Hq, Hk, D, page, "bf16"), "bf16")


@pytest.mark.parametrize("rows,Hq,Hk", [(16, 2, 2), (17, 2, 2), (33, 4, 4), (13, 10, 2), (64, 5, 1), (65, 3, 3), (130, 2, 1)])
def test_tiles_of_rows(rows, Hq, Hk):
    g = torch.Generator().manual_seed(rows)
    kv_len = [300 + int(torch.randint(0, 40, (1,), generator=g)) for _ in range(rows)]
    check(case([rows], [290], kv_len, Hq, Hk, 128, 32, "bf16"), "bf16")
    check(case([rows], [290], kv_len, Hq, Hk, 64, 32, "f16"), "f32")


def test_requests_that_are_shorter_than_their_prefix():
    # idle ones, some of a prefix, all of it; in front of and behind those that have it all
    for kv_len in ([0, 150, 40, 100, 200, 0], [0, 0, 0, 0, 0, 0], [99, 17, 1, 64, 98, 32], [160, 0, 0, 0, 0, 0], [0, 0, 0, 0, 0, 130]):
        c = case([6], [100], kv_len, 4, 2, 64, 16, "bf16")
        check(c, "f32")
        check(c, "bf16")
    kv_len = [0, 150, 40, 100, 200, 0, 700, 13, 0, 0, 0, 500, 512, 511, 513, 0]
    check(case([5, 1, 3, 7], [100, 0, 512, 500], kv_len, 8, 2, 128, 16, "f16"), "f16")


def test_requests_outside_groups():
    kv_len = [50, 0, 33, 120, 130, 200, 90, 210]
    check(case([3], [100], kv_len, 4, 4, 64, 16, "bf16", outside=(3, 2)), "bf16")
    c = case([], [], [50, 0, 700], 4, 4, 64, 16, "bf16", outside=(3, 0))
    c["start"] = [0]
    o = check(c, "bf16")
    c["shared"], c["start"] = [0, 0], [0, 0, 3]
    assert torch.equal(o, run(c, "bf16")[0])


def test_many_groups():
    g = torch.Generator().manual_seed(1)
    for groups in (63, 64, 65, 200):
        sizes = torch.randint(0, 3, (groups,), generator=g).tolist()
        shared = torch.randint(0, 40, (groups,), generator=g).tolist()
        kv_len = [s + int(torch.randint(0, 9, (1,), generator=g)) for n, s in zip(sizes, shared) for _ in range(n)]
        check(case(sizes, shared, kv_len, 2, 1, 64, 8, "bf16"), "f32")
    sizes = [1 if i % 9 == 0 else 0 for i in range(5000)]
    shared = [i % 20 for i in range(5000)]
    check(case(sizes, shared, [1 + s for n, s in zip(sizes, shared) if n], 2, 1, 64, 8, "f16"), "f32")


def test_bounds_cut_what_is_attended():
    kv_len = [140, 250, 101, 100, 30]
    c = case([5], [100], kv_len, 4, 2, 64, 16, "bf16")
    for max_shared, max_own in ((100, 200), (256, 256), (100, 40), (100, 1), (100, 0), (64, 256), (33, 70), (0, 256), (0, 0), (1, 5)):
        check(c, "f32", max_shared=max_shared, max_own=max_own)
    c["kv_len"][1] = 2 ** 31 - 1  # past the table's row
    c["kv_len"][0] = -5
    c["shared"][0] = 2 ** 31 - 1
    cut = dict(c, kv_len=[0, 256, 101, 100, 30], shared=[256])
    got = run(c, "f32", max_shared=256, max_own=256)
    want = run(cut, "f32", max_shared=256, max_own=256)
    assert torch.isnan(want[1][1]).all()  # rows that the cache has as NaN are attended
    assert all(torch.allclose(a, b, rtol=0, atol=0, equal_nan=True) for a, b in zip(got, want))


def test_pages_that_are_none():
    for where in ((0, 1), (0, 6), (1, 7), (2, 6)):
        c = case([3], [100], [150, 140, 200], 4, 2, 64, 16, "bf16")
        for bad in (-1, c["k"].shape[0], 2 ** 31 - 1):
            c["table"][where] = bad
            check(c, "f32")
    c["table"][:] = -1
    o, lse = run(c, "f32")
    assert (o == 0).all() and (lse == -INF).all()


def test_values_that_are_not_finite():
    c = case([4], [100], [150, 140, 60, 101], 2, 2, 64, 16, "bf16")
    base, lbase = run(c, "f32")
    page = c["table"][0, 4].item()  # tokens 64 .. 79, past request 2
    c["v"][page, 0, 3, 5] = INF
    c["v"][page, 1, 4, 7] = -INF
    o, lse = run(c, "f32")
    assert torch.equal(lse, lbase)
    full = [0, 1, 3]
    assert (o[full, 0, 5] == INF).all() and (o[full, 1, 7] == -INF).all() and torch.isfinite(o[2]).all()
    # what is beside them differs by the order of its sum: one row was formed token by token, 100 products
    keep = torch.ones_like(o, dtype=torch.bool)
    keep[full, 0, 5] = keep[full, 1, 7] = False
    assert (o - base)[keep].abs().max() <= 256 * 2.0 ** -24 * 8
    c["v"][page, 0, 3, 5] = NAN
    o, lse = run(c, "f32")
    assert torch.isnan(o[full, 0, 5]).all() and torch.isfinite(o[2]).all() and torch.equal(lse, lbase)
    # a NaN key makes a NaN score for those that attend it
    c["k"][page, 0, 3, 5] = NAN
    o, lse = run(c, "f32")
    assert torch.isnan(o[full, 0]).all() and torch.isnan(lse[full, 0]).all() and torch.isfinite(lse[:, 1]).all()
    assert torch.isfinite(o[2]).all()
    # own tokens
    c = case([2], [32], [40, 50], 2, 1, 128, 16, "f16")
    c["v"][c["table"][1, 2].item(), 0, 1, 9] = INF
    o, _ = run(c, "f16")
    assert torch.isfinite(o[0]).all() and (o[1, :, 9] == INF).all() and torch.isfinite(o[1, :, 10:]).all()


def test_scores_of_all_sizes():
    # a shared token far above and far below the own ones, and queries that make every score one value
    for factor in (40.0, -40.0, 0.0):
        c = case([3], [70], [90, 71, 70], 4, 2, 64, 16, "bf16")
        c["q"] = (c["q"].float() * factor).to(torch.bfloat16)
        check(c, "f32")
        check(c, "bf16")


def test_strided_queries_and_a_larger_workspace():
    c = case([3, 2], [70, 20], [90, 71, 70, 25, 200], 4, 2, 64, 16, "f16")
    R, Hq, D = c["q"].shape
    wide = torch.randn((R, Hq + 5, D), generator=torch.Generator().manual_seed(2)).half().cuda()
    wide[:, 2:2 + Hq] = c["q"].cuda()
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    ws = B.alloc_attn_shared_workspace(200, 40, Hq, kv, 9000, 500)
    a, la = run(c, "f16")
    b, lb = run(c, "f16", q=wide[:, 2:2 + Hq], ws=ws)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_equals_the_paged_attention():
    g = torch.Generator().manual_seed(6)
    kv_len = [2000 + int(torch.randint(0, 300, (1,), generator=g)) for _ in range(12)]
    c = case([12], [1984], kv_len, 8, 2, 128, 32, "bf16")
    o, lse = run(c, "f32")
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    p, pl = torch.empty_like(o), torch.empty_like(lse)
    most = c["table"].shape[1] * 32
    B.sq_attn_paged(c["q"].cuda(), kv, c["table"].cuda(), i32(kv_len), most, 0, c["scale"], p, B.SQ_OUT_F32, pl,
                    B.alloc_attn_workspace(12, 8, kv, most))
    _, _, bo, bl = reference(c, "f32")
    assert ((o - p).cpu().double().abs() <= 2 * bo + 2.0 ** -23 * p.cpu().double().abs()).all()
    assert ((lse - pl).cpu().double().abs() <= 2 * bl).all()


def test_no_requests():
    kv = B.KVCache(torch.zeros((2, 1, 8, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 1, 8, 64), dtype=torch.float16, device="cuda"))
    q = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    B.sq_attn_shared(q, kv, i32([[0]])[:0], i32([0])[:0], i32([0, 0]), i32([5]), 8, 8, 1.0, q.clone(), B.SQ_OUT_F16, None,
                     B.alloc_attn_shared_workspace(0, 1, 2, kv, 8, 8))


def test_graph_replays_with_other_lengths():
    c = case([4, 3], [300, 77], [400] * 4 + [150] * 3, 8, 2, 128, 16, "bf16")
    R, Hq, D = c["q"].shape
    kv = B.KVCache(c["k"].cuda(), c["v"].cuda())
    q, table, kv_len = c["q"].cuda(), c["table"].cuda(), i32(c["kv_len"])
    start, shared = i32(c["start"]), i32(c["shared"])
    o = torch.empty((R, Hq, D), device="cuda")
    ws = B.alloc_attn_shared_workspace(R, 2, Hq, kv, 300, 400)

    def call(out, w):
        B.sq_attn_shared(q, kv, table, kv_len, start, shared, 300, 400, c["scale"], out, B.SQ_OUT_F32, None, w)

    call(o, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, ws)
    eager, ws2 = torch.empty_like(o), torch.empty_like(ws)
    side = torch.cuda.Stream()
    for kv_now, shared_now in (([310, 300, 301, 400, 77, 78, 150], [300, 77]), ([5, 0, 390, 16, 90, 12, 150], [288, 64]), ([0] * 7, [300, 77])):
        kv_len.copy_(i32(kv_now))
        shared.copy_(i32(shared_now))
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):  # at the same time, on a workspace of its own
            call(eager, ws2)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(o, eager)


def test_cache_offsets_past_32_bits():
    # the pages of a small case at both ends of a cache whose byte and element offsets both pass 2^32
    c = case([5, 3], [700, 64], [720, 701, 900, 700, 640, 64, 65, 300], 4, 2, 128, 64, "bf16", seed=3)
    o, lse = run(c, "f32")
    n, many = c["k"].shape[0], 140000
    ids = torch.cat([torch.arange(n // 2), torch.arange(many - (n - n // 2), many)])
    big = {}
    for x in "kv":
        big[x] = torch.empty((many, *c[x].shape[1:]), dtype=torch.bfloat16, device="cuda")
        big[x][ids.cuda()] = c[x].cuda()
    assert big["k"].numel() > 1 << 31 and big["k"].nbytes > 1 << 32
    kv = B.KVCache(big["k"], big["v"])
    table = torch.where(c["table"] < 0, c["table"], ids.to(torch.int32)[c["table"].long().clamp(min=0)]).cuda()
    R, Hq, D = c["q"].shape
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    B.sq_attn_shared(c["q"].cuda(), kv, table, i32(c["kv_len"]), i32(c["start"]), i32(c["shared"]), 700, 900, c["scale"], o2,
                     B.SQ_OUT_F32, lse2, B.alloc_attn_shared_workspace(R, 2, Hq, kv, 700, 900))
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_two_graphs_share_a_workspace():
    cases = [case([4, 3], [300, 77], [400] * 4 + [150] * 3, 8, 2, 128, 16, "bf16", seed=1),
             case([40], [1500], [1500 + 7 * r for r in range(40)], 8, 2, 128, 64, "bf16", seed=2)]
    want = [run(c, "bf16")[0] for c in cases]
    kvs = [B.KVCache(c["k"].cuda(), c["v"].cuda()) for c in cases]
    ws = B.alloc_attn_shared_workspace(40, 2, 8, kvs[1], 1500, 2000)
    graphs, outs, keep = [], [], []
    for c, kv, w in zip(cases, kvs, want):
        o = torch.zeros_like(w)
        args = (c["q"].cuda(), kv, c["table"].cuda(), i32(c["kv_len"]), i32(c["start"]), i32(c["shared"]), max(c["shared"]),
                max(c["kv_len"]), c["scale"], o, B.SQ_OUT_BF16, None, ws)
        B.sq_attn_shared(*args)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.sq_attn_shared(*args)
        graphs.append(graph), outs.append(o), keep.append(args)
    for i in (0, 1, 0, 0, 1, 1, 0):
        outs[i].zero_()
        graphs[i].replay()
        assert torch.equal(outs[i], want[i])
