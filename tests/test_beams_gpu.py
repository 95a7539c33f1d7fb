"""The operators of beams on the GPU (choice of continuations, tables that follow
it, copies of pages) against plain forms, at the sizes and contents where they can
go wrong."""
import math

import numpy as np
import pytest
import torch

import beam_ref as R
from paper_2609_39056_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ choice
def select(logits, scores, done, end, beams, width):
    rows, V = logits.shape
    wide = torch.full((rows, -(-V // 8) * 8 + 8), INF, dtype=logits.dtype)  # what stands past the vocabulary is not read
    wide[:, :V] = logits
    G = rows // beams
    out = dict(parent=i32([[77] * width] * G), token=i32([[77] * width] * G), score=torch.full((G, width), 77.0, device="cuda"),
               done=i32([[77] * width] * G))
    ws = torch.full((B.sq_beam_workspace_bytes(rows, beams, V, width),), 0xA5, dtype=torch.uint8, device="cuda")
    B.sq_beam_select(wide.cuda()[:, :V], beams, scores.cuda(), None if done is None else done.cuda(), end, out["parent"],
                     out["token"], out["score"], out["done"], ws)
    return out


def check_select(logits, scores, done, end, beams, width):
    """The selected continuations are the best ones in exact order wherever their totals differ by more than
    fp32 exponentials allow: each is off by 2 units and its argument's rounding, |x - top| units; a thread adds 16
    of them, the rest is fp64.  The sum is off by what its terms are, largest for terms of e^-2 or so: 24 units."""
    out = {k: v.cpu() for k, v in select(logits, scores, done, end, beams, width).items()}
    total = R.beam_totals(logits, scores, done, end)
    want = R.beam_select(total, logits, done, beams, width)
    eps = 24 * R.U32
    for g, best in enumerate(want):
        got = list(zip(out["parent"][g].tolist(), out["token"][g].tolist()))
        assert got[len(best):] == [(-1, -1)] * (width - len(best))
        assert (out["score"][g, len(best):] == -INF).all() and (out["done"][g, len(best):] == 0).all()
        got = got[:len(best)]
        assert len(set(got)) == len(got)
        for i, ((r, t), (wr, wt, wv)) in enumerate(zip(got, best)):
            assert g * beams <= r < (g + 1) * beams and 0 <= t < logits.shape[1]
            v = total[r, t].item()
            assert (r, t) == (wr, wt) or (r != wr and abs(v - wv) <= 2 * eps), (g, i, (r, t), (wr, wt))
            assert abs(out["score"][g, i].item() - v) <= eps + R.U32 * abs(v)
            ended = (done is not None and done[r] != 0) or t == end
            assert out["done"][g, i].item() == int(ended)
        # within a row the order is that of its logits
        for r in {r for r, _ in got}:
            if done is None or done[r] == 0:
                mine = [t for q, t in got if q == r]
                order = torch.sort(logits[r].double(), descending=True, stable=True).indices[:width].tolist()
                assert mine == order[:len(mine)]


@pytest.mark.parametrize("groups,beams,V,width", [
    (1, 1, 1, 1), (2, 1, 5, 8), (1, 4, 8, 4), (3, 2, 100, 4), (2, 4, 511, 4), (2, 3, 4095, 6), (1, 4, 4096, 4), (2, 2, 4097, 2),
    (1, 4, 8192, 4), (5, 5, 12289, 5), (2, 8, 50257, 16), (1, 64, 700, 64), (2, 33, 70, 33), (1, 2, 131071, 64), (1, 1, 1 << 20, 3)])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
def test_select(groups, beams, V, width, dt):
    g = torch.Generator().manual_seed(groups + beams + V)
    rows = groups * beams
    logits = (torch.randn((rows, V), generator=g) * 2.5).to(DT[dt])
    scores = -torch.rand((rows,), generator=g) * 20
    check_select(logits, scores, None, 0, beams, width)
    done = (torch.rand((rows,), generator=g) < 0.4).to(torch.int32) * 5
    check_select(logits, scores, done, V // 2, beams, width)


def test_select_ties():
    # equal logits: the lowest tokens; equal rows and scores: the lowest rows first
    for V in (10, 4096, 10000):
        logits = torch.zeros((4, V))
        out = select(logits, torch.zeros(4), None, 0, 4, 6)
        assert out["parent"].tolist() == [[0] * 6] and out["token"].tolist() == [list(range(6))]
        logits[:, V - 1] = 1.0
        logits[:, 3] = 1.0
        out = select(logits, torch.zeros(4), None, 0, 2, 5)
        assert out["parent"].tolist() == [[0, 0, 1, 1, 0], [2, 2, 3, 3, 2]]
        assert out["token"].tolist() == [[3, V - 1, 3, V - 1, 0]] * 2
    # zeros of both signs are equal
    logits = torch.full((1, 300), -5.0)
    logits[0, 7], logits[0, 9], logits[0, 11] = -0.0, 0.0, -0.0
    assert select(logits, torch.zeros(1), None, 0, 1, 3)["token"].tolist() == [[7, 9, 11]]


@pytest.mark.parametrize("at", [0, 4000, 8100, 20000])
def test_select_neighbours(at):
    # the best tokens next to each other, rising, falling and equal
    V, n = 20200, 200
    base = torch.randn((3, V), generator=torch.Generator().manual_seed(at))
    base[0, at:at + n] = 20.0 + torch.arange(n) * 0.25
    base[1, at:at + n] = 20.0 - torch.arange(n) * 0.03125
    base[2, at:at + n] = 20.0
    for width in (1, 8, 33, 64):
        check_select(base, torch.tensor([0.0, -1.0, -2.0]), None, 3, 3, width)
        check_select(base.to(torch.bfloat16), torch.tensor([0.0, -40.0, -40.0]), None, 3, 1, width)


def test_select_values_that_are_never_taken():
    g = torch.Generator().manual_seed(8)
    logits = torch.randn((8, 5000), generator=g)
    logits[0, 17] = NAN
    logits[1, 4999] = INF
    logits[2] = -INF
    logits[3, 1:] = -INF
    logits[4, ::2] = -INF
    logits[6, :] = -INF
    logits[6, 4200] = NAN
    logits[7, :] = NAN
    scores = torch.zeros(8)
    check_select(logits, scores, None, 0, 8, 8)
    check_select(logits, scores, None, 0, 4, 4)  # one continuation in all of the first group
    check_select(logits, scores, None, 0, 1, 3)
    # rows without a finite score: as in a search's first step
    scores = torch.tensor([0.0, -INF, -INF, -INF, -INF, NAN, INF, -1.0])
    check_select(torch.randn((8, 600), generator=g), scores, None, 0, 4, 6)
    done = torch.tensor([1, 1, 0, 0, 1, 1, 1, 0], dtype=torch.int32)
    check_select(torch.randn((8, 600), generator=g), scores, done, 599, 4, 6)
    # a done row's logits do not count
    x = torch.randn((2, 600), generator=g)
    x[0] = NAN
    check_select(x, torch.tensor([-3.0, -1.0]), torch.tensor([1, 0], dtype=torch.int32), 5, 2, 4)


def test_select_large_logits_and_far_scores():
    g = torch.Generator().manual_seed(12)
    x = torch.randn((6, 9000), generator=g) * 300
    check_select(x, torch.tensor([0.0, -1e4, -1.0, -1e30, 5.0, 4.0]), None, 1, 3, 12)


def test_select_in_place_and_graph():
    g = torch.Generator().manual_seed(21)
    G, W, V = 3, 4, 9001
    logits = torch.randn((G * W, 9008), generator=g).cuda()
    scores, done = torch.zeros(G * W, device="cuda"), torch.zeros(G * W, dtype=torch.int32, device="cuda")
    ws = B.alloc_beam_workspace(G * W, W, V, W)
    parent, token = i32([[0] * W] * G), i32([[0] * W] * G)

    def call(s, d):
        B.sq_beam_select(logits[:, :V], W, scores, done, 9, parent, token, s, d, ws)

    apart = torch.empty((G, W), device="cuda"), i32([[0] * W] * G)
    call(*apart)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(scores.view(G, W), done.view(G, W))
    for _ in range(4):
        call(*apart)
        want = parent.clone(), token.clone(), apart[0].clone(), apart[1].clone()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, (parent, token, scores.view(G, W), done.view(G, W))))
        logits.copy_(torch.randn((G * W, 9008), generator=g))


# ------------------------------------------------------------------ tables
def run_reorder(parent, kv_len, page, num_pages, free, head, table, use_head=True, fill=-9):
    n, max_pages = len(parent), len(table[0])
    d = dict(table=torch.full((n, max_pages), fill, dtype=torch.int32, device="cuda"), free=i32(free) if free else i32([0])[:0])
    for k in ("kv_len", "src", "dst", "rows"):
        d[k] = i32([77] * n)
    d["head"] = i32([77])
    ws = torch.full((B.sq_kv_reorder_workspace_bytes(n, num_pages),), 0x5A, dtype=torch.uint8, device="cuda")
    B.sq_kv_reorder(i32(parent), i32(kv_len), page, num_pages, d["free"], i32([head]) if use_head else None, i32(table), d["table"],
                    d["kv_len"], d["src"], d["dst"], d["rows"], d["head"], ws)
    return d


def check_reorder(parent, kv_len, page, num_pages, free, head, table, use_head=True):
    d = run_reorder(parent, kv_len, page, num_pages, free, head, table, use_head)
    want = R.reorder(parent, kv_len, page, num_pages, free, head if use_head else 0, table, [[-9] * len(table[0])] * len(table))
    for name, w in zip(("table", "kv_len", "src", "dst", "rows", "free"), want):
        assert d[name].tolist() == w, name
    assert d["head"].item() == want[6]
    return want


def beams_state(rng, groups, beams, page, prompt, own, spare):
    """Tables of groups whose beams share the prompt's full pages, a free list whose first entries are taken."""
    ids = iter(rng.permutation(groups * (prompt // page + 1) + groups * beams * (own // page + 3) + spare).tolist())
    table, kv_len = [], []
    most = -(-(prompt + own) // page) + 1
    for _ in range(groups):
        n = int(rng.integers(0, prompt + 1))
        common = [next(ids) for _ in range(n // page)]
        more = int(rng.integers(0, own + 1))
        for _ in range(beams):
            length = len(common) * page + n % page + more
            row = common + [next(ids) for _ in range(-(-length // page) - len(common))]
            table.append(row + [-1] * (most - len(row)))
            kv_len.append(length)
    rest = list(ids)
    used = sorted({p for row in table for p in row if p >= 0})
    num_pages = max(used + rest, default=0) + 1
    return table, kv_len, used, rest, num_pages


@pytest.mark.parametrize("groups,beams,page,prompt,own,spare", [
    (1, 1, 8, 0, 0, 0), (1, 1, 16, 30, 5, 1), (1, 2, 8, 20, 3, 2), (4, 4, 16, 100, 40, 20), (16, 4, 16, 300, 60, 64), (3, 16, 64, 500, 200, 0),
    (60, 3, 8, 90, 30, 10), (200, 4, 32, 600, 70, 300), (7, 5, 1024, 3000, 900, 4)])
def test_reorder_after_a_choice(groups, beams, page, prompt, own, spare):
    rng = np.random.default_rng([groups, beams, page])
    for trial in range(3):
        table, kv_len, used, rest, num_pages = beams_state(rng, groups, beams, page, prompt, own, spare)
        parent = []
        for g in range(groups):
            parent += [int(g * beams + rng.integers(0, beams)) if rng.random() < 0.95 else -1 for _ in range(beams)]
        head = len(used)
        check_reorder(parent, kv_len, page, num_pages, used + rest, head, table)


def test_reorder_forks_frees_and_moves():
    rng = np.random.default_rng(3)
    table, kv_len, used, rest, num_pages = beams_state(rng, 12, 1, 16, 200, 20, 40)
    free, head = used + rest, len(used)
    n = len(table)
    # nothing changes; everything is freed; every row to one; rows move together; a prompt is forked into empty rows
    table_id = check_reorder(list(range(n)), kv_len, 16, num_pages, free, head, table)
    assert table_id[6] == head and table_id[1] == kv_len
    gone = check_reorder([-1] * n, kv_len, 16, num_pages, free, head, table)
    assert gone[6] == 0 and sorted(gone[5]) == sorted(free)
    check_reorder([4] * n, kv_len, 16, num_pages, free, head, table)
    check_reorder([r for r in range(n) if r % 3] + [-1] * 4, kv_len, 16, num_pages, free, head, table)
    kv_len[5:] = [0] * (n - 5)
    check_reorder([0, 1, 2, 3, 4, 2, 2, 2, 0, -7, 99, n], kv_len, 16, num_pages, free, head, table)


def test_reorder_without_room():
    # copies find freed pages first, then the list's, then none: those rows are empty, the others go on
    page = 8
    table = [[0, 1], [0, 2], [3, 4], [5, -1]]
    kv_len = [12, 13, 16, 3]
    for free, head in (([6, 7], 0), ([6, 7], 1), ([6, 7], 2), ([], 0), ([6, 7], 5), ([6, 7], -3)):
        check_reorder([0, 0, 0, 0], kv_len, page, 8, free, head, table)
        check_reorder([1, 1, 3, 3], kv_len, page, 8, free, head, table)
        check_reorder([2, 2, 2, 2], kv_len, page, 8, free, head, table)
        check_reorder([3, 3, 3, 3], kv_len, page, 8, free, head, table, use_head=False)
    # more pages come free than the list has room in front of its head for
    check_reorder([-1] * 4, kv_len, page, 8, [6, 7, 9, 9], 2, table)
    check_reorder([1, -1, -1, -1], kv_len, page, 8, [6, 7], 0, table)


def test_reorder_entries_that_are_no_pages():
    page = 8
    table = [[0, -1, 7], [100, 2, 2], [3, 99, -5], [2, 3, 0]]
    for parent in ([0, 0, 1, 1], [2, 2, 2, 2], [3, 2, 1, 0], [-1, -1, -1, -1], [0, 2, 2, 0], [1, 1, 1, -1]):
        for kv_len in ([17, 9, 10, 24], [16, 24, 20, 100], [-3, 2 ** 31 - 1, 0, 5], [11, 22, 23, 1]):
            check_reorder(parent, kv_len, page, 8, [4, 5, 6, 1, 1], 3, table)


def test_reorder_many_rows():
    rng = np.random.default_rng(11)
    n, page, most = 8192, 8, 3
    table = rng.integers(0, 30000, (n, most)).tolist()
    kv_len = rng.integers(0, page * most + 1, n).tolist()
    parent = rng.integers(-200, n, n).tolist()
    check_reorder(parent, kv_len, page, 30000, list(range(30000)), 15000, table)
    check_reorder([-1] * n, kv_len, page, 30000, list(range(30000)), 29000, table)
    check_reorder([8191] * n, kv_len, page, 30000, list(range(30000)), 29000, table)


def test_reorder_graph_and_stream():
    rng = np.random.default_rng(5)
    table, kv_len, used, rest, num_pages = beams_state(rng, 10, 4, 16, 200, 40, 40)
    n = len(table)
    t, length, head = i32(table), i32(kv_len), i32([len(used)])
    parent = i32([-1] * n)
    free0 = i32(used + rest)
    free = free0.clone()
    ws = B.alloc_reorder_workspace(n, num_pages)
    out = torch.full_like(t, -9)
    o = [i32([0] * n) for _ in range(4)] + [i32([0])]

    def call():
        B.sq_kv_reorder(parent, length, 16, num_pages, free, head, t, out, o[0], o[1], o[2], o[3], o[4], ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        p = [int(r // 4 * 4 + rng.integers(0, 4)) if rng.random() < 0.9 else -1 for r in range(n)]
        parent.copy_(i32(p))
        free.copy_(free0)
        out.fill_(-9)
        graph.replay()
        want = R.reorder(p, kv_len, 16, num_pages, used + rest, len(used), table, [[-9] * len(table[0])] * n)
        assert [out.tolist()] + [x.tolist() for x in o[:4]] + [free.tolist(), o[4].item()] == list(want)


# ------------------------------------------------------------------ copies
@pytest.mark.parametrize("layers,pages,heads,page,dim,dt", [(1, 9, 1, 8, 64, "bf16"), (3, 20, 2, 16, 96, "f16"), (2, 12, 5, 64, 128, "bf16"),
                                                           (66, 8, 1, 8, 64, "f16"), (1, 6, 3, 1024, 192, "bf16"), (2, 30, 40, 32, 256, "bf16")])
def test_copy_pages(layers, pages, heads, page, dim, dt):
    g = torch.Generator().manual_seed(pages + page)
    k = torch.randn((layers, pages, heads, page, dim), generator=g).to(DT[dt])
    v = torch.randn((layers, pages, heads, page, dim), generator=g).to(DT[dt])
    k[:, :, :, page // 2], v[:, 1] = NAN, INF  # bits are copied
    ids = torch.randperm(pages, generator=g).tolist()
    half = pages // 2
    src = ids[:half] + [-1, pages, ids[0], ids[0], 2 ** 31 - 1]
    dst = ids[half:2 * half] + [ids[0], ids[0], -1, ids[0], ids[0]]
    src[1] = src[0]  # a page may be copied to several
    rows = torch.randint(0, page + 1, (len(src),), generator=g).tolist()
    rows[0], rows[-1] = page + 7, 5
    rows[2 % half] = -2 if half > 2 else rows[2 % half]
    for use_rows in (True, False):
        wk, wv = k.clone(), v.clone()
        for a, b, n in zip(src, dst, rows):
            if 0 <= a < pages and 0 <= b < pages:
                n = min(max(n, 0), page) if use_rows else page
                wk[:, b, :, :n], wv[:, b, :, :n] = k[:, a, :, :n], v[:, a, :, :n]
        dk, dv = k.cuda(), v.cuda()
        caches = [B.KVCache(dk[i], dv[i]) for i in range(layers)]
        B.sq_kv_copy_pages(caches, i32(src), i32(dst), i32(rows) if use_rows else None)
        for got, want in ((dk, wk), (dv, wv)):
            assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))


def test_copy_nothing():
    k = torch.randn((4, 1, 8, 64)).to(torch.bfloat16).cuda()
    kv = B.KVCache(k, k.clone())
    was = k.clone()
    B.sq_kv_copy_pages([kv], i32([0])[:0], i32([0])[:0], None)
    B.sq_kv_copy_pages([], i32([0]), i32([1]), None)
    B.sq_kv_copy_pages([kv], i32([0, 1]), i32([2, 3]), i32([0, -1]))
    assert torch.equal(k, was)


def test_copy_past_32_bits():
    # element offsets beyond 2^31 and byte offsets beyond 2^32, both ways
    n, shape = 140000, (2, 64, 128)
    k, v = (torch.empty((n, *shape), dtype=torch.float16, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 31 and k.nbytes > 1 << 32
    g = torch.Generator().manual_seed(4)
    src, dst, rows = [n - 1, 3, n - 5], [2, n - 2, n - 9], [64, 17, 33]
    for t in (k, v):
        for p in src:
            t[p] = torch.randn(shape, generator=g).half().cuda()
        for p in dst:
            t[p] = 7.0
    want = [[torch.cat([t[s][:, :r], t[d][:, r:]], 1) for s, d, r in zip(src, dst, rows)] for t in (k, v)]
    B.sq_kv_copy_pages([B.KVCache(k, v)], i32(src), i32(dst), i32(rows))
    for t, w in zip((k, v), want):
        assert all(torch.equal(t[d], x) for d, x in zip(dst, w))


def test_reorder_two_graphs_share_a_workspace():
    # one of a small table (one launch), one of a large one (four)
    rng = np.random.default_rng(8)
    calls = []
    for n, most, num_pages in ((12, 5, 64), (1500, 40, 40000)):
        table = rng.integers(0, num_pages, (n, most)).tolist()
        kv_len, parent = rng.integers(0, most * 16 + 1, n).tolist(), rng.integers(0, n, n).tolist()
        calls.append(dict(parent=i32(parent), kv_len=i32(kv_len), table=i32(table), free0=i32(list(range(num_pages))), num=num_pages,
                          head=i32([num_pages // 2]), out=[torch.full((n, most), -9, dtype=torch.int32, device="cuda")] +
                          [i32([0] * n) for _ in range(4)] + [i32([0])]))
    shared = B.alloc_reorder_workspace(1500, 40000)

    def call(c, ws):
        o = c["out"]
        B.sq_kv_reorder(c["parent"], c["kv_len"], 16, c["num"], c["free"], c["head"], c["table"], o[0], o[1], o[2], o[3], o[4], o[5], ws)

    for c in calls:
        c["free"] = c["free0"].clone()
        call(c, torch.full_like(B.alloc_reorder_workspace(len(c["parent"]), c["num"]), 0x5A))
        c["want"] = [t.clone() for t in c["out"] + [c["free"]]]
        c["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(c["graph"]):
            call(c, shared)
    for i in (0, 1, 1, 0, 1, 0):
        c = calls[i]
        c["free"].copy_(c["free0"])
        c["graph"].replay()
        assert all(torch.equal(a, b) for a, b in zip(c["out"] + [c["free"]], c["want"]))
