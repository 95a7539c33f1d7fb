"""Performance cases of a decoder that follows several continuations of a prompt
at once: the choice of the best continuations of every group of beams, the page
tables that follow that choice with the pages it copies and frees, attention of
beams or requests over a prefix that they share, and the residual norm between
the layers' parts with 8-bit codes for the quantized linears.

kinds
  beam     sq_beam_select: `groups` of `beams` rows of logits over `vocab` tokens,
           the `width` best continuations of each group
  reorder  sq_kv_reorder: page tables of `groups` of `beams` after such a choice
  copy     sq_kv_copy_pages: the partly filled pages of `copies` forked beams in
           the caches of `layers` layers
  shared   sq_attn_shared: one query per request, `groups` of `beams` requests with
           up to `prefix` tokens in common and up to `length` of their own
  norm     sq_add_rmsnorm: `tokens` rows of `K` channels added to their residual
           and normed, to 16 bits or to 8-bit codes with a scale per row

`own` False computes the operators in elementary torch operations; True calls
the library.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
OUT = {"f32": 0, "bf16": 1, "f16": 2}  # the library's SQ_OUT_*
EPS = 1e-6
STREAMS, STEPS = 3, 10  # of the codes' gain tables


def listed():
    return [
        # one prompt's beams over a small vocabulary of action tokens: latency
        dict(name="beam_one", kind="beam", groups=1, beams=4, vocab=8192, width=4, dtype="f32", done=False),
        # a batch of prompts with many beams over a large vocabulary of an odd size, some beams finished
        dict(name="beam_batch", kind="beam", groups=16, beams=8, vocab=131071, width=8, dtype="bf16", done=True),
        # the tables of a decoding step of 16 prompts with 4 beams each
        dict(name="reorder_step", kind="reorder", groups=16, beams=4, prefix=2048, length=200, page=16),
        # a large batch with long prompts
        dict(name="reorder_many", kind="reorder", groups=256, beams=4, prefix=8192, length=1000, page=32),
        # the forked beams of a step, in one layer
        dict(name="copy_step", kind="copy", copies=48, layers=1, page=16, heads=8, dim=128, dtype="bf16"),
        # large pages, in every layer of a 28-layer decoder
        dict(name="copy_layers", kind="copy", copies=128, layers=28, page=64, heads=8, dim=128, dtype="bf16"),
        # four beams of one short prompt: latency
        dict(name="shared_beams", kind="shared", groups=1, beams=4, prefix=1024, length=60, heads=16, kv_heads=16,
             dim=128, page=16, dtype="bf16", out="bf16", lse=False),
        # a serving batch behind one long instruction, grouped heads
        dict(name="shared_batch", kind="shared", groups=1, beams=64, prefix=8192, length=500, heads=40, kv_heads=8,
             dim=128, page=64, dtype="bf16", out="bf16", lse=False),
        # many prompts of different lengths with beams each, small heads, f16
        dict(name="shared_groups", kind="shared", groups=24, beams=8, prefix=4001, length=150, heads=14, kv_heads=2,
             dim=64, page=16, dtype="f16", out="f32", lse=True),
        # one token of hidden 2048, to codes: latency
        dict(name="norm_one", kind="norm", tokens=1, K=2048, dtype="bf16", residual="bf16", to="codes", static=False),
        # the 4192 tokens of the 2B class into its quantized linears
        dict(name="norm_codes", kind="norm", tokens=4192, K=2048, dtype="bf16", residual="bf16", to="codes",
             static=False),
        # the 8384 tokens of the 14B class with an fp32 residual stream, to 16 bits
        dict(name="norm_sequence", kind="norm", tokens=8384, K=5120, dtype="bf16", residual="f32", to="bf16",
             static=False),
    ]


# (query heads, kv heads, head dim): one kv head per query head, groups, one kv head for all
HEADS = [(16, 16, 128), (40, 40, 128), (40, 8, 128), (32, 8, 128), (14, 2, 64), (25, 5, 64), (20, 20, 96),
         (8, 1, 256), (32, 1, 128), (12, 12, 192)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """A case of the same ranges: 1 to 256 groups of 1 to 32 beams, vocabularies
    of 100 to 131071 tokens, prefixes of 8 to 32768 tokens, 1 to 8384 rows of 128
    to 13824 channels."""
    kind = rng.choice(["beam", "reorder", "copy", "shared", "shared", "norm"])
    if kind == "beam":
        vocab, beams = _log_int(rng, 100, 131071), _log_int(rng, 1, 32)
        groups = _log_int(rng, 1, max(1, min(256, 128 * 131071 // (vocab * beams))))
        return dict(kind=kind, groups=groups, beams=beams, vocab=vocab, width=beams * rng.choice([1, 1, 2]),
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]) if groups * beams * vocab <= 64 * 131071 else "bf16",
                    done=rng.random() < 0.5)
    if kind == "reorder":
        groups, beams, page = _log_int(rng, 1, 256), _log_int(rng, 2, 16), rng.choice([8, 16, 32, 64, 128])
        most = 1024 * 9192 // 32 * page // (groups * beams)  # tokens of a request
        prefix = _log_int(rng, 8, min(32768, most - most // 8))
        return dict(kind=kind, groups=groups, beams=beams, prefix=prefix,
                    length=_log_int(rng, 1, max(1, min(4096, most // 8))), page=page)
    heads, kv_heads, dim = rng.choice(HEADS)
    page = rng.choice([8, 16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "copy":
        layers = rng.choice([1, 1, 28, _log_int(rng, 1, 40)])
        most = 28 * 128 * 64 * 8 * 128 // (layers * page * kv_heads * dim)
        return dict(kind=kind, copies=_log_int(rng, 1, max(1, min(1024, most))), layers=layers, page=page, heads=kv_heads,
                    dim=dim, dtype=dtype)
    if kind == "shared":
        most, most_kv = 64 * 8192 * 40 * 128, 1 << 26  # products and keys
        prefix = _log_int(rng, 8, min(32768, most_kv // (kv_heads * dim)))
        beams = _log_int(rng, 1, max(1, min(64, most // (prefix * heads * dim))))
        groups = _log_int(rng, 1, max(1, min(64, most // (prefix * heads * dim * beams),
                                             most_kv // (prefix * kv_heads * dim))))
        own_most = max(1, min(1000, prefix, most // (8 * groups * beams * kv_heads * dim)))
        return dict(kind=kind, groups=groups, beams=beams, prefix=prefix, length=_log_int(rng, 1, own_most), heads=heads,
                    kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, out=rng.choice([dtype, dtype, "f32"]),
                    lse=rng.random() < 0.5)
    K = 128 * _log_int(rng, 1, 108)
    tokens = _log_int(rng, 1, min(8384, 8384 * 5120 // K))
    return dict(kind=kind, tokens=tokens, K=K, dtype=dtype, residual=rng.choice(["none", dtype, dtype, "f32"]),
                to=rng.choice(["codes", "codes", dtype, "f32"]), static=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand_int(g, lo, hi, n):
    """n int32 values in [lo, hi]."""
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def _cdiv(a, b):
    return (a + b - 1) // b


def _normal(g, shape, dtype):
    """Standard normal values of the type, made in pieces of the first axis."""
    t = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, t[0].numel()))
    for i in range(0, shape[0], step):
        t[i:i + step] = torch.randn(t[i:i + step].shape, generator=g, device="cuda")
    return t


def _beam_inputs(case, seed):
    g, G, W, V = _gen(seed), case["groups"], case["beams"], case["vocab"]
    # rows as a linear of 64-channel multiples leaves them, the vocabulary in front
    wide = 64 * _cdiv(V, 64)
    logits = (torch.randn((G * W, wide), generator=g, device="cuda") * 2.5).to(DT[case["dtype"]])
    scores = -40.0 * torch.rand((G, W), generator=g, device="cuda")
    # beams of a prompt are near each other, in order
    scores = (scores[:, :1] - torch.rand((G, W), generator=g, device="cuda").cumsum(1)).view(-1).contiguous()
    done = (torch.rand((G * W,), generator=g, device="cuda") < 0.15).to(torch.int32) if case["done"] else None
    return dict(logits=logits[:, :V], scores=scores, done=done, end=V // 3)


def _tables(g, G, W, P, prefix, length, ragged_own):
    """Tables of G groups of W requests: the group's full pages of the prefix, then each request's own."""
    R = G * W
    frac = torch.exp2(-2.0 * torch.rand((G,), generator=g, device="cuda"))
    frac[0] = 1.0
    common = (frac * prefix).long().clamp_(min=1) // P  # full pages that are shared
    if ragged_own:
        more = torch.randint(1, length + 1, (R,), generator=g, device="cuda")
    else:  # the beams of a prompt have taken the same steps
        more = torch.randint(1, length + 1, (G,), generator=g, device="cuda").repeat_interleave(W)
    each = common.repeat_interleave(W)
    kv_len = each * P + more
    pages = _cdiv(kv_len, P)
    mine = pages - each
    first_common, first_mine = common.cumsum(0) - common, mine.cumsum(0) - mine
    used, shared = int(mine.sum()) + int(common.sum()), int(common.sum())
    # a pool as large as the longest prefixes and histories need, some pages more
    total = G * _cdiv(prefix, P) + R * (_cdiv(length, P) + 2)
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    j = torch.arange(_cdiv(prefix + length, P) + 1, device="cuda")
    at = torch.where(j < each[:, None], first_common.repeat_interleave(W)[:, None] + j,
                     shared + first_mine[:, None] + j - each[:, None])
    held = j < pages[:, None]
    table = torch.where(held, ids[torch.where(held, at, 0)], -1).contiguous()
    return dict(table=table, kv_len=kv_len.to(torch.int32), shared_len=(common * P).to(torch.int32), ids=ids, used=used,
                num_pages=total)


def _reorder_inputs(case, seed):
    g, G, W = _gen(seed), case["groups"], case["beams"]
    s = _tables(g, G, W, case["page"], case["prefix"], case["length"], False)
    # a beam mostly goes on from itself or from a better one; a few groups have ended
    pick = (torch.rand((G, W), generator=g, device="cuda") ** 2 * W).long().sort(1).values
    parent = pick + torch.arange(G, device="cuda")[:, None] * W
    ended = torch.rand((G, 1), generator=g, device="cuda") < 0.05
    parent = torch.where(ended, -1, parent).view(-1).to(torch.int32)
    return dict(s, parent=parent, free=s["ids"].clone(),
                head=torch.full((1,), s["used"], dtype=torch.int32, device="cuda"))


def _copy_inputs(case, seed):
    g, n, P = _gen(seed), case["copies"], case["page"]
    pages = 2 * n + 8
    ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    # entries without a copy stand between the others
    go = torch.rand((n,), generator=g, device="cuda") < 0.9
    shape = (case["layers"], pages, case["heads"], P, case["dim"])
    dt = DT[case["dtype"]]
    return dict(k=_normal(g, shape, dt), v=_normal(g, shape, dt), src=torch.where(go, ids[:n], -1),
                dst=torch.where(go, ids[n:2 * n], -1), rows=_rand_int(g, 1, P - 1, n))


def _shared_inputs(case, seed):
    g, G, W, P = _gen(seed), case["groups"], case["beams"], case["page"]
    s = _tables(g, G, W, P, case["prefix"], case["length"], True)
    dt = DT[case["dtype"]]
    shape = (s["num_pages"], case["kv_heads"], P, case["dim"])
    start = torch.arange(G + 1, dtype=torch.int32, device="cuda") * W
    return dict(s, q=_normal(g, (G * W, case["heads"], case["dim"]), dt), k=_normal(g, shape, dt), v=_normal(g, shape, dt),
                start=start, scale=1.0 / math.sqrt(case["dim"]))


def _norm_inputs(case, seed):
    g, M, K = _gen(seed), case["tokens"], case["K"]
    # a layer's output, and a residual stream with a few large channels
    x = torch.randn((M, K), generator=g, device="cuda").to(DT[case["dtype"]])
    chan = torch.where(torch.rand((K,), generator=g, device="cuda") < 0.02, 12.0, 1.0)
    res = None
    if case["residual"] != "none":
        res = (torch.randn((M, K), generator=g, device="cuda") * chan).to(DT[case["residual"]])
    s = dict(x=x, res=res, w=torch.randn((K,), generator=g, device="cuda") * 0.2 + 1.0)
    if case["to"] == "codes":
        s["dinv"] = (torch.rand((K,), generator=g, device="cuda") + 0.5) / chan
        s["gamma"] = torch.exp(torch.randn((STEPS, STREAMS), generator=g, device="cuda") * 0.3)
        s["clip"] = torch.rand((STEPS,), generator=g, device="cuda") + 3.0 if case["static"] else None
        s["stream"] = torch.arange(M, device="cuda", dtype=torch.int32) * STREAMS // M
        s["step"] = 4
    return s


_INPUTS = {"beam": _beam_inputs, "reorder": _reorder_inputs, "copy": _copy_inputs, "shared": _shared_inputs,
           "norm": _norm_inputs}


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    if case["kind"] == "reorder":  # entries past a row's pages are left as they are
        s["table_out"] = torch.full_like(s["table"], -1)
    if not own:
        return s
    from paper_2609_39056_amd import binding as B

    def i32(*shape):
        return torch.empty(shape, dtype=torch.int32, device="cuda")

    s["B"] = B
    if case["kind"] == "beam":
        G, n = case["groups"], case["width"]
        s["parent"], s["token"], s["score"] = i32(G, n), i32(G, n), torch.empty((G, n), device="cuda")
        s["done_out"] = i32(G, n) if case["done"] else None
        s["ws"] = B.alloc_beam_workspace(G * case["beams"], case["beams"], case["vocab"], n)
    elif case["kind"] == "reorder":
        R = case["groups"] * case["beams"]
        s["len_out"], s["src"], s["dst"], s["rows"], s["head_out"] = i32(R), i32(R), i32(R), i32(R), i32(1)
        s["ws"] = B.alloc_reorder_workspace(R, s["num_pages"])
    elif case["kind"] == "copy":
        s["caches"] = [B.KVCache(k=s["k"][i], v=s["v"][i]) for i in range(case["layers"])]
    elif case["kind"] == "shared":
        s["cache"] = B.KVCache(k=s["k"], v=s["v"])
        s["out"] = torch.empty(s["q"].shape, dtype=DT[case["out"]], device="cuda")
        s["lse"] = torch.empty(s["q"].shape[:2], device="cuda") if case["lse"] else None
        s["ws"] = B.alloc_attn_shared_workspace(case["groups"] * case["beams"], case["groups"], case["heads"], s["cache"],
                                                case["prefix"], case["length"])
    else:
        M, K = case["tokens"], case["K"]
        s["sum"] = None if s["res"] is None else torch.empty_like(s["res"])
        s["y"] = s["act"] = s["qx"] = s["r"] = None
        if case["to"] == "codes":
            s["act"] = B.ActParams(tok2stream=s["stream"], gamma=s["gamma"], step=s["step"], act_bits=8,
                                   range_mode=int(case["static"]), clip=s["clip"], dinv=s["dinv"])
            s["qx"], s["r"] = B.act_buffers(M, K, 8)
            s["values"] = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
        else:
            s["y"] = torch.empty((M, K), dtype=DT[case["to"]], device="cuda")
    return s


# ------------------------------------------------------------------ run: the plain forms
def _plain_beam(s):
    case = s["case"]
    G, W, V, n = case["groups"], case["beams"], case["vocab"], case["width"]
    x = s["logits"].float() + 0.0
    # 64-bit sums: the beams' scores are next to each other
    d = x.double()
    top = d.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(d - top).sum(1, keepdim=True))
    # a row's best by logit, ties to the lowest token: whole numbers in that order
    bits = x.view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) + (V - 1 - torch.arange(V, device="cuda"))
    k = min(n, V)
    token = torch.topk(order, k, dim=1).indices
    total = s["scores"].double()[:, None] + (d.gather(1, token) - lse)
    if s["done"] is not None:
        done = s["done"].bool()[:, None]
        only = (torch.arange(k, device="cuda") == 0)[None, :]
        total = torch.where(done, torch.where(only, s["scores"].double()[:, None], -math.inf), total)
        token = torch.where(done & only, s["end"], token)
    total, token = total.view(G, W * k), token.view(G, W * k)
    score, at = torch.sort(total, dim=1, descending=True, stable=True)
    score, at = score[:, :n], at[:, :n]
    parent = at // k + torch.arange(G, device="cuda")[:, None] * W
    token = token.gather(1, at)
    none = score == -math.inf
    i32 = torch.int32
    out = dict(parent=torch.where(none, -1, parent).to(i32), token=torch.where(none, -1, token).to(i32),
               score=score.float())
    if s["done"] is not None:
        ended = (s["done"][parent] != 0) | (token == s["end"])
        out["done"] = (ended & ~none).to(i32)
    if score.shape[1] < n:  # fewer continuations than asked for
        pad = n - score.shape[1]
        fill = dict(parent=-1, token=-1, score=-math.inf, done=0)
        out = {key: torch.nn.functional.pad(t, (0, pad), value=fill[key]) for key, t in out.items()}
    return out


def _plain_reorder(s):
    P, (R, max_pages) = s["case"]["page"], s["table"].shape
    pages_all, free, F = s["num_pages"], s["free"], s["free"].numel()
    n, parent, table = s["kv_len"].long(), s["parent"].long(), s["table"]
    r = torch.arange(R, device="cuda")
    j = torch.arange(max_pages, device="cuda")[None, :]
    ok = (parent >= 0) & (parent < R)
    par = parent.clamp(0, R - 1)
    first = torch.full((R + 1,), R, device="cuda").scatter_reduce(0, torch.where(ok, par, R), r, "amin")[:R]
    held = j < _cdiv(n, P)[:, None]
    # the pages of rows that nobody goes on from, unless another row holds them, in the order of the rows
    i = r[:, None] * max_pages + j
    page = torch.where(held & (table >= 0) & (table < pages_all), table, pages_all).long()
    keep = (first < R)[:, None]
    mark = torch.full((pages_all + 1,), R * max_pages, device="cuda").scatter_reduce(
        0, page.view(-1), torch.where(keep, -1, i).view(-1), "amin")
    freed = (~keep & (page < pages_all) & (mark[page] == i)).view(-1)
    rank = freed.cumsum(0) - 1
    m = freed.sum()
    # beams behind the first of a parent copy its last page where that is partly filled
    last = (n // P).clamp(max=max_pages - 1)
    last_page = table.gather(1, last[:, None])[:, 0].long()
    part = (n % P > 0) & (last_page >= 0) & (last_page < pages_all)
    copies = ok & (first[par] != r) & part[par]
    c = copies.cumsum(0) - copies.long()
    head = s["head"].long()
    fits = copies & (c < m + F - head)
    # copies take the freed pages first, then those of the free list
    by_rank = torch.full((R * max_pages + 1,), -1, dtype=torch.int32, device="cuda")
    by_rank = by_rank.scatter(0, torch.where(freed, rank, R * max_pages), page.view(-1).to(torch.int32))
    fresh = torch.where(c < m, by_rank[c], free[(head + c - m).clamp(0, F - 1)])
    rows = torch.where(held[par] & ok[:, None], table[par], s["table_out"])
    at_last = j == last[par][:, None]
    s["table_out"] = torch.where(at_last & fits[:, None], fresh[:, None],
                                 torch.where(at_last & (copies & ~fits)[:, None], -1, rows))
    taken = fits.sum()
    back = m - taken  # freed pages that go back to the list, in front of its head
    pos = torch.arange(F, device="cuda")
    new_head = (head + taken - m).clamp(min=0)
    returned = (pos >= new_head) & (pos < new_head + torch.minimum(back, head))
    free_out = torch.where(returned, by_rank[(taken + pos - new_head).clamp(0, R * max_pages)], free)
    i32 = torch.int32
    return dict(table=s["table_out"], kv_len=torch.where(ok & ~(copies & ~fits), n[par], 0).to(i32),
                src=torch.where(fits, last_page[par], -1).to(i32), dst=torch.where(fits, fresh, -1).to(i32),
                rows=torch.where(fits, n[par] % P, 0).to(i32), free=free_out, head=new_head.to(i32))


def _plain_copy(s):
    go = s["src"] >= 0
    src, dst, rows = s["src"][go].long(), s["dst"][go].long(), s["rows"][go]
    take = (torch.arange(s["case"]["page"], device="cuda") < rows[:, None])[None, :, None, :, None]
    s["k"][:, dst] = torch.where(take, s["k"][:, src], s["k"][:, dst])
    s["v"][:, dst] = torch.where(take, s["v"][:, src], s["v"][:, dst])
    return dict(k=s["k"], v=s["v"])


def _plain_shared(s):
    case = s["case"]
    G, W, P = case["groups"], case["beams"], case["page"]
    R, Hq, D = s["q"].shape
    Hk = s["k"].shape[1]
    h = Hq // Hk
    common, n = s["shared_len"].long(), s["kv_len"].long()

    def gathered(c, pages):
        B, m = pages.shape
        return c[pages.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, Hk, m * P, D).float()

    # the prefix, once for a group: [G, Hk, requests x heads, tokens]
    pages = s["table"][::W, :_cdiv(case["prefix"], P)]
    q = s["q"].float().view(G, W, Hk, h, D).transpose(1, 2).reshape(G, Hk, W * h, D) * s["scale"]
    j = torch.arange(pages.shape[1] * P, device="cuda")
    a = torch.matmul(q, gathered(s["k"], pages).transpose(2, 3))
    a = torch.where((j < common[:, None])[:, None, None], a, -math.inf)
    a = a.view(G, Hk, W, h, -1).transpose(1, 2).reshape(R, Hk, h, -1)
    # each request's own tokens
    each = common.repeat_interleave(W)
    at = (each // P)[:, None] + torch.arange(_cdiv(case["length"], P), device="cuda")[None, :]
    mine = s["table"].gather(1, at.clamp(max=s["table"].shape[1] - 1))
    t = each[:, None] + torch.arange(mine.shape[1] * P, device="cuda")[None, :]
    qr = s["q"].float().view(R, Hk, h, D) * s["scale"]
    b = torch.matmul(qr, gathered(s["k"], mine).transpose(2, 3))
    b = torch.where((t < n[:, None])[:, None, None], b, -math.inf)
    top = torch.maximum(a.amax(-1, keepdim=True), b.amax(-1, keepdim=True))
    ea, eb = torch.exp(a - top), torch.exp(b - top)
    total = ea.sum(-1, keepdim=True) + eb.sum(-1, keepdim=True)
    pa = ea.view(G, W, Hk, h, -1).transpose(1, 2).reshape(G, Hk, W * h, -1)
    va = torch.matmul(pa, gathered(s["v"], pages)).view(G, Hk, W, h, D).transpose(1, 2).reshape(R, Hk, h, D)
    out = ((va + torch.matmul(eb, gathered(s["v"], mine))) / total).reshape(R, Hq, D).to(DT[case["out"]])
    if not case["lse"]:
        return out
    return dict(out=out, lse=(top + torch.log(total)).view(R, Hq))


def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    out = {}
    if s["res"] is not None:
        h = h + s["res"].float()
        out["sum"] = h.to(s["res"].dtype)
    u = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["w"]
    if case["to"] != "codes":
        out["y"] = u.to(DT[case["to"]])
        return out
    u = u * s["dinv"]
    g = s["gamma"][s["step"]][s["stream"].long()][:, None]
    c = s["clip"][s["step"]] if case["static"] else u.abs().amax(-1, keepdim=True)
    delta = c / 127.0
    code = torch.round(torch.clamp((u * g) * (1.0 / delta), -127.0, 127.0))
    r = delta / g
    # the values that codes and row scales stand for
    out["values"], out["r"] = (code * r).to(torch.bfloat16), r.view(-1)
    return out


_PLAIN = {"beam": _plain_beam, "reorder": _plain_reorder, "copy": _plain_copy, "shared": _plain_shared, "norm": _plain_norm}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return _PLAIN[kind](s)
    B = s["B"]
    if kind == "beam":
        B.sq_beam_select(s["logits"], case["beams"], s["scores"], s["done"], s["end"], s["parent"], s["token"], s["score"],
                         s["done_out"], s["ws"])
        out = dict(parent=s["parent"], token=s["token"], score=s["score"])
        return out if s["done"] is None else dict(out, done=s["done_out"])
    if kind == "reorder":
        B.sq_kv_reorder(s["parent"], s["kv_len"], case["page"], s["num_pages"], s["free"], s["head"], s["table"],
                        s["table_out"], s["len_out"], s["src"], s["dst"], s["rows"], s["head_out"], s["ws"])
        return dict(table=s["table_out"], kv_len=s["len_out"], src=s["src"], dst=s["dst"], rows=s["rows"], free=s["free"],
                    head=s["head_out"])
    if kind == "copy":
        B.sq_kv_copy_pages(s["caches"], s["src"], s["dst"], s["rows"])
        return dict(k=s["k"], v=s["v"])
    if kind == "shared":
        B.sq_attn_shared(s["q"], s["cache"], s["table"], s["kv_len"], s["start"], s["shared_len"], case["prefix"],
                         case["length"], s["scale"], s["out"], OUT[case["out"]], s["lse"], s["ws"])
        return s["out"] if s["lse"] is None else dict(out=s["out"], lse=s["lse"])
    B.sq_add_rmsnorm(s["x"], s["res"], s["w"], EPS, s["sum"], s["y"], OUT.get(case["to"], 0), s["act"], s["qx"], s["r"])
    out = {} if s["res"] is None else dict(sum=s["sum"])
    if case["to"] != "codes":
        return dict(out, y=s["y"])
    torch.mul(s["qx"], s["r"][:, None], out=s["values"])
    return dict(out, values=s["values"], r=s["r"])


# ------------------------------------------------------------------ floors
_BYTES = {"bf16": 2, "f16": 2, "f32": 4, "none": 0}


def _mean_prefix(case):
    """Expected tokens of a prefix: log-uniform over a factor of four (the first is the longest)."""
    mean = case["prefix"] * 0.75 / math.log(4.0)
    return max(1.0, (case["prefix"] + (case["groups"] - 1) * mean) / case["groups"])


def work(case):
    kind = case["kind"]
    if kind == "beam":
        R, n = case["groups"] * case["beams"], case["groups"] * case["width"]
        return dict(bytes=R * case["vocab"] * _BYTES[case["dtype"]] + 8 * R + 16 * n, flops=4 * R * case["vocab"])
    if kind == "reorder":
        R = case["groups"] * case["beams"]
        entries = R * (_mean_prefix(case) + case["length"] / 2) / case["page"]
        # the old entries and the new ones; parents and lengths, the copies
        return dict(bytes=8 * entries + 8 * R + 16 * R, flops=4 * entries)
    if kind == "copy":
        return dict(bytes=0.9 * case["copies"] * case["layers"] * case["page"] / 2 * case["heads"] * case["dim"] * 8,
                    flops=1)
    if kind == "shared":
        R, D, Hk = case["groups"] * case["beams"], case["dim"], case["kv_heads"]
        prefix, mine = _mean_prefix(case), case["length"] / 2
        q = R * case["heads"] * D
        return dict(bytes=4 * D * Hk * (case["groups"] * prefix + R * mine) + q * (2 + _BYTES[case["out"]])
                    + 4 * R * (prefix + mine) / case["page"], flops=4 * q * (prefix + mine))
    M, K = case["tokens"], case["K"]
    each = _BYTES[case["dtype"]] + 2 * _BYTES[case["residual"]]
    if case["to"] == "codes":
        return dict(bytes=M * K * (each + 1) + 8 * K + 8 * M, flops=12 * M * K)
    return dict(bytes=M * K * (each + _BYTES[case["to"]]) + 4 * K, flops=6 * M * K)


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_beam(case, s):
    """Group after group; every continuation of a row that can be among the best is looked at."""
    G, W, V, n = case["groups"], case["beams"], case["vocab"], case["width"]
    parent, token, score, done = [], [], [], []
    ends = [0] * (G * W) if s["done"] is None else s["done"].tolist()
    base = s["scores"].tolist()
    x = s["logits"].double()
    lse = torch.logsumexp(x, 1)
    floor = x.topk(min(n, V), dim=1).values[:, -1:]
    row, col = (x >= floor).nonzero(as_tuple=True)  # row by row, tokens in order
    value = (x[row, col] - lse[row]).tolist()
    found = [[] for _ in range(G)]
    for r, t, v in zip(row.tolist(), col.tolist(), value):
        if not ends[r]:
            found[r // W].append((-(base[r] + v), r, t))
    for r in range(G * W):
        if ends[r]:
            found[r // W].append((-base[r], r, s["end"]))
    for g in range(G):
        best = sorted(found[g])[:n]
        parent.append([b[1] for b in best] + [-1] * (n - len(best)))
        token.append([b[2] for b in best] + [-1] * (n - len(best)))
        score.append([-b[0] for b in best] + [-math.inf] * (n - len(best)))
        done.append([int(bool(ends[b[1]]) or b[2] == s["end"]) for b in best] + [0] * (n - len(best)))

    def i32(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    out = dict(parent=i32(parent), token=i32(token), score=torch.tensor(score, dtype=torch.float64, device="cuda"))
    return out if s["done"] is None else dict(out, done=i32(done))


def _exact_reorder(case, s):
    """One row after another, as the definition reads."""
    P, F, total = case["page"], s["free"].numel(), s["num_pages"]
    table, n, parent, free = (s[k].tolist() for k in ("table", "kv_len", "parent", "free"))
    head, R, max_pages = int(s["head"]), len(table), len(table[0])
    rows = [row[:-(-length // P)] for row, length in zip(table, n)]
    alive = {p for p in parent if 0 <= p < R}
    kept = {page for p in alive for page in rows[p]}
    freed = []
    for r in range(R):
        if r not in alive:
            for page in rows[r]:
                if 0 <= page < total and page not in kept:
                    kept.add(page)
                    freed.append(page)
    pool = freed + free[head:]
    out, length, src, dst, copied, seen, asked = [], [], [], [], [], set(), 0
    for p in parent:
        row, take, frm, to = [], 0, -1, -1
        if 0 <= p < R:
            row, take = list(rows[p]), n[p]
            if p in seen and n[p] % P:
                if asked < len(pool):
                    frm, to = row[-1], pool[asked]
                    row[-1] = to
                else:
                    row[-1], take = -1, 0
                asked += 1
            seen.add(p)
        out.append(row + [-1] * (max_pages - len(row)))
        length.append(take)
        src.append(frm)
        dst.append(to)
        copied.append(n[p] % P if to >= 0 else 0)
    taken = min(asked, len(pool))
    back = freed[taken:]
    new_head = max(0, head + taken - len(freed))
    back = back[:head]
    free[new_head:new_head + len(back)] = back

    def i32(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    return dict(table=i32(out), kv_len=i32(length), src=i32(src), dst=i32(dst), rows=i32(copied), free=i32(free),
                head=i32([new_head]))


def _exact_copy(case, s):
    k, v = s["k"].double(), s["v"].double()
    for a, b, n in zip(s["src"].tolist(), s["dst"].tolist(), s["rows"].tolist()):
        if a >= 0:
            k[:, b, :, :n] = k[:, a, :, :n]
            v[:, b, :, :n] = v[:, a, :, :n]
    return dict(k=k, v=v)


def _exact_shared(case, s):
    R, Hq, D = s["q"].shape
    Hk, P = s["k"].shape[1:3]
    group = Hq // Hk
    out = torch.zeros((R, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((R, Hq), dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["kv_len"].tolist()):
        j = torch.arange(n, device="cuda")
        page, at = s["table"][r].long()[j // P], j % P
        k = s["k"][page, :, at].double().permute(1, 2, 0).contiguous()  # [Hk, D, n]
        v = s["v"][page, :, at].double().transpose(0, 1).contiguous()
        sc = torch.matmul(s["q"][r].double().view(Hk, group, D), k) * s["scale"]
        lse[r] = torch.logsumexp(sc, 2).view(Hq)
        out[r] = torch.matmul(torch.softmax(sc, 2), v).view(Hq, D)
    return dict(out=out, lse=lse) if case["lse"] else out


def _exact_norm(case, s):
    out = {}
    h = s["x"].double()
    if s["res"] is not None:
        h = h + s["res"].double()
        out["sum"] = h
    u = h / (h.square().sum(1, keepdim=True) / case["K"] + EPS).sqrt() * s["w"].double()
    if case["to"] != "codes":
        out["y"] = u
        return out
    u = u * s["dinv"].double()
    gain = s["gamma"].double()[s["step"], s["stream"].long()].unsqueeze(1)
    top = s["clip"].double()[s["step"]].expand(case["tokens"], 1) if case["static"] else u.abs().max(1, keepdim=True).values
    step = top / 127
    out["r"] = (step / gain).squeeze(1)
    out["values"] = (u * gain / step).clamp(-127, 127).round() * step / gain
    return out


_EXACT = {"beam": _exact_beam, "reorder": _exact_reorder, "copy": _exact_copy, "shared": _exact_shared, "norm": _exact_norm}


def exact(case, seed):
    return _EXACT[case["kind"]](case, _INPUTS[case["kind"]](case, seed))
