"""Performance cases of a decoder's token step on int4 weights: block tables and
slot maps from request lengths, the per-head norm of queries and keys with the
position rotation and the cache write, attention of one new token over a paged
key-value cache, and the few-token linear on packed int4 weights whose
activations stay in bf16.

kinds
  plan    sq_kv_plan: `requests` requests with cached tokens get `new` tokens
          each (0: none or one, a decoding step with idle requests)
  rope    sq_qk_norm_rope: `tokens` rows of a fused qkv linear's output, keys
          and values written to their slots of the cache
  attn    sq_attn_paged: one query per request over up to `length` cached tokens
  linear  sq_linear_w4a16: `tokens` rows against a packed weight [N][K/2]

`own` False computes the operators in elementary torch operations in fp32;
True calls the library.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
OUT = {"f32": 0, "bf16": 1, "f16": 2}  # the library's SQ_OUT_*
EPS = 1e-6


def listed():
    return [
        # one decoding step of a batch of requests, most of them with one new token
        dict(name="plan_step", kind="plan", requests=64, new=0, page=16, length=4096),
        # admission of a large batch of prompts in one call
        dict(name="plan_prompts", kind="plan", requests=512, new=1024, page=64, length=1024),
        # one new token of one request, 16 heads of 128 (hidden 2048): latency
        dict(name="rope_one", kind="rope", tokens=1, requests=1, heads=16, kv_heads=16, dim=128, rot=128, inter=False,
             norm=True, page=16, dtype="bf16"),
        # a decoding step of 64 requests, grouped heads, half of each head rotated in adjacent pairs
        dict(name="rope_step", kind="rope", tokens=64, requests=64, heads=40, kv_heads=8, dim=128, rot=64, inter=True,
             norm=True, page=64, dtype="f16"),
        # the benchmark's 8384 tokens at hidden 5120 as one long sequence
        dict(name="rope_sequence", kind="rope", tokens=8384, requests=1, heads=40, kv_heads=40, dim=128, rot=128,
             inter=False, norm=True, page=64, dtype="bf16"),
        # one request with a short history: latency
        dict(name="attn_one", kind="attn", requests=1, length=211, heads=16, kv_heads=16, dim=128, page=16, window=0,
             dtype="bf16", out="bf16", lse=False),
        # a serving batch with ragged histories and grouped heads
        dict(name="attn_batch", kind="attn", requests=64, length=8192, heads=40, kv_heads=8, dim=128, page=64,
             window=0, dtype="bf16", out="bf16", lse=False),
        # every query head with its own keys and values, small heads, f16, a sliding window
        dict(name="attn_window", kind="attn", requests=48, length=4001, heads=16, kv_heads=16, dim=64, page=16,
             window=1024, dtype="f16", out="f32", lse=True),
        # few requests with long histories: the split over the cache's length
        dict(name="attn_long", kind="attn", requests=2, length=131072, heads=32, kv_heads=8, dim=128, page=32,
             window=0, dtype="bf16", out="bf16", lse=True),
        # one token through the output projection of the 2B class
        dict(name="linear_one", kind="linear", tokens=1, K=2048, N=2048, group=128, dinv=True, bias=True, out="bf16"),
        # one token through the up projection of the 14B class, one step per output channel
        dict(name="linear_up", kind="linear", tokens=1, K=5120, N=13824, group=0, dinv=False, bias=True, out="bf16"),
        # a batch of 16 requests through its down projection, fp32 out
        dict(name="linear_batch", kind="linear", tokens=16, K=13824, N=5120, group=128, dinv=True, bias=False,
             out="f32"),
    ]


# (query heads, kv heads, head dim): one kv head per query head, groups, one kv head for all
HEADS = [(16, 16, 128), (40, 40, 128), (40, 8, 128), (32, 8, 128), (14, 2, 64), (25, 5, 64), (20, 20, 96),
         (8, 1, 256), (32, 1, 128), (12, 12, 192)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: 1 to 4096 requests planned, 1 to 8384 tokens
    rotated, histories of 1 to 131072 tokens, 1 to 64 rows against weights of
    256 to 13824 channels."""
    kind = rng.choice(["plan", "rope", "attn", "attn", "linear", "linear"])
    if kind == "plan":
        requests = _log_int(rng, 1, 4096)
        new = 0 if rng.random() < 0.5 else _log_int(rng, 1, max(1, min(8192, (512 << 10) // requests)))
        return dict(kind=kind, requests=requests, new=new, page=rng.choice([8, 16, 32, 64, 128]),
                    length=_log_int(rng, 1, 8192))
    heads, kv_heads, dim = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    page = rng.choice([8, 16, 32, 64, 128])
    if kind == "rope":
        tokens = _log_int(rng, 1, 8384)
        return dict(kind=kind, tokens=tokens, requests=rng.choice([1, tokens, max(1, tokens // 37)]), heads=heads,
                    kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim, dim // 2, 0]), inter=rng.random() < 0.4,
                    norm=rng.random() < 0.8, page=page, dtype=dtype)
    if kind == "attn":
        most = 2 * 131072 * 8 * 128  # the longest listed case's keys
        length = _log_int(rng, 1, 131072)
        requests = _log_int(rng, 1, max(1, min(256, most // (length * kv_heads * dim))))
        if requests * length * kv_heads * dim > most:
            length = most // (requests * kv_heads * dim)
        return dict(kind=kind, requests=requests, length=length, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                    window=rng.choice([0, 0, _log_int(rng, 1, length)]), dtype=dtype,
                    out=rng.choice([dtype, dtype, "f32"]), lse=rng.random() < 0.5)
    K, N = 128 * _log_int(rng, 2, 108), 64 * _log_int(rng, 4, 216)
    return dict(kind=kind, tokens=_log_int(rng, 1, 64), K=K + 128 * (K == 24 * 128), N=N + 64 * (N == 24 * 128),
                group=rng.choice([128, 128, 0]), dinv=rng.random() < 0.5, bias=rng.random() < 0.5,
                out=rng.choice(["bf16", "bf16", "f32", "f16"]))


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


def _plan_inputs(case, seed):
    g, R, P = _gen(seed), case["requests"], case["page"]
    if case["new"] == 0:
        cached = _rand_int(g, 1, case["length"], R)
        new = (torch.rand((R,), generator=g, device="cuda") < 0.9).to(torch.int32)
        most_new = 1
    else:
        cached = torch.where(torch.rand((R,), generator=g, device="cuda") < 0.5, 0, _rand_int(g, 0, case["length"], R))
        cached = cached.to(torch.int32)
        new = _rand_int(g, _cdiv(case["new"], 4), case["new"], R)
        most_new = case["new"]
    max_pages = _cdiv(case["length"] + most_new, P)
    pool = torch.randperm(R * max_pages, generator=g, device="cuda").to(torch.int32)
    table = pool[:R * max_pages].view(R, max_pages)
    have = _cdiv(cached, P)
    j = torch.arange(max_pages, device="cuda", dtype=torch.int32)
    held = j[None, :] < have[:, None]
    free = table[~held].contiguous()
    head = torch.full((1,), min(3, free.numel()), dtype=torch.int32, device="cuda")
    return dict(cached=cached, new=new, table=torch.where(held, table, -1).contiguous(), free=free, head=head,
                max_tokens=R * most_new)


def _rope_inputs(case, seed):
    g, T, R, P = _gen(seed), case["tokens"], case["requests"], case["page"]
    Hq, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    dt = DT[case["dtype"]]
    # R runs of consecutive tokens, each at its place in its own pages
    per = _cdiv(T, R)
    pages_each = _cdiv(per, P) + 1
    pages = torch.randperm(R * pages_each, generator=g, device="cuda").to(torch.int32).view(R, pages_each)
    start = _rand_int(g, 0, P - 1, R)
    t = torch.arange(T, device="cuda")
    at = start[t // per].long() + t % per
    slot = (pages[t // per, at // P] * P + (at % P).to(torch.int32)).to(torch.int32)
    num_pos = T + 4096
    base = _rand_int(g, 0, num_pos - per, R)
    pos = (base[t // per] + (t % per).to(torch.int32)).to(torch.int32)
    rot = case["rot"]
    if rot:
        inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
        ang = torch.arange(num_pos, dtype=torch.float64, device="cuda")[:, None] * inv[None, :]
        cos, sin = ang.cos().float().contiguous(), ang.sin().float().contiguous()
    else:
        cos = sin = None
    qw = kw = None
    if case["norm"]:
        qw = torch.randn((D,), generator=g, device="cuda") * 0.2 + 1.0
        kw = torch.randn((D,), generator=g, device="cuda") * 0.2 + 1.0
    qkv = (torch.randn((T, (Hq + 2 * Hk) * D), generator=g, device="cuda") * 1.5).to(dt)
    shape = (R * pages_each, Hk, P, D)
    return dict(qkv=qkv, qw=qw, kw=kw, cos=cos, sin=sin, pos=pos, slot=slot,
                k=torch.zeros(shape, dtype=dt, device="cuda"), v=torch.zeros(shape, dtype=dt, device="cuda"))


def _split_qkv(case, qkv):
    Hq, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D], dim=1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hk, D)), v.unflatten(1, (Hk, D))


def _attn_inputs(case, seed):
    g, R, P = _gen(seed), case["requests"], case["page"]
    Hq, Hk, D, L = case["heads"], case["kv_heads"], case["dim"], case["length"]
    dt = DT[case["dtype"]]
    # ragged histories: from an eighth of the longest to the longest
    frac = torch.exp2(-3.0 * torch.rand((R,), generator=g, device="cuda"))
    frac[0] = 1.0
    kv_len = (frac * L).to(torch.int32).clamp_(1, L)
    need = _cdiv(kv_len, P)
    max_pages = _cdiv(L, P)
    total = int(need.sum())
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    j = torch.arange(max_pages, device="cuda", dtype=torch.int32)
    held = j[None, :] < need[:, None]
    table = torch.full((R, max_pages), -1, dtype=torch.int32, device="cuda")
    table[held] = ids
    # keys and queries as a per-head norm leaves them, scores of a spread of about one
    return dict(q=_normal(g, (R, Hq, D), dt), k=_normal(g, (total, Hk, P, D), dt), v=_normal(g, (total, Hk, P, D), dt),
                table=table, kv_len=kv_len, scale=1.0 / math.sqrt(D))


def _linear_inputs(case, seed):
    g, M, K, N = _gen(seed), case["tokens"], case["K"], case["N"]
    G = case["group"] or K
    codes = (torch.randn((N, K), generator=g, device="cuda") * 2.5).round_().clamp_(-7, 7).to(torch.int32)
    c = (codes & 15).view(N, K // 8, 2, 4)
    qw = (c[:, :, 0] | (c[:, :, 1] << 4)).to(torch.uint8).reshape(N, K // 2).contiguous()
    step = torch.exp2(torch.randn((K // G, N), generator=g, device="cuda") * 0.4) / (2.5 * math.sqrt(K))
    # activations with outlier channels that the channel scaling evens out
    chan = torch.where(torch.rand((K,), generator=g, device="cuda") < 0.02, 12.0, 1.0)
    x = (torch.randn((M, K), generator=g, device="cuda") * chan).to(torch.bfloat16)
    dinv = (torch.rand((K,), generator=g, device="cuda") + 0.5) / chan if case["dinv"] else None
    bias = torch.randn((N,), generator=g, device="cuda").to(torch.bfloat16) if case["bias"] else None
    return dict(x=x, qw=qw, step=step.half().contiguous(), G=G, dinv=dinv, bias=bias)


_INPUTS = {"plan": _plan_inputs, "rope": _rope_inputs, "attn": _attn_inputs, "linear": _linear_inputs}


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_2609_39056_amd import binding as B

    i32 = dict(dtype=torch.int32, device="cuda")
    s["B"] = B
    if case["kind"] == "plan":
        R = case["requests"]
        s["slot"], s["pos"] = torch.empty((s["max_tokens"],), **i32), torch.empty((s["max_tokens"],), **i32)
        s["token_start"], s["kv_len"] = torch.empty((R + 1,), **i32), torch.empty((R,), **i32)
        s["head_out"] = torch.empty((1,), **i32)
    elif case["kind"] == "rope":
        s["cache"] = B.KVCache(k=s["k"], v=s["v"])
        s["rope"] = B.RopeParams(q_weight=s["qw"], k_weight=s["kw"], eps=EPS, cos=s["cos"], sin=s["sin"],
                                 interleaved=case["inter"])
        s["q_out"] = torch.empty((case["tokens"], case["heads"], case["dim"]), dtype=DT[case["dtype"]], device="cuda")
    elif case["kind"] == "attn":
        s["cache"] = B.KVCache(k=s["k"], v=s["v"])
        s["out"] = torch.empty(s["q"].shape, dtype=DT[case["out"]], device="cuda")
        s["lse"] = torch.empty(s["q"].shape[:2], device="cuda") if case["lse"] else None
        s["ws"] = B.alloc_attn_workspace(case["requests"], case["heads"], s["cache"], case["length"])
    else:
        s["w"] = B.Weight(qw=s["qw"], w_scale=s["step"], w_group=s["G"], bias=s["bias"])
        s["y"] = torch.empty((case["tokens"], case["N"]), dtype=DT[case["out"]], device="cuda")
    return s


# ------------------------------------------------------------------ run: the plain forms
def _plain_plan(s):
    P, (R, max_pages), T = s["case"]["page"], s["table"].shape, s["max_tokens"]
    cached, new = s["cached"].long(), s["new"].long()
    have, need = _cdiv(cached, P), _cdiv(cached + new, P)
    take = torch.where(need > max_pages, 0, need - have)
    first = take.cumsum(0) - take
    end = new.cumsum(0)
    start = end - new
    head = s["head"].long()
    fits = (need <= max_pages) & ((take == 0) | (head + first + take <= s["free"].numel())) & (end <= T)
    j = torch.arange(max_pages, device="cuda")[None, :]
    fresh = fits[:, None] & (j >= have[:, None]) & (j < (have + take)[:, None])
    at = (head + first[:, None] + j - have[:, None]).clamp(0, s["free"].numel() - 1)
    table = torch.where(fresh, s["free"][at], s["table"])
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(end, t, right=True).clamp(max=R - 1)
    ok = (t < end[-1]) & fits[r]
    pos = torch.where(ok, cached[r] + t - start[r], 0)
    slot = torch.where(ok, table[r, pos // P].long() * P + pos % P, -1)
    pos = torch.where(ok, pos, -1)
    used = torch.where(fits & (take > 0), first + take, 0).max()
    i32 = torch.int32
    return dict(table=table, slot=slot.to(i32), pos=pos.to(i32), token_start=torch.cat([start, end[-1:]]).to(i32),
                kv_len=torch.where(fits, cached + new, cached).to(i32), head=(head + used).to(i32))


def _plain_norm_rotate(x, w, s):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    rot = s["case"]["rot"]
    if rot == 0:
        return x
    pos = s["pos"].long()
    c, n = s["cos"][pos][:, None, :], s["sin"][pos][:, None, :]
    y = x.clone()
    if s["case"]["inter"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * n, b * c + a * n
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * n, b * c + a * n
    return y


def _plain_rope(s):
    q, k, v = _split_qkv(s["case"], s["qkv"])
    slot, P = s["slot"].long(), s["case"]["page"]
    s["k"][slot // P, :, slot % P] = _plain_norm_rotate(k, s["kw"], s).to(s["k"].dtype)
    s["v"][slot // P, :, slot % P] = v
    return dict(q=_plain_norm_rotate(q, s["qw"], s).to(q.dtype), k=s["k"], v=s["v"])


def _plain_attn(s):
    case = s["case"]
    R, Hq, D = s["q"].shape
    Hk, P = s["k"].shape[1:3]
    pages = s["table"].clamp(min=0).long()
    L = pages.shape[1] * P

    def gathered(c):
        return c[pages].permute(0, 2, 1, 3, 4).reshape(R, Hk, L, D).float()

    q = s["q"].float().view(R, Hk, Hq // Hk, D)
    score = torch.matmul(q, gathered(s["k"]).transpose(2, 3)) * s["scale"]
    j, n = torch.arange(L, device="cuda")[None, :], s["kv_len"].long()[:, None]
    live = j < n
    if case["window"]:
        live &= j >= n - case["window"]
    score = torch.where(live[:, None, None, :], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - top)
    total = e.sum(-1, keepdim=True)
    out = (torch.matmul(e, gathered(s["v"])) / total).view(R, Hq, D).to(DT[case["out"]])
    if not case["lse"]:
        return out
    return dict(out=out, lse=(top + torch.log(total)).view(R, Hq))


def _plain_linear(s):
    N, K = s["qw"].shape[0], s["qw"].shape[1] * 2
    b = s["qw"].view(N, K // 8, 1, 4)
    nib = torch.cat([b & 15, b >> 4], dim=2).view(N, K).to(torch.int8)
    code = torch.where(nib > 7, nib - 16, nib).float()
    w = (code.view(N, K // s["G"], s["G"]) * s["step"].float().t()[:, :, None]).view(N, K)
    x = s["x"].float()
    if s["dinv"] is not None:
        x = x * s["dinv"]
    y = torch.matmul(x, w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(DT[s["case"]["out"]])


_PLAIN = {"plan": _plain_plan, "rope": _plain_rope, "attn": _plain_attn, "linear": _plain_linear}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return _PLAIN[kind](s)
    B = s["B"]
    if kind == "plan":
        B.sq_kv_plan(s["cached"], s["new"], case["page"], s["free"], s["head"], s["table"], s["slot"], s["pos"],
                     s["token_start"], s["kv_len"], s["head_out"])
        return dict(table=s["table"], slot=s["slot"], pos=s["pos"], token_start=s["token_start"], kv_len=s["kv_len"],
                    head=s["head_out"])
    if kind == "rope":
        q, k, v = _split_qkv(case, s["qkv"])
        B.sq_qk_norm_rope(q, k, v, s["rope"], s["pos"], s["slot"], s["q_out"], None, s["cache"])
        return dict(q=s["q_out"], k=s["k"], v=s["v"])
    if kind == "attn":
        B.sq_attn_paged(s["q"], s["cache"], s["table"], s["kv_len"], case["length"], case["window"], s["scale"],
                        s["out"], OUT[case["out"]], s["lse"], s["ws"])
        return s["out"] if s["lse"] is None else dict(out=s["out"], lse=s["lse"])
    B.sq_linear_w4a16(s["x"], s["dinv"], s["w"], s["y"], OUT[case["out"]])
    return s["y"]


# ------------------------------------------------------------------ floors
def _mean_live(case):
    """Expected attended tokens of a request: lengths are log-uniform over a
    factor of eight (the first is the longest)."""
    n = 24
    lens = [case["length"] * 2.0 ** (-3.0 * (i + 0.5) / n) for i in range(n)]
    w = case["window"] or case["length"]
    mean = sum(min(v, w) for v in lens) / n
    first = min(case["length"], w)
    return max(1.0, (first + (case["requests"] - 1) * mean) / case["requests"])


def work(case):
    kind = case["kind"]
    if kind == "plan":
        R, P = case["requests"], case["page"]
        slots = R * max(1, case["new"])
        tokens = 0.9 * R if case["new"] == 0 else R * case["new"] * 0.625
        pages = tokens / P
        # lengths, pages taken, the entries of the pages that are continued; slots and positions, new entries, the rest
        return dict(bytes=8 * R + 4 * pages + 4 * R + 8 * slots + 4 * pages + 8 * R + 12, flops=4 * slots)
    if kind == "rope":
        T, D = case["tokens"], case["dim"]
        n = (case["heads"] + 2 * case["kv_heads"]) * D
        rotated = (case["heads"] + case["kv_heads"]) * D
        return dict(bytes=4 * T * n + 8 * T + 4 * T * case["rot"] + (8 * D if case["norm"] else 0),
                    flops=8 * T * rotated)
    if kind == "attn":
        R, live = case["requests"], _mean_live(case)
        q = R * case["heads"] * case["dim"]
        return dict(bytes=4 * R * live * case["kv_heads"] * case["dim"] + 2 * q + q * (4 if case["out"] == "f32" else 2)
                    + 4 * R * live / case["page"] + 4 * R, flops=4 * live * q)
    M, K, N = case["tokens"], case["K"], case["N"]
    G = case["group"] or K
    return dict(bytes=N * K // 2 + 2 * N * (K // G) + 2 * M * K + (4 * K if case["dinv"] else 0)
                + (2 * N if case["bias"] else 0) + M * N * (4 if case["out"] == "f32" else 2), flops=2 * M * N * K)


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_plan(case, s):
    """One request after another, as the definition reads."""
    P, T = case["page"], s["max_tokens"]
    cached, new, table, free = (s[k].tolist() for k in ("cached", "new", "table", "free"))
    head, max_pages = int(s["head"]), len(table[0])
    slot, pos, start, kv_len = [-1] * T, [-1] * T, [0], []
    asked, used = 0, 0
    for r, (c, n) in enumerate(zip(cached, new)):
        held, wanted = -(-c // P), -(-(c + n) // P)
        room = wanted <= max_pages
        more = wanted - held if room else 0
        room = room and (more == 0 or head + asked + more <= len(free)) and start[-1] + n <= T
        if room:
            for i in range(more):
                table[r][held + i] = free[head + asked + i]
            for i in range(n):
                pos[start[-1] + i] = c + i
                slot[start[-1] + i] = table[r][(c + i) // P] * P + (c + i) % P
            used = asked + more if more else used
        kv_len.append(c + n if room else c)
        asked += more
        start.append(start[-1] + n)

    def i32(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    return dict(table=i32(table), slot=i32(slot), pos=i32(pos), token_start=i32(start), kv_len=i32(kv_len),
                head=i32([head + used]))


def _exact_head(case, x, w, s):
    x = x.double()
    if w is not None:
        x = x / (x.square().sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * w.double()
    rot = case["rot"]
    if rot == 0:
        return x
    i = torch.arange(rot // 2, device="cuda")
    lo, hi = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
    c, n = s["cos"].double()[s["pos"].long()].unsqueeze(1), s["sin"].double()[s["pos"].long()].unsqueeze(1)
    y = x.clone()
    y[:, :, lo] = x[:, :, lo] * c - x[:, :, hi] * n
    y[:, :, hi] = x[:, :, hi] * c + x[:, :, lo] * n
    return y


def _exact_rope(case, s):
    q, k, v = _split_qkv(case, s["qkv"])
    P, at = case["page"], s["slot"].long()
    ck, cv = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda"), s["v"].double()
    rows = torch.arange(case["kv_heads"], device="cuda")
    ck[(at // P)[:, None], rows[None, :], (at % P)[:, None]] = _exact_head(case, k, s["kw"], s)
    cv[(at // P)[:, None], rows[None, :], (at % P)[:, None]] = v.double()
    return dict(q=_exact_head(case, q, s["qw"], s), k=ck, v=cv)


def _exact_attn(case, s):
    R, Hq, D = s["q"].shape
    Hk, P = s["k"].shape[1:3]
    group = Hq // Hk
    out = torch.zeros((R, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((R, Hq), dtype=torch.float64, device="cuda")
    lens = s["kv_len"].tolist()
    for r, n in enumerate(lens):
        first = max(0, n - case["window"]) if case["window"] else 0
        j = torch.arange(first, n, device="cuda")
        page, at = s["table"][r].long()[j // P], j % P
        for h in range(Hk):
            k, v = s["k"][page, h, at].double(), s["v"][page, h, at].double()
            for g in range(h * group, (h + 1) * group):
                sc = (k * s["q"][r, g].double()).sum(1) * s["scale"]
                lse[r, g] = torch.logsumexp(sc, 0)
                out[r, g] = (torch.exp(sc - lse[r, g])[:, None] * v).sum(0)
    return dict(out=out, lse=lse) if case["lse"] else out


def _exact_linear(case, s):
    N, K, G = case["N"], case["K"], s["G"]
    k = torch.arange(K, device="cuda")
    at, high = (k // 8) * 4 + k % 4, (k % 8) >= 4
    x = s["x"].double()
    if s["dinv"] is not None:
        x = x * s["dinv"].double()
    y = torch.zeros((case["tokens"], N), dtype=torch.float64, device="cuda")
    for n0 in range(0, N, 2048):
        byte = s["qw"][n0:n0 + 2048][:, at].int()
        nib = torch.where(high[None, :], byte // 16, byte % 16)
        w = (nib - 16 * (nib >= 8)).double() * s["step"].double()[k // G, n0:n0 + 2048].t()
        y[:, n0:n0 + 2048] = x @ w.t()
    return y if s["bias"] is None else y + s["bias"].double()


_EXACT = {"plan": _exact_plan, "rope": _exact_rope, "attn": _exact_attn, "linear": _exact_linear}


def exact(case, seed):
    return _EXACT[case["kind"]](case, _INPUTS[case["kind"]](case, seed))
