"""The token step's operators on the GPU with inputs whose exact result is known
to more than a general bound can tell: sums that cancel, values that mark every
token, infinities and NaN where they are read."""
import math

import numpy as np
import pytest
import torch

from paper_2609_39056_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
OUT = {"bf16": B.SQ_OUT_BF16, "f16": B.SQ_OUT_F16, "f32": B.SQ_OUT_F32}
U = 2.0 ** -24  # the fp32 unit


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def attend(q, k, v, lens, page, out, window=0, scale=1.0, longest=None):
    """q [R, Hq, D]; k, v [R, L, Hk, D] on the host, put into pages in a shuffled
    order; the tokens past a request's length hold NaN.  Returns out and lse."""
    R, L, Hk, D = k.shape
    n = -(-L // page)
    ids = torch.randperm(R * n, generator=torch.Generator().manual_seed(R + L)).view(R, n)
    cache = []
    for t in (k, v):
        pages = torch.full((R, n * page, Hk, D), float("nan"), dtype=t.dtype)
        for r, m in enumerate(lens):
            pages[r, :m] = t[r, :m]
        c = torch.empty((R * n, Hk, page, D), dtype=t.dtype)
        c[ids.flatten()] = pages.view(R * n, page, Hk, D).transpose(1, 2)
        cache.append(c.cuda())
    kv = B.KVCache(*cache)
    Hq = q.shape[1]
    longest = L if longest is None else longest
    y = torch.full((R, Hq, D), 77.0, dtype=DT[out], device="cuda")
    lse = torch.full((R, Hq), 77.0, device="cuda")
    ws = B.alloc_attn_workspace(R, Hq, kv, longest)
    ws.fill_(255)  # NaN patterns
    B.sq_attn_paged(q.cuda(), kv, ids.to(torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                    longest, window, scale, y, OUT[out], lse, ws)
    return y.cpu(), lse.cpu()


# ------------------------------------------------------------------ probabilities
def halves(x, dtype, parts):
    """x (float32 numpy) as the sum of this many values of a 16-bit type, each
    taking what the ones before left, and what they leave."""
    rest, total = x.astype(np.float32), np.zeros(x.shape)
    for _ in range(parts):
        p = torch.from_numpy(rest).to(dtype).float().numpy()
        total += p
        rest = rest - p
    return total, x - total


def cancelling(D, dtype, seed):
    """Twelve keys whose probabilities two bf16 parts hold worst (0.5 .. 0.6 of
    the largest, with a residual of nearly 2^-18), values with the residuals'
    signs, and four keys of probability one whose values cancel the sum."""
    rng = np.random.default_rng(seed)
    s = -np.arange(64, 90, dtype=np.float64) / 128  # exact in both types
    p = np.exp(s)
    _, rest = halves(p.astype(np.float32), torch.bfloat16, 2)
    best = np.argsort(-np.abs(rest) / p)[:12]
    v = np.sign(rest[best])[:, None] * torch.from_numpy(rng.uniform(0.5, 1, (12, D))).to(dtype).double().numpy()
    scores, values = list(s[best]), list(v)
    for _ in range(4):
        total = sum(math.exp(a) * b for a, b in zip(scores, values))
        scores.append(0.0)
        values.append(-torch.from_numpy(total).to(dtype).double().numpy())
    return np.array(scores), np.stack(values), np.abs(rest[best])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L,at", [(16, 0), (300, 96), (700, 640), (5000, 1536)])
def test_attn_probabilities_are_whole(dtype, L, at):
    """16-bit outputs like fp32 ones are sums over fp32 probabilities: a score's three
    roundings in units of log 2 make 6 units of p (|s| < 1 and a factor of log2 e),
    the exponential 2, the parts 1, sixteen sums of exact products up to 18 and the
    quotient and rounding of a result that cancels to nothing none; 32 in all, of
    the sum of magnitudes.  The other tokens' probabilities are 0."""
    D, dt = 64, DT[dtype]
    s, v, rest = cancelling(D, dt, L)
    p = np.exp(s)
    bound = 32 * U * (p[:, None] * np.abs(v)).sum(0)
    assert ((rest[:, None] * np.abs(v[:12])).sum(0) > 1.3 * bound).all()  # what two bf16 parts would leave is outside
    k = torch.zeros((1, L, 1, D))
    k[0, :, 0, 0] = -200.0
    k[0, at:at + 16, 0, 0] = torch.from_numpy(s).float()
    vals = torch.ones((1, L, 1, D))
    vals[0, at:at + 16, 0] = torch.from_numpy(v).float()
    q = torch.zeros((1, 3, D))
    q[:, :, 0] = 1.0
    want = (p[:, None] * v).sum(0) / p.sum()
    bound = bound / p.sum()
    for out in (dtype, "f32"):
        y, _ = attend(q.to(dt), k.to(dt), vals.to(dt), [L], 16, out)
        err = np.abs(y[0].double().numpy() - want[None])
        assert (err <= bound + np.abs(want) * 2.0 ** -8).all(), f"{out}: {(err / bound).max():.3g} of the bound"


# ------------------------------------------------------------------ values that are not finite
def spread(R, L, Hq, Hk, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g).to(DT[dtype]) for s in ((R, Hq, D), (R, L, Hk, D), (R, L, Hk, D))]


LENGTHS = [(24, 64), (60, 64), (300, 128), (700, 96), (2500, 64), (2500, 256)]  # one wave and more, whole and split


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L,D", LENGTHS)
def test_attn_nan_that_is_read_is_not_an_empty_row(dtype, L, D):
    """A NaN in an attended key or a query, or a score of +infinity, makes out and
    lse NaN; only a row that attends nothing has lse -infinity."""
    q, k, v = spread(5, L, 4, 2, D, dtype, L)
    k[0, L // 2, 1, 5] = float("nan")
    q[1, 2, 7] = float("nan")
    k[2, L - 1, 0, 0], k[2, L - 1, 0, 1] = float("inf"), float("-inf")
    k[4, 0, 1, 3] = float("inf")
    q[2, :2], q[4, 2:] = 1.0, 1.0
    y, lse = attend(q, k, v, [L, L, L, 0, L - 1], 16, dtype, scale=D ** -0.5)
    bad = torch.zeros((5, 4), dtype=torch.bool)
    bad[0, 2:], bad[1, 2], bad[2, :2], bad[4, 2:] = True, True, True, True
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(y), bad[:, :, None].expand_as(y))
    assert torch.isfinite(lse[[0, 1, 2, 4]][~bad[[0, 1, 2, 4]]]).all()
    assert (lse[3] == -math.inf).all() and (y[3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L,D", LENGTHS)
def test_attn_infinite_values_of_probability_zero(dtype, L, D):
    """0 times an infinity: a value whose key's score is -infinity."""
    q, k, v = spread(2, L, 4, 2, D, dtype, L + 3)
    q[:, :, 2] = 1.0
    k[:, L // 2, 0, 2] = float("-inf")
    want, _ = attend(q, k, v, [L, L], 16, "f32", scale=D ** -0.5)
    v[0, L // 2, 0, 7], v[1, L // 2, 0, 7], v[1, 0, 0, 7] = float("inf"), float("-inf"), float("-inf")
    v[1, 3, 0, 6] = float("inf")
    want[:, :2, 7], want[1, :2, 6] = float("nan"), float("inf")
    y, _ = attend(q, k, v, [L, L], 16, "f32", scale=D ** -0.5)
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y.nan_to_num(5.0, math.inf, -math.inf), want.nan_to_num(5.0, math.inf, -math.inf))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L,D", LENGTHS)
def test_attn_scores_of_minus_infinity(dtype, L, D):
    """An attended key whose score is -infinity has probability 0; a row of
    nothing else is like one that attends nothing."""
    q, k, v = spread(2, L, 2, 1, D, dtype, 2 * L + D)
    q[:, :, 0] = 1.0
    ref = attend(q, k[:, :L - 1], v[:, :L - 1], [L - 1, L - 1], 16, "f32", scale=D ** -0.5, longest=L)
    k[0, L - 1, 0, 0] = float("-inf")
    k[1, :, 0, 0] = float("-inf")
    y, lse = attend(q, k, v, [L, L], 16, "f32", scale=D ** -0.5)
    assert torch.equal(y[0], ref[0][0]) and torch.equal(lse[0], ref[1][0])
    assert (y[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f32"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("L,D", LENGTHS)
def test_attn_infinite_values(dtype, out, L, D):
    """An infinite value that is attended makes its dimension infinite, with its
    sign; both signs, or a NaN, make it NaN; the other dimensions do not change."""
    q, k, v = spread(3, L, 6, 2, D, dtype, L + D)
    lens = [L, L - 1, L - 5]
    want, lse = attend(q, k, v, lens, 16, out, scale=D ** -0.5)
    inf = float("inf")
    v[0, L // 3, 0, 3], v[0, L // 2, 1, 9], v[0, 0, 1, D - 1] = inf, -inf, inf
    v[1, L - 2, 0, 0], v[1, 1, 0, 0], v[1, 2, 0, 1], v[1, L // 2, 0, 1] = inf, -inf, inf, inf
    v[2, 0, 1, 40], v[2, 0, 1, 41] = float("nan"), -inf
    want[0, :3, 3], want[0, 3:, 9], want[0, 3:, D - 1] = inf, -inf, inf
    want[1, :3, 0], want[1, :3, 1] = float("nan"), inf
    want[2, 3:, 40], want[2, 3:, 41] = float("nan"), -inf
    y, lse2 = attend(q, k, v, lens, 16, out, scale=D ** -0.5)
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y.nan_to_num(5.0, inf, -inf), want.nan_to_num(5.0, inf, -inf))
    assert torch.equal(lse, lse2)


# ------------------------------------------------------------------ linear
def packed(codes, step, group, bias=None):
    """Codes int [N, K], steps [K / group, N] -> the weight on the device."""
    N, K = codes.shape
    c = (codes & 15).view(N, K // 8, 2, 4)
    qw = (c[:, :, 0] | (c[:, :, 1] << 4)).to(torch.uint8).reshape(N, K // 2)
    return B.Weight(qw.cuda(), step.half().cuda(), group, None if bias is None else bias.cuda())


ROWS = [(1, 1280, 64), (3, 1280, 320), (5, 640, 4160), (16, 1280, 320), (20, 1280, 5120), (64, 256, 8256)]


@pytest.mark.parametrize("M,K,N", ROWS)
@pytest.mark.parametrize("use_d", [True, False])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_linear_infinite_rows(M, K, N, use_d, out):
    """An infinite activation gives what its products do: an infinity with the
    code's sign, NaN where the code is 0 or two of them have both signs; a NaN
    gives NaN.  The other rows do not change."""
    g = torch.Generator().manual_seed(M + N)
    codes = torch.randint(-7, 8, (N, K), generator=g)
    step = torch.rand((K // 128, N), generator=g) + 0.1
    x = torch.randn((M, K), generator=g).to(torch.bfloat16)
    dinv = torch.rand((K,), generator=g) + 0.5 if use_d else None
    bias = torch.randn((N,), generator=g).to(torch.bfloat16)
    W = packed(codes, step, 128, bias)

    def run():
        y = torch.full((M, N), 77.0, dtype=DT[out], device="cuda")
        B.sq_linear_w4a16(x.cuda(), None if dinv is None else dinv.cuda(), W, y, OUT[out])
        return y.cpu()

    want = run()
    inf = float("inf")
    changed = {0: [(0, inf)], M // 2: [(130, -inf), (K - 1, inf)], M - 1: [(7, inf), (K - 5, inf)]}
    if M > 4:
        changed[1] = [(99, float("nan"))]
    for m, at in changed.items():
        x[m] = torch.randn((K,), generator=g).to(torch.bfloat16)
        row = torch.zeros((N,))
        for k, val in at:
            x[m, k] = val
            row = row + val * codes[:, k].float()
        want[m] = row.to(DT[out])
    y = run()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y.nan_to_num(5.0, inf, -inf), want.nan_to_num(5.0, inf, -inf))


@pytest.mark.parametrize("M", [1, 2, 20])
def test_linear_largest_values(M):
    """Activations near the type's largest and a scaling that takes them past it
    stay what fp32 makes of them."""
    K, N = 256, 64
    codes = torch.zeros((N, K), dtype=torch.long)
    codes[:, 3], codes[:, 200] = torch.arange(N) % 8 - 1, 1
    W = packed(codes, torch.full((2, N), 2.0 ** -10), 128)
    x = torch.zeros((M, K), dtype=torch.bfloat16)
    x[:, 3], x[:, 200] = 3.3e38, 1.0
    y = torch.empty((M, N), device="cuda")
    for d in (3.4e38 / x[0, 3].item(), 1.0, 0.5):  # the first is past bf16's range, within fp32's
        dinv = torch.full((K,), d)
        B.sq_linear_w4a16(x.cuda(), dinv.cuda(), W, y, B.SQ_OUT_F32)
        want = ((x.float() * dinv).double() @ (codes.double() * 2.0 ** -10).t())
        assert torch.isfinite(want).all()
        # two products, each good to some units of the 15 |x~| that a code is met with
        assert ((y.cpu().double() - want).abs() <= 64 * U * 15 * 2.0 ** -10 * 3.4e38 * d).all()


# ------------------------------------------------------------------ the batch drains
def test_attn_workspace_serves_smaller_batches():
    """One workspace, sized for the largest batch, through a batch that gets
    smaller and shorter: the same results as with one of its own."""
    Hq, Hk, D, L = 16, 4, 64, 1000
    q, k, v = spread(130, L, Hq, Hk, D, "bf16", 3)
    kv = B.KVCache(*(t.view(130 * L // 8, 8, Hk, D).transpose(1, 2).contiguous().cuda() for t in (k, v)))
    table = torch.arange(130 * L // 8, dtype=torch.int32, device="cuda").view(130, L // 8)
    ws = B.alloc_attn_workspace(130, Hq, kv, L)
    q = q.cuda()
    for R, n in ((130, 1000), (64, 1000), (40, 900), (24, 700), (7, 500), (1, 385)):
        lens = torch.full((R,), n, dtype=torch.int32, device="cuda")
        out = [torch.full((R, Hq, D), 77.0, device="cuda") for _ in range(2)]
        for o, w in zip(out, (ws, B.alloc_attn_workspace(R, Hq, kv, n))):
            B.sq_attn_paged(q[:R], kv, table[:R], lens, n, 0, 0.125, o, B.SQ_OUT_F32, None, w)
        assert torch.equal(*out) and not (out[0] == 77.0).any()


# ------------------------------------------------------------------ every token once
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("R,L,Hq,Hk,D,page,window", [
    (3, 31, 2, 2, 64, 8, 0), (3, 1280, 2, 1, 128, 16, 0), (2, 5000, 8, 2, 96, 8, 0), (2, 5000, 32, 1, 128, 64, 1999),
    (1, 20011, 4, 4, 192, 16, 0), (1, 66003, 32, 32, 64, 128, 0), (1, 66003, 2, 1, 256, 32, 65601), (70, 1300, 34, 2, 64, 16, 0),
    (400, 64, 4, 4, 64, 8, 0), (300, 61, 6, 3, 96, 16, 7), (260, 48, 3, 3, 128, 8, 33), (200, 40, 4, 4, 192, 32, 0),
    (200, 63, 5, 5, 256, 8, 20)])
def test_attn_takes_every_token_once(R, L, Hq, Hk, D, page, window, dtype):
    """Scores of 0 make every probability 1, and values of small integers make all
    sums exact: a token left out, taken twice or from another place changes an
    integer.  Out and lse carry a quotient, a logarithm and their roundings."""
    g = torch.Generator().manual_seed(L)
    lens = ([L, L - 1, max(0, L - 129), L // 2, 0, 33, 32, 1] + [(53 * r) % (L + 1) for r in range(R)])[:R]
    k = torch.zeros((R, L, Hk, D), dtype=DT[dtype])
    v = torch.randint(-3, 4, (R, L, Hk, D), generator=g, dtype=torch.int8)
    q = torch.randn((R, Hq, D), generator=g)
    y, lse = attend(q.to(DT[dtype]), k, v.to(DT[dtype]), lens, page, "f32", window=window)
    for r, n in enumerate(lens):
        first = max(0, n - window) if window else 0
        total = v[r, first:n].sum(0).double().repeat_interleave(Hq // Hk, 0)
        if n == 0:
            assert (y[r] == 0).all() and (lse[r] == -math.inf).all()
            continue
        assert ((y[r].double() * (n - first) - total).abs() <= 4 * U * total.abs()).all(), (r, n)
        # log2 to an ulp, of the sum in the kernel's units (f16: probabilities times 2^11),
        # its product with ln 2 (rounded) and the result's rounding
        size = math.log(n - first) + (11 * math.log(2) if dtype == "f16" else 0.0)
        assert ((lse[r].double() - math.log(n - first)).abs() <= 6 * U * max(1.0, size)).all(), (r, n)


# ------------------------------------------------------------------ norm and rotation of prompts
@pytest.mark.parametrize("T", [511, 512, 513])
@pytest.mark.parametrize("Hq,Hk,D,rot", [(33, 11, 128, 128), (40, 8, 128, 64), (12, 12, 192, 96), (5, 5, 96, 96),
                                         (24, 7, 256, 256), (70, 35, 64, 64), (1, 1, 64, 0)])
def test_rope_of_prompts(T, Hq, Hk, D, rot):
    """From 512 tokens on a workgroup takes all heads of a token in several rounds,
    queries, keys and values in turn, the last one ragged; below it one round."""
    from test_token_step_gpu import check_rope, rope_case

    for dtype, inter, norm in (("bf16", False, True), ("f16", True, True), ("bf16", True, False)):
        c = rope_case(T, Hq, Hk, D, rot, dtype, T + D + Hq, norm=norm)
        n = c["shape"][0] * c["shape"][2]
        skip = dict(skip_pos=((3, -1), (T - 2, 50)), skip_slot=((0, -1), (7, n), (T - 1, 2 ** 31 - 1))) if rot else {}
        check_rope(c, T, Hq, Hk, D, dtype, inter, use_k_out=inter, **skip)


# ------------------------------------------------------------------ a product at a time
@pytest.mark.parametrize("M,K,N", ROWS)
def test_linear_keeps_every_bit_of_a_scaled_row(M, K, N):
    """fp32 outputs take all 24 bits of x * dinv.  One channel of a row is not 0 and
    its codes are 7 or -7, so y is 7 x~ step: three parts, the sums with code + 8
    and of the -8, their difference and the step's product come to at most
    (3 * 2 (15 + 8)) / 7 + 2 = 22 units.  Two parts of these x~ leave more."""
    g = torch.Generator().manual_seed(M * N)
    # x~ in (1, 2) whose two leading bf16 parts miss at least 2^-18.4
    cand = (1 + torch.rand((20000,), generator=g)).numpy()
    _, rest = halves(cand, torch.bfloat16, 2)
    cand = torch.from_numpy(cand[np.abs(rest) > 48 * U * cand])
    dinv = cand[torch.arange(K) % cand.numel()]
    codes = torch.where(torch.rand((N, K), generator=g) < 0.5, 7, -7)
    W = packed(codes, torch.full((K // 128, N), 0.25), 128)
    x = torch.zeros((M, K), dtype=torch.bfloat16)
    at = torch.randint(0, K, (M,), generator=g)
    x[torch.arange(M), at] = 1.0
    y = torch.empty((M, N), device="cuda")
    B.sq_linear_w4a16(x.cuda(), dinv.cuda(), W, y, B.SQ_OUT_F32)
    want = dinv[at].double()[:, None] * codes[:, at].t().double() * 0.25
    assert ((y.cpu().double() - want).abs() <= 22 * U * want.abs()).all()
