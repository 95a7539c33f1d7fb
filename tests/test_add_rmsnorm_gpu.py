"""The residual norm on the GPU against its 64-bit form, and its codes against
the quantizer's chain, at sizes, types, strides and contents where they can go
wrong."""
import pytest
import torch

import beam_ref as R
import token_ref as T
from paper_2609_39056_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
OUT = {"bf16": B.SQ_OUT_BF16, "f16": B.SQ_OUT_F16, "f32": B.SQ_OUT_F32}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def rand(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def act_of(g, M, K, static, dinv, streams=3, steps=4):
    return dict(t2s=torch.randint(0, streams, (M,), generator=g, dtype=torch.int32), gamma=torch.rand((steps, streams), generator=g) + 0.5,
                clip=torch.rand((steps,), generator=g) + 2.0 if static else None,
                dinv=torch.rand((K,), generator=g) + 0.5 if dinv else None, step=2)


def dev(t):
    return None if t is None else t.cuda()


def params(a):
    return B.ActParams(tok2stream=dev(a["t2s"]), gamma=dev(a["gamma"]), step=a["step"], act_bits=8,
                       range_mode=int(a["clip"] is not None), clip=dev(a["clip"]), dinv=dev(a["dinv"]))


def check_codes(qx, r, y32, a):
    q, s = R.codes(y32.cpu(), a["dinv"], a["gamma"][a["step"]][a["t2s"].long()], None if a["clip"] is None else a["clip"][a["step"]].item())
    assert torch.equal(qx.cpu(), q) and torch.equal(r.cpu(), s)


SIZES = [(1, 8), (3, 64), (5, 72), (7, 512), (4, 520), (9, 2048), (2, 2056), (33, 5120), (3, 6152), (2, 8192), (3, 8200),
         (2, 13824), (2, 16392), (1, 32768), (1030, 256), (2050, 1024)]


@pytest.mark.parametrize("M,K", SIZES)
@pytest.mark.parametrize("dt,res,out", [("bf16", "bf16", "bf16"), ("f16", "f32", "f16"), ("f32", None, "f32"), ("bf16", "f32", "f32"),
                                        ("f32", "bf16", "bf16")])
def test_norm(M, K, dt, res, out):
    g = torch.Generator().manual_seed(M + K)
    x = rand(g, M, K, scale=1.5, dtype=DT[dt])
    residual = None if res is None else rand(g, M, K, scale=4.0, dtype=DT[res])
    w = rand(g, K, scale=0.3) + 1.0
    h, u, bh, bu = R.add_rmsnorm(x, residual, w, EPS)
    y = torch.full((M, K), 7.0, dtype=DT[out], device="cuda")
    s = None if res is None else torch.full((M, K), 7.0, dtype=DT[res], device="cuda")
    B.sq_add_rmsnorm(x.cuda(), dev(residual), w.cuda(), EPS, s, y, OUT[out], None, None, None)
    T.check(y, u, bu, DT[out], "y")
    if res is not None:
        T.check(s, h, bh, DT[res], "sum")


@pytest.mark.parametrize("M,K", [(1, 128), (5, 512), (4, 640), (9, 2048), (33, 5120), (2, 13824), (1, 32768), (1030, 256),
                                 (3, 1024), (2, 4096), (4, 6144), (2, 8192), (1024, 5120), (1025, 4224), (1025, 6144), (1025, 6272)])
@pytest.mark.parametrize("static,dinv,res,weight", [(False, True, "bf16", True), (True, True, None, True), (False, False, "f32", False),
                                                    (True, False, "f16", True)])
def test_codes(M, K, static, dinv, res, weight):
    g = torch.Generator().manual_seed(3 * M + K)
    x = rand(g, M, K, dtype=DT["f16" if res == "f16" else "bf16"])
    residual = None if res is None else rand(g, M, K, scale=3.0, dtype=DT[res])
    w = rand(g, K, scale=0.3) + 1.0 if weight else None
    if M > 2:  # rows of zeros: their codes and, with a dynamic range, their scales are 0
        x[1] = 0
        if residual is not None:
            residual[1] = 0
    a = act_of(g, M, K, static, dinv)
    qx, r = B.act_buffers(M, K, 8)
    y = torch.empty((M, K), device="cuda")
    B.sq_add_rmsnorm(x.cuda(), dev(residual), dev(w), EPS, None, y, B.SQ_OUT_F32, params(a), qx, r)
    check_codes(qx, r, y, a)
    _, u, _, bu = R.add_rmsnorm(x, residual, w, EPS)
    T.check(y, u, bu, torch.float32, "y")
    # without y the codes are the same
    q2, r2 = B.act_buffers(M, K, 8)
    B.sq_add_rmsnorm(x.cuda(), dev(residual), dev(w), EPS, None, None, 0, params(a), q2, r2)
    assert torch.equal(q2, qx) and torch.equal(r2, r)


def test_codes_feed_the_quantized_linear():
    # codes of a row that 16 bits hold exactly are the quantizer's own, and so is the linear on them
    g = torch.Generator().manual_seed(5)
    M, K, N = 20, 256, 128
    a = act_of(g, M, K, False, True)
    y = torch.empty((M, K), device="cuda")
    x = rand(g, M, K, dtype=torch.bfloat16).cuda()
    qx, r = B.act_buffers(M, K, 8)
    B.sq_add_rmsnorm(x, None, None, 0.0, None, y, B.SQ_OUT_F32, params(a), qx, r)
    W = B.prepare_weight(rand(g, N, K, scale=0.02).cuda(), None, 128)
    out = torch.empty((M, N), device="cuda")
    B.sq_gemm_w4a8(qx, r, W, out, B.SQ_OUT_F32)
    want, bound = T.linear(qx.cpu().double() * r.cpu().double()[:, None], None, W.qw.cpu().numpy(), W.w_scale.cpu(), 128, None,
                           torch.float32)
    T.check(out, want, bound + 4 * R.U32 * want.abs(), torch.float32, "linear")


@pytest.mark.parametrize("dt,res", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
def test_strides_and_places(dt, res):
    g = torch.Generator().manual_seed(9)
    M, K, wide = 6, 520, 1536
    xb, rb = rand(g, M, wide, dtype=DT[dt]).cuda(), rand(g, M, wide, dtype=DT[res]).cuda()
    x, residual = xb[:, 8:8 + K], rb[:, 16:16 + K]
    w = (rand(g, K) + 1.0).cuda()
    h, u, bh, bu = R.add_rmsnorm(x.cpu(), residual.cpu(), w.cpu(), EPS)
    keep, rkeep = xb.clone(), rb.clone()
    y = torch.empty((M, K), device="cuda")
    # the sum in the residual's place
    B.sq_add_rmsnorm(x, residual, w, EPS, residual, y, B.SQ_OUT_F32, None, None, None)
    T.check(y, u, bu, torch.float32, "y")
    T.check(residual, h, bh, DT[res], "sum")
    rkeep[:, 16:16 + K] = residual
    assert torch.equal(rb, rkeep) and torch.equal(xb, keep)  # nothing beside the rows
    # y in the place of x, of one type
    x2 = x.contiguous()
    B.sq_add_rmsnorm(x2, None, w, EPS, None, x2, OUT[dt], None, None, None)
    _, u2, _, bu2 = R.add_rmsnorm(x.cpu(), None, w.cpu(), EPS)
    T.check(x2, u2, bu2, DT[dt], "y in the place of x")
    # only the sum
    s = torch.empty((M, K), dtype=DT[res], device="cuda")
    rb.copy_(rkeep)
    B.sq_add_rmsnorm(x, residual, None, EPS, s, None, 0, None, None, None)
    T.check(s, x.cpu().double() + residual.cpu().double(), R.U32 * (x.cpu().double() + residual.cpu().double()).abs(), DT[res], "sum")


def test_no_rows_and_rows_past_the_last():
    g = torch.Generator().manual_seed(2)
    w = rand(g, 256).cuda()
    empty = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    B.sq_add_rmsnorm(empty, None, w, EPS, None, empty.clone(), B.SQ_OUT_BF16, None, None, None)
    for M in (1, 2, 3, 5):
        y = torch.full((M + 4, 256), 3.0, dtype=torch.bfloat16, device="cuda")
        B.sq_add_rmsnorm(rand(g, M, 256, dtype=torch.bfloat16).cuda(), None, w, EPS, None, y[:M], B.SQ_OUT_BF16, None, None, None)
        assert (y[M:] == 3.0).all() and (y[:M] != 3.0).any()


def test_weights_and_scales_are_applied_where_they_belong():
    # whole powers of two: exact results
    M, K = 3, 1024
    x = torch.ones((M, K), dtype=torch.bfloat16)
    x[1] = 2.0
    w = 2.0 ** (torch.arange(K) % 7).float()
    y = torch.empty((M, K), device="cuda")
    B.sq_add_rmsnorm(x.cuda(), None, w.cuda(), 0.0, None, y, B.SQ_OUT_F32, None, None, None)
    assert torch.equal(y.cpu(), w.expand(M, K))


def test_graph_replays():
    g = torch.Generator().manual_seed(4)
    M, K = 40, 2048
    x, residual = rand(g, M, K, dtype=torch.bfloat16).cuda(), rand(g, M, K, dtype=torch.bfloat16).cuda()
    w = (rand(g, K) + 1.0).cuda()
    a = params(act_of(g, M, K, False, True))
    qx, r = B.act_buffers(M, K, 8)
    s = torch.empty_like(x)

    def call():
        B.sq_add_rmsnorm(x, residual, w, EPS, s, None, 0, a, qx, r)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        x.copy_(rand(g, M, K, dtype=torch.bfloat16))
        graph.replay()
        got = qx.clone(), r.clone(), s.clone()
        call()
        assert all(torch.equal(p, q) for p, q in zip(got, (qx, r, s)))
