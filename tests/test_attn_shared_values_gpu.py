"""Attention over shared prefixes on the GPU with inputs whose exact result is
known to more than a general bound can tell."""
import numpy as np
import pytest
import torch

from paper_2609_39056_amd import binding as B
from test_token_step_values_gpu import DT, OUT, U, cancelling

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,L,at", [(1, 16, 0), (3, 300, 96), (9, 5000, 1536), (40, 300, 96)])
def test_probabilities_of_the_prefix_are_whole(rows, L, at, dtype, out):
    """16-bit outputs too are sums over fp32 probabilities: a score's three
    roundings in units of log 2 make 6 units of p (|s| < 1 and a factor of log2 e),
    the exponential 2, the parts 1, sixteen sums of exact products up to 18 and the
    quotient and rounding of a result that cancels to nothing none; 32 in all, of
    the sum of magnitudes.  The other tokens' probabilities are 0."""
    D, dt, page = 64, DT[dtype], 16
    s, v, rest = cancelling(D, dt, L)
    p = np.exp(s)
    bound = 32 * U * (p[:, None] * np.abs(v)).sum(0)
    assert ((rest[:, None] * np.abs(v[:12])).sum(0) > 1.3 * bound).all()  # what two bf16 parts would leave is outside
    n = -(-L // page) * page
    k, vals = torch.zeros((n, D)), torch.ones((n, D))
    k[:, 0] = -200.0
    k[at:at + 16, 0] = torch.from_numpy(s).float()
    vals[at:at + 16] = torch.from_numpy(v).float()
    kv = B.KVCache(*(t.to(dt).view(n // page, 1, page, D).cuda() for t in (k, vals)))
    q = torch.zeros((rows, 3, D), dtype=dt, device="cuda")
    q[:, :, 0] = 1.0

    def ints(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    y = torch.full((rows, 3, D), 77.0, dtype=DT[out], device="cuda")
    ws = B.alloc_attn_shared_workspace(rows, 1, 3, kv, L, 1)
    ws.fill_(255)  # NaN patterns
    B.sq_attn_shared(q, kv, ints([list(range(n // page))] * rows), ints([L] * rows), ints([0, rows]), ints([L]), L, 1, 1.0, y,
                     OUT[out], None, ws)
    want = (p[:, None] * v).sum(0) / p.sum()
    bound = bound / p.sum()
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= bound + np.abs(want) * 2.0 ** -8).all(), f"{(err / bound).max():.3g} of the bound"
