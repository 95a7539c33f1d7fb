"""Plain 64-bit forms of the token step's operators on the CPU, written from
their definitions in include/sq.h, and the error bounds of their outputs.

Bounds: u = 2^-24 is the fp32 unit.  A 16-bit output adds its own rounding,
half a unit in the last place: of 8 significant bits (bf16) at most 2^-8 of the
value, of 11 (f16) at most 2^-11, and at most 2^-25 below f16's normal range."""
import math

import numpy as np
import torch

U32 = 2.0 ** -24
HALF = {torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.float32: (0.0, 2.0 ** -149)}


def out_rounding(y, dtype):
    """Bound of rounding y (float64) to dtype."""
    rel, tiny = HALF[dtype]
    return rel * y.abs() + tiny


def check(got, want, bound, dtype, what):
    """|got - want| within the bound and the output's rounding (1 % on top for
    the rounding of a value that is already off by the bound)."""
    got = got.detach().cpu().double()
    err = (got - want).abs()
    lim = bound * 1.01 + out_rounding(want.abs() + bound, dtype)
    assert not torch.isnan(got).any(), f"{what}: NaN"
    bad = err > lim
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {(err / lim).max():.3g} of the bound"


# ------------------------------------------------------------------ plan
def plan(cached, new, page, free, head, table, max_tokens):
    """One request after another; lists and ints in, the operator's outputs out."""
    table = [list(row) for row in table]
    max_pages = len(table[0])
    slot, pos, start, kv_len = [-1] * max_tokens, [-1] * max_tokens, [0], []
    head = min(max(head, 0), len(free))
    first = used = 0
    for r in range(len(cached)):
        c, n = max(cached[r], 0), max(new[r], 0)
        have, need = -(-c // page), -(-(c + n) // page)
        take = need - have if need <= max_pages else 0
        ok = need <= max_pages and (take == 0 or head + first + take <= len(free)) and start[-1] + n <= max_tokens
        if ok:
            table[r][have:have + take] = free[head + first:head + first + take]
            for t in range(n):
                p = c + t
                pos[start[-1] + t] = p
                slot[start[-1] + t] = table[r][p // page] * page + p % page
            used = first + take if take else used
        kv_len.append(c + n if ok else c)
        first += take
        start.append(start[-1] + n)
    cap = 2 ** 31 - 1
    return table, slot, pos, [min(s, cap) for s in start], kv_len, head + used


# ------------------------------------------------------------------ norm and rotation
def norm_rope(x, w, eps, cos, sin, pos, interleaved):
    """x [T, H, D] (any type) -> float64 result and the bound of its fp32
    computation: the norm's factor is good to a few units (a sum of D squares
    in pairs, a division, a root), each product and the rotation's sum add one
    each; 16 units of the magnitudes that enter cover them."""
    x = x.double()
    D = x.shape[-1]
    if w is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + eps) * w.double()
    y, mag = x.clone(), x.abs()
    if cos is not None:
        h = cos.shape[1]
        c, s = cos.double()[pos.long()][:, None], sin.double()[pos.long()][:, None]
        ia = torch.arange(h) * 2 if interleaved else torch.arange(h)
        ib = ia + 1 if interleaved else ia + h
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        both = a.abs() + b.abs()
        mag = mag.clone()
        mag[..., ia], mag[..., ib] = both, both
    return y, (16 + D / 16) * U32 * mag


# ------------------------------------------------------------------ attention
def attn(q, k, v, table, kv_len, window, scale, max_kv_len, out_dtype):
    """q [R, Hq, D]; k, v the pages [num_pages, Hk, P, D].  Returns out, lse
    (float64) and their bounds: a score is a fp32 sum of D exact products, off
    by at most (D + 4) units of scale * sum |q k|; an exponential by 4 units
    and its argument's own rounding; a sum of n terms by (n / 32 + 64) units;
    a probability enters its product with 16 bits (2^-16) where the output has
    16, with 21 where it is fp32."""
    R, Hq, D = q.shape
    num_pages, Hk, P, _ = k.shape
    G = Hq // Hk
    out, lse = torch.zeros((R, Hq, D), dtype=torch.float64), torch.full((R, Hq), -math.inf, dtype=torch.float64)
    b_out, b_lse = torch.zeros_like(out), torch.zeros_like(lse)
    part = 2.0 ** -21 if out_dtype == torch.float32 else 2.0 ** -16
    for r in range(R):
        n = min(max(int(kv_len[r]), 0), max_kv_len)
        j = torch.arange(max(0, n - window) if window else 0, n)
        page = table[r].long()[j // P]
        live = (page >= 0) & (page < num_pages)
        page, at = page[live], (j % P)[live]
        if page.numel() == 0:
            continue
        for h in range(Hk):
            kk, vv = k[page, h, at].double(), v[page, h, at].double()
            qq = q[r, h * G:(h + 1) * G].double()
            s = qq @ kk.t() * scale
            mag = (qq.abs() @ kk.abs().t() * abs(scale)).amax(1)
            ds = (D + 4) * U32 * mag
            top = s.amax(1, keepdim=True)
            e = torch.exp(s - top)
            total = e.sum(1)
            A = (e @ vv.abs()) / total[:, None]
            N = page.numel()
            rel = 2 * (ds + (8 + 4 * mag) * U32) + (N / 32 + 64) * U32
            out[r, h * G:(h + 1) * G] = (e @ vv) / total[:, None]
            lse[r, h * G:(h + 1) * G] = top[:, 0] + torch.log(total)
            b_out[r, h * G:(h + 1) * G] = A * (rel + part)[:, None]
            b_lse[r, h * G:(h + 1) * G] = rel + 4 * U32 * (top[:, 0].abs() + torch.log(total).abs() + 1)
    return out, lse, b_out, b_lse


# ------------------------------------------------------------------ linear
def unpack(qw):
    """Packed uint8 [N, K/2] -> codes int64 [N, K]."""
    b = np.asarray(qw).astype(np.int64)
    N = b.shape[0]
    b = b.reshape(N, -1, 1, 4)
    nib = np.concatenate([b & 15, b >> 4], axis=2).reshape(N, -1)
    return torch.from_numpy(np.where(nib > 7, nib - 16, nib))


def linear(x, dinv, qw, w_scale, group, bias, out_dtype):
    """x [M, K] bf16; w_scale fp16 [K/group, N].  The codes may be met as
    code + 8 (sums up to 16 |x~| per channel cancel), fp32 sums of 128 channels
    and then of the groups; 16-bit outputs take x~ with 16 bits."""
    x64 = x.double()
    if dinv is not None:
        x64 = x64 * dinv.double()
    codes = unpack(qw)
    N, K = codes.shape
    step = w_scale.double().t().repeat_interleave(group, dim=1)
    w = codes.double() * step
    y = x64 @ w.t()
    wide = x64.abs() @ ((codes.abs() + 16).double() * step).t()
    bound = (48 + K / 128) * U32 * wide
    if dinv is not None:
        bound = bound + (0.0 if out_dtype == torch.float32 else 2.0 ** -16) * (x64.abs() @ w.abs().t())
    if bias is not None:
        y = y + bias.double()
        bound = bound + U32 * (y.abs() + bias.double().abs())
    return y, bound
