"""Plain 64-bit forms of the operators of beams and of the residual norm, on the
CPU, written from their definitions in include/sq.h, with the error bounds of
their outputs (u = 2^-24 is the fp32 unit)."""
import math

import torch

U32 = 2.0 ** -24


# ------------------------------------------------------------------ norm
def add_rmsnorm(x, residual, weight, eps):
    """Returns h, u (float64) and the bounds of their fp32 values.  h is rounded
    once.  A row's sum of squares is formed of at most 32 values in turn in a lane,
    six halvings and 16 waves: 54 roundings, and 2 of each h^2; the mean, eps, the
    root and the division add 2 and halve what came before, 30 units in all; the two
    products and h add 3."""
    h = x.double()
    b = torch.zeros_like(h)
    if residual is not None:
        h = h + residual.double()
        b = U32 * h.abs()
    u = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    if weight is not None:
        u = u * weight.double()
    return h, u, b, 36 * U32 * u.abs()


def codes(u32, dinv, gain, clip):
    """The quantizer's chain in single fp32 operations on fp32 rows u32 [M, K]: codes and row scales."""
    v = u32 if dinv is None else u32 * dinv
    c = v.abs().amax(1, keepdim=True) if clip is None else torch.full((v.shape[0], 1), clip)
    delta = c / torch.tensor(127.0)
    inv = 1.0 / delta
    inv = torch.where(torch.isinf(inv), torch.zeros_like(inv), inv)
    q = torch.round(torch.clamp((v * gain[:, None]) * inv, -127.0, 127.0))
    return q.to(torch.int8), (delta / gain[:, None])[:, 0]


# ------------------------------------------------------------------ choice of beams
def beam_totals(logits, scores, done, end_token):
    """float64 totals [R, V]: -infinity for what is never taken."""
    x = logits.double()
    total = scores.double()[:, None] + (x - torch.logsumexp(x, 1, keepdim=True))
    bad = torch.isnan(x).any(1) | (x == math.inf).any(1)
    total[bad] = -math.inf
    for r in range(x.shape[0]):
        if done is not None and done[r] != 0:
            total[r] = -math.inf
            total[r, end_token] = scores[r].double()
        if not math.isfinite(scores[r]):
            total[r] = -math.inf
    return torch.where(torch.isnan(total), torch.full_like(total, -math.inf), total)


def beam_select(total, logits, done, beams, width):
    """Groups of (row, token, total), best first, of totals as beam_totals gives them."""
    out = []
    R, V = total.shape
    keep = min(width, V)
    x = logits.double()
    for g in range(R // beams):
        found = []
        for r in range(g * beams, (g + 1) * beams):
            if done is not None and done[r] != 0:
                found += [(-total[r, t].item(), r, i, t) for i, t in enumerate((total[r] > -math.inf).nonzero()[:, 0].tolist())]
                continue
            order = torch.sort(x[r], descending=True, stable=True).indices[:keep].tolist()
            found += [(-total[r, t].item(), r, i, t) for i, t in enumerate(order)]
        best = sorted(f for f in found if f[0] < math.inf)[:width]
        out.append([(r, t, -v) for v, r, _, t in best])
    return out


# ------------------------------------------------------------------ tables
def reorder(parent, kv_len, page, num_pages, free, head, table, table_out):
    """One row after another; lists and ints in, the operator's outputs out."""
    R, max_pages = len(table), len(table[0])
    free, out = list(free), [list(row) for row in table_out]
    head = min(max(head, 0), len(free))
    n = [min(max(v, 0), max_pages * page) for v in kv_len]
    rows = [table[s][:-(-n[s] // page)] for s in range(R)]
    alive = {p for p in parent if 0 <= p < R}
    held = {p for s in alive for p in rows[s]}
    freed = []
    for s in range(R):
        for p in rows[s] if s not in alive else ():
            if 0 <= p < num_pages and p not in held and p not in freed:
                freed.append(p)
    pool = freed + free[head:]
    length, src, dst, copied = [0] * R, [-1] * R, [-1] * R, [0] * R
    seen, asked = set(), 0
    for r, s in enumerate(parent):
        if not 0 <= s < R:
            continue
        new, m = list(rows[s]), n[s] % page
        length[r] = n[s]
        if s in seen and m and 0 <= new[-1] < num_pages:
            if asked < len(pool):
                src[r], dst[r], copied[r] = new[-1], pool[asked], m
                new[-1] = pool[asked]
            else:
                length[r], new[-1] = 0, -1
            asked += 1
        seen.add(s)
        out[r][:len(new)] = new
    taken = min(asked, len(pool))
    head_out = max(0, head + taken - len(freed))
    back = freed[taken:][:head]
    free[head_out:head_out + len(back)] = back
    return out, length, src, dst, copied, free, head_out
