"""One attention layer of an autoregressive action decoder on the library's int4
weights: prompts are placed in a paged cache, then every step of a captured HIP
graph takes one new token per request through

    page plan -> qkv linear -> head norm, rotation, cache write -> paged
    attention -> out linear -> residual

with the step's lengths and free pages kept on the GPU.  Synthetic weights and
inputs.  At the end the cache and the last outputs are compared with a plain
fp32 form on the same weights.

    python examples/token_step.py [--requests 16 --hidden 2048 --heads 16 --steps 64]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_39056_amd import binding as B  # noqa: E402

PAGE, EPS = 16, 1e-6


def int32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


class Layer:
    """Weights, cache and the buffers that the captured step works on."""

    def __init__(self, requests, hidden, heads, kv_heads, capacity, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.R, self.h, self.Hq, self.Hk, self.D, self.cap = requests, hidden, heads, kv_heads, hidden // heads, capacity
        D, qkv = self.D, (heads + 2 * kv_heads) * self.D
        self.dinv = torch.rand((hidden,), generator=g, device="cuda") + 0.5
        self.w_qkv, self.w_out = (
            B.prepare_weight(torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k), d, 128)
            for n, k, d in ((qkv, hidden, 1 / self.dinv), (hidden, heads * D, None)))
        inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
        angle = torch.arange(capacity, dtype=torch.float64, device="cuda")[:, None] * inv
        self.rope = B.RopeParams(torch.randn((D,), generator=g, device="cuda") * 0.1 + 1,
                                 torch.randn((D,), generator=g, device="cuda") * 0.1 + 1, EPS,
                                 angle.cos().float().contiguous(), angle.sin().float().contiguous())
        pages = requests * (capacity // PAGE)
        shape = (pages, kv_heads, PAGE, D)
        self.kv = B.KVCache(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"),
                            torch.zeros(shape, dtype=torch.bfloat16, device="cuda"))
        self.free = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.table = int32(requests, capacity // PAGE) - 1
        self.cached, self.kv_len, self.start = int32(requests), int32(requests), int32(requests + 1)
        self.head, self.head_out = int32(1), int32(1)
        self.one = int32(requests) + 1
        self.slot, self.pos = int32(requests), int32(requests)
        self.x = torch.zeros((requests, hidden), dtype=torch.bfloat16, device="cuda")
        self.qkv = torch.empty((requests, qkv), dtype=torch.bfloat16, device="cuda")
        self.q, self.attn = (torch.empty((requests, heads, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.y = torch.empty((requests, hidden), dtype=torch.bfloat16, device="cuda")
        self.ws = B.alloc_attn_workspace(requests, heads, self.kv, capacity)

    def heads_of(self, qkv):
        q, k, v = qkv.split([self.Hq * self.D, self.Hk * self.D, self.Hk * self.D], dim=1)
        return q.unflatten(1, (-1, self.D)), k.unflatten(1, (-1, self.D)), v.unflatten(1, (-1, self.D))

    def advance(self):
        """The next call starts from this call's lengths and free pages."""
        torch.add(self.kv_len, 0, out=self.cached)
        torch.add(self.head_out, 0, out=self.head)

    def prompts(self, lengths, x):
        """Keys and values of the prompts (x [tokens, hidden], request after request) into the cache."""
        T = x.shape[0]
        new = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        slot, pos = int32(T), int32(T)
        B.sq_kv_plan(self.cached, new, PAGE, self.free, self.head, self.table, slot, pos, self.start, self.kv_len,
                     self.head_out)
        qkv = torch.empty((T, self.qkv.shape[1]), dtype=torch.bfloat16, device="cuda")
        for t in range(0, T, 64):  # (a prompt's many tokens would take sq_linear_w4a8)
            B.sq_linear_w4a16(x[t:t + 64], self.dinv, self.w_qkv, qkv[t:t + 64], B.SQ_OUT_BF16)
        q, k, v = self.heads_of(qkv)
        B.sq_qk_norm_rope(q, k, v, self.rope, pos, slot, torch.empty_like(q, memory_format=torch.contiguous_format), None,
                          self.kv)
        self.advance()

    def step(self):
        """One token per request: x becomes x + the layer's output."""
        B.sq_kv_plan(self.cached, self.one, PAGE, self.free, self.head, self.table, self.slot, self.pos, self.start,
                     self.kv_len, self.head_out)
        B.sq_linear_w4a16(self.x, self.dinv, self.w_qkv, self.qkv, B.SQ_OUT_BF16)
        q, k, v = self.heads_of(self.qkv)
        B.sq_qk_norm_rope(q, k, v, self.rope, self.pos, self.slot, self.q, None, self.kv)
        B.sq_attn_paged(self.q, self.kv, self.table, self.kv_len, self.cap, 0, 1 / math.sqrt(self.D), self.attn,
                        B.SQ_OUT_BF16, None, self.ws)
        B.sq_linear_w4a16(self.attn.view(self.R, -1), None, self.w_out, self.y, B.SQ_OUT_BF16)
        self.x.add_(self.y)
        self.advance()

    # -------------------------------------------------------------- the plain form, fp32
    def plain_weight(self, w):
        b = w.qw.view(w.N, -1, 1, 4).int()
        nib = torch.cat([b & 15, b >> 4], 2).view(w.N, w.K)
        return torch.where(nib > 7, nib - 16, nib).float() * w.w_scale.float().t().repeat_interleave(w.w_group, 1)

    def plain_heads(self, x, weight, pos):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
        c, s = self.rope.cos[pos][:, None], self.rope.sin[pos][:, None]
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1).to(torch.bfloat16)

    def plain_step(self, x, pos, history):
        """The step's output for x at positions pos, given each request's (keys, values) so far; extends them."""
        qkv = ((x.float() * self.dinv) @ self.plain_weight(self.w_qkv).t()).to(torch.bfloat16)
        q, k, v = self.heads_of(qkv)
        q, k = self.plain_heads(q, self.rope.q_weight, pos), self.plain_heads(k, self.rope.k_weight, pos)
        out = torch.empty_like(q)
        group = self.Hq // self.Hk
        for r in range(self.R):
            hk, hv = history[r]
            history[r] = hk, hv = torch.cat([hk, k[r:r + 1]]), torch.cat([hv, v[r:r + 1]])
            kk, vv = (t.float().repeat_interleave(group, 1).transpose(0, 1).contiguous() for t in (hk, hv))
            s = torch.matmul(kk, q[r].float()[:, :, None]).squeeze(2) / math.sqrt(self.D)
            out[r] = torch.matmul(torch.softmax(s, 1)[:, None, :], vv).squeeze(1).to(torch.bfloat16)
        y = (out.reshape(self.R, -1).float() @ self.plain_weight(self.w_out).t()).to(torch.bfloat16)
        return x + y

    def history(self, r, n):
        """(keys, values) [n, kv_heads, D] of request r from the cache."""
        page = self.table[r].long()[torch.arange(n, device="cuda") // PAGE]
        at = torch.arange(n, device="cuda") % PAGE
        return self.kv.k[page, :, at], self.kv.v[page, :, at]


def run(requests=16, hidden=2048, heads=16, kv_heads=None, steps=64, longest=300, seed=0):
    """Places prompts, captures the step, replays it; returns us a step and the worst error of the last
    step's output against the plain form on the cache before it, relative to the output's own size."""
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(1, longest + 1, (requests,), generator=g).tolist()
    capacity = -(-(longest + steps + 4) // PAGE) * PAGE
    L = Layer(requests, hidden, heads, kv_heads or heads, capacity, seed)
    dev = torch.Generator(device="cuda")
    dev.manual_seed(seed + 1)
    L.prompts(lengths, torch.randn((sum(lengths), hidden), generator=dev, device="cuda").to(torch.bfloat16))
    L.x.normal_(generator=dev)
    L.step()  # eagerly, before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.step()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    us = begin.elapsed_time(end) * 1e3 / steps
    n = [v + 1 + steps for v in lengths]
    assert L.cached.tolist() == n, "lengths on the GPU"
    x = L.x.clone()
    history = [L.history(r, n[r]) for r in range(requests)]
    graph.replay()
    torch.cuda.synchronize()
    want = L.plain_step(x, torch.tensor(n, device="cuda"), history)
    written = [L.history(r, n[r] + 1) for r in range(requests)]
    scale = want.float().abs().amax()
    err = ((L.x.float() - want.float()).abs().amax() / scale).item()
    cache = max(((a.float() - b.float()).abs().amax() / b.float().abs().amax()).item()
                for got, ref in zip(written, history) for a, b in zip(got, ref))
    return us, err, cache


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--requests", type=int, default=16)
    p.add_argument("--hidden", type=int, default=2048)
    p.add_argument("--heads", type=int, default=16)
    p.add_argument("--kv-heads", type=int, default=None)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--longest", type=int, default=300)
    a = p.parse_args()
    us, err, cache = run(a.requests, a.hidden, a.heads, a.kv_heads, a.steps, a.longest)
    print(f"{a.requests} requests, hidden {a.hidden}: {us:.1f} us a step (one layer, captured), "
          f"{a.requests / us * 1e6:.0f} tokens/s; last step against the plain form: output {err:.1e}, cache {cache:.1e}")


if __name__ == "__main__":
    main()
