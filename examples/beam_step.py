"""Beam search with a decoder on the library's int4 weights: prompts are placed in
paged caches once and forked into beams, then every step of a captured HIP graph
takes one token per beam through

    embedding -> layers (residual norm to 8-bit codes, quantized qkv linear, page
    plan, head norm, rotation and cache write, attention over the prompt that the
    beams share, out linear) -> residual norm -> logits -> choice of continuations
    -> page tables that follow it -> copies of pages in every layer

with scores, lengths, tables and free pages kept on the GPU.  Synthetic weights.
Every step's choice is made again in plain torch operations from the step's own
logits, and the logits are compared with a plain fp32 form that attends the
history which the page tables name.

    python examples/beam_step.py [--prompts 4 --beams 4 --hidden 1024 --layers 2 --steps 16]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_39056_amd import binding as B  # noqa: E402

PAGE, EPS, END = 16, 1e-6, 2


def int32(*shape, value=0):
    return torch.full(shape, value, dtype=torch.int32, device="cuda")


class Decoder:
    """Weights, caches and the buffers that the captured step works on: request g * beams + b is beam b of prompt g."""

    def __init__(self, prompts, beams, hidden, heads, kv_heads, layers, vocab, capacity, longest, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rand(*shape, scale=1.0):
            return torch.randn(shape, generator=g, device="cuda") * scale

        self.G, self.W, self.h, self.L, self.V, self.cap = prompts, beams, hidden, layers, vocab, capacity
        self.Hq, self.Hk, self.D, self.longest = heads, kv_heads, hidden // heads, longest
        R = self.R = prompts * beams
        D, qkv = self.D, (heads + 2 * kv_heads) * self.D
        self.embed = rand(vocab, hidden).to(torch.bfloat16)
        self.layers = []
        per = capacity // PAGE
        pages = prompts * per + R * per
        for _ in range(layers):
            dinv = torch.rand((hidden,), generator=g, device="cuda") + 0.5
            w_qkv = B.prepare_weight(rand(qkv, hidden, scale=hidden ** -0.5), 1 / dinv, 128)
            w_out = B.prepare_weight(rand(hidden, heads * D, scale=(heads * D) ** -0.5), None, 128)
            kv = B.KVCache(*(torch.zeros((pages, kv_heads, PAGE, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
            self.layers.append((rand(hidden, scale=0.1) + 1, dinv, w_qkv, w_out, kv))
        self.norm = rand(hidden, scale=0.1) + 1
        self.w_vocab = B.prepare_weight(rand(-(-vocab // 64) * 64, hidden, scale=2.0 * hidden ** -0.5), None, 128)
        inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
        angle = torch.arange(capacity, dtype=torch.float64, device="cuda")[:, None] * inv
        self.rope = B.RopeParams(rand(D, scale=0.1) + 1, rand(D, scale=0.1) + 1, EPS, angle.cos().float().contiguous(),
                                 angle.sin().float().contiguous())
        # one stream with a gain of one: the plain quantized linear
        self.gamma = torch.ones((1, 1), device="cuda")
        self.num_pages = pages
        self.free = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.head, self.head_out, self.head_next = int32(1), int32(1), int32(1)
        self.table, self.table_next = int32(R, per, value=-1), int32(R, per, value=-1)
        self.cached, self.kv_len, self.len_next, self.start = int32(R), int32(R), int32(R), int32(R + 1)
        self.src, self.dst, self.rows = int32(R), int32(R), int32(R)
        self.group, self.shared = torch.arange(prompts + 1, device="cuda").to(torch.int32) * beams, int32(prompts)
        self.token, self.parent, self.done = int32(prompts, beams), int32(prompts, beams), int32(R)
        self.scores = torch.zeros(R, device="cuda")
        self.logits = torch.empty((R, self.w_vocab.N), device="cuda")
        self.live = int32(R, value=1)
        self.ws = torch.empty(max(
            B.sq_attn_shared_workspace_bytes(R, prompts, heads, self.layers[0][4], longest, capacity),
            B.sq_beam_workspace_bytes(R, beams, vocab, beams), B.sq_kv_reorder_workspace_bytes(R, pages),
            B.sq_workspace_bytes(B.SQ_VARIANT_GEMM, R, hidden, qkv, 8)), dtype=torch.uint8, device="cuda")

    def forward(self, token, table, kv, new, buffers, shared):
        """One new token per request (or a prompt's tokens) into the caches; logits of every row into self.logits.
        `kv`: lengths before and after, `shared`: whether groups share their prompts' pages."""
        T = token.shape[0]
        x = self.embed[token.long().clamp(0, self.V - 1)]
        act = B.ActParams(tok2stream=buffers["stream"], gamma=self.gamma, step=0)
        B.sq_kv_plan(kv[0], new, PAGE, self.free, self.head, table, buffers["slot"], buffers["pos"], buffers["start"], kv[1],
                     self.head_out)
        res, y = x.float(), None
        for i, (norm, dinv, w_qkv, w_out, cache) in enumerate(self.layers):
            act.dinv = dinv
            if y is None:
                B.sq_add_rmsnorm(res, None, norm, EPS, None, None, 0, act, buffers["qx"], buffers["r"])
            else:
                B.sq_add_rmsnorm(y, res, norm, EPS, res, None, 0, act, buffers["qx"], buffers["r"])
            qkv = torch.empty((T, w_qkv.N), dtype=torch.bfloat16, device="cuda")
            B.sq_gemm_w4a8(buffers["qx"], buffers["r"], w_qkv, qkv, B.SQ_OUT_BF16, None)
            q, k, v = (t.unflatten(1, (-1, self.D)) for t in qkv.split([self.Hq * self.D] + 2 * [self.Hk * self.D], 1))
            q_out = torch.empty((T, self.Hq, self.D), dtype=torch.bfloat16, device="cuda")
            B.sq_qk_norm_rope(q, k, v, self.rope, buffers["pos"], buffers["slot"], q_out, None, cache)
            if not shared:
                y = torch.zeros((T, self.h), dtype=torch.bfloat16, device="cuda")
                continue
            attn = torch.empty_like(q_out)
            B.sq_attn_shared(q_out, cache, table, kv[1], self.group, self.shared, self.longest, self.cap,
                             self.D ** -0.5, attn, B.SQ_OUT_BF16, None, self.ws)
            y = torch.empty((T, self.h), dtype=torch.bfloat16, device="cuda")
            B.sq_linear_w4a16(attn.view(T, -1), None, w_out, y, B.SQ_OUT_BF16)
        if shared:
            last = torch.empty((T, self.h), dtype=torch.bfloat16, device="cuda")
            B.sq_add_rmsnorm(y, res, self.norm, EPS, None, last, B.SQ_OUT_BF16, None, None, None)
            B.sq_linear_w4a16(last, None, self.w_vocab, self.logits, B.SQ_OUT_F32)

    def buffers(self, T):
        qx, r = B.act_buffers(T, self.h, 8)
        return dict(qx=qx, r=r, slot=int32(T), pos=int32(T), start=int32(self.R + 1), stream=int32(T))

    def follow(self):
        """Tables go on from self.parent; the caches copy what cannot be shared."""
        B.sq_kv_reorder(self.parent.view(-1), self.kv_len, PAGE, self.num_pages, self.free, self.head_out, self.table,
                        self.table_next, self.len_next, self.src, self.dst, self.rows, self.head_next, self.ws)
        B.sq_kv_copy_pages([layer[4] for layer in self.layers], self.src, self.dst, self.rows)
        # (copies by kernels: the step is captured)
        torch.add(self.table_next, 0, out=self.table)
        torch.add(self.len_next, 0, out=self.cached)
        torch.add(self.head_next, 0, out=self.head)

    def prompts(self, lengths, tokens):
        """Caches of the prompts (tokens [sum of lengths], prompt after prompt) in the rows of their first beams, then
        the fork: every beam goes on from it.  (The prompts' own attention is left out: their layers see the embeddings.)"""
        new = int32(self.R)
        new[::self.W] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.forward(tokens, self.table, (self.cached, self.kv_len), new, self.buffers(tokens.shape[0]), False)
        self.parent.copy_(self.group[:-1, None].expand(-1, self.W))
        self.follow()
        self.shared.copy_(torch.tensor([n // PAGE * PAGE for n in lengths]))
        # all beams are the prompt now: only the first may go on
        self.scores.fill_(-math.inf)
        self.scores[::self.W] = 0.0
        ends = torch.tensor(lengths, device="cuda").cumsum(0) - 1
        self.token.copy_(tokens[ends][:, None].expand(-1, self.W))
        self.step_buffers = self.buffers(self.R)

    def step(self):
        self.forward(self.token.view(-1), self.table, (self.cached, self.kv_len), self.live, self.step_buffers, True)
        B.sq_beam_select(self.logits[:, :self.V], self.W, self.scores, self.done, END, self.parent, self.token,
                         self.scores.view(self.G, self.W), self.done.view(self.G, self.W), self.ws)
        self.follow()

    # -------------------------------------------------------------- the plain form, fp32
    def plain_weight(self, w):
        b = w.qw.view(w.N, -1, 1, 4).int()
        nib = torch.cat([b & 15, b >> 4], 2).view(w.N, w.K)
        return torch.where(nib > 7, nib - 16, nib).float() * w.w_scale.float().t().repeat_interleave(w.w_group, 1)

    @staticmethod
    def plain_norm(x, w):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w

    def plain_logits(self, token, table, cached, caches):
        """Logits of one token per beam, its history read from `caches` (keys and values of every layer before the step)
        through `table`; the new keys and values are formed here."""
        x = self.embed[token.long()].float()
        pos = cached.long()
        c, s = self.rope.cos[pos][:, None], self.rope.sin[pos][:, None]

        def rotated(x, w):
            x = self.plain_norm(x, w)
            a, b = x.chunk(2, -1)
            return torch.cat([a * c - b * s, b * c + a * s], -1).to(torch.bfloat16).float()

        for (norm, dinv, w_qkv, w_out, _), (ck, cv) in zip(self.layers, caches):
            u = self.plain_norm(x, norm) * dinv
            delta = u.abs().amax(1, keepdim=True) / 127
            qkv = ((u / delta).round() * delta @ self.plain_weight(w_qkv).t()).to(torch.bfloat16).float()
            q, k, v = (t.unflatten(1, (-1, self.D)) for t in qkv.split([self.Hq * self.D] + 2 * [self.Hk * self.D], 1))
            q, k = rotated(q, self.rope.q_weight), rotated(k, self.rope.k_weight)
            out = torch.empty((self.R, self.Hq, self.D), device="cuda")
            for r in range(self.R):
                at = torch.arange(int(cached[r]), device="cuda")
                page = table[r].long()[at // PAGE]
                kk = torch.cat([ck[page, :, at % PAGE].float(), k[r:r + 1]]).repeat_interleave(self.Hq // self.Hk, 1)
                vv = torch.cat([cv[page, :, at % PAGE].float(), v[r:r + 1]]).repeat_interleave(self.Hq // self.Hk, 1)
                p = torch.softmax((kk * q[r]).sum(-1) * self.D ** -0.5, 0)
                out[r] = (p[..., None] * vv).sum(0)
            y = (out.to(torch.bfloat16).float().flatten(1) @ self.plain_weight(w_out).t()).to(torch.bfloat16).float()
            x = x + y
        last = self.plain_norm(x, self.norm).to(torch.bfloat16).float()
        return last @ self.plain_weight(self.w_vocab).t()

    def plain_choice(self, logits, scores, done):
        """(rows, tokens, totals) of the best continuations of each prompt, best first."""
        total = scores.double()[:, None] + torch.log_softmax(logits[:, :self.V].double(), 1)
        only = torch.full_like(total, -math.inf)
        only[:, END] = scores.double()
        total = torch.where(done.bool()[:, None], only, total).view(self.G, -1)
        best, at = torch.sort(total, dim=1, descending=True, stable=True)
        at, best = at[:, :self.W], best[:, :self.W]
        return at // self.V + self.group[:-1, None], at % self.V, best


def run(prompts=4, beams=4, hidden=1024, heads=8, kv_heads=2, layers=2, vocab=2000, steps=16, longest=120, seed=0, check=4):
    """Decodes; returns us a step, how often a choice differed from the plain one (by totals that are not within fp32 of
    each other), and the worst error of the last steps' logits relative to their size."""
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(1, longest + 1, (prompts,), generator=g).tolist()
    lengths[0] = longest
    capacity = -(-(longest + steps + check + 4) // PAGE) * PAGE
    d = Decoder(prompts, beams, hidden, heads, kv_heads, layers, vocab, capacity, longest, seed)
    d.prompts(lengths, torch.randint(3, vocab, (sum(lengths),), generator=g).to(torch.int32).cuda())
    d.step()  # eagerly, before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.step()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    us = begin.elapsed_time(end) * 1e3 / steps
    wrong, err = 0, 0.0
    for _ in range(check):
        token, table, cached = d.token.view(-1).clone(), d.table.clone(), d.cached.clone()
        scores, done = d.scores.clone(), d.done.clone()
        caches = [(layer[4].k.clone(), layer[4].v.clone()) for layer in d.layers]
        graph.replay()
        torch.cuda.synchronize()
        want = d.plain_logits(token, table, cached, caches)
        err = max(err, ((d.logits - want).abs().amax() / want.abs().amax()).item())
        rows, tokens, totals = d.plain_choice(d.logits, scores, done)
        wrong += int((((d.parent != rows) | (d.token != tokens)) & ((d.scores.view(d.G, d.W) - totals).abs() > 1e-5)).sum())
        pages = [row[:-(-n // PAGE)] for row, n in zip(d.table.tolist(), d.cached.tolist())]
        held, free = {p for row in pages for p in row}, d.free[int(d.head):].tolist()
        assert held.isdisjoint(free) and len(held) + len(free) == d.num_pages, "pages are held or free"
    return us, wrong, err


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("prompts", 4), ("beams", 4), ("hidden", 1024), ("heads", 8), ("kv-heads", 2), ("layers", 2),
                        ("vocab", 2000), ("steps", 16), ("longest", 120)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    us, wrong, err = run(a.prompts, a.beams, a.hidden, a.heads, a.kv_heads, a.layers, a.vocab, a.steps, a.longest)
    print(f"{a.prompts} prompts of {a.beams} beams, {a.layers} layers of hidden {a.hidden}: {us:.1f} us a step (captured); "
          f"choices unlike the plain form's: {wrong}, logits against it: {err:.1e}")


if __name__ == "__main__":
    main()
