"""The calls that README prints go through the binding as they stand: its own checks of
types and sizes, with host tensors in the place of device tensors and nothing launched."""
import os
import re
from collections import defaultdict

import pytest
import torch

from paper_2609_39056_amd import _build
from paper_2609_39056_amd import binding as B

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


class Library:
    """Notes what is called and takes it; sizes of workspaces are the library's own."""

    def __init__(self, real):
        self.real, self.called, self.sq_address = real, [], defaultdict(int)

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)

        def call(*args):
            self.called.append(name)
            return B.SQ_OK

        return call


@pytest.fixture
def library(monkeypatch):
    if not os.path.exists(B.LIB_PATH):
        _build.build()
    stub = Library(B.lib())
    monkeypatch.setattr(B, "_lib", stub)
    monkeypatch.setattr(B, "_call", B._NoCall())
    monkeypatch.setattr(B, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    return stub


def block(heading):
    """The first indented block with calls under a heading."""
    if not os.path.exists(README):
        pytest.skip("no README here")
    text = open(README).read().split(f"## {heading}\n", 1)[1].split("\n## ")[0]
    return next(b for b in re.findall(r"(?:^    .*\n|^\n)+", text, re.M) if "B.sq_" in b)


def run(code, names):
    exec("\n".join(line[4:] for line in code.splitlines()), names)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def common():
    R, heads, kv_heads, head_dim, page, num_pages, max_pages, K = 6, 4, 2, 64, 16, 40, 5, 256
    bf16 = torch.bfloat16
    pages = [torch.zeros((num_pages, kv_heads, page, head_dim), dtype=bf16) for _ in range(2)]
    return dict(B=B, R=R, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, num_pages=num_pages, eps=1e-6,
                k_pages=pages[0], v_pages=pages[1], kv=B.KVCache(*pages), kv_len=ints(R), free=ints(num_pages), head=ints(1),
                head_out=ints(1), table=ints(R, max_pages), q_out=torch.zeros((R, heads, head_dim), dtype=bf16),
                attn=torch.zeros((R, heads, head_dim), dtype=bf16), K=K, bf16=bf16)


def test_token_step(library):
    n = common()
    R, K, rows = n["R"], n["K"], (n["heads"] + 2 * n["kv_heads"]) * n["head_dim"]

    def weight(N, K):
        return B.Weight(torch.zeros((N, K // 2), dtype=torch.uint8), torch.zeros((K // 128, N), dtype=torch.float16), 128)

    n.update(q_weight=torch.ones(64), k_weight=torch.ones(64), cos=torch.ones(100, 32), sin=torch.ones(100, 32), capacity=80,
             cached=ints(R), new=ints(R), slot=ints(R), pos=ints(R), token_start=ints(R + 1), x=torch.zeros((R, K), dtype=n["bf16"]),
             dinv=torch.ones(K), W_qkv=weight(rows, K), W_out=weight(K, K), qkv=torch.zeros((R, rows), dtype=n["bf16"]),
             y=torch.zeros((R, K), dtype=n["bf16"]))
    run(block("A decoder's token step"), n)
    assert library.called == ["sq_kv_plan", "sq_linear_w4a16", "sq_qk_norm_rope", "sq_attn_paged", "sq_linear_w4a16"]


def test_several_continuations(library):
    n = common()
    R, K, beams, V = n["R"], n["K"], 3, 104
    n.update(x=torch.zeros((R, K), dtype=n["bf16"]), h=torch.zeros(R, K), w=torch.ones(K), qx=torch.zeros((R, K), dtype=torch.int8),
             r=torch.zeros(R), act=B.ActParams(tok2stream=ints(R), gamma=torch.ones(1, 1), step=0, act_bits=8),
             ws=torch.zeros(256, dtype=torch.uint8), beam_ws=torch.zeros(256, dtype=torch.uint8),
             reorder_ws=torch.zeros(256, dtype=torch.uint8), group_start=ints(R // beams + 1), shared_len=ints(R // beams),
             shared_cap=32, own_cap=32, beams=beams, logits=torch.zeros(R, V), scores=torch.zeros(R), done=ints(R), end_token=2,
             parent=ints(R // beams, beams), token=ints(R // beams, beams), table_out=ints(R, 5),
             kv_len_out=ints(R), src=ints(R), dst=ints(R), rows=ints(R), caches=[n["kv"], n["kv"]])
    run(block("Several continuations of a prompt"), n)
    assert library.called == ["sq_add_rmsnorm", "sq_attn_shared", "sq_beam_select", "sq_kv_reorder", "sq_kv_copy_pages"]
