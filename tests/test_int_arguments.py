"""Integers that do not fit the library's 32 bits are refused by the ctypes
path, which every argument that is not plain takes; its low bits would be
another, valid argument."""
import ctypes

import pytest
import torch

from paper_2609_39056_amd import binding as B

WIDE = 1 << 32


def test_arguments_past_32_bits_are_refused():
    L = B.lib()
    assert B.sq_workspace_bytes(B.SQ_VARIANT_FUSED, 88, 256, 256, 8) > 0
    for args in ((WIDE, 88, 256, 256, 8), (0, WIDE + 88, 256, 256, 8), (0, 88, 256 - WIDE, 256, 8), (0, 88, 256, 256, 8 + 3 * WIDE)):
        with pytest.raises(ctypes.ArgumentError, match="32 bits"):
            B.sq_workspace_bytes(*args)
    kv = B.sq_kv_cache(k=4096, v=4096, num_pages=10, num_heads=2, page_size=16, head_dim=64, dtype=B.SQ_OUT_BF16)
    assert L.sq_attn_workspace_bytes(1, 2, ctypes.byref(kv), 2**31 - 1) > 0
    assert L.sq_attn_workspace_bytes(1, 2, ctypes.byref(kv), -2**31) == 0
    for args in ((1 + WIDE, 2, 100), (1, 2 + WIDE, 100), (1, 2, 100 + WIDE), (1, 2, 2**31), (1, 2, -2**31 - 1)):
        with pytest.raises(ctypes.ArgumentError, match="32 bits"):
            L.sq_attn_workspace_bytes(*args[:2], ctypes.byref(kv), args[2])


@pytest.mark.gpu
def test_calls_refuse_integers_past_32_bits():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bf, i = dict(dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.int32, device="cuda")
    kv = B.KVCache(torch.zeros((4, 1, 16, 64), **bf), torch.zeros((4, 1, 16, 64), **bf))
    q, out = torch.zeros((1, 1, 64), **bf), torch.full((1, 1, 64), 7.0, **bf)
    table, n = torch.zeros((1, 4), **i), torch.full((1,), 60, **i)
    ws = B.alloc_attn_workspace(1, 1, kv, 64)
    for longest, window in ((64 + WIDE, 0), (64, 1 + WIDE), (64 - WIDE, 0)):
        with pytest.raises(ctypes.ArgumentError, match="32 bits"):
            B.sq_attn_paged(q, kv, table, n, longest, window, 1.0, out, B.SQ_OUT_BF16, None, ws)
    with pytest.raises(ctypes.ArgumentError, match="32 bits"):
        B.alloc_attn_workspace(1, 1, kv, 64 + WIDE)
    slot = torch.full((2,), 7, **i)
    with pytest.raises(ctypes.ArgumentError, match="32 bits"):
        B.sq_kv_plan(n, n, 16 + WIDE, n, None, table, slot, slot.clone(), torch.zeros((2,), **i), torch.zeros((1,), **i),
                     torch.zeros((1,), **i))
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (slot == 7).all()
