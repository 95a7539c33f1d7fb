"""The example of the token step runs, and its captured steps give what the
plain fp32 form gives."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads", [(10, 10), (10, 2)])
def test_example(heads, kv_heads):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("token_step", os.path.join(ROOT, "examples", "token_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    us, err, cache = m.run(requests=5, hidden=1280, heads=heads, kv_heads=kv_heads, steps=20, longest=70)
    # both sides round qkv, rotated heads, attention and output to bf16 (2^-8 of a value each) and may differ by one
    # unit where the fp32 sums before a rounding differ; four roundings in a chain, each of at most the largest value
    assert err <= 4 * 2.0 ** -7 and cache <= 2 * 2.0 ** -7
    assert us > 0
