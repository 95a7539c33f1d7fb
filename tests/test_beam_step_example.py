"""The example of beam search runs: captured steps of all operators together
choose what plain operations choose from the same logits, logits agree with a plain
form over the history that the page tables name, and every page is held or free."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("prompts,beams,heads,kv_heads", [(3, 4, 8, 2), (1, 7, 4, 4)])
def test_example(prompts, beams, heads, kv_heads):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("beam_step", os.path.join(ROOT, "examples", "beam_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    us, wrong, err = m.run(prompts, beams, hidden=512, heads=heads, kv_heads=kv_heads, vocab=777, steps=20, longest=70)
    assert us > 0 and wrong == 0
    # Both sides round codes to 8 bits and qkv, rotated heads, attention, the layer's output and the last norm to bf16
    # (2^-8 of a value each).  A value that lies at a rounding's border may fall to either side: one unit of 2^-7 in
    # bf16, 1/127 of a row's largest in a code.  Two layers of five such roundings and the last norm, each of at most
    # the largest value.
    assert err <= (2 * 5 + 1) * 2.0 ** -7
