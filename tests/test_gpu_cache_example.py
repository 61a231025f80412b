"""The example that runs the cache operators together, against the plain 64-bit form where it ends (needs a B200)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_prompts_a_block_and_decoded_tokens_on_one_4_bit_cache():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rotated_4bit_cache.py")
    spec = importlib.util.spec_from_file_location("rotated_4bit_cache", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    block, decoded = example.run(prompts=(70, 3, 300), steps=3, decode=2)
    again = example.run(prompts=(70, 3, 300), steps=3, decode=2)
    assert block.isfinite().all() and decoded.isfinite().all()
    assert (block == again[0]).all() and (decoded == again[1]).all()
    # a cache of random values averages them: an output's size is that of a mean over the tokens it attends to
    assert 0.01 < float(decoded.float().abs().mean()) < 1.0
    assert torch.cuda.is_available()
