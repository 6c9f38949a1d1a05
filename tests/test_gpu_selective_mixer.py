"""The example mixer: it trains, and decoding token by token continues prompts of several lengths as one pass does."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_trains_and_decodes():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import selective_mixer as m
    finally:
        sys.path.pop(0)
    torch.manual_seed(0)
    mixer = m.SelectiveMixer(128)
    losses = m.train(mixer, steps=12)
    assert all(map(lambda v: v == v, losses)) and losses[-1] < 0.9 * losses[0], losses
    # the projections round to bf16 after sums whose order differs between one token and many: a few 2^-9 of an output
    assert m.decode_error(mixer) <= 2e-2
    exact = m.SelectiveMixer(64, dtype=torch.float32)
    assert m.decode_error(exact) <= 1e-4
