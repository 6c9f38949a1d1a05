"""The example mixer over a cache: with gradients on, a prompt has the whole graph that it has without a cache, and the
cache is brought up to its end as without gradients."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_gradients_over_a_cache():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import selective_mixer as m
    finally:
        sys.path.pop(0)
    torch.manual_seed(1)
    mixer = m.SelectiveMixer(64, dtype=torch.float32)
    h = torch.randn((2, 45, 64), device="cuda")
    n = torch.tensor([45, 30], dtype=torch.int32, device="cuda")

    def grads(cache):
        mixer.zero_grad()
        y = mixer(h, lengths=n, cache=cache)
        y.square().sum().backward()
        return y.detach(), {k: p.grad.clone() for k, p in mixer.named_parameters()}

    y, want = grads(None)
    cache = mixer.new_cache(2)
    y_cached, got = grads(cache)
    assert torch.equal(y, y_cached)
    assert set(got) == set(want)  # every parameter has one
    for k in want:
        # the same kernels on the same values: the sums of the projections' products may differ in order
        assert (got[k] - want[k]).abs().max() <= 1e-5 * want[k].abs().max(), k
    # a second pass continues the first, in the same tensors
    places = {k: t.data_ptr() for k, t in cache.items()}
    plain = mixer.new_cache(2)
    with torch.no_grad():
        mixer(h, lengths=n, cache=plain)
    for k in cache:
        assert torch.equal(cache[k], plain[k]), k
    grads(cache)
    with torch.no_grad():
        mixer(h, lengths=n, cache=plain)
    for k in cache:
        assert torch.equal(cache[k], plain[k]) and cache[k].data_ptr() == places[k], k
        assert not cache[k].requires_grad
