"""The decay attention's states over many tokens, on the GPU against float64: what a bound that grows with the tokens does
not see.

u = 2^-24, half a step of fp32.  A rounding is at most u of its value, and to either side: the mean over N elements of n
roundings each is below 6 u sqrt(n / N) but for one in 10^8, while what a factor is off by moves all of them alike."""

import numpy as np
import pytest

from oracle import layer
from tests.gpu_util import to_dev, torch_dtype

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_04761_amd  # noqa: F401  (fails loudly if the library is missing)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# 1 - g = 2^-12.5 in both; heads that remember thousands of tokens
DECAYS = np.array([np.log1p(-2.0 ** -12.5), -2.0 ** -12.5, -3e-4, -1e-4, -0.0011, -0.003, -0.0007, -5e-5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inplace", [True, False])
def test_decoding_forgets_at_the_rate_of_the_decay(inplace, dtype):
    """4096 tokens whose keys are zero: the state times g^4096, off by their roundings alone."""
    from paper_2506_04761_amd import block as ll
    import torch
    n, H, dk, dv = 4096, len(DECAYS), 64, 48
    r = np.random.default_rng(1)
    q, v = (to_dev(r.standard_normal((1, H, d)), dtype) for d in (dk, dv))
    k, ld = torch.zeros_like(q), to_dev(DECAYS)
    first = to_dev(r.standard_normal((1, H, dk, dv)))
    state, other, out = first.clone(), torch.empty_like(first), torch.empty_like(v)
    for _ in range(n // 2):
        new = None if inplace else other
        ll.ll_decay_attention_step(q, k, v, ld, state, 1.0, new, out)
        ll.ll_decay_attention_step(q, k, v, ld, state if inplace else other, 1.0, None if inplace else state, out)
    want = _np(first)[0] * np.exp(_np(ld) * n)[:, None, None]
    off = (_np(state)[0] / want - 1).reshape(H, -1)
    assert (np.abs(off) <= 2 * n * U).all()
    # two roundings a token (of lo S, which is none to speak of, and of the sum), and 2 u
    assert (np.abs(off.mean(1)) <= 2 * U + 6 * U * np.sqrt(n / off.shape[1])).all(), off.mean(1) / U
