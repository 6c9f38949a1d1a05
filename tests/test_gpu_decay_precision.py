"""The decay attention's states over many tokens, on the GPU against float64: what a bound that grows with the tokens does
not see.

u = 2^-24, half a step of fp32.  A rounding is at most u of its value, and to either side: the mean over N elements of n
roundings each is below 6 u sqrt(n / N) but for one in 10^8, while what a factor is off by moves all of them alike."""

import numpy as np
import pytest

from oracle import layer
from tests.gpu_util import to_dev
from tests.test_gpu_decay_attention import HALF, _Case

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


@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (33, 80), (128, 128), (101, 143), (128, 48), (256, 128), (200, 50)])
@pytest.mark.parametrize("T", [65, 150, 600])
def test_short_sequences_of_a_longer_batch_are_rounded_once(T, dk, dv):
    """bf16 sequences of one chunk (64 tokens) take scores and states in two parts, which leave 2^-16 of them, whatever
    stands beside them in the batch: (2 n + 64) u A for the sums, 2^-16 A for the operands, the results' own rounding."""
    ends = [1, T, 3, 64, 0, 17, 65]
    c = _Case(dk + T, len(ends), T, 2, 1, dk, dv, "bf16", ends=ends)
    h = [np.nan_to_num(_np(t)) for t in (c.q, c.k, c.v)] + [_np(c.ld)]
    d, i, f = np.nan_to_num(_np(c.d_o)), _np(c.initial), _np(c.d_final)
    mag = [np.abs(x) for x in h[:3]] + [h[3]]
    o, final, g = c.run()
    wants = [*layer.decay_attention(*h, c.scale, i, ends), *layer.decay_attention_grad(*h, d, c.scale, i, ends, f)]
    bounds = [*layer.decay_attention(*mag, c.scale, np.abs(i), ends),
              *layer.decay_attention_grad(*mag, np.abs(d), c.scale, np.abs(i), ends, np.abs(f))]
    for name, got, want, bound in zip(("o", "final", "dq", "dk", "dv", "dinitial"), (o, final, *g), wants, bounds):
        got = _np(got)
        for b, n in enumerate(ends):
            if n > 64:
                continue
            tol = (2 * n + 64) * U * bound[b]
            if name not in ("final", "dinitial"):
                tol += 2.0 ** -16 * bound[b]
                tol += HALF["bf16"] * (np.abs(want[b]) + tol)
            assert (np.abs(got[b] - want[b]) <= tol + 1e-36).all(), (name, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,B,H,dk,dv", [(16384, 1, 8, 64, 48), (16400, 1, 8, 128, 128), (8192, 50, 8, 16, 16)])
def test_prompts_forget_at_the_rate_of_the_decay(T, B, H, dk, dv, dtype):
    """Tokens whose keys are zero, in 128 segments and in one: the state times g^T.  A rounding for each chunk or segment,
    not for a factor's error in each."""
    from paper_2506_04761_amd import block as ll
    import torch
    r = np.random.default_rng(2)
    k = torch.zeros((B, T, H, dk), device="cuda", dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    v = torch.ones((B, T, H, dv), device="cuda", dtype=k.dtype)
    ld, first = to_dev(DECAYS), to_dev(r.standard_normal((B, H, dk, dv)))
    final = torch.empty_like(first)
    ll.ll_decay_attention_fwd(k, k, v, ld, 1.0, first, final)
    want = _np(first) * np.exp(_np(ld) * T)[None, :, None, None]
    off = (_np(final) / want - 1).swapaxes(0, 1).reshape(H, -1)
    steps = T // 32 + 2
    assert (np.abs(off) <= 2 * steps * U).all()
    assert (np.abs(off.mean(1)) <= 2 * U + 6 * U * np.sqrt(steps / off.shape[1])).all(), off.mean(1) / U


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(16, 24), (33, 47), (64, 128), (128, 128), (101, 143), (256, 200)])
@pytest.mark.parametrize("T", [64, 400, 640, 1100])
def test_states_of_few_tokens_keep_the_bits_of_fp32(T, dk, dv, dtype):
    """States, and gradients of states, that a few tokens make.  In u of the same sums of absolute values A: a power of the
    decay 5 (exp2's 2, its exponent of up to 1.3), the products with it, with the scale and in parts 3, their sums 3 for each
    of two tokens of a chunk, a chunk's factor 1 and a segment's 1: 24 + T / 32.  (Two parts of bf16 would leave 2^-14.)"""
    from paper_2506_04761_amd import block as ll
    import torch
    c = _Case(T + dk, 2, T, 2, 1, dk, dv, dtype, decays=[-0.003, -0.02], state=False)
    at = sorted({3 % T, 40 % T, T // 3, T // 2, T - 70 if T > 70 else 0, T - 1})
    keep = torch.zeros(T, dtype=torch.bool, device="cuda")
    keep[at] = True
    c.k = c.k.masked_fill(~keep[None, :, None, None], 0)
    c.d_o = c.d_o.masked_fill(~keep[None, :, None, None], 0)
    final = torch.empty((2, 2, dk, dv), device="cuda")
    states = ll.ll_decay_attention_states(c.q, c.v)
    a = (c.q, c.k, c.v, c.ld)
    ll.ll_decay_attention_fwd(*a, c.scale, None, final, states=states)
    g = ll.ll_decay_attention_bwd(*a, states, c.d_o, c.scale, initial_state_grad=True)
    h, d = [_np(t) for t in a], _np(c.d_o)
    mag = [np.abs(x) for x in h[:3]] + [h[3]]
    wants = layer.decay_attention(*h, c.scale)[1], layer.decay_attention_grad(*h, d, c.scale)[3]
    bounds = layer.decay_attention(*mag, c.scale)[1], layer.decay_attention_grad(*mag, np.abs(d), c.scale)[3]
    for name, got, want, bound in zip(("final", "d_initial"), (final, g.initial_state), wants, bounds):
        off = np.abs(_np(got) - want) / ((24 + T / 32) * U * bound + 1e-36)
        assert (off <= 1).all(), (name, float(off.max()))
