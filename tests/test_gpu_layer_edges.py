"""The operators around a mixer at the edges of their inputs, against the float64 oracle: sequences without a token whose
states hold NaN, axes of one token with any stride, values near the top of float32's range, arguments that are not
tensors; and second derivatives, which none of the differentiable functions has."""

import numpy as np
import pytest

from oracle import layer
from tests.test_gpu_layer import SCAN_TOL, TOL, _device, _Draw, _lengths, _np, _ok, _scan_inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,bad", [(5, float("nan")), (5, float("inf")), (70, float("nan"))])
def test_conv_gradients_without_a_token(T, bad, dtype):
    """A sequence of no token has a part in no sum, whatever its state holds (a slot of a cache that nothing has
    written); its state's gradient is the final state's."""
    import paper_2506_04761_amd as ll
    B, D, W, ns = 3, 66, 4, [T, 0, 2]
    d = _Draw(T, dtype)
    x, w, b, init, dy, df = d.rows(B, T, D), d.f32(D, W), d.f32(D), d.rows(B, W - 1, D), d.rows(B, T, D), d.rows(B, W - 1, D)
    init[1] = bad
    g = ll.ll_causal_conv_bwd(x, w, b, dy, ll.LL_ACT_SILU, init, _lengths(ns), df)
    want = layer.conv_grad(_np(x), _np(w), _np(dy), _np(b), True, _np(init), ns, _np(df))
    for got, v, name in zip(g, want, ("dx", "dweight", "dbias", "dinitial")):
        _ok(got, v, TOL[dtype] if got.dtype == x.dtype else TOL["f32"], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N", [(5, 16), (70, 7), (70, 40)])
def test_scan_gradients_without_a_token(T, N, dtype):
    """As above, with NaN in the state, in the final state's gradient, or in both."""
    import paper_2506_04761_amd as ll
    B, D, ns = 4, 36, [T, 0, 0, 0]
    d = _Draw(T + N, dtype)
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, 1, None)
    dy, df = d.rows(B, T, D), d.f32(B, D, N)
    init[1] = init[3] = float("nan")
    df[2] = df[3] = float("nan")
    states = ll.ll_selective_scan_states(x, Bm)
    ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, None, _lengths(ns), states)
    g = ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, skip, z, bias, True, _lengths(ns), df, True)
    want = layer.scan_grad(_np(x), _np(dt), _np(A), _np(Bm)[:, :, None], _np(Cm)[:, :, None], _np(dy), _np(skip), _np(z),
                           _np(bias), True, _np(init), ns, _np(df))
    for name, got in zip(("x", "dt", "A", "B", "C", "D", "z", "dt_bias"), g):
        _ok(got, want[name].reshape(got.shape), SCAN_TOL[dtype] if got.dtype == x.dtype else SCAN_TOL["f32"], "d" + name)
    assert np.array_equal(_np(g.initial_state)[1:], _np(df)[1:], equal_nan=True)
    _ok(g.initial_state[0], want["initial"][0], SCAN_TOL["f32"], "dinitial")


def test_axes_of_one_token_have_any_stride():
    """[T, 1, D] of the rows of one long sequence, turned: the stride of its single token is the sequence's size, which
    is beyond what a token stride may be."""
    import torch
    import paper_2506_04761_amd as ll
    R, D, N = 8200, 2048, 4
    d = _Draw(2, "bf16")
    x = torch.randn((1, R, D), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16().transpose(0, 1)
    assert x.shape == (R, 1, D) and x.stride(1) >= 1 << 24
    dense = x.clone(memory_format=torch.contiguous_format)
    assert dense.stride(1) == D
    w, A, bias = d.f32(D, 4), -torch.exp(d.f32(D, N)), d.f32(D)
    BC = torch.randn((1, R, (1 << 24) // R + N + 1), device="cuda").bfloat16().transpose(0, 1)[..., :N]
    assert BC.stride(1) >= 1 << 24
    stats = ll.ll_group_norm_stats(x, 16)
    results = []
    for t, bc in ((x, BC), (dense, BC.clone(memory_format=torch.contiguous_format))):
        states = ll.ll_selective_scan_states(t, bc)
        out = [ll.ll_group_norm_fwd(t, 16, gate=t, stats=stats), ll.ll_causal_conv_fwd(t, w),
               ll.ll_selective_scan_fwd(t, t, A, bc, bc, bias, t, states=states)]
        out += ll.ll_group_norm_bwd(t, 16, bias, None, stats, dense, gate=t)
        out += ll.ll_causal_conv_bwd(t, w, None, dense)
        out += ll.ll_selective_scan_bwd(t, t, A, bc, bc, states, dense, bias, t)
        results.append([o for o in out if o is not None])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("S", [1, 40])
def test_norm_of_large_values(S):
    """Means whose square is beyond float32, with a spread whose square is not.  A mean is off by a few roundings of
    2^-24 of 300 spreads, 2e-5 each."""
    import paper_2506_04761_amd as ll
    d = _Draw(S, "f32")
    x = d.rows(3, S, 64, scale=1e17) + 3e19
    y = ll.ll_group_norm_fwd(x, 8, act=ll.LL_ACT_NONE)
    _ok(y, layer.norm(_np(x), 8, silu=False), 1e-4, "y")


def test_scan_refuses_what_are_no_tensors_of_its_axes():
    import torch
    import paper_2506_04761_amd as ll
    x, A, BC = torch.zeros((2, 8, 64), device="cuda"), torch.zeros((64, 16), device="cuda"), torch.zeros((2, 8, 16), device="cuda")
    states = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    for b, c in ((None, BC), (BC, None), (BC[0, 0], BC), (BC, BC[0, 0]), (3.0, BC), (BC[0], BC[0]), (BC[:, :, None], BC)):
        with pytest.raises((TypeError, ValueError)):
            ll.ll_selective_scan_fwd(x, x, A, b, c)
        with pytest.raises((TypeError, ValueError)):
            ll.ll_selective_scan_bwd(x, x, A, b, c, states, x)
        with pytest.raises((TypeError, ValueError)):
            ll.selective_scan(x, x, A, b, c)
    for b in (None, BC[0, 0], 3.0, BC[0]):
        with pytest.raises((TypeError, ValueError)):
            ll.ll_selective_scan_workspace(x, b)
        with pytest.raises((TypeError, ValueError)):
            ll.ll_selective_scan_states(x, b)
    for w in (None, A[0], 3.0):
        with pytest.raises((TypeError, ValueError)):
            ll.ll_causal_conv_bwd_workspace(x, w)


def test_second_derivatives_are_refused():
    """The gradients are no functions that can be differentiated: an expression that would need it says so, where the
    terms through the operators would be missing from it otherwise."""
    import torch
    import paper_2506_04761_amd as ll
    d = _Draw(4, "f32")
    x, w, A, BC, n = d.f32(2, 9, 32), d.f32(32, 4), -torch.exp(d.f32(32, 8)), d.f32(2, 9, 8), d.f32(32)
    q, la, lam = d.f32(1, 32, 1, 16), -torch.rand((1, 32, 1), device="cuda"), torch.rand((1, 32, 1, ll.ll_num_levels(32)), device="cuda")
    for f, v in ((lambda t: ll.causal_conv(t, w), x), (lambda t: ll.selective_scan(t, x, A, BC, BC), x),
                 (lambda t: ll.group_norm(t, 4, n), x), (lambda t: ll.log_linear_mamba2(t, q, q, la, lam, 16), q)):
        t = v.clone().requires_grad_()
        g, = torch.autograd.grad(f(t).sum(), t, create_graph=True)
        plain, = torch.autograd.grad(f(t).sum(), t)
        assert torch.equal(g, plain)
        with pytest.raises(RuntimeError, match="second derivatives"):
            (g * t).sum().backward()
        g, = torch.autograd.grad(f(t).square().sum(), t, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            (g * t).sum().backward()
