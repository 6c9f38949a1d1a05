"""Pins of the float64 oracle of the convolution, the selective scan and the group norm: closed forms, and every
gradient against central differences of the forward."""

import numpy as np
import pytest

from oracle import layer


def _differences(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * step)
    return g


def _close(got, want):
    # a central difference of step 1e-5 is off by 1e-10 of the third derivative and 1e-11 of rounding
    assert np.max(np.abs(got - want)) <= 1e-7 * max(1.0, float(np.max(np.abs(want))))


def test_conv_closed_forms():
    x = np.arange(1.0, 7.0).reshape(1, 6, 1)
    y, final = layer.conv(x, np.array([[0.0, 0.0, 1.0]]), silu=False)  # the last tap: the token itself
    assert np.array_equal(y, x) and np.array_equal(final[0, :, 0], [5.0, 6.0])
    y, final = layer.conv(x, np.array([[1.0, 0.0, 0.0]]), silu=False, initial=np.array([[[8.0], [9.0]]]), lengths=[1])
    assert np.array_equal(y[0, :, 0], [8.0, 0, 0, 0, 0, 0]) and np.array_equal(final[0, :, 0], [9.0, 1.0])


def test_scan_closed_forms():
    T = 5
    one = np.ones((1, T, 1))
    # A = 0 counts: h_t = sum of dt x B
    y, final = layer.scan(one, 2 * one, np.zeros((1, 1)), one[..., None], one[..., None], with_softplus=False)
    assert np.array_equal(y[0, :, 0], 2.0 * np.arange(1, T + 1)) and final[0, 0, 0] == 2.0 * T
    # an initial state alone decays by exp(dt A) a token
    y, _ = layer.scan(0 * one, one, np.array([[-0.5]]), one[..., None], one[..., None], with_softplus=False,
                      initial=np.ones((1, 1, 1)))
    assert np.allclose(y[0, :, 0], np.exp(-0.5 * np.arange(1, T + 1)), rtol=1e-14)


def test_norm_closed_forms():
    x = np.array([[[1.0, 3.0, 10.0, 14.0]]])
    assert np.allclose(layer.norm(x, 2, eps=0.0, silu=False), [[[-1, 1, -1, 1]]])
    assert np.allclose(layer.norm(np.full((1, 4, 2), 7.0), 1, b=np.array([1.0, 2.0]), silu=False), [1.0, 2.0])


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("lengths", [None, [3, 1]])
def test_conv_gradients(silu, lengths):
    r = np.random.default_rng(1)
    x, w, b, i = r.standard_normal((2, 5, 2)), r.standard_normal((2, 3)), r.standard_normal(2), r.standard_normal((2, 2, 2))
    dy, df = r.standard_normal((2, 5, 2)), r.standard_normal((2, 2, 2))

    def f():
        y, final = layer.conv(x, w, b, silu, i, lengths)
        return (y * dy).sum() + (final * df).sum()

    for got, of in zip(layer.conv_grad(x, w, dy, b, silu, i, lengths, df), (x, w, b, i)):
        _close(got, _differences(f, of))


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("lengths", [None, [4, 0]])
def test_scan_gradients(softplus, gate, lengths):
    r = np.random.default_rng(2)
    B, T, D, G, N = 2, 4, 4, 2, 3
    a = {"x": r.standard_normal((B, T, D)), "dt": r.standard_normal((B, T, D)) * 0.3 + 0.5, "A": -np.exp(r.standard_normal((D, N))),
         "B": r.standard_normal((B, T, G, N)), "C": r.standard_normal((B, T, G, N)), "D": r.standard_normal(D),
         "z": r.standard_normal((B, T, D)), "dt_bias": r.standard_normal(D) * 0.1, "initial": r.standard_normal((B, D, N))}
    dy, df = r.standard_normal((B, T, D)), r.standard_normal((B, D, N))
    z = a["z"] if gate else None

    def f():
        y, final = layer.scan(a["x"], a["dt"], a["A"], a["B"], a["C"], a["D"], z, a["dt_bias"], softplus, a["initial"], lengths)
        return (y * dy).sum() + (final * df).sum()

    got = layer.scan_grad(a["x"], a["dt"], a["A"], a["B"], a["C"], dy, a["D"], z, a["dt_bias"], softplus, a["initial"], lengths, df)
    for k, v in a.items():
        if k != "z" or gate:
            _close(got[k], _differences(f, v))


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("S", [1, 3])
def test_norm_gradients(silu, gate, S):
    r = np.random.default_rng(3)
    x, w, b = r.standard_normal((2, S, 6)), r.standard_normal(6), r.standard_normal(6)
    z, dy = r.standard_normal((2, S, 6)) if gate else None, r.standard_normal((2, S, 6))

    def f():
        return (layer.norm(x, 2, w, b, z, silu=silu) * dy).sum()

    for got, of in zip(layer.norm_grad(x, 2, dy, w, b, z, silu=silu), (x, w, b, z)):
        if of is not None:
            _close(got, _differences(f, of))
