"""The convolution, the selective scan and the group norm on the GPU against the float64 oracle: forward, gradients,
one token at a time; lengths from none to several tiles and segments, odd sizes, columns of wider rows at any start,
sequences that end early with NaN behind their ends, states continued in place.

Tolerances on max|got - want| / max|want|, set from the arithmetic (float32 throughout, one rounding at the end):
  bf16 results  2^-8 + 1e-4: a value of 8 significant bits is off by at most half a unit of the last, 2^-8 of a
                power of two, and 1e-4 is left for what comes before
  float32       conv, norm 2e-5: about ten roundings of 2^-24, in sums of up to 1e3 terms of either sign
                scan 1e-4: three roundings of 2^-24 a token, carried over at most 550 tokens"""

import numpy as np
import pytest

from oracle import layer
from tests.gpu_util import rel_err, to_dev, torch_dtype

pytestmark = pytest.mark.gpu

TOL = {"f32": 2e-5, "bf16": 2.0 ** -8 + 1e-4}
SCAN_TOL = {"f32": 1e-4, "bf16": 2.0 ** -8 + 1e-4}


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_04761_amd  # noqa: F401  (fails loudly if the library is missing)


def _np(t):
    return None if t is None else t.detach().float().cpu().numpy().astype(np.float64)


def _ok(got, want, tol, name):
    e = rel_err(_np(got), want)
    assert e <= tol, (name, e)


class _Draw:
    """Seeded inputs on the device; `dtype` rounds to storage, `off` places the columns of [B, T, D] at that start of
    wider rows."""

    def __init__(self, seed, dtype):
        self.r, self.dtype = np.random.default_rng(seed), dtype

    def rows(self, *shape, off=None, scale=1.0):
        x = to_dev(self.r.standard_normal(shape) * scale, self.dtype)
        if off is None:
            return x
        import torch
        wide = torch.full((*shape[:-1], shape[-1] + off + 3), float("nan"), device="cuda", dtype=x.dtype)
        wide[..., off:off + shape[-1]] = x
        return wide[..., off:off + shape[-1]]

    def f32(self, *shape, scale=1.0):
        return to_dev(self.r.standard_normal(shape) * scale)


def _lengths(ns):
    import torch
    return None if ns is None else torch.tensor(ns, dtype=torch.int32, device="cuda")


def _blank(ns, *tensors):
    """NaN behind the ends; returns the tensors' float64 values with zeros there for the oracle."""
    out = []
    for t in tensors:
        v = _np(t)
        if ns is not None and t is not None:
            for b, n in enumerate(ns):
                t[b, max(n, 0):] = float("nan")
        out.append(v)
    return out


# ------------------------------------------------------------------------------------ convolution

CONV = [  # B, T, D, W, lengths, start of the columns
    (1, 1, 1, 2, None, None), (2, 1, 8, 4, None, 8), (1, 2, 24, 4, None, 1), (3, 7, 65, 3, [7, 0, 1], 3),
    (2, 33, 64, 4, [2, 33], 8), (1, 150, 16, 2, None, None), (2, 41, 130, 4, None, 2), (5, 64, 520, 3, [64, 63, 3, 2, 1], 8),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("case", CONV, ids=str)
def test_conv(case, silu, dtype):
    import torch
    import paper_2506_04761_amd as ll
    B, T, D, W, ns, off = case
    d = _Draw(T * 7 + D, dtype)
    x, w, b, init = d.rows(B, T, D, off=off), d.f32(D, W), d.f32(D), d.rows(B, W - 1, D)
    dy, df = d.rows(B, T, D), d.rows(B, W - 1, D)
    xr, dyr = _blank(ns, x, dy)
    act = ll.LL_ACT_SILU if silu else ll.LL_ACT_NONE
    final = torch.empty_like(init)
    y = ll.ll_causal_conv_fwd(x, w, b, act, init, final, _lengths(ns))
    g = ll.ll_causal_conv_bwd(x, w, b, dy, act, init, _lengths(ns), df)
    wy, wf = layer.conv(xr, _np(w), _np(b), silu, _np(init), ns)
    _ok(y, wy, TOL[dtype], "y")
    assert np.array_equal(_np(final), wf)  # copies
    for got, want, name in zip(g, layer.conv_grad(xr, _np(w), dyr, _np(b), silu, _np(init), ns, _np(df)),
                               ("dx", "dweight", "dbias", "dinitial")):
        _ok(got, want, TOL[dtype] if got.dtype == x.dtype else TOL["f32"], name)
    # without the optional inputs
    y = ll.ll_causal_conv_fwd(x, w, None, act, lengths=_lengths(ns))
    _ok(y, layer.conv(xr, _np(w), None, silu, None, ns)[0], TOL[dtype], "y without bias and state")
    # the final state in place of the initial one
    y2 = ll.ll_causal_conv_fwd(x, w, b, act, init, init, _lengths(ns))
    _ok(y2, wy, TOL[dtype], "y in place")
    assert torch.equal(init, final)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("D", [1, 64, 77])
def test_conv_tokens_continue_a_prompt(D, W, dtype):
    import torch
    import paper_2506_04761_amd as ll
    B, T, P = 3, 12, 5
    d = _Draw(D + W, dtype)
    x, w, b = d.rows(B, T, D, off=1), d.f32(D, W), d.f32(D)
    whole = ll.ll_causal_conv_fwd(x, w, b)
    state = torch.empty((B, W - 1, D), dtype=x.dtype, device="cuda")
    ll.ll_causal_conv_fwd(x[:, :P], w, b, final_state=state)
    for t in range(P, T):
        if t % 2:  # in place, and into another buffer
            y = ll.ll_causal_conv_step(x[:, t], w, b, state)
        else:
            old, new = state.clone(), torch.empty_like(state)
            y = ll.ll_causal_conv_step(x[:, t], w, b, state, new_state=new)
            assert torch.equal(state, old)
            state = new
        assert torch.equal(y, whole[:, t])
    assert torch.equal(state, x[:, T - W + 1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_long_runs(dtype):
    """Enough tokens for lanes that walk several groups of four, and an end inside a run.  The parameters' sums are
    of 6322 terms, formed with at most 50 roundings of 2^-24 of sums of magnitudes, which are some 80 times the sum of
    terms of either sign: 2.4e-4."""
    import paper_2506_04761_amd as ll
    B, T, D, W, ns = 2, 4100, 1030, 4, [4100, 2222]
    d = _Draw(9, dtype)
    x, w, b, dy = d.rows(B, T, D, off=1), d.f32(D, W), d.f32(D), d.rows(B, T, D)
    xr, dyr = _blank(ns, x, dy)
    y = ll.ll_causal_conv_fwd(x, w, b, lengths=_lengths(ns))
    g = ll.ll_causal_conv_bwd(x, w, b, dy, lengths=_lengths(ns))
    _ok(y, layer.conv(xr, _np(w), _np(b), True, None, ns)[0], TOL[dtype], "y")
    want = layer.conv_grad(xr, _np(w), dyr, _np(b), True, None, ns, None)
    _ok(g[0], want[0], TOL[dtype], "dx")
    _ok(g[1], want[1], 2.4e-4, "dweight")
    _ok(g[2], want[2], 2.4e-4, "dbias")


# ------------------------------------------------------------------------------------ selective scan

SCAN = [  # B, T, D, N, groups, lengths, start of the columns
    (1, 1, 1, 1, 1, None, None), (2, 1, 16, 16, 1, [1, 0], None), (1, 7, 20, 16, 1, None, 4), (2, 16, 64, 16, 1, None, 8),
    (3, 37, 65, 7, 1, [37, 0, 16], 1), (2, 70, 96, 16, 3, [1, 70], 4), (1, 130, 40, 24, 2, None, 3), (2, 81, 36, 33, 1, [81, 64], 4),
    (1, 72, 130, 64, 1, None, 2), (2, 550, 132, 16, 1, [550, 300], 4), (1, 540, 34, 20, 1, None, None),
]


def _scan_inputs(d, B, T, D, N, G, off):
    import torch
    x, dt, z = d.rows(B, T, D, off=off), d.rows(B, T, D, off=off, scale=0.5), d.rows(B, T, D, off=off)
    BC = d.rows(B, T, 2 * G * N + 5)
    Bm, Cm = (BC[..., 5 + i * G * N:5 + (i + 1) * G * N].unflatten(-1, (G, N)) for i in (0, 1))
    if G == 1:
        Bm, Cm = Bm[..., 0, :], Cm[..., 0, :]
    A = -torch.exp(d.f32(D, N))
    return x, dt, z, Bm, Cm, A, d.f32(D), d.f32(D, scale=0.5) - 1.0, d.f32(B, D, N)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan(case, gate, dtype):
    import torch
    import paper_2506_04761_amd as ll
    B, T, D, N, G, ns, off = case
    d = _Draw(T * 11 + D + N, dtype)
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, G, off)
    dy, df = d.rows(B, T, D), d.f32(B, D, N)
    xr, dtr, zr, Br, Cr, dyr = _blank(ns, x, dt, z, Bm, Cm, dy)
    Br, Cr = Br.reshape(B, T, G, N), Cr.reshape(B, T, G, N)
    if not gate:
        z = zr = None
    tol = SCAN_TOL[dtype]
    final = torch.empty_like(init)
    states = ll.ll_selective_scan_states(x, Bm)
    y = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, final, _lengths(ns), states)
    g = ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, skip, z, bias, True, _lengths(ns), df, True)
    wy, wf = layer.scan(xr, dtr, _np(A), Br, Cr, _np(skip), zr, _np(bias), True, _np(init), ns)
    want = layer.scan_grad(xr, dtr, _np(A), Br, Cr, dyr, _np(skip), zr, _np(bias), True, _np(init), ns, _np(df))
    _ok(y, wy, tol, "y")
    _ok(final, wf, SCAN_TOL["f32"], "final state")
    for name, got in zip(("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "initial"), g):
        if got is None:
            assert name == "z" and not gate
            continue
        _ok(got, want[name].reshape(got.shape), tol if got.dtype == x.dtype else SCAN_TOL["f32"], "d" + name)
    if ns is not None:  # nothing behind the ends
        for b, n in enumerate(ns):
            for t in (y, g.x, g.dt, g.B, g.C) + ((g.z,) if gate else ()):
                assert not t[b, n:].any()
    # the final state in place of the initial one; without the states for a backward
    y2 = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, init, _lengths(ns))
    assert torch.equal(y2, y) and torch.equal(init, final)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,D,N", [(1, 4300, 20, 16), (2, 300, 1100, 16), (1, 4200, 9, 24)])
def test_scan_in_many_segments(B, T, D, N, dtype):
    """Few channels (hundreds of segments a channel, joined in runs) and many (joined in one).  Three roundings of 2^-24
    a token, carried over at most T tokens."""
    import paper_2506_04761_amd as ll
    d = _Draw(T + D, dtype)
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, 1, None)
    dy, df = d.rows(B, T, D), d.f32(B, D, N)
    carried = max(1e-4, 3 * T * 2.0 ** -24)
    tol = {"f32": carried, "bf16": 2.0 ** -8 + carried}
    final, states = init.clone(), ll.ll_selective_scan_states(x, Bm)
    y = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, final, None, states)
    g = ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, skip, z, bias, True, None, df, True)
    args = (_np(x), _np(dt), _np(A), _np(Bm)[:, :, None], _np(Cm)[:, :, None])
    wy, wf = layer.scan(*args, _np(skip), _np(z), _np(bias), True, _np(init), None)
    want = layer.scan_grad(*args, _np(dy), _np(skip), _np(z), _np(bias), True, _np(init), None, _np(df))
    _ok(y, wy, tol[dtype], "y")
    _ok(final, wf, tol["f32"], "final state")
    for name, got in zip(("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "initial"), g):
        _ok(got, want[name].reshape(got.shape), tol[dtype] if got.dtype == x.dtype else tol["f32"], "d" + name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [5, 300])
def test_scan_without_options(T, dtype):
    """No skip, gate, bias, softplus, initial or final state, length or wanted sum."""
    import paper_2506_04761_amd as ll
    B, D, N = 2, 48, 16
    d = _Draw(T, dtype)
    x, dt, _, Bm, Cm, A, _, _, _ = _scan_inputs(d, B, T, D, N, 1, None)
    dt = dt.abs()
    dy = d.rows(B, T, D)
    states = ll.ll_selective_scan_states(x, Bm)
    y = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, delta_softplus=False, states=states)
    g = ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, delta_softplus=False)
    Br, Cr = _np(Bm)[:, :, None], _np(Cm)[:, :, None]
    _ok(y, layer.scan(_np(x), _np(dt), _np(A), Br, Cr, with_softplus=False)[0], SCAN_TOL[dtype], "y")
    want = layer.scan_grad(_np(x), _np(dt), _np(A), Br, Cr, _np(dy), with_softplus=False)
    for name in ("x", "dt", "A", "B", "C"):
        got = getattr(g, name)
        _ok(got, want[name].reshape(got.shape), SCAN_TOL[dtype] if got.dtype == x.dtype else SCAN_TOL["f32"], "d" + name)
    assert g.D is None and g.z is None and g.dt_bias is None and g.initial_state is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,N,G", [(1, 1, 1), (64, 16, 1), (70, 16, 2), (33, 23, 1), (24, 64, 3)])
def test_scan_tokens_continue_a_prompt(D, N, G, dtype):
    import torch
    import paper_2506_04761_amd as ll
    B, T, P = 2, 9, 4
    d = _Draw(D + N, dtype)
    x, dt, z, Bm, Cm, A, skip, bias, state = _scan_inputs(d, B, T, D, N, G, 1)
    Br, Cr = _np(Bm).reshape(B, T, G, N), _np(Cm).reshape(B, T, G, N)
    want, wf = layer.scan(_np(x), _np(dt), _np(A), Br, Cr, _np(skip), _np(z), _np(bias), True, _np(state))
    more = {"D": skip, "z": z, "dt_bias": bias}
    first = {**more, "z": z[:, :P]}
    ll.ll_selective_scan_fwd(x[:, :P], dt[:, :P], A, Bm[:, :P], Cm[:, :P], **first, initial_state=state, final_state=state)
    got = []
    for t in range(P, T):
        more["z"] = z[:, t]
        old, new = state.clone(), torch.empty_like(state)
        y = ll.ll_selective_scan_step(x[:, t], dt[:, t], A, Bm[:, t], Cm[:, t], state, **more, new_state=new)
        assert torch.equal(state, old)
        y2 = ll.ll_selective_scan_step(x[:, t], dt[:, t], A, Bm[:, t], Cm[:, t], state, **more)  # in place
        assert torch.equal(state, new) and torch.equal(y, y2)
        got.append(y)
    _ok(torch.stack(got, 1), want[:, P:], SCAN_TOL[dtype], "y")
    _ok(state, wf, SCAN_TOL["f32"], "state")


def test_scan_step_sizes_of_any_size():
    """softplus far below and above zero, and rates that forget a state within a token."""
    import paper_2506_04761_amd as ll
    B, T, D, N = 1, 64, 16, 16
    d = _Draw(3, "f32")
    x, _, z, Bm, Cm, A, skip, _, _ = _scan_inputs(d, B, T, D, N, 1, None)
    v = np.concatenate([np.linspace(-110, -30, 20), np.linspace(-30, 30, 30), [1e3, 3e4, 0.0, -0.0], np.linspace(-1e-3, 1e-3, 10)])
    dt = to_dev(np.broadcast_to(v[None, :, None], (B, T, D)))
    y = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z)
    want = layer.scan(_np(x), _np(dt), _np(A), _np(Bm)[:, :, None], _np(Cm)[:, :, None], _np(skip), _np(z))[0]
    for t in range(T):  # token by token: step sizes span many orders of magnitude
        _ok(y[:, t], want[:, t], SCAN_TOL["f32"], t)


# ------------------------------------------------------------------------------------ group norm

NORM = [  # N, S, C, groups, start of the columns
    (1, 1, 1, 1, None), (5, 1, 64, 4, None), (3, 1, 24, 3, 1), (7, 1, 96, 1, 8), (300, 1, 2048, 16, 8), (9, 1, 257, 1, 3),
    (4, 1, 4112, 1, 8), (3, 1, 1285, 5, None), (2, 1, 9000, 1, None), (2, 1, 5000, 1, 1), (2, 3, 40, 5, 8), (3, 130, 80, 1, 8),
    (2, 50, 64, 4, 1), (1, 333, 771, 3, None), (4, 64, 1024, 32, 8), (1, 2000, 8, 1, None),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("silu,gate", [(True, False), (True, True), (False, True), (False, False)])
@pytest.mark.parametrize("case", NORM, ids=str)
def test_norm(case, silu, gate, dtype):
    import paper_2506_04761_amd as ll
    N, S, C, G, off = case
    d = _Draw(S * 5 + C, dtype)
    x, w, b = d.rows(N, S, C, off=off, scale=2.0), d.f32(C) + 1.0, d.f32(C)
    z, dy = d.rows(N, S, C, off=off) if gate else None, d.rows(N, S, C)
    act = ll.LL_ACT_SILU if silu else ll.LL_ACT_NONE
    stats = ll.ll_group_norm_stats(x, G)
    y = ll.ll_group_norm_fwd(x, G, w, b, z, 1e-5, act, stats)
    g = ll.ll_group_norm_bwd(x, G, w, b, stats, dy, z, act)
    _ok(y, layer.norm(_np(x), G, _np(w), _np(b), _np(z), silu=silu), TOL[dtype], "y")
    want = layer.norm_grad(_np(x), G, _np(dy), _np(w), _np(b), _np(z), silu=silu)
    for got, v, name in zip(g, want, ("dx", "dweight", "dbias", "dgate")):
        if v is None:
            assert got is None
        elif C == G and name in ("dx", "dweight"):  # a group of one value is its mean: nothing is left of it
            assert not got.any()
        else:
            _ok(got, v, TOL[dtype] if got.dtype == x.dtype else TOL["f32"], name)
    y = ll.ll_group_norm_fwd(x, G, None, None, z, 1e-5, act)
    if C != G:
        _ok(y, layer.norm(_np(x), G, None, None, _np(z), silu=silu), TOL[dtype], "y without weight and bias")


@pytest.mark.parametrize("S", [1, 200])
def test_norm_keeps_its_precision_at_a_large_mean(S):
    """Values of spread 1 around 1000: their float32 storage keeps 3e-5 of the spread, sums of squares would keep 0.1."""
    import paper_2506_04761_amd as ll
    d = _Draw(S, "f32")
    x = d.rows(3, S, 512) + 1000.0
    y = ll.ll_group_norm_fwd(x, 8, act=ll.LL_ACT_NONE)
    # the mean is off by at most 2^-24 of 1000, 6e-5 of the spread, the largest value is about 4
    _ok(y, layer.norm(_np(x), 8, silu=False), 6e-5, "y")


# ------------------------------------------------------------------------------------ together

def _directional(f, tensors, grads, seed):
    """A central difference of f along a random direction against the gradients' product with it."""
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    vs = [torch.randn(t.shape, generator=g, device="cuda") for t in tensors]
    step = 1e-2
    with torch.no_grad():
        up = f(*[t + step * v for t, v in zip(tensors, vs)])
        down = f(*[t - step * v for t, v in zip(tensors, vs)])
    along = sum((a.double() * v.double()).sum() for a, v in zip(grads, vs)).item()
    scale = sum(((a.double() * v.double()) ** 2).sum() for a, v in zip(grads, vs)).sqrt().item()
    # third derivatives leave some 1e-4 of the terms' size, sums in float32 1e-3 of a step's difference
    assert abs((up - down) / (2 * step) - along) <= 5e-3 * max(scale, abs(along)), ((up - down) / (2 * step), along, scale)


def test_functions_are_differentiable():
    import torch
    import paper_2506_04761_amd as ll
    d = _Draw(5, "f32")
    B, T, D, N = 2, 100, 32, 8
    c, s0 = d.f32(B, T, D), d.f32(B, D, N)
    conv = [d.f32(B, T, D), d.f32(D, 4), d.f32(D), d.f32(B, 3, D)]
    scan = [d.f32(B, T, D), d.f32(B, T, D, scale=0.3), -torch.exp(d.f32(D, N, scale=0.3)), d.f32(B, T, N), d.f32(B, T, N),
            d.f32(D), d.f32(B, T, D), d.f32(D, scale=0.3) - 2.0, s0]
    norm = [d.f32(B, T, D), d.f32(D) + 1.0, d.f32(D), d.f32(B, T, D)]
    cs, cf = d.f32(B, 3, D), d.f32(B, D, N)

    def f_conv(x, w, b, i):
        y, final = ll.causal_conv(x, w, b, initial_state=i, return_final_state=True)
        return (y.double() * c).sum() + (final.double() * cs).sum()

    def f_scan(x, dt, A, Bm, Cm, D_, z, bias, h):
        y, final = ll.selective_scan(x, dt, A, Bm, Cm, D_, z, bias, initial_state=h, return_final_state=True)
        return (y.double() * c).sum() + (final.double() * cf).sum()

    def f_norm(x, w, b, z):
        return (ll.group_norm(x, 4, w, b, z).double() * c).sum()

    for f, args in ((f_conv, conv), (f_scan, scan), (f_norm, norm)):
        leaves = [t.clone().requires_grad_() for t in args]
        f(*leaves).backward()
        for k in range(3):
            _directional(lambda *a: f(*a).item(), args, [t.grad for t in leaves], k)


def test_repeats_are_bit_equal():
    import torch
    import paper_2506_04761_amd as ll
    d = _Draw(9, "bf16")
    B, T, D, N = 2, 700, 272, 16
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, 1, 4)
    dy, w, b = d.rows(B, T, D), d.f32(D, 4), d.f32(D)

    def run():
        states, stats = ll.ll_selective_scan_states(x, Bm), ll.ll_group_norm_stats(x, 17)
        out = [ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, None, None, states)]
        out += ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, skip, z, bias)[:8]
        out += ll.ll_causal_conv_bwd(x, w, b, dy)[:3]
        out.append(ll.ll_group_norm_fwd(x, 17, skip, bias, z, stats=stats))
        return out + list(ll.ll_group_norm_bwd(x, 17, skip, bias, stats, dy, z))

    first = run()
    for _ in range(3):
        for u, v in zip(first, run()):
            assert torch.equal(u, v)


def test_other_streams_and_graphs():
    """Work on a stream of the caller's, and replays of a captured graph with eager work in between."""
    import torch
    import paper_2506_04761_amd as ll
    d = _Draw(10, "bf16")
    B, T, D, N = 1, 600, 128, 16
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, 1, None)
    w, dy = d.f32(D, 4), d.rows(B, T, D)
    u = torch.empty_like(x)
    states, stats = ll.ll_selective_scan_states(x, Bm), ll.ll_group_norm_stats(x, 8)
    ws = [ll.ll_selective_scan_workspace(x, Bm), ll.ll_selective_scan_workspace(x, Bm, True),
          ll.ll_group_norm_workspace(x, 8), ll.ll_causal_conv_bwd_workspace(x, w)]
    v, y = torch.empty_like(x), torch.empty_like(x)
    gs = ll.ScanGrads(*(torch.empty_like(t) for t in (x, dt, A, Bm.contiguous(), Cm.contiguous(), skip, x, bias)), None)
    gc = ll.ConvGrads(torch.empty_like(x), torch.empty_like(w), None, None)

    def run(stream=None):
        ll.ll_causal_conv_fwd(x, w, out=u, stream=stream)
        ll.ll_selective_scan_fwd(u, dt, A, Bm, Cm, skip, z, bias, states=states, out=v, workspace=ws[0], stream=stream)
        ll.ll_group_norm_fwd(v, 8, stats=stats, out=y, workspace=ws[2], stream=stream)
        ll.ll_selective_scan_bwd(u, dt, A, Bm, Cm, states, dy, skip, z, bias, grads=gs, workspace=ws[1], stream=stream)
        ll.ll_causal_conv_bwd(x, w, None, gs.x, grads=gc, workspace=ws[3], stream=stream)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (y, *gs[:8], *gc[:2])]

    run()
    want = results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y.zero_()
    torch.cuda.synchronize()
    run(side)
    for a, b in zip(results(), want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(4):
        x.copy_(torch.roll(x, 1, 1))
        graph.replay()
        got = results()
        run()
        for a, b in zip(got, results()):
            assert torch.equal(a, b), k


def test_offsets_beyond_32_bits():
    """More than 2^31 elements: the end of one long call against a call of the end alone."""
    import torch
    import paper_2506_04761_amd as ll
    T, D, N, E = (1 << 20) + 37, 2080, 8, 4096
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.empty((1, T, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.randn((D, 4), generator=g, device="cuda")
    end = slice(T - E, T)
    y = ll.ll_causal_conv_fwd(x, w)
    assert x.numel() > 1 << 31
    assert torch.equal(y[:, end], ll.ll_causal_conv_fwd(x[:, end].contiguous(), w, initial_state=x[:, T - E - 3:T - E].contiguous()))
    del y
    y = ll.ll_group_norm_fwd(x.view(T, 1, D), 13)
    assert torch.equal(y[end], ll.ll_group_norm_fwd(x.view(T, 1, D)[end].contiguous(), 13))
    del y
    # rates of at least 0.69 a token: the state 4096 tokens back has no part in the last 2048 tokens
    A = -torch.ones((D, N), device="cuda")
    BC = torch.randn((1, T, 2 * N), generator=g, device="cuda").bfloat16()
    dt = torch.zeros((1, 1, D), dtype=torch.bfloat16, device="cuda").expand(1, T, D)  # a token stride of zero
    y = ll.ll_selective_scan_fwd(x, dt, A, BC[..., :N], BC[..., N:], z=x)
    part = ll.ll_selective_scan_fwd(x[:, end].contiguous(), dt[:, :E], A, BC[:, end, :N], BC[:, end, N:], z=x[:, end])
    assert rel_err(_np(y[:, T - 2048:]), _np(part[:, E - 2048:])) <= 2.0 ** -8  # one unit of the last place


def test_refusals_on_the_device():
    import torch
    import paper_2506_04761_amd as ll
    x = torch.zeros((2, 8, 64), device="cuda")
    w, A, BC = torch.zeros((64, 4), device="cuda"), torch.zeros((64, 16), device="cuda"), torch.zeros((2, 8, 16), device="cuda")
    bad = [
        lambda: ll.ll_causal_conv_fwd(x, w.double()), lambda: ll.ll_causal_conv_fwd(x, w[:32]),
        lambda: ll.ll_causal_conv_fwd(x.transpose(1, 2), torch.zeros((8, 4), device="cuda")),
        lambda: ll.ll_causal_conv_fwd(x.half(), w), lambda: ll.ll_causal_conv_fwd(x, torch.zeros((64, 9), device="cuda")),
        lambda: ll.ll_causal_conv_fwd(x, w, lengths=torch.tensor([1, 2], device="cuda")),
        lambda: ll.ll_causal_conv_step(x[:, 0], w, None, torch.zeros((2, 2, 64), device="cuda")),
        lambda: ll.ll_selective_scan_fwd(x, x[:, :4], A, BC, BC), lambda: ll.ll_selective_scan_fwd(x, x, A[:, :3], BC, BC),
        lambda: ll.ll_selective_scan_fwd(x, x, A, BC.bfloat16(), BC),
        lambda: ll.ll_selective_scan_fwd(x, x, torch.zeros((64, 65), device="cuda"), *[torch.zeros((2, 8, 65), device="cuda")] * 2),
        lambda: ll.ll_selective_scan_fwd(x, x, A, *[torch.zeros((2, 8, 5, 16), device="cuda")] * 2),
        lambda: ll.ll_selective_scan_bwd(x, x, A, BC, BC, torch.empty(8, dtype=torch.uint8, device="cuda"), x),
        lambda: ll.ll_group_norm_fwd(x, 5), lambda: ll.ll_group_norm_fwd(x, 4, gate=x[:1]), lambda: ll.ll_group_norm_fwd(x[0], 4),
        lambda: ll.ll_group_norm_fwd(x, 4, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
    ]
    for f in bad:
        with pytest.raises((TypeError, ValueError, ll.LLError)):
            f()
