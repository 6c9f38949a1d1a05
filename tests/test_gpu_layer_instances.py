"""The operators around a mixer at the sizes that training and wide layers have, against the float64 oracle: every
instance of the norm's and the scan's kernels, loops of more than one round, segments of several chunks, and backward
passes beyond 2^31 elements.

Tolerances on max|got - want| / max|want|.  Outputs: as in tests/test_gpu_layer.py.  Sums over rows (dweight, dbias of a
norm): a chain of at most 1400 additions, each rounded to 2^-24 of a partial sum no larger than the largest total, 8e-5,
and as much again for the terms: 2.4e-4 in all.  The scan: three roundings of 2^-24 a token, carried over at most T."""

import numpy as np
import pytest

from oracle import layer
from tests.gpu_util import rel_err
from tests.test_gpu_layer import TOL, _device, _Draw, _lengths, _np, _ok, _scan_inputs  # noqa: F401

pytestmark = pytest.mark.gpu

SUM_TOL = 2.4e-4


# ------------------------------------------------------------------------------------ norm of single tokens

def _norm_case(N, C, G, dtype, gate, silu=True, off=None):
    import paper_2506_04761_amd as ll
    d = _Draw(N + C, dtype)
    x, w, b = d.rows(N, 1, C, off=off, scale=2.0), d.f32(C) + 1.0, d.f32(C)
    z, dy = d.rows(N, 1, C, off=off) if gate else None, d.rows(N, 1, C)
    act = ll.LL_ACT_SILU if silu else ll.LL_ACT_NONE
    stats = ll.ll_group_norm_stats(x, G)
    y = ll.ll_group_norm_fwd(x, G, w, b, z, 1e-5, act, stats)
    g = ll.ll_group_norm_bwd(x, G, w, b, stats, dy, z, act)
    _ok(y, layer.norm(_np(x), G, _np(w), _np(b), _np(z), silu=silu), TOL[dtype], "y")
    want = layer.norm_grad(_np(x), G, _np(dy), _np(w), _np(b), _np(z), silu=silu)
    for got, v, name in zip(g, want, ("dx", "dweight", "dbias", "dgate")):
        if v is not None:
            _ok(got, v, TOL[dtype] if got.dtype == x.dtype else SUM_TOL, name)


# channels of a group -> lanes x vectors of the forward and the backward, bf16: 300 64x1 64x2, 512 64x1 64x2, 600 64x2 64x4,
# 1024 64x2 64x4, 1025 64x4 256x2, 2047 64x4 256x2, 2048 the same, 2100 and 4096 256x2 256x4, 5001 and 8192 256x4 both;
# float32: 200 64x1 64x2, 300 64x2 64x4, 600 and 1000 64x4 256x2, 1025 and 2048 256x2 256x4, 2100 and 4096 256x4 both, 5001
# and 8192 as sequences of one token
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("cg", [200, 300, 512, 600, 1000, 1024, 1025, 2047, 2048, 2100, 4096, 5001, 8192])
def test_norm_of_wide_groups(cg, gate, dtype):
    _norm_case(5, cg, 1, dtype, gate)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G,cg,off", [(4, 1024, 8), (2, 2048, 8), (5, 700, 4), (3, 1501, 1), (2, 4097, 3)])
def test_norm_of_several_wide_groups(G, cg, off, dtype):
    """Rows that take several workgroups, at any start."""
    _norm_case(7, G * cg, G, dtype, cg % 2 == 1, off=off)


# a round of the backward is 2048 rows of workgroups of 256 lanes, 1024 of 512 lanes, 86016 of 6 (bf16; 43008 of 12 in float32)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("N,C,G", [(2500, 2048, 16), (2100, 4112, 1), (4200, 1500, 1), (2300, 768, 1), (100000, 15, 3),
                                   (2049, 257, 1), (3000, 520, 4)])
def test_norm_of_more_rows_than_a_round(N, C, G, gate, dtype):
    _norm_case(N, C, G, dtype, gate)


def test_norm_forward_of_more_rows_than_two_rounds():
    """16384 workgroups of one row of four groups of 257 channels (64 lanes each)."""
    import paper_2506_04761_amd as ll
    N, C, G = 40000, 1028, 4
    d = _Draw(7, "bf16")
    x, z, w, b = d.rows(N, 1, C), d.rows(N, 1, C), d.f32(C), d.f32(C)
    y = ll.ll_group_norm_fwd(x, G, w, b, z)
    for part in (slice(0, N, 97), slice(16384 - 40, 16384 + 40), slice(2 * 16384 - 40, 2 * 16384 + 40), slice(N - 200, N)):
        _ok(y[part], layer.norm(_np(x[part]), G, _np(w), _np(b), _np(z[part])), TOL["bf16"], part)


# ------------------------------------------------------------------------------------ scan

def _up(a, b):
    return -(-a // b)


def _bwd_split(B, T, D, N, G):
    """Tokens of a segment and of a fine one, fine segments of a segment, chunks of a segment, and the workspace's bytes:
    the rule by which the backward splits the length."""
    NP = 16 if N <= 16 else (32 if N <= 32 else 64)
    waves, rev = _up(D // G, 32), B * G * _up(D // G, 64)
    blocks = _up(waves, 4)
    wgs, most = B * G * blocks, _up(T, 16)
    want, fine = min(most, _up(2048 // _up(waves, blocks), wgs)), min(most, _up(4096, rev))
    fine = max(fine, want)
    flen = _up(_up(T, fine), 16) * 16
    R = _up(_up(T, want), flen)
    S, F, T4 = _up(T, R * flen), _up(T, flen), _up(T, 16) * 4

    def al(v):
        return _up(v, 256) * 256

    total = (al(B * F * D * NP * 4) + al(B * F * D * 4) if F > 1 else 0) + al(2 * wgs * T4 * NP * 16) + al(B * S * D * (NP + 2) * 4)
    return R * flen, flen, R, R * flen // 16, total


# B, T, D, N, groups, lengths; segments' tokens, fine ones' tokens
TRAINING = [
    (2, 2100, 1985, 16, 1, [2100, 1111], 144, 48),  # fine segments of more than a tile of 32 tokens, an end inside a segment
    (1, 3000, 1056, 16, 3, None, 64, 16),
    (1, 1500, 1000, 24, 1, [1490], 32, 16),
    (1, 1400, 1024, 40, 1, None, 32, 16),
    (2, 700, 1000, 8, 1, [700, 0], 32, 16),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("case", TRAINING, ids=str)
def test_scan_in_segments_of_several_chunks(case, gate, dtype):
    import paper_2506_04761_amd as ll
    B, T, D, N, G, ns, tokens, fine = case
    split = _bwd_split(B, T, D, N, G)
    need = ll.lib.ll_selective_scan_workspace_size
    assert split[:2] == (tokens, fine) and split[3] > 1 and split[2] > 1
    assert need(B, T, D, N, G, 1) == max(split[4], need(B, T, D, N, G, 0))
    d = _Draw(T + D + N, dtype)
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, G, None)
    dy, df = d.rows(B, T, D), d.f32(B, D, N)
    xr, dtr, zr, Br, Cr, dyr = (np.nan_to_num(_np(t)) for t in (x, dt, z, Bm, Cm, dy))
    if ns is not None:
        for t in (x, dt, z, dy):
            for b, n in enumerate(ns):
                t[b, n:] = float("nan")
    if not gate:
        z = zr = None
    Br, Cr = Br.reshape(B, T, G, N), Cr.reshape(B, T, G, N)
    carried = max(1e-4, 3 * T * 2.0 ** -24)
    tol = {"f32": carried, "bf16": 2.0 ** -8 + carried}
    final, states = init.clone(), ll.ll_selective_scan_states(x, Bm)
    y = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, final, _lengths(ns), states)
    g = ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, skip, z, bias, True, _lengths(ns), df, True)
    wy, wf = layer.scan(xr, dtr, _np(A), Br, Cr, _np(skip), zr, _np(bias), True, _np(init), ns)
    want = layer.scan_grad(xr, dtr, _np(A), Br, Cr, dyr, _np(skip), zr, _np(bias), True, _np(init), ns, _np(df))
    _ok(y, wy, tol[dtype], "y")
    _ok(final, wf, tol["f32"], "final state")
    for name, got in zip(("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "initial"), g):
        if got is not None:
            _ok(got, want[name].reshape(got.shape), tol[dtype] if got.dtype == x.dtype else tol["f32"], "d" + name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("N", [5, 8, 9, 17, 24, 25, 27, 32, 33, 64])
def test_scan_of_any_number_of_states(N, gate, dtype):
    """8, 16, 24, 32 and 64 states of a lane forward, 16, 32 and 64 backward; 144 tokens in segments of 8 and more."""
    import paper_2506_04761_amd as ll
    B, T, D = 2, 144, 75
    d = _Draw(N, dtype)
    x, dt, z, Bm, Cm, A, skip, bias, init = _scan_inputs(d, B, T, D, N, 1, 1)
    z = z if gate else None
    dy, df = d.rows(B, T, D), d.f32(B, D, N)
    tol = {"f32": 1e-4, "bf16": 2.0 ** -8 + 1e-4}
    final, states = init.clone(), ll.ll_selective_scan_states(x, Bm)
    y = ll.ll_selective_scan_fwd(x, dt, A, Bm, Cm, skip, z, bias, True, init, final, None, states)
    g = ll.ll_selective_scan_bwd(x, dt, A, Bm, Cm, states, dy, skip, z, bias, True, None, df, True)
    args = (_np(x), _np(dt), _np(A), _np(Bm)[:, :, None], _np(Cm)[:, :, None])
    wy, wf = layer.scan(*args, _np(skip), _np(z), _np(bias), True, _np(init), None)
    want = layer.scan_grad(*args, _np(dy), _np(skip), _np(z), _np(bias), True, _np(init), None, _np(df))
    _ok(y, wy, tol[dtype], "y")
    _ok(final, wf, tol["f32"], "final state")
    for name, got in zip(("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "initial"), g):
        if got is not None:
            _ok(got, want[name].reshape(got.shape), tol[dtype] if got.dtype == x.dtype else tol["f32"], "d" + name)


# ------------------------------------------------------------------------------------ beyond 2^31 elements

LONG, WIDE, END = (1 << 20) + 37, 2080, 4096


def _long(seed):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.empty((1, LONG, WIDE), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    assert x.numel() > 1 << 31
    return g, x


def test_conv_gradients_beyond_32_bits():
    """The end of one long call against a call of the end alone; the taps' gradients against those of two parts."""
    import torch
    import paper_2506_04761_amd as ll
    g, x = _long(2)
    w = torch.randn((WIDE, 4), generator=g, device="cuda")
    whole = ll.ll_causal_conv_bwd(x, w, None, x)
    end, before = slice(LONG - END, LONG), x[:, LONG - END - 3:LONG - END].contiguous()
    tail = ll.ll_causal_conv_bwd(x[:, end].contiguous(), w, None, x[:, end].contiguous(), initial_state=before)
    assert torch.equal(whole.x[:, end], tail.x)
    head = ll.ll_causal_conv_bwd(x[:, :LONG - END], w, None, x[:, :LONG - END].contiguous())
    # chains of at most 600 additions
    assert rel_err(_np(whole.weight), _np(head.weight) + _np(tail.weight)) <= 1e-4


def test_scan_gradients_beyond_32_bits():
    """Rates of at least 0.69 a token: the state 4096 tokens back has no part in the last 2048 tokens' gradients."""
    import torch
    import paper_2506_04761_amd as ll
    g, x = _long(3)
    N = 8
    A = -torch.ones((WIDE, N), device="cuda")
    BC = torch.randn((1, LONG, 2 * N), generator=g, device="cuda").bfloat16()
    dt = torch.zeros((1, 1, WIDE), dtype=torch.bfloat16, device="cuda").expand(1, LONG, WIDE)
    a = (dt, A, BC[..., :N], BC[..., N:])
    states = ll.ll_selective_scan_states(x, a[2])
    ll.ll_selective_scan_fwd(x, *a, z=x, states=states)
    whole = ll.ll_selective_scan_bwd(x, *a, states, x, z=x)
    whole = {n: getattr(whole, n)[:, LONG - 2048:].clone() for n in ("x", "dt", "B", "C", "z")}
    del states
    end = slice(LONG - END, LONG)
    xe = x[:, end].contiguous()
    a = (dt[:, :END], A, BC[:, end, :N], BC[:, end, N:])
    states = ll.ll_selective_scan_states(xe, a[2])
    ll.ll_selective_scan_fwd(xe, *a, z=xe, states=states)
    tail = ll.ll_selective_scan_bwd(xe, *a, states, xe, z=xe)
    for n, t in whole.items():
        assert rel_err(_np(t), _np(getattr(tail, n)[:, END - 2048:])) <= 2.0 ** -8, n  # one unit of the last place


def test_norm_beyond_32_bits():
    """Single tokens: the end of one long call against a call of the end alone.  Over tokens: statistics and group sums
    of all tokens in float64, and with them the end of the output and of the gradient."""
    import torch
    import paper_2506_04761_amd as ll
    _, x = _long(4)
    G, end = 13, slice(LONG - 300, LONG)
    rows, dy = x.view(LONG, 1, WIDE), x.view(LONG, 1, WIDE)
    stats = ll.ll_group_norm_stats(rows, G)
    ll.ll_group_norm_fwd(rows, G, stats=stats)
    whole = ll.ll_group_norm_bwd(rows, G, None, None, stats, dy).x[end].clone()
    tail = ll.ll_group_norm_bwd(rows[end].contiguous(), G, None, None, stats[end].contiguous(), dy[end].contiguous())
    assert torch.equal(whole, tail.x)
    # without an activation: dx = r (dy - mean dy - xh mean(dy xh)), here with dy = x
    cg = WIDE // G
    s, q = torch.zeros(G, dtype=torch.float64, device="cuda"), torch.zeros(G, dtype=torch.float64, device="cuda")
    for part in x[0].split(1 << 14):
        v = part.double().view(-1, G, cg)
        s += v.sum((0, 2))
        q += (v * v).sum((0, 2))
    n = LONG * cg
    mean = s / n
    r = 1 / torch.sqrt(q / n - mean * mean + 1e-5)
    stats = ll.ll_group_norm_stats(x, G)
    y = ll.ll_group_norm_fwd(x, G, act=ll.LL_ACT_NONE, stats=stats)[:, end].clone()
    dx = ll.ll_group_norm_bwd(x, G, None, None, stats, x, act=ll.LL_ACT_NONE).x[:, end].clone()
    v = x[0, end].double().view(-1, G, cg)
    xh = (v - mean[:, None]) * r[:, None]
    _ok(stats[0, :, 1], _np(r), 1e-5, "rstd")
    _ok(y[0], _np(xh.reshape(-1, WIDE)), TOL["bf16"], "y")
    # mean(x xh) = (mean x^2 - (mean x)^2) r; what is left of dx is the rounding of x by eps and the mean
    left = r[:, None] * (v - mean[:, None] - xh * ((q / n - mean * mean) * r)[:, None])
    err = (dx[0].double() - left.reshape(-1, WIDE)).abs().max().item()
    # of values of about 5: x and xh times their mean product, each within a few 2^-24 of sums over 1e8 values (1e-5)
    assert err <= 5 * 4e-5, err
