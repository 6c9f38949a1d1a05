"""Host-only checks of the convolution, selective scan and group norm entry points: every argument check returns its
status before anything is launched (dummy, never-dereferenced pointers), and the size functions."""

import ctypes

import pytest

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")
lib = ll.lib
OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = (ll._lib.LL_OK, ll._lib.LL_ERR_NULL_ARG, ll._lib.LL_ERR_BAD_SHAPE,
                                           ll._lib.LL_ERR_UNSUPPORTED, ll._lib.LL_ERR_WORKSPACE)
FAKE = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4096 + 4)
BIG = 1 << 40


def _conv(x=FAKE, bs=64, ts=8, w=FAKE, y=FAKE, B=2, T=8, D=8, W=4, act=1, dtype=1):
    return lib.ll_causal_conv_fwd(x, bs, ts, w, None, None, None, None, y, B, T, D, W, act, dtype, None)


def _conv_step(x=FAKE, state=FAKE, new=FAKE, y=FAKE, W=4, act=1, dtype=1):
    return lib.ll_causal_conv_step(x, 8, FAKE, None, state, new, y, 2, 8, W, act, dtype, None)


def _conv_bwd(x=FAKE, dy=FAKE, dx=FAKE, dw=FAKE, W=4, ws=FAKE, wsb=BIG, T=8):
    return lib.ll_causal_conv_bwd(x, 64, 8, FAKE, None, None, None, dy, None, dx, dw, None, None, 2, T, 8, W, 1, 1, ws,
                                  wsb, None)


def test_conv_checks_return_before_launch():
    assert _conv(x=None) == NULL and _conv(w=None) == NULL and _conv(y=None) == NULL
    assert _conv(B=0) == SHAPE and _conv(T=0) == SHAPE and _conv(D=0) == SHAPE and _conv(W=0) == SHAPE
    assert _conv(bs=-1) == SHAPE and _conv(ts=-8) == SHAPE
    assert _conv(W=1) == UNSUPPORTED and _conv(W=5) == UNSUPPORTED
    assert _conv(act=2) == UNSUPPORTED and _conv(dtype=2) == UNSUPPORTED
    assert _conv(ts=1 << 24) == UNSUPPORTED and _conv(D=1 << 24) == UNSUPPORTED and _conv(T=1 << 45) == UNSUPPORTED
    assert _conv_step(x=None) == NULL and _conv_step(state=None) == NULL and _conv_step(new=None) == NULL
    assert _conv_step(y=None) == NULL and _conv_step(W=5) == UNSUPPORTED and _conv_step(dtype=-1) == UNSUPPORTED
    assert _conv_bwd(x=None) == NULL and _conv_bwd(dy=None) == NULL and _conv_bwd(dx=None) == NULL
    assert _conv_bwd(dw=None) == NULL and _conv_bwd(ws=None) == NULL
    assert _conv_bwd(T=0) == SHAPE and _conv_bwd(W=7) == UNSUPPORTED
    assert _conv_bwd(wsb=64) == WORKSPACE and _conv_bwd(ws=ctypes.c_void_p(4096 + 128)) == WORKSPACE


def test_conv_workspace_size():
    size = lib.ll_causal_conv_bwd_workspace_size
    assert size(ll.LL_BF16, 2, 100, 64, 4) > 0
    assert size(ll.LL_BF16, 2, 0, 64, 4) == 0 and size(ll.LL_BF16, 2, 100, 64, 5) == 0 and size(7, 2, 100, 64, 4) == 0


def _inputs(**kw):
    s = ll._layer._ScanInputs()
    for n in ("x", "dt", "z", "B", "C", "A"):
        setattr(s, n, 4096)
    s.batch, s.T, s.channels, s.N, s.groups, s.delta_softplus, s.dtype = 2, 8, 64, 16, 1, 1, 1
    for k, v in kw.items():
        if k.endswith("_strides"):
            name = k[:-len("_strides")]
            setattr(s, name + "_batch", v[0]), setattr(s, name + "_token", v[1])
        else:
            setattr(s, k, v)
    return s


def _scan(y=FAKE, states=None, ws=FAKE, wsb=BIG, none=False, **kw):
    return lib.ll_selective_scan_fwd(None if none else _inputs(**kw), None, y, None, states, ws, wsb, None)


def _scan_step(state=FAKE, new=FAKE, y=FAKE, **kw):
    return lib.ll_selective_scan_step(_inputs(**{"T": 1, **kw}), state, new, y, None)


def _scan_bwd(states=FAKE, dy=FAKE, dx=FAKE, dz=FAKE, dA=FAKE, dB=FAKE, ws=FAKE, wsb=BIG, **kw):
    return lib.ll_selective_scan_bwd(_inputs(**kw), states, dy, None, dx, FAKE, dz, dA, dB, FAKE, None, None, None, ws,
                                     wsb, None)


def test_scan_checks_return_before_launch():
    assert _scan(none=True) == NULL and _scan(y=None) == NULL
    for n in ("x", "dt", "A", "B", "C"):
        assert _scan(**{n: None}) == NULL, n
    assert _scan(batch=0) == SHAPE and _scan(T=0) == SHAPE and _scan(channels=0) == SHAPE and _scan(N=0) == SHAPE
    assert _scan(groups=0) == SHAPE and _scan(groups=3) == SHAPE  # 64 channels do not split into 3 groups
    for n in ("x", "dt", "z", "B", "C"):
        assert _scan(**{n + "_strides": (-1, 8)}) == SHAPE and _scan(**{n + "_strides": (8, 1 << 24)}) == UNSUPPORTED
    assert _scan(N=65) == UNSUPPORTED and _scan(dtype=2) == UNSUPPORTED and _scan(batch=1 << 33) == UNSUPPORTED
    assert _scan(states=ODD) == WORKSPACE
    # one sequence of 64 channels is split over its length: it needs a workspace
    assert _scan(T=8192, ws=None) == NULL and _scan(T=8192, wsb=64) == WORKSPACE
    assert _scan(T=8192, ws=ctypes.c_void_p(4096 + 16)) == WORKSPACE
    assert _scan_step(state=None) == NULL and _scan_step(new=None) == NULL and _scan_step(y=None) == NULL
    assert _scan_step(T=2) == SHAPE and _scan_step(lengths=4096) == SHAPE and _scan_step(N=65) == UNSUPPORTED
    assert _scan_bwd(states=None) == NULL and _scan_bwd(dy=None) == NULL and _scan_bwd(dx=None) == NULL
    assert _scan_bwd(dz=None) == NULL and _scan_bwd(dA=None) == NULL and _scan_bwd(dB=None) == NULL
    assert _scan_bwd(ws=None) == NULL and _scan_bwd(wsb=64) == WORKSPACE and _scan_bwd(states=ODD) == WORKSPACE


def test_scan_sizes():
    states, ws = lib.ll_selective_scan_states_bytes, lib.ll_selective_scan_workspace_size
    # the state of 16 (padded) float32 values before every 16th token
    assert states(2, 65, 8, 5) == 2 * 5 * 8 * 16 * 4 and states(1, 16, 8, 16) == 8 * 16 * 4
    assert states(1, 64, 8, 17) == 4 * 8 * 32 * 4 and states(1, 64, 8, 64) == 4 * 8 * 64 * 4
    assert states(1, 64, 8, 65) == 0 and states(1, 0, 8, 16) == 0
    assert ws(1, 8, 64, 16, 1, 0) == 0 and ws(1, 64, 64, 16, 1, 1) > 0 and ws(1, 8192, 64, 16, 1, 0) > 0
    assert ws(1, 64, 64, 16, 3, 1) == 0 and ws(0, 64, 64, 16, 1, 1) == 0


def _norm(x=FAKE, gate=None, y=FAKE, stats=None, N=4, S=1, C=64, G=4, act=1, dtype=1, bs=64, ts=64, gbs=64, ws=FAKE,
          wsb=BIG):
    return lib.ll_group_norm_fwd(x, bs, ts, gate, gbs, 64, None, None, y, stats, N, S, C, G, 1e-5, act, dtype, ws, wsb, None)


def _norm_bwd(x=FAKE, gate=None, stats=FAKE, dy=FAKE, dx=FAKE, dgate=None, G=4, ws=FAKE, wsb=BIG):
    return lib.ll_group_norm_bwd(x, 64, 64, gate, 64, 64, None, None, stats, dy, dx, dgate, None, None, 4, 1, 64, G, 1, 1,
                                 ws, wsb, None)


def test_norm_checks_return_before_launch():
    assert _norm(x=None) == NULL and _norm(y=None) == NULL
    assert _norm(N=0) == SHAPE and _norm(S=0) == SHAPE and _norm(G=0) == SHAPE and _norm(G=3) == SHAPE
    assert _norm(bs=-1) == SHAPE and _norm(gate=FAKE, gbs=-1) == SHAPE and _norm(ts=1 << 24) == UNSUPPORTED
    assert _norm(act=5) == UNSUPPORTED and _norm(dtype=5) == UNSUPPORTED
    assert _norm(S=64, ws=None) == NULL and _norm(S=64, wsb=8) == WORKSPACE and _norm(stats=ODD) == WORKSPACE
    assert _norm_bwd(x=None) == NULL and _norm_bwd(stats=None) == NULL and _norm_bwd(dy=None) == NULL
    assert _norm_bwd(dx=None) == NULL and _norm_bwd(gate=FAKE) == NULL
    assert _norm_bwd(ws=None) == NULL and _norm_bwd(wsb=8) == WORKSPACE and _norm_bwd(stats=ODD) == WORKSPACE
    assert _norm_bwd(G=5) == SHAPE


def test_norm_workspace_size():
    size = lib.ll_group_norm_workspace_size
    assert size(ll.LL_BF16, 4, 1, 64, 4, 0) == 0  # tokens by themselves: statistics stay on chip
    assert size(ll.LL_BF16, 4, 64, 64, 4, 0) > 0 and size(ll.LL_BF16, 4, 1, 64, 4, 1) > 0
    assert size(ll.LL_BF16, 4, 1, 64, 3, 1) == 0 and size(9, 4, 1, 64, 4, 1) == 0


def test_wrappers_refuse_what_is_not_on_the_device():
    import torch
    x = torch.zeros(2, 8, 64)
    with pytest.raises(TypeError):
        ll.ll_causal_conv_fwd(x, torch.zeros(64, 4))
    with pytest.raises(ValueError):
        ll.ll_causal_conv_fwd(x[0], torch.zeros(64, 4))
    with pytest.raises(TypeError):
        ll.ll_selective_scan_fwd(x, x, torch.zeros(64, 16), torch.zeros(2, 8, 16), torch.zeros(2, 8, 16))
    with pytest.raises(TypeError):
        ll.ll_group_norm_fwd(x, 4)
