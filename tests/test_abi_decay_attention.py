"""Host-only checks of the entry points of the linear attention with a decay for each head: every argument check returns its
status before anything is launched (dummy, never-dereferenced pointers), the size functions, and the oracle's pins."""

import ctypes

import numpy as np
import pytest

from oracle import layer

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")
lib = ll.lib
NULL, SHAPE, UNSUPPORTED, WORKSPACE = (ll._lib.LL_ERR_NULL_ARG, ll._lib.LL_ERR_BAD_SHAPE, ll._lib.LL_ERR_UNSUPPORTED,
                                       ll._lib.LL_ERR_WORKSPACE)
FAKE, ODD, ODD4 = ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 128), ctypes.c_void_p(4096 + 4)
BIG = 1 << 50


def _inputs(**kw):
    s = ll.block._DecayInputs()
    for n in ("q", "k", "v", "log_decay"):
        setattr(s, n, 4096)
    s.batch, s.T, s.heads, s.qk_heads, s.d_k, s.d_v, s.scale, s.dtype = 2, 4096, 4, 2, 64, 32, 1.0, 1
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _fwd(o=FAKE, states=None, ws=FAKE, wsb=BIG, none=False, **kw):
    return lib.ll_decay_attention_fwd(None if none else _inputs(**kw), None, o, None, states, ws, wsb, None)


def _step(state=FAKE, new=FAKE, o=FAKE, **kw):
    return lib.ll_decay_attention_step(_inputs(**{"T": 1, **kw}), state, new, o, None)


def _bwd(states=FAKE, d_o=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, wsb=BIG, **kw):
    return lib.ll_decay_attention_bwd(_inputs(**kw), states, d_o, None, dq, dk, dv, None, ws, wsb, None)


@pytest.mark.parametrize("call", [_fwd, _step, _bwd])
def test_checks_return_before_launch(call):
    for n in ("q", "k", "v", "log_decay"):
        assert call(**{n: None}) == NULL
    for n in ("batch", "T", "heads", "qk_heads", "d_k", "d_v"):
        assert call(**{n: 0}) == SHAPE and call(**{n: -3}) == SHAPE
    assert call(qk_heads=3) == SHAPE and call(qk_heads=8) == SHAPE
    for n in "qkv":
        assert call(**{n + "_batch": -1}) == SHAPE and call(**{n + "_token": -1}) == SHAPE
        assert call(**{n + "_token": 1 << 24}) == UNSUPPORTED
    assert call(d_k=257) == UNSUPPORTED and call(d_v=257) == UNSUPPORTED and call(dtype=2) == UNSUPPORTED
    assert call(heads=1 << 24, qk_heads=1) == UNSUPPORTED and call(batch=1 << 40) == UNSUPPORTED
    # launches of 2^32 threads
    assert call(batch=1 << 30) == UNSUPPORTED


def test_checks_of_each():
    assert _fwd(none=True) == NULL and _fwd(o=None) == NULL and _fwd(T=1 << 45) == UNSUPPORTED
    assert _fwd(ws=None) == NULL and _fwd(wsb=256) == WORKSPACE and _fwd(ws=ODD) == WORKSPACE
    assert _fwd(states=ODD4) == WORKSPACE
    assert _step(state=None) == NULL and _step(new=None) == NULL and _step(o=None) == NULL
    assert _step(T=2) == SHAPE and _step(lengths=4096) == SHAPE
    for n in ("states", "d_o", "dq", "dk", "dv", "ws"):
        assert _bwd(**{n: None}) == NULL
    assert _bwd(wsb=256) == WORKSPACE and _bwd(ws=ODD) == WORKSPACE and _bwd(states=ODD4) == WORKSPACE


def test_sizes():
    size, states = lib.ll_decay_attention_workspace_size, lib.ll_decay_attention_states_bytes
    assert size(2, 300, 4, 4, 64, 32, 0) == 0  # one segment: no workspace
    assert states(2, 300, 4, 64, 32) == 2 * 4 * 64 * 32 * 4
    assert states(1, 65536, 4, 64, 32) >= 64 * 4 * 64 * 32 * 4
    for s in ((2, 300, 4, 2, 64, 32), (1, 65536, 4, 4, 64, 32), (64, 8192, 32, 1, 128, 128)):
        assert size(*s, 1) >= size(*s, 0)
    assert size(2, 300, 4, 2, 64, 32, 1) >= 2 * 300 * 4 * 64 * 4  # gradients of shared heads, one by one
    for bad in ((0, 300, 4, 4, 64, 32), (2, 0, 4, 4, 64, 32), (2, 300, 4, 3, 64, 32), (2, 300, 4, 4, 512, 32)):
        assert size(*bad, 1) == 0
    assert states(2, 300, 4, 64, 300) == 0


def test_oracle_is_the_masked_product():
    r = np.random.default_rng(0)
    q, k, v = (r.standard_normal((2, 9, h, d)) for h, d in ((2, 3), (2, 3), (4, 5)))
    ld = -np.array([0.1, 0.7, 0.0, 3.0])
    o, final = layer.decay_attention(q, k, v, ld, 0.5)
    t = np.arange(9)
    for h in range(4):
        mask = np.where(t[:, None] >= t, np.exp(ld[h] * (t[:, None] - t)), 0.0)
        want = 0.5 * (q[:, :, h // 2] @ k[:, :, h // 2].transpose(0, 2, 1) * mask) @ v[:, :, h]
        assert np.abs(o[:, :, h] - want).max() <= 1e-12
        weight = np.exp(ld[h] * (8 - t))
        assert np.abs(final[:, h] - (k[:, :, h // 2] * weight[:, None]).transpose(0, 2, 1) @ v[:, :, h]).max() <= 1e-12


def test_oracle_gradients_against_differences():
    r = np.random.default_rng(1)
    q, k, v = (r.standard_normal((2, 4, h, d)) for h, d in ((1, 2), (1, 2), (2, 3)))
    ld, first, n = -np.array([0.1, 0.6]), r.standard_normal((2, 2, 2, 3)), [4, 2]
    do, df = r.standard_normal((2, 4, 2, 3)), r.standard_normal((2, 2, 2, 3))

    def loss():
        o, final = layer.decay_attention(q, k, v, ld, 0.5, first, n)
        return (o * do).sum() + (final * df).sum()

    for t, g in zip((q, k, v, first), layer.decay_attention_grad(q, k, v, ld, do, 0.5, first, n, df)):
        for i in np.ndindex(t.shape):
            at, ends = t[i], []
            for s in (1e-4, -1e-4):
                t[i] = at + s
                ends.append(loss())
            t[i] = at
            assert abs((ends[0] - ends[1]) / 2e-4 - g[i]) <= 1e-8
