"""Host-only checks of the projections' entry points: every argument check returns its status before anything is launched
(dummy, never-dereferenced pointers), and the size function."""

import ctypes

import numpy as np
import pytest

from oracle import layer

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")
lib = ll.lib
NULL, SHAPE, UNSUPPORTED, WORKSPACE = (ll._lib.LL_ERR_NULL_ARG, ll._lib.LL_ERR_BAD_SHAPE, ll._lib.LL_ERR_UNSUPPORTED,
                                       ll._lib.LL_ERR_WORKSPACE)
FAKE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 128)
BIG = 1 << 40


def _fwd(x=FAKE, xs=64, w=FAKE, res=None, rs=0, y=FAKE, M=300, K=4096, N=64, act=0, dtype=1, ws=FAKE, wsb=BIG):
    return lib.ll_projection_fwd(x, xs, w, None, res, rs, y, None, M, K, N, act, dtype, ws, wsb, None)


def _bwd(x=FAKE, xs=64, w=FAKE, pre=FAKE, dy=FAKE, M=300, K=64, N=64, act=1, dtype=1, ws=FAKE, wsb=BIG):
    return lib.ll_projection_bwd(x, xs, w, pre, dy, FAKE, FAKE, None, M, K, N, act, dtype, ws, wsb, None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_checks_return_before_launch(call):
    assert call(x=None) == NULL and call(w=None) == NULL
    assert call(M=0) == SHAPE and call(K=0) == SHAPE and call(N=0) == SHAPE and call(M=-1) == SHAPE and call(xs=-1) == SHAPE
    assert call(act=2) == UNSUPPORTED and call(dtype=2) == UNSUPPORTED and call(xs=1 << 24) == UNSUPPORTED
    assert call(K=1 << 24) == UNSUPPORTED and call(N=1 << 24) == UNSUPPORTED and call(M=1 << 40) == UNSUPPORTED
    assert call(ws=None) == NULL and call(wsb=256) == WORKSPACE and call(ws=ODD) == WORKSPACE


def test_checks_of_either():
    assert _fwd(y=None) == NULL
    assert _fwd(res=FAKE, rs=-1) == SHAPE and _fwd(res=FAKE, rs=1 << 24) == UNSUPPORTED
    assert _bwd(dy=None) == NULL and _bwd(pre=None) == NULL
    # launches of 2^32 threads
    assert _fwd(M=1 << 36, K=8, N=8) == UNSUPPORTED and _bwd(M=1 << 36, K=8, N=8) == UNSUPPORTED


def test_workspace_size():
    size = lib.ll_projection_workspace_size
    assert size(ll.LL_BF16, 1, 64, 64, 0, 0) == 0  # none needed
    assert size(ll.LL_BF16, 300, 4096, 64, 0, 0) >= 2 * 300 * 64 * 4
    assert size(ll.LL_BF16, 300, 64, 64, 1, 1) >= 300 * 64 * 2
    for bad in ((7, 300, 4096, 64, 0, 1), (1, 0, 64, 64, 0, 1), (1, 300, 1 << 24, 64, 0, 1), (1, 300, 64, 64, 5, 1)):
        assert size(*bad) == 0
    for s in ((1, 300, 4096, 64), (0, 8064, 257, 1000), (1, 70, 64, 8192)):
        assert size(*s, 1, 1) >= size(*s, 1, 0)


def test_oracle_gradients_against_differences():
    r = np.random.default_rng(0)
    x, w, b, d = (r.standard_normal(s) for s in ((5, 3), (4, 3), (4,), (5, 4)))
    grads = layer.projection_grad(x, w, d, b, True)
    for t, g in zip((x, w, b), grads):
        for i in np.ndindex(t.shape):
            at, ends = t[i], []
            for s in (1e-5, -1e-5):
                t[i] = at + s
                ends.append((layer.projection(x, w, b, None, True)[0] * d).sum())
            t[i] = at
            assert abs((ends[0] - ends[1]) / 2e-5 - g[i]) <= 1e-8
