"""Host-only checks of the largest sizes: what the arithmetic of sizes or a launch cannot hold is refused before
anything is enqueued (dummy, never-dereferenced pointers)."""

import ctypes

import pytest

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")
lib = ll.lib
UNSUPPORTED = ll._lib.LL_ERR_UNSUPPORTED
FAKE = ctypes.c_void_p(4096)
BIG = (1 << 63) - 1


@pytest.mark.parametrize("B,T", [(1 << 39, 1 << 39), (1 << 36, 1 << 36), (1 << 36, 1 << 35), (1 << 25, 1 << 39), ((1 << 40) - 1, 300)])
def test_sizes_beyond_64_bits_are_invalid(B, T):
    """Tensors of more than 2^44 elements, most of which wrap in 64 bits: no bytes, and refused by every call."""
    for D in (1, 64, (1 << 24) - 1):
        assert lib.ll_causal_conv_bwd_workspace_size(ll.LL_BF16, B, T, D, 4) == 0
        assert lib.ll_selective_scan_states_bytes(B, T, D, 64) == 0
        for backward in (0, 1):
            assert lib.ll_selective_scan_workspace_size(B, T, D, 64, 1, backward) == 0
            assert lib.ll_group_norm_workspace_size(ll.LL_BF16, B, T, D, 1, backward) == 0
        assert lib.ll_causal_conv_fwd(FAKE, 64, 8, FAKE, None, None, None, None, FAKE, B, T, D, 4, 1, 1, None) == UNSUPPORTED
        assert lib.ll_group_norm_fwd(FAKE, 64, 8, None, 0, 0, None, None, FAKE, None, B, T, D, 1, 1e-5, 1, 1, FAKE, BIG,
                                     None) == UNSUPPORTED


def test_sizes_of_the_largest_tensors():
    """2^40 elements, beyond any GPU's memory, still have a size."""
    B, T, D = 1 << 10, 1 << 20, 1 << 10
    assert lib.ll_causal_conv_bwd_workspace_size(ll.LL_BF16, B, T, D, 4) > 0
    assert lib.ll_selective_scan_states_bytes(B, T, D, 64) == (1 << 40) // 16 * 64 * 4
    assert lib.ll_selective_scan_workspace_size(B, T, D, 64, 1, 1) > 0
    assert lib.ll_group_norm_workspace_size(ll.LL_BF16, B, T, D, 1, 1) > 0


def _scan_inputs(B, T, D, N, G):
    s = ll._layer._ScanInputs()
    for n in ("x", "dt", "z", "B", "C", "A"):
        setattr(s, n, 4096)
    s.batch, s.T, s.channels, s.N, s.groups, s.delta_softplus, s.dtype = B, T, D, N, G, 1, 1
    return s


def _norm(N, S, C, G, dtype=1):
    a = (N, S, C, G)
    return (lib.ll_group_norm_fwd(FAKE, 64, 64, None, 0, 0, None, None, FAKE, None, *a, 1e-5, 1, dtype, FAKE, BIG, None),
            lib.ll_group_norm_bwd(FAKE, 64, 64, None, 0, 0, None, None, FAKE, FAKE, FAKE, None, FAKE, FAKE, *a, 1, dtype, FAKE,
                                  BIG, None))


def _conv(B, T, D, dtype=1):
    return lib.ll_causal_conv_fwd(FAKE, 64, 8, FAKE, None, None, None, None, FAKE, B, T, D, 4, 1, dtype, None)


def _conv_bwd(B, T, D, dtype=1):
    return lib.ll_causal_conv_bwd(FAKE, 64, 8, FAKE, None, None, None, FAKE, None, FAKE, FAKE, None, None, B, T, D, 4, 1,
                                  dtype, FAKE, BIG, None)


def test_launches_of_too_many_threads_are_refused():
    """A launch holds fewer than 2^32 threads.  Each of these calls has one that would hold more, some behind others that
    would not."""
    # a workgroup of 256 to a sequence and group
    assert _norm(1 << 20, 2, 64, 16) == (UNSUPPORTED,) * 2 and _norm(1 << 24, 3, 8, 1, dtype=0) == (UNSUPPORTED,) * 2
    # a thread to a run and channel vector
    assert _conv(1 << 32, 1, 1) == UNSUPPORTED and _conv(1 << 20, 1, (1 << 24) - 1, dtype=0) == UNSUPPORTED
    assert _conv_bwd(1 << 32, 1, 1) == UNSUPPORTED
    # a workgroup of the backward to a sequence, of which each has only a channel (the forward would take these)
    assert _conv_bwd(1 << 24, 4, 1) == UNSUPPORTED
    # sequences of one token
    assert lib.ll_causal_conv_step(FAKE, 8, FAKE, None, FAKE, FAKE, FAKE, 1 << 30, 64, 4, 1, 1, None) == UNSUPPORTED
    assert lib.ll_selective_scan_step(_scan_inputs(1 << 24, 1, 64, 16, 1), FAKE, FAKE, FAKE, None) == UNSUPPORTED

    def bwd(*a):
        return lib.ll_selective_scan_bwd(_scan_inputs(*a), FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None,
                                         None, FAKE, BIG, None)

    def fwd(*a):
        return lib.ll_selective_scan_fwd(_scan_inputs(*a), None, FAKE, None, None, FAKE, BIG, None)

    assert bwd(1, 1 << 27, 64, 16, 1) == UNSUPPORTED                # dB and dC, by a lane an element
    assert bwd(1 << 20, 16, 64, 16, 16) == UNSUPPORTED
    assert bwd(1, 16, (1 << 24) - 64, 64, 1) == UNSUPPORTED         # dA
    assert fwd(1 << 26, 8, 64, 16, 1) == UNSUPPORTED and fwd(1 << 20, 8, 64, 1, 64) == UNSUPPORTED
    assert fwd(1 << 24, 64, 2048, 16, 1) == UNSUPPORTED
