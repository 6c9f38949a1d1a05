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
