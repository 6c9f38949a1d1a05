"""The backward of an activation with few values of du in bf16: they enter their products in two parts at any width, in a
workspace that does not jump between one size and the next."""

import pytest

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")


def test_the_workspace_has_no_cliff():
    size = ll.lib.ll_projection_workspace_size
    for K in (64, 1024, 8192, 65536, 65537, 1 << 20):
        few, more = (size(ll.LL_BF16, 1, K, N, 1, 1) for N in (1023, 1024))
        # du twice, the sums over strips, and splits of 1 x K at most
        assert few <= more + 2 * 1024 * 2 + 32 * K * 4, (K, few, more)
        few, more = (size(ll.LL_BF16, M, K, 31, 1, 1) for M in (33, 34))
        assert few <= more + 2 * 1024 * 2 + 32 * 33 * K * 4, (K, few, more)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,off", [(1, 65536, 16, None), (1, 65537, 16, None), (3, 70000, 40, None), (31, 66000, 33, 3),
                                       (1, 100001, 3, 3), (600, 1024, 1, None), (1, 8192, 1023, None)])
def test_wide_ones_are_rounded_once(M, K, N, off):
    """From sums `pre` that are inputs.  du in fp32 is off by (8 + |pre|) 2^-23 |dy| (exp2, rcp, a few roundings), its two
    parts leave 2^-16 of it, n products are added in fp32, and the results are rounded once."""
    import numpy as np
    from oracle import layer
    from tests.gpu_util import to_dev
    from tests.test_gpu_projection import _host, _inputs, _within
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    i = _inputs(M + N, M, K, N, "bf16", off, residual=False)
    u = np.random.default_rng(K).standard_normal((M, N))
    pre, h = to_dev(u), _host(i)
    u = pre.cpu().double().numpy()
    ws = ll.block.ll_projection_workspace(i["x"], i["w"], ll.block.LL_ACT_SILU, True)
    ws.fill_(255)
    g = ll.block.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.block.LL_ACT_SILU, pre, workspace=ws)
    du = h["dy"] * layer.act_grad(u, True)
    d = (8 + np.abs(u)) * 2.0 ** -23 * np.abs(h["dy"]) + 2.0 ** -16 * np.abs(du)
    for name, got, a, off_a, b, n in (("dx", g.x, du, d, h["w"], N), ("dw", g.weight, du.T, d.T, h["x"], M)):
        want = a @ b
        tol = (n + 8) * 2.0 ** -24 * ((np.abs(a) + off_a) @ np.abs(b)) + off_a @ np.abs(b)
        _within(got, want, tol + 2.0 ** -8 * (np.abs(want) + tol), name)
