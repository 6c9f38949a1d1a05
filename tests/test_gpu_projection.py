"""Projections on the GPU against the float64 oracle: forward and gradients at single rows, odd sizes, sizes of several
tiles and of split reductions, columns of wider rows at any start, with each part of the epilogue.

Tolerances are bounds, element by element, with e = 2^-8 (bf16) or 2^-24 (fp32), half a step of the storage type:
  sums       (n + 8) 2^-24 sum |a b| for n terms added in fp32 in some order, bias and residual among them
  SiLU       |v| (8 + |v|) 2^-23 for the value and (8 + |v|) 2^-23 for the factor: exp2 and rcp are off by a unit or two
             each, the exponent v log2 e by half a unit, and the sums' error passes with a slope below 1.1
  du         enters its products rounded: e |du|
  results    one rounding: e |want|"""

import numpy as np
import pytest

from oracle import layer
from tests.gpu_util import to_dev

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_04761_amd  # noqa: F401  (fails loudly if the library is missing)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _rows(r, M, N, dtype, off):
    """[M, N], or with `off` its columns from there on in wider rows full of NaN."""
    x = to_dev(r.standard_normal((M, N)), dtype)
    if off is None:
        return x
    import torch
    wide = torch.full((M, N + off + 3), float("nan"), device="cuda", dtype=x.dtype)
    wide[:, off:off + N] = x
    return wide[:, off:off + N]


def _within(got, want, tol, name):
    got = _np(got)
    assert got.shape == want.shape, (name, got.shape)
    bad = ~(np.abs(got - want) <= tol + 1e-37)
    assert not bad.any(), (name, int(bad.sum()), float(np.max(np.abs(got - want) / (tol + 1e-37))))


def _sum_tol(a, b, n):
    return (n + 8) * 2.0 ** -24 * (np.abs(a) @ np.abs(b))


def _inputs(seed, M, K, N, dtype, off, bias=True, residual=True):
    r = np.random.default_rng(seed)
    return {"x": _rows(r, M, K, dtype, off), "w": to_dev(r.standard_normal((N, K)) / np.sqrt(K), dtype),
            "b": to_dev(r.standard_normal(N)) if bias else None,
            "r": _rows(r, M, N, dtype, off) if residual else None, "dy": to_dev(r.standard_normal((M, N)), dtype)}


def _host(i):
    return {k: None if t is None else _np(t) for k, t in i.items()}


def _check_fwd(y, pre, h, dtype, silu, K):
    want, u = layer.projection(h["x"], h["w"], h["b"], h["r"], silu)
    tol = _sum_tol(h["x"], h["w"].T, K) + 8 * 2.0 ** -24 * np.abs(u)
    if h["b"] is not None:
        tol += 8 * 2.0 ** -24 * np.abs(h["b"])
    if pre is not None:
        _within(pre, u, tol, "pre")
    if silu:
        tol = 1.1 * tol + np.abs(u) * (8 + np.abs(u)) * 2.0 ** -23
    if h["r"] is not None:
        tol += 2.0 ** -23 * (np.abs(h["r"]) + np.abs(want))
    _within(y, want, tol + HALF[dtype] * (np.abs(want) + tol), "y")


def _check_bwd(g, h, dtype, silu, K, into_e=None):
    e = HALF[dtype]
    into_e = e if into_e is None else into_e
    M, N = h["dy"].shape
    dx, dw, db = layer.projection_grad(h["x"], h["w"], h["dy"], h["b"], silu)
    u = layer.projection(h["x"], h["w"], h["b"])[1]
    du = np.abs(h["dy"] * layer.act_grad(u, silu))
    off = np.zeros_like(du)  # of du in fp32
    if silu:
        off = np.abs(h["dy"]) * (0.5 * _sum_tol(h["x"], h["w"].T, K) + (8 + np.abs(u)) * 2.0 ** -23)
    into = off + (into_e * (du + off) if silu else 0)  # of du in the products
    for name, got, want, a, b, n in (("dx", g[0], dx, du, h["w"], N), ("dw", g[1], dw, du.T, h["x"], M)):
        d = into if name == "dx" else into.T
        tol = (n + 8) * 2.0 ** -24 * ((a + d) @ np.abs(b)) + d @ np.abs(b)
        _within(got, want, tol + e * (np.abs(want) + tol), name)
    if g[2] is not None:
        _within(g[2], db, off.sum(0) + (M + 8) * 2.0 ** -24 * (du + off).sum(0), "dbias")


#        M, K, N
SIZES = [(1, 1, 1), (1, 8, 16), (1, 2048, 40), (5, 40, 24), (16, 64, 64), (17, 100, 33), (33, 257, 130), (64, 520, 48),
         (65, 64, 64), (100, 1000, 129), (129, 72, 257), (300, 2056, 64), (1000, 136, 520), (700, 1, 9), (513, 33, 5),
         (2100, 72, 2000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("off", [None, 8, 3])
def test_sizes(M, K, N, dtype, off):
    from paper_2506_04761_amd import block as ll
    import torch
    i = _inputs(M + K + N, M, K, N, dtype, off)
    h = _host(i)
    pre = torch.full((M, N), float("nan"), device="cuda")
    y = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], ll.LL_ACT_SILU, pre)
    _check_fwd(y, pre, h, dtype, True, K)
    _check_bwd(ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, pre), h, dtype, True, K)


@pytest.mark.parametrize("M,K,N", [(1, 8, 8), (1, 2048, 40), (1, 100, 1023), (7, 257, 130), (31, 64, 33), (3, 8192, 64),
                                   (1000, 65, 1), (15, 1000, 64)])
@pytest.mark.parametrize("off", [None, 3])
def test_few_gradients_are_rounded_once(off, M, K, N):
    """bf16, fewer than 1024 values of du: du enters its products in two parts, which leave 2^-8 of 2^-8, so the head's
    bounds with 2^-16 |du| for 2^-8 |du|."""
    from paper_2506_04761_amd import block as ll
    i = _inputs(M + N, M, K, N, "bf16", off, residual=False)
    h = _host(i)
    import torch
    pre = torch.empty((M, N), device="cuda")
    ll.ll_projection_fwd(i["x"], i["w"], i["b"], None, ll.LL_ACT_SILU, pre)
    ws = ll.ll_projection_workspace(i["x"], i["w"], ll.LL_ACT_SILU, True)
    ws.fill_(255)
    _check_bwd(ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, pre, workspace=ws), h, "bf16", True, K,
               into_e=2.0 ** -16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(3, 72, 40), (70, 200, 136), (400, 1100, 64)])
@pytest.mark.parametrize("silu,bias,residual", [(False, False, False), (False, True, False), (True, False, True),
                                                (False, False, True), (True, True, False)])
def test_epilogue(M, K, N, dtype, silu, bias, residual):
    from paper_2506_04761_amd import block as ll
    import torch
    i = _inputs(7, M, K, N, dtype, None, bias, residual)
    h = _host(i)
    act = ll.LL_ACT_SILU if silu else ll.LL_ACT_NONE
    pre = torch.empty((M, N), device="cuda") if silu else None
    y = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], act, pre)
    _check_fwd(y, pre, h, dtype, silu, K)
    g = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], act, pre)
    assert (g.bias is None) == (not bias)
    _check_bwd(g, h, dtype, silu, K)
    # without `pre`, and the same call again: the same bits
    again = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], act)
    assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(4090, 1032, 2816), (4090, 1031, 2810), (2050, 2048, 1030), (700, 4104, 1000), (20, 8200, 8200)])
def test_tiles_of_every_size(M, K, N, dtype):
    """Sizes that take tiles of 64, 128 and 256 outputs, whole and in splits, of aligned and unaligned rows.  The reference
    is in 64 bits on the GPU; bounds as above."""
    from paper_2506_04761_amd import block as ll
    i = _inputs(M, M, K, N, dtype, None)
    h = {k: t.double() for k, t in i.items()}
    u24, e = 2.0 ** -24, HALF[dtype]
    y = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"])
    g = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"])
    more = (h["b"].abs() + h["r"].abs()) * 16 * u24
    for name, got, a, b, n, add, tol in (("y", y, h["x"], h["w"].T, K, h["b"] + h["r"], more), ("dx", g.x, h["dy"], h["w"], N, 0, 0),
                                         ("dw", g.weight, h["dy"].T, h["x"], M, 0, 0)):
        want = a @ b + add
        bound = (n + 8) * u24 * (a.abs() @ b.abs()) + tol
        assert ((got.double() - want).abs() <= bound + e * (want.abs() + bound)).all(), name
    want, bound = h["dy"].sum(0), (M + 8) * u24 * h["dy"].abs().sum(0)
    assert ((g.bias.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype,M", [("bf16", 260), ("f32", 131)])
def test_the_widest_rows(dtype, M):
    """Rows as far apart as strides may be: a tile spans more than 2^32 bytes."""
    import paper_2506_04761_amd as ll
    import torch
    from tests.gpu_util import torch_dtype
    step = (1 << 24) - 8
    if torch.cuda.mem_get_info()[0] < 3 * M * step * 4:
        pytest.skip("memory")
    i = _inputs(12, M, 72, 264, dtype, None)
    wide = torch.empty(M * step, dtype=torch_dtype(dtype), device="cuda").as_strided((M, 72), (step, 1))
    wide.copy_(i["x"])
    i["x"] = wide
    h = _host(i)
    pre = torch.empty((M, 264), device="cuda")
    y = ll.block.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], ll.LL_ACT_SILU, pre)
    _check_fwd(y, pre, h, dtype, True, 72)
    _check_bwd(ll.block.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, pre), h, dtype, True, 72)


def test_rows_that_are_one_row():
    """Strides of zero: one input row, and one residual row, for every output row."""
    from paper_2506_04761_amd import block as ll
    i = _inputs(13, 1, 200, 72, "bf16", None)
    h = _host(i)
    y = ll.ll_projection_fwd(i["x"].expand(150, -1), i["w"], i["b"], i["r"].expand(150, -1))
    h = {**h, "x": np.repeat(h["x"], 150, 0), "r": np.repeat(h["r"], 150, 0)}
    _check_fwd(y, None, h, "bf16", False, 200)


def test_only_the_gradients_that_are_wanted():
    from paper_2506_04761_amd import block as ll
    import torch
    i = _inputs(9, 90, 64, 72, "bf16", None)
    full = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"])
    for keep in range(3):
        some = ll.ProjectionGrads(*(torch.empty_like(t) if k == keep else None for k, t in enumerate(full)))
        got = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], grads=some)
        assert torch.equal(got[keep], full[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [7, 200])
def test_inf_and_nan_stay_in_their_rows(dtype, M):
    from paper_2506_04761_amd import block as ll
    import torch
    i = _inputs(3, M, 100, 50, dtype, None)
    y = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"])
    x = i["x"].clone()
    x[2, 99] = float("nan")
    x[5, 0] = float("inf")
    z = ll.ll_projection_fwd(x, i["w"], i["b"], i["r"])
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[2] = rows[5] = False
    assert torch.equal(z[rows], y[rows])
    assert z[2].isnan().all() and not z[5].isfinite().any()


def test_differentiable_over_leading_axes():
    from paper_2506_04761_amd import block as ll
    import torch
    r = np.random.default_rng(5)
    wide = to_dev(r.standard_normal((3, 7, 96))).requires_grad_()
    w, b = (to_dev(r.standard_normal(s) / 8).requires_grad_() for s in ((40, 48), (40,)))
    res = to_dev(r.standard_normal((3, 7, 40))).requires_grad_()
    dy = to_dev(r.standard_normal((3, 7, 40)))
    y = ll.projection(wide[..., :48], w, b, res, ll.LL_ACT_SILU)
    y.backward(dy)
    x = _np(wide)[..., :48].reshape(21, 48)
    want, _ = layer.projection(x, _np(w), _np(b), _np(res).reshape(21, 40), True)
    dx, dw, db = layer.projection_grad(x, _np(w), _np(dy).reshape(21, 40), _np(b), True)
    for got, ref in ((y.reshape(21, 40), want), (wide.grad[..., :48].reshape(21, 48), dx), (w.grad, dw), (b.grad, db)):
        # about 50 roundings of 2^-24 of terms no larger than a few of the largest result
        assert np.abs(_np(got) - ref).max() <= 1e-5 * np.abs(ref).max()
    assert torch.equal(res.grad, dy) and not wide.grad[..., 48:].any()


def test_gradients_against_differences():
    from paper_2506_04761_amd import block as ll
    import torch
    r = np.random.default_rng(6)
    x, w, b = (to_dev(r.standard_normal(s)).requires_grad_() for s in ((6, 5), (4, 5), (4,)))
    d = to_dev(r.standard_normal((6, 4)))

    def loss():
        return (ll.projection(x, w, b, None, ll.LL_ACT_SILU) * d).double().sum()

    loss().backward()
    step = 2.0 ** -7
    for t in (x, w, b):
        flat, grad = t.data.view(-1), t.grad.view(-1)
        for i in range(0, flat.numel(), 3):
            at = flat[i].item()
            ends = []
            for s in (step, -step):
                flat[i] = at + s
                ends.append(loss().item())
            flat[i] = at
            # the third derivative's share step^2 / 6 of up to 10 terms, and rounding 2^-22 of 24 values over 2 step
            assert abs((ends[0] - ends[1]) / (2 * step) - grad[i].item()) <= 5e-3


def test_second_derivatives_are_refused_but_the_residual_is_linear():
    from paper_2506_04761_amd import block as ll
    import torch
    x, w = (torch.randn(s, device="cuda", requires_grad=True) for s in ((4, 8), (8, 8)))
    y = ll.projection(x, w, residual=x)
    g, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        g.sum().backward()


def test_on_another_stream_and_in_a_graph():
    from paper_2506_04761_amd import block as ll
    import torch
    i = _inputs(11, 300, 1032, 136, "bf16", None)
    pre = torch.empty((300, 136), device="cuda")
    want = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], ll.LL_ACT_SILU, pre)
    wants = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, pre)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], ll.LL_ACT_SILU, pre, stream=side)
    grads = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, pre, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(grads, wants))
    out, ws = torch.empty_like(want), ll.ll_projection_workspace(i["x"], i["w"], ll.LL_ACT_SILU, backward=True)
    made = ll.ProjectionGrads(*(torch.empty_like(t) for t in wants))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], ll.LL_ACT_SILU, pre, out=out, workspace=ws)
        ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, pre, grads=made, workspace=ws)
    for scale in (1.0, -0.5, 2.0):
        i["x"].mul_(scale)
        for t in (out, pre, *made):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        eager_pre = torch.empty_like(pre)
        assert torch.equal(out, ll.ll_projection_fwd(i["x"], i["w"], i["b"], i["r"], ll.LL_ACT_SILU, eager_pre))
        eager = ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU, eager_pre)
        assert all(torch.equal(a, b) for a, b in zip(made, eager))


def test_refusals():
    from paper_2506_04761_amd import block as ll
    import torch
    i = _inputs(1, 4, 8, 16, "bf16", None)
    f = ll.ll_projection_fwd
    with pytest.raises(ValueError, match="weight has shape"):
        f(i["x"][:, :7], i["w"])
    with pytest.raises(TypeError, match="weight must be"):
        f(i["x"], i["w"].float())
    with pytest.raises(TypeError, match="bias must be"):
        f(i["x"], i["w"], i["b"].bfloat16())
    with pytest.raises(ValueError, match="residual has shape"):
        f(i["x"], i["w"], None, i["r"][:, 1:])
    with pytest.raises(ValueError, match="adjacent channels"):
        f(i["x"].t().contiguous().t(), i["w"])
    with pytest.raises(TypeError, match="device tensor"):
        f(i["x"].cpu(), i["w"])
    with pytest.raises(TypeError, match="unsupported dtype"):
        f(i["x"].half(), i["w"].half())
    with pytest.raises(ValueError, match="out has shape"):
        f(i["x"], i["w"], out=torch.empty((4, 8), device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ll.LLError):  # no rows
        f(i["x"][:0], i["w"])
    with pytest.raises(ll.LLError):  # an activation's gradient needs its sums
        ll.ll_projection_bwd(i["x"], i["w"], i["b"], i["dy"], ll.LL_ACT_SILU)
    with pytest.raises(ll.LLError):  # no such activation
        f(i["x"], i["w"], act=7)
    big = _inputs(1, 300, 4096, 64, "bf16", None)
    with pytest.raises(ll.LLError):
        f(big["x"], big["w"], workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
