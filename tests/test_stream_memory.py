"""Memory that a call with `stream` allocates by itself belongs to that stream: a block of the current stream could be
handed out there again, or still be in use there, while the kernels run on the other one.

Without a GPU the allocations are watched: CPU tensors, an entry point that does nothing in place of each of the
library's, and a context in place of torch.cuda.stream.  On the GPU the results are."""

import contextlib
import inspect

import pytest

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")


class _Side:
    cuda_stream, device = 1234, None


def _calls(t):
    """name -> (wrapper, its arguments); `t(*shape)` makes a tensor, `t.f32` a float32 one.  Nothing that a wrapper
    can allocate is passed."""
    B, T, D, N, H, d, L = 2, 8, 8, 4, 1, 16, 4
    x, f = t(B, T, D), t.f32
    w, bias, A, BC = f(D, 4), f(D), f(D, N), t(B, T, N)
    q, la, lam = t(B, T, H, d), f(B, T, H), f(B, T, H, L)
    states, stats = t.u8(1 << 20), f(B, 2, 2)
    one, s = t(B, H, d), f(B, D, N)
    return {
        "ll_causal_conv_fwd": (x, w), "ll_causal_conv_step": (x[:, 0], w, None, t(B, 3, D)),
        "ll_causal_conv_bwd": (x, w, bias, x, 1, t(B, 3, D)),
        "ll_selective_scan_fwd": (x, x, A, BC, BC), "ll_selective_scan_step": (x[:, 0], x[:, 0], A, BC[:, 0], BC[:, 0], s),
        "ll_selective_scan_bwd": (x, x, A, BC, BC, states, x, bias, x, bias, True, None, None, True),
        "ll_group_norm_fwd": (x, 2), "ll_group_norm_bwd": (x, 2, bias, bias, stats, x, x),
        "ll_mamba2_fwd": (q, q, q, la, lam, 16), "ll_mamba2_fwd_grouped": (q, q, q, la, lam, 16),
        "ll_mamba2_fwd_matrix_lambda": (q, q, q, la, f(B, T, H, L, d), 16), "ll_mamba2_bwd": (q, q, q, la, lam, q, 16),
        "ll_mamba2_decode_step": (one, one, one, f(B, H), None, states, 0, L),
        "ll_gdn_fwd": (q, q, q, la, la, lam, 16), "ll_gdn_decode_step": (one, one, one, f(B, H), f(B, H), None, states, 0, L),
    }


class _Cpu:
    def __call__(self, *shape):
        return self.f32(*shape)

    def f32(self, *shape):
        import torch
        return torch.zeros(shape)

    def u8(self, n):
        import torch
        return torch.zeros(n, dtype=torch.uint8)


class _Lib:
    """Every entry point succeeds, every size is 256."""

    def __getattr__(self, name):
        return lambda *a: 256 if name.endswith(("_size", "_bytes")) else 0


def test_every_wrapper_with_a_stream_is_called_here():
    named = {n for n in dir(ll) if n.startswith("ll_") and "stream" in inspect.signature(getattr(ll, n)).parameters}
    # no memory of their own: the caller's states, scratch and workspaces; staged forms share the others' code; a debug map
    own = {"ll_mamba2_decode_init", "ll_gdn_decode_init", "ll_mamba2_fwd_noalloc", "ll_mamba2_bwd_after_fwd",
           "ll_debug_level_map"}
    assert {n for n in named if not n.endswith("_staged")} - own == set(_calls(_Cpu()))


@pytest.mark.parametrize("name", sorted(_calls(_Cpu())))
def test_allocations_are_made_under_the_stream(name, monkeypatch):
    import torch
    from torch.utils._python_dispatch import TorchDispatchMode
    from paper_2506_04761_amd import _layer, _lib
    within, elsewhere, recorded = [], [], []
    active = []

    @contextlib.contextmanager
    def stream(s):
        active.append(s)
        yield
        active.pop()

    class Watch(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            out = func(*args, **(kwargs or {}))
            if "empty" in str(func):
                (within if active else elsewhere).append(out.data_ptr())
            return out

    def rows(t, name, dtype, shape):
        return t.stride()

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: recorded.append((self.data_ptr(), s)))
    for m in (_layer, _lib):
        monkeypatch.setattr(m, "lib", _Lib())
        monkeypatch.setattr(m, "_check", lambda *a, **k: None)
        monkeypatch.setattr(m, "_stream", lambda stream: 0)
    monkeypatch.setattr(_layer, "_rows", rows)
    args = _calls(_Cpu())[name]
    with Watch():
        out = getattr(ll, name)(*args, stream=_Side)
    assert not elsewhere and within
    # what the caller gets may be used on the current stream when it dies
    outs = [out] if isinstance(out, torch.Tensor) else [t for t in out if t is not None]
    assert sorted(recorded) == sorted((t.data_ptr(), "current") for t in outs)
    within.clear()
    with Watch():
        getattr(ll, name)(*args)
    assert elsewhere and not within


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["ll_causal_conv_bwd", "ll_selective_scan_fwd", "ll_selective_scan_bwd", "ll_group_norm_fwd",
                                  "ll_group_norm_bwd", "ll_mamba2_fwd", "ll_mamba2_bwd", "ll_gdn_fwd"])
def test_results_on_another_stream_with_memory_of_its_own(name):
    """Two streams, each behind other work, and allocations on the current stream meanwhile, which are written at once."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator("cuda").manual_seed(5)

    def r(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

    B, T, D, N, H, d = 2, 640, 256, 16, 2, 128
    x, dt, z, dy, BC = r(B, T, D), r(B, T, D, scale=0.5), r(B, T, D), r(B, T, D), r(B, T, 2 * N)
    w, bias = torch.randn((D, 4), generator=g, device="cuda"), torch.randn(D, generator=g, device="cuda")
    A = -torch.exp(torch.randn((D, N), generator=g, device="cuda"))
    scan = (x, dt, A, BC[..., :N], BC[..., N:])
    states, stats = ll.ll_selective_scan_states(x, scan[3]), ll.ll_group_norm_stats(x, 8)
    ll.ll_selective_scan_fwd(*scan, bias, z, bias, states=states)
    ll.ll_group_norm_fwd(x, 8, w[:, 0].contiguous(), bias, stats=stats)
    q, k, v = (r(B, T, H, d, scale=0.1) for _ in range(3))
    la, lam = -torch.rand((B, T, H), generator=g, device="cuda"), torch.rand((B, T, H, ll.ll_num_levels(T)), generator=g, device="cuda")
    args = {
        "ll_causal_conv_bwd": (x, w, bias, dy), "ll_selective_scan_fwd": (*scan, bias, z, bias),
        "ll_selective_scan_bwd": (*scan, states, dy, bias, z, bias), "ll_group_norm_fwd": (x, 8, w[:, 0].contiguous(), bias),
        "ll_group_norm_bwd": (x, 8, w[:, 0].contiguous(), bias, stats, dy), "ll_mamba2_fwd": (q, k, v, la, lam, 64),
        "ll_mamba2_bwd": (q, k, v, la, lam, v, 64), "ll_gdn_fwd": (q, k, v, la, torch.sigmoid(la), lam, 64),
    }[name]
    fn = getattr(ll, name)

    def listed(out):
        return [out] if isinstance(out, torch.Tensor) else [t for t in out if t is not None]

    want = [t.clone() for t in listed(fn(*args))]
    work = torch.ones((4096, 4096), device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            for _ in range(4):
                work @ work  # a few ms
        outs.append(listed(fn(*args, stream=s)))
        junk = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 8, 1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 22)]
        del junk
    torch.cuda.synchronize()
    for out in outs:
        assert len(out) == len(want)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
