"""Memory that a call of the block's operators allocates by itself belongs to the stream it runs on: without a GPU the
allocations are watched (CPU tensors, an entry point that does nothing in place of each of the library's, a context in
place of torch.cuda.stream), on the GPU the results are."""

import contextlib
import inspect

import pytest

block = pytest.importorskip("paper_2506_04761_amd.block", reason="libloglinear.so not built")


def _calls(t, u8):
    """name -> the wrapper's arguments, nothing that it can allocate among them; t(*shape) float32, u8(n) bytes."""
    B, T, H, d, M, K, N = 2, 640, 2, 16, 600, 2048, 24
    q, ld, state = t(B, T, H, d), t(H), t(B, H, d, d)
    x, w, b, y = t(M, K), t(N, K), t(N), t(M, N)
    return {
        "ll_decay_attention_fwd": (q, q, q, ld), "ll_decay_attention_step": (q[:, 0], q[:, 0], q[:, 0], ld, state),
        "ll_decay_attention_bwd": (q, q, q, ld, u8(1 << 20), q, 1.0, None, state, True),
        "ll_projection_fwd": (x, w, b), "ll_projection_bwd": (x, w, b, y, block.LL_ACT_SILU, y),
    }


def _cpu_calls():
    import torch
    return _calls(lambda *s: torch.zeros(s), lambda n: torch.zeros(n, dtype=torch.uint8))


class _Lib:
    def __getattr__(self, name):
        return lambda *a: 256 if name.endswith(("_size", "_bytes")) else 0


def test_every_wrapper_with_a_stream_is_called_here():
    named = {n for n in dir(block) if n.startswith("ll_") and "stream" in inspect.signature(getattr(block, n)).parameters}
    assert named == set(_cpu_calls())


@pytest.mark.parametrize("name", sorted(_cpu_calls()))
def test_allocations_are_made_under_the_stream(name, monkeypatch):
    import torch
    from torch.utils._python_dispatch import TorchDispatchMode
    from paper_2506_04761_amd import _layer, _lib
    within, elsewhere, recorded, active = [], [], [], []

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

    class Side:
        cuda_stream, device = 1234, None

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: recorded.append((self.data_ptr(), s)))
    for m in (block, _layer, _lib):
        monkeypatch.setattr(m, "lib", _Lib())
        monkeypatch.setattr(m, "_check", lambda *a, **k: None)
        monkeypatch.setattr(m, "_stream", lambda stream: 0)
    monkeypatch.setattr(block, "_rows", lambda t, name, dtype, shape: t.stride())
    args = _cpu_calls()[name]
    with Watch():
        out = getattr(block, name)(*args, stream=Side)
    assert not elsewhere and within
    outs = [out] if isinstance(out, torch.Tensor) else [t for t in out if t is not None]
    assert sorted(recorded) == sorted((t.data_ptr(), "current") for t in outs)
    within.clear()
    with Watch():
        getattr(block, name)(*args)
    assert elsewhere and not within


@pytest.mark.gpu
@pytest.mark.parametrize("name", sorted(_cpu_calls()))
def test_results_on_another_stream_with_memory_of_its_own(name):
    """Two streams, each behind other work, and allocations on the current stream meanwhile, which are written at once."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator("cuda").manual_seed(5)
    args = list(_calls(lambda *s: torch.randn(s, generator=g, device="cuda"),
                       lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda"))[name])
    if name.startswith("ll_decay"):
        args[3] = -args[3].abs()
    if name == "ll_decay_attention_step":
        def fn(*a, stream=None):
            new = torch.empty_like(a[4])
            return block.ll_decay_attention_step(*a, new_state=new, stream=stream), new
    else:
        fn = getattr(block, name)

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
        if name != "ll_decay_attention_step":  # whose new state is the test's own
            junk = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 8, 1 << 12, 1 << 16, 1 << 18, 1 << 20)]
            del junk
    torch.cuda.synchronize()
    for out in outs:
        assert len(out) == len(want)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
