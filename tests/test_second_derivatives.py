"""Gradients that kernels form have no graph: where a backward runs for a graph of itself, what differentiates its
results fails, and everything else stays as it is."""

import pytest

torch = pytest.importorskip("torch")
ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")


class _Square(torch.autograd.Function):
    """x^2 and y^2, with gradients outside the graph, of which the second may be None."""

    @staticmethod
    def forward(ctx, x, y):
        ctx.save_for_backward(x, y)
        return x * x, y * y

    @staticmethod
    def backward(ctx, dx, dy):
        x, y = ctx.saved_tensors
        with torch.no_grad():
            grads = (2 * x * dx, 2 * y * dy if ctx.needs_input_grad[1] else None)
        return ll._lib._once(grads)


@pytest.mark.parametrize("both", [True, False])
def test_first_derivatives_stay(both):
    x, y = torch.tensor([3.0], requires_grad=True), torch.tensor([4.0], requires_grad=both)
    for graph in (False, True):
        wanted = (x, y) if both else (x,)
        u, v = _Square.apply(x, y)
        g = torch.autograd.grad((u + v).sum(), wanted, create_graph=graph)
        assert [t.item() for t in g] == [6.0, 8.0][:len(wanted)] and all(t.requires_grad == graph for t in g)
        # as numbers they are of use in a graph too
        h, = torch.autograd.grad((g[0].detach() * x).sum(), x)
        assert h.item() == 6.0


def test_second_derivatives_fail():
    x, y = torch.tensor([3.0], requires_grad=True), torch.tensor([4.0], requires_grad=True)
    for scale in (1.0, x):  # whether what comes in depends on x or not
        g, _ = torch.autograd.grad((scale * sum(_Square.apply(x, y))).sum(), (x, y), create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            (g * x).sum().backward()
