"""The operators as a block uses them: a projection to queries, keys, values and a gate, attention over its columns, the
group norm of the heads with the gate, and a projection back with the residual.  A prompt of several lengths goes on token by
token as one pass does; gradients of every parameter are those of the same block in 64 bits."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2506_04761_amd  # noqa: F401  (fails loudly if the library is missing)


H, HQK, DK, DV, D = 4, 2, 32, 48, 72
COLS = 2 * HQK * DK + 2 * H * DV


def _parameters(dtype):
    import torch
    r = np.random.default_rng(3)

    def new(*shape, scale=1.0):
        return torch.from_numpy(r.standard_normal(shape) * scale).float().cuda()

    return {"into": new(COLS, D, scale=D ** -0.5).to(dtype), "into_b": new(COLS, scale=0.1),
            "out": new(D, H * DV, scale=(H * DV) ** -0.5).to(dtype), "norm_w": 1 + new(H * DV, scale=0.1),
            "norm_b": new(H * DV, scale=0.1), "ld": -torch.exp2(torch.arange(H).float().cuda() - 7)}


def _split(p):
    a, b = HQK * DK, 2 * HQK * DK
    return (p[..., :a].unflatten(-1, (HQK, DK)), p[..., a:b].unflatten(-1, (HQK, DK)),
            p[..., b:b + H * DV].unflatten(-1, (H, DV)), p[..., b + H * DV:])


def _block(w, x, state=None, lengths=None):
    """x [B, T, D]; (y, final state)."""
    import paper_2506_04761_amd as ll
    q, k, v, gate = _split(ll.projection(x, w["into"], w["into_b"]))
    o, final = ll.decay_attention(q, k, v, w["ld"], DK ** -0.5, state, lengths, return_final_state=True)
    rows = x.shape[0] * x.shape[1]
    o = ll.group_norm(o.reshape(rows, 1, H * DV), H, w["norm_w"], w["norm_b"], gate.reshape(rows, 1, H * DV))
    return ll.projection(o.view(*x.shape[:2], H * DV), w["out"], residual=x), final


def _reference(w, x, state, lengths):
    """The same in 64 bits, token by token."""
    import torch
    q, k, v, gate = _split(x @ w["into"].T + w["into_b"])
    q, k = (t.repeat_interleave(H // HQK, 2) for t in (q, k))
    g = torch.exp(w["ld"])[:, None, None]
    ys, ends = [], []
    for b in range(x.shape[0]):
        S, os = state[b], []
        for t in range(lengths[b]):
            S = g * S + k[b, t, :, :, None] * v[b, t, :, None, :]
            os.append(DK ** -0.5 * (q[b, t, :, :, None] * S).sum(1))
        o = torch.stack(os + [torch.zeros_like(os[0])] * (x.shape[1] - lengths[b]))
        ys.append(o)
        ends.append(S)
    o = torch.stack(ys)
    o = (o - o.mean(-1, keepdim=True)) / torch.sqrt(o.var(-1, correction=0, keepdim=True) + 1e-5)
    o = (o.flatten(2) * w["norm_w"] + w["norm_b"]) * (gate * torch.sigmoid(gate))
    return o @ w["out"].T + x, torch.stack(ends)


def test_gradients_of_a_block():
    """float32: about 1e3 roundings of 2^-24 a value, of terms a few times the largest result."""
    import torch
    r = np.random.default_rng(1)
    lengths = [70, 33]
    w = _parameters(torch.float32)
    x = torch.from_numpy(r.standard_normal((2, 70, D))).float().cuda()
    x[1, 33:] = 0
    state = torch.from_numpy(r.standard_normal((2, H, DK, DV))).float().cuda()
    dy = torch.from_numpy(r.standard_normal((2, 70, D))).float().cuda()
    dy[1, 33:] = 0
    ds = torch.from_numpy(r.standard_normal((2, H, DK, DV))).float().cuda()
    leaves = {**{k: t for k, t in w.items() if k != "ld"}, "x": x, "state": state}
    for t in leaves.values():
        t.requires_grad_()
    y, end = _block(w, x, state, torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    ((y * dy).sum() + (end * ds).sum()).backward()
    w64 = {k: t.detach().double().cpu().requires_grad_(k != "ld") for k, t in w.items()}
    x64, s64 = (t.detach().double().cpu().requires_grad_() for t in (x, state))
    y64, end64 = _reference(w64, x64, s64, lengths)
    ((y64 * dy.double().cpu()).sum() + (end64 * ds.double().cpu()).sum()).backward()
    for b, n in enumerate(lengths):
        assert (y[b, :n].double().cpu() - y64[b, :n]).abs().max() <= 2e-5 * y64.abs().max()
    assert (end.double().cpu() - end64).abs().max() <= 2e-5 * end64.abs().max()
    for name, t in leaves.items():
        want = {**w64, "x": x64, "state": s64}[name].grad
        assert (t.grad.double().cpu() - want).abs().max() <= 1e-4 * want.abs().max(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_goes_on_token_by_token(dtype):
    import paper_2506_04761_amd as ll
    import torch
    from tests.gpu_util import torch_dtype
    block = ll.block
    w = _parameters(torch_dtype(dtype))
    prompts, more = [150, 1, 77], 12
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn((3, max(prompts) + more, D), generator=g, device="cuda").to(torch_dtype(dtype))
    with torch.no_grad():
        n = torch.tensor(prompts, dtype=torch.int32, device="cuda")
        want, end = _block(w, x, lengths=n + more)
        _, state = _block(w, x[:, :max(prompts)], lengths=n)
        got = []
        for t in range(more):
            h = torch.stack([x[b, p + t] for b, p in enumerate(prompts)])
            q, k, v, gate = _split(block.ll_projection_fwd(h, w["into"], w["into_b"]))
            o = block.ll_decay_attention_step(q, k, v, w["ld"], state, DK ** -0.5)
            o = ll.ll_group_norm_fwd(o.view(3, 1, H * DV), H, w["norm_w"], w["norm_b"], gate.unsqueeze(1))
            got.append(block.ll_projection_fwd(o.view(3, H * DV), w["out"], residual=h))
    got = torch.stack(got, 1).float()
    want = torch.stack([want[b, p:p + more] for b, p in enumerate(prompts)]).float()
    # bf16: the roundings of the projections, the attention and the norm, each 2^-8 of its values, differ between the two
    # paths where the sums before them do; fp32: as above
    assert (got - want).abs().max() <= (6e-2 if dtype == "bf16" else 2e-5) * want.abs().max()
    assert (state - end).abs().max() <= (2.0 ** -7 if dtype == "bf16" else 2e-5) * end.abs().max()
