"""The operators around a recurrent token mixer, as cases to be timed and checked: the short causal
convolution, the selective state space scan and the group norm with its activation.

Each case is one pass through one operator, as a layer's prompt, training step or single decoded token
makes it.  Tensors have the shapes and strides that a layer's projections leave: x and the gate z are
halves of one projection's rows, the scan's B and C are columns of another's.

`run` computes the operator in plain torch (32 bits, rounded once at the end), or, with `own` set, through
the entry points of paper_2506_04761_amd.  `exact` computes it in 64 bits, token by token, from the
definitions alone.

Definitions, with t a token, d a channel, n a state, W taps, act(v) = v sigmoid(v) or v:
  convolution   y_td = act(b_d + sum_j w_dj x_(t-W+1+j)d); tokens before the first come from a state
  scan          D_td = softplus(dt_td + bias_d), h_tdn = exp(D_td A_dn) h_(t-1)dn + D_td x_td B_tn,
                y_td = (sum_n C_tn h_tdn + skip_d x_td) z_td sigmoid(z_td)
  group norm    y = act(u), or u act(z) with a gate z; u = (x - mean) / sqrt(var + eps) w + b, mean and
                variance over the tokens and the channels of a group
A sequence shorter than its batch's longest ends at its length: outputs after it are zero.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


# ------------------------------------------------------------------------------------ the cases

def _conv(name, kind, B, T, D, W=4, dtype="bf16", act=True, ragged=False):
    c = {"op": "conv", "kind": kind, "dtype": dtype, "B": B, "T": T, "D": D, "W": W, "act": act, "ragged": ragged}
    return {"name": name, **c} if name else c


def _scan(name, kind, B, T, D, N=16, dtype="bf16", gate=True, ragged=False):
    c = {"op": "scan", "kind": kind, "dtype": dtype, "B": B, "T": T, "D": D, "N": N, "gate": gate, "ragged": ragged}
    return {"name": name, **c} if name else c


def _norm(name, kind, N, S, C, G, dtype="bf16", act=True, gate=True):
    c = {"op": "norm", "kind": kind, "dtype": dtype, "N": N, "S": S, "C": C, "G": G, "act": act, "gate": gate}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the convolution of a batch of prompts: 32 heads of 64 channels, 8192 tokens
        _conv("conv_prompt", "fwd", 4, 8192, 2048),
        # its training step at a ragged medium length
        _conv("conv_train", "train", 2, 4032, 2048),
        # one token for 64 sequences
        _conv("conv_step", "step", 64, 1, 2048),
        # one short prompt through one small layer: latency and launches
        _scan("scan_short", "fwd", 1, 320, 512),
        # a layer's prompts at full batch
        _scan("scan_8k", "fwd", 4, 8192, 2048),
        # one long context
        _scan("scan_64k", "fwd", 1, 65536, 2048),
        # float32, sequences of different lengths, an odd number of channels, a cached state to start from
        _scan("scan_f32", "fwd", 3, 1984, 1000, dtype="f32", ragged=True),
        # the training step at a ragged medium length
        _scan("scan_train", "train", 2, 4032, 2048),
        # one token for 64 sequences
        _scan("scan_step", "step", 64, 1, 2048),
        # the mixer's output norm: 16 heads of 128 channels at each of 65536 tokens, gated
        _norm("norm_tokens", "fwd", 65536, 1, 2048, 16),
        # its training step
        _norm("norm_train", "train", 8064, 1, 2048, 16),
        # statistics over the tokens too: 4 sequences of 8192 tokens, 32 groups of 32 channels
        _norm("norm_seq", "fwd", 4, 8192, 1024, 32, gate=False),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v if v != 3072 else v - 1


def _channels(rng):
    """Channel counts from a toy layer to a wide one: multiples of 64 mostly, some odd."""
    d = _log_int(rng, 48, 4160)
    d = d if rng.random() < 0.35 else max(64, d // 64 * 64)
    return d if d != 3072 else d - 64


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    D = _channels(rng)
    if op == "norm":
        kind = rng.choice(["fwd", "train"])
        cg = rng.choice([16, 32, 64, 80, 128, 257])
        G = max(1, min(64, D // cg))
        G -= G * cg == 3072
        C = G * cg
        rows = max(1, min(65536, (1 << 27) // C // (4 if kind == "train" else 1)))
        rows = _log_int(rng, 1, rows)
        S = 1 if rng.random() < 0.6 else _log_int(rng, 1, rows)
        return _norm(None, kind, max(1, rows // S), S, C, G, dtype, act=rng.random() < 0.8, gate=rng.random() < 0.5)
    kind = rng.choice(["fwd", "fwd", "train", "step"])
    if kind == "step":
        B = _log_int(rng, 1, 256)
        if op == "conv":
            return _conv(None, kind, B, 1, D, rng.choice([2, 3, 4]), dtype, act=rng.random() < 0.8)
        return _scan(None, kind, B, 1, D, rng.choice([8, 16, 16, 24]), dtype, gate=rng.random() < 0.8)
    # tokens of the whole batch, up to the work of the largest listed cases
    most = (1 << 26) // D // (4 if kind == "train" else 1)
    N = rng.choice([8, 16, 16, 16, 24]) if op == "scan" else 0
    if N > 16:
        most //= 2
    T = _log_int(rng, 1, min(65536, max(1, most)))
    B = _log_int(rng, 1, max(1, min(32, most // T)))
    ragged = rng.random() < 0.4
    if op == "conv":
        return _conv(None, kind, B, T, D, rng.choice([2, 3, 4]), dtype, act=rng.random() < 0.8, ragged=ragged)
    return _scan(None, kind, B, T, D, N, dtype, gate=rng.random() < 0.8, ragged=ragged)


# ------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _normal(g, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _lengths(case, seed):
    """Lengths of the batch's sequences: the longest fills the batch, the others are shorter, down to none."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return None
    r = torch.Generator().manual_seed(seed + 1)
    n = (torch.rand(B, generator=r) * (T + 1)).to(torch.int32)
    n[0] = T
    return n.cuda()


def _blank(x, lengths):
    """What stands after a sequence's end is no input: it is filled with NaN."""
    if lengths is not None:
        gone = torch.arange(x.shape[1], device=x.device)[None, :] >= lengths[:, None]
        x.masked_fill_(gone.view(*gone.shape, *([1] * (x.dim() - 2))), float("nan"))
    return x


def _conv_inputs(case, seed):
    B, T, D, W, dt = case["B"], case["T"], case["D"], case["W"], DTYPES[case["dtype"]]
    g = _gen(seed)
    s = {"case": case, "lengths": _lengths(case, seed)}
    s["x"] = _blank(_normal(g, (B, T, 2 * D), dt), s["lengths"])[..., :D]  # the other half of the rows is the gate
    s["weight"] = _normal(g, (D, W), scale=1 / math.sqrt(W))
    s["bias"] = _normal(g, (D,), scale=0.1)
    s["initial"] = _normal(g, (B, W - 1, D), dt)
    if case["kind"] == "step":
        s["x"] = s["x"][:, 0]
    if case["kind"] == "train":
        s["initial"] = None
        s["d_y"] = _blank(_normal(g, (B, T, D), dt), s["lengths"])
    return s


def _scan_inputs(case, seed):
    B, T, D, N, dt = case["B"], case["T"], case["D"], case["N"], DTYPES[case["dtype"]]
    R = max(1, D // 16)  # columns of the step sizes' low-rank projection, before those of B and C
    g = _gen(seed)
    s = {"case": case, "lengths": _lengths(case, seed)}
    ln = s["lengths"]
    s["z"] = _blank(_normal(g, (B, T, 2 * D), dt), ln)[..., D:] if case["gate"] else None
    s["x"] = _blank(_normal(g, (B, T, D), dt), ln)
    s["dt"] = _blank(_normal(g, (B, T, D), dt, 0.5), ln)
    p = _blank(_normal(g, (B, T, R + 2 * N), dt), ln)
    s["B"], s["C"] = p[..., R:R + N], p[..., R + N:]
    # channels remember a few to a thousand tokens: step sizes of 0.001 to 0.1, rates about 1 .. N
    s["A"] = -torch.arange(1, N + 1, device="cuda") * torch.exp(_normal(g, (D, N), scale=0.2))
    step = torch.exp(torch.rand(D, generator=g, device="cuda") * math.log(100.0) + math.log(0.001))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["skip"] = 1 + _normal(g, (D,), scale=0.1)
    s["initial"] = _normal(g, (B, D, N), scale=0.5)
    if case["kind"] == "step":
        s.update({k: s[k][:, 0] for k in ("x", "dt", "B", "C")}, z=s["z"][:, 0] if case["gate"] else None)
    if case["kind"] == "train":
        s["initial"] = None
        s["d_y"] = _blank(_normal(g, (B, T, D), dt), ln)
    return s


def _norm_inputs(case, seed):
    N, S, C, dt = case["N"], case["S"], case["C"], DTYPES[case["dtype"]]
    g = _gen(seed)
    s = {"case": case}
    # values with a mean that differs by channel, as a mixer's outputs have
    s["x"] = (_normal(g, (N, S, C)) * 1.5 + _normal(g, (C,), scale=0.5)).to(dt)
    s["gate"] = _normal(g, (N, S, 2 * C), dt)[..., C:] if case["gate"] else None
    s["weight"] = 1 + _normal(g, (C,), scale=0.1)
    s["bias"] = _normal(g, (C,), scale=0.1)
    if case["kind"] == "train":
        s["d_y"] = _normal(g, (N, S, C), dt)
    return s


_INPUTS = {"conv": _conv_inputs, "scan": _scan_inputs, "norm": _norm_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    if own:
        _prepare_own(s)
    return s


# ------------------------------------------------------------------------------------ through the library

def _prepare_own(s):
    """The buffers that a program keeps from call to call: outputs, states and workspaces."""
    import paper_2506_04761_amd as ll
    case = s["case"]
    op, kind = case["op"], case["kind"]
    s["ll"] = ll
    s["act"] = ll.LL_ACT_SILU if op == "scan" or case["act"] else ll.LL_ACT_NONE
    if op == "conv":
        s["out"] = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda")
        s["final"] = torch.empty_like(s["initial"]) if s["initial"] is not None else None
        if kind == "train":
            s["ws"] = ll.ll_causal_conv_bwd_workspace(s["x"], s["weight"])
    elif op == "scan":
        s["out"] = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda")
        s["final"] = torch.empty_like(s["initial"]) if s["initial"] is not None else None
        if kind == "fwd":
            s["ws"] = ll.ll_selective_scan_workspace(s["x"], s["B"])
        if kind == "train":
            s["states"] = ll.ll_selective_scan_states(s["x"], s["B"])
            s["ws"] = ll.ll_selective_scan_workspace(s["x"], s["B"], backward=True)
    else:
        s["out"] = torch.empty_like(s["x"])
        s["ws"] = ll.ll_group_norm_workspace(s["x"], case["G"], backward=kind == "train")
        s["stats"] = ll.ll_group_norm_stats(s["x"], case["G"]) if kind == "train" else None


def _own_conv(s):
    ll, kind = s["ll"], s["case"]["kind"]
    if kind == "step":
        y = ll.ll_causal_conv_step(s["x"], s["weight"], s["bias"], s["initial"], act=s["act"], new_state=s["final"],
                                   out=s["out"])
        return {"y": y, "state": s["final"]}
    y = ll.ll_causal_conv_fwd(s["x"], s["weight"], s["bias"], act=s["act"], initial_state=s["initial"],
                              final_state=s["final"], lengths=s["lengths"], out=s["out"])
    if kind == "fwd":
        return {"y": y, "state": s["final"]}
    g = ll.ll_causal_conv_bwd(s["x"], s["weight"], s["bias"], s["d_y"], act=s["act"], lengths=s["lengths"],
                              workspace=s["ws"])
    return {"y": y, "dx": g.x, "dweight": g.weight, "dbias": g.bias}


def _own_scan(s):
    ll, kind = s["ll"], s["case"]["kind"]
    a = (s["x"], s["dt"], s["A"], s["B"], s["C"])
    more = {"D": s["skip"], "z": s["z"], "dt_bias": s["dt_bias"]}
    if kind == "step":
        y = ll.ll_selective_scan_step(*a, s["initial"], **more, new_state=s["final"], out=s["out"])
        return {"y": y, "state": s["final"]}
    if kind == "fwd":
        y = ll.ll_selective_scan_fwd(*a, **more, initial_state=s["initial"], final_state=s["final"],
                                     lengths=s["lengths"], out=s["out"], workspace=s["ws"])
        return {"y": y, "state": s["final"]}
    y = ll.ll_selective_scan_fwd(*a, **more, lengths=s["lengths"], states=s["states"], out=s["out"],
                                 workspace=s["ws"])
    g = ll.ll_selective_scan_bwd(*a, s["states"], s["d_y"], **more, lengths=s["lengths"], workspace=s["ws"])
    out = {"y": y, "dx": g.x, "ddt": g.dt, "dA": g.A, "dB": g.B, "dC": g.C, "dskip": g.D, "ddt_bias": g.dt_bias}
    if s["z"] is not None:
        out["dz"] = g.z
    return out


def _own_norm(s):
    ll, case = s["ll"], s["case"]
    a = (s["x"], case["G"], s["weight"], s["bias"])
    y = ll.ll_group_norm_fwd(*a, gate=s["gate"], eps=EPS, act=s["act"], stats=s["stats"], out=s["out"],
                             workspace=s["ws"])
    if case["kind"] == "fwd":
        return {"y": y}
    g = ll.ll_group_norm_bwd(*a, s["stats"], s["d_y"], gate=s["gate"], act=s["act"], workspace=s["ws"])
    out = {"y": y, "dx": g.x, "dweight": g.weight, "dbias": g.bias}
    if s["gate"] is not None:
        out["dgate"] = g.gate
    return out


# ------------------------------------------------------------------------------------ the plain form

def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _act(v, on):
    return v * _sigmoid(v) if on else v


def _act_grad(v, on):
    if not on:
        return torch.ones_like(v)
    p = _sigmoid(v)
    return p * (1 + v * (1 - p))


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _live(case, lengths):
    """Which tokens are inputs, [B, T, 1]; None where all are."""
    if lengths is None:
        return None
    return (torch.arange(case["T"], device="cuda")[None, :] < lengths[:, None])[..., None]


def _only(x, live):
    return x if live is None else torch.where(live, x, torch.zeros((), device=x.device, dtype=x.dtype))


def _tail(ext, lengths, T, W):
    """The W - 1 tokens before each sequence's end, of the sequence with its state in front."""
    if lengths is None:
        return ext[:, T:]
    at = lengths.long()[:, None] + torch.arange(W - 1, device=ext.device)
    return torch.gather(ext, 1, at[..., None].expand(-1, -1, ext.shape[2]))


def _plain_conv(s):
    case, x, w, b = s["case"], s["x"], s["weight"], s["bias"]
    W, kind, on = case["W"], case["kind"], case["act"]
    if kind == "step":
        x = x[:, None]
    live = _live(case, s["lengths"])
    xf = _only(x.float(), live)
    first = s["initial"].float() if s["initial"] is not None else xf.new_zeros((xf.shape[0], W - 1, xf.shape[2]))
    ext = torch.cat([first, xf], 1)
    T = xf.shape[1]
    v = b.expand_as(xf).clone()
    for j in range(W):
        v += w[:, j] * ext[:, j:j + T]
    y = _only(_act(v, on), live).to(x.dtype)
    if kind != "train":
        return {"y": y[:, 0] if kind == "step" else y, "state": _tail(ext, s["lengths"], T, W).to(x.dtype)}
    dv = _only(_only(s["d_y"].float(), live) * _act_grad(v, on), live)
    dext = torch.zeros_like(ext)
    dw = []
    for j in range(W):
        dext[:, j:j + T] += w[:, j] * dv
        dw.append((dv * ext[:, j:j + T]).sum((0, 1)))
    return {"y": y, "dx": dext[:, W - 1:].to(x.dtype), "dweight": torch.stack(dw, 1), "dbias": dv.sum((0, 1))}


SPAN = 256  # tokens that the plain scan works on at a time


def _doubling(a, h):
    """h_i += a_i h_(i-1) along the first axis, in rounds of doubled reach; a is used up."""
    k = 1
    while k < h.shape[0]:
        h[k:] += a[k:] * h[:-k]
        if 2 * k < h.shape[0]:
            a[k:] = a[k:] * a[:-k]
        k *= 2
    return h


def _plain_scan(s):
    case = s["case"]
    kind, A = case["kind"], s["A"]
    names = ("x", "dt", "B", "C") + (("z",) if s["z"] is not None else ())
    live = _live(case, s["lengths"])
    f = {}
    for k in names:
        v = s[k] if kind != "step" else s[k][:, None]
        # token first; what is no input has a step size of zero and leaves the state as it is
        f[k] = _only(v.float(), live).transpose(0, 1).contiguous()
    pre = f["dt"] + s["dt_bias"]
    delta = _softplus(pre)
    if live is not None:
        delta = _only(delta, live.transpose(0, 1))
    x, Bm, Cm = f["x"], f["B"], f["C"]
    T, nb, D = x.shape
    h0 = s["initial"].clone() if s["initial"] is not None else x.new_zeros((nb, D, A.shape[1]))
    y = torch.empty_like(x)
    keep = x.new_empty((T, *h0.shape)) if kind == "train" else None  # every state, for the gradients
    h = h0
    for t in range(0, T, SPAN):
        r = slice(t, min(T, t + SPAN))
        a = torch.exp(delta[r, ..., None] * A)
        u = (delta[r] * x[r])[..., None] * Bm[r, :, None]
        u[0] += a[0] * h
        u = _doubling(a, u)
        y[r] = (u * Cm[r, :, None]).sum(-1)
        h = u[-1].clone()
        if keep is not None:
            keep[r] = u
    inner = y + s["skip"] * x
    out = inner * _act(f["z"], True) if "z" in f else inner
    out = _only(out.transpose(0, 1), live).to(s["x"].dtype)
    if kind != "train":
        return {"y": out[:, 0] if kind == "step" else out.contiguous(), "state": h}
    dy = _only(s["d_y"].float(), live).transpose(0, 1)
    got = {}
    if "z" in f:
        got["dz"] = dy * inner * _act_grad(f["z"], True)
        dy = dy * _act(f["z"], True)
    dx, ddelta = torch.empty_like(x), torch.empty_like(x)
    dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
    dA = torch.zeros_like(A)
    carry = torch.zeros_like(h0)
    for t in range((T - 1) // SPAN * SPAN, -1, -SPAN):
        r = slice(t, min(T, t + SPAN))
        a = torch.exp(delta[r, ..., None] * A)
        g = dy[r, ..., None] * Cm[r, :, None]
        g[-1] += carry
        # g_t += a_(t+1) g_(t+1): the same rounds, backwards
        g = _doubling(torch.cat([a[1:], torch.zeros_like(a[:1])]).flip(0), g.flip(0)).flip(0)
        carry = a[0] * g[0]
        before = torch.cat([(keep[t - 1] if t else h0)[None], keep[t:r.stop - 1]])
        q = a * before * g
        gb = (g * Bm[r, :, None]).sum(-1)
        dx[r] = gb * delta[r]
        ddelta[r] = gb * x[r] + (q * A).sum(-1)
        dA += (q * delta[r, ..., None]).sum((0, 1))
        dB[r] = (g * (delta[r] * x[r])[..., None]).sum(2)
        dC[r] = (keep[r] * dy[r, ..., None]).sum(2)
    ddt = ddelta * _sigmoid(pre)
    if live is not None:
        ddt = _only(ddt, live.transpose(0, 1))
    got.update(dx=dx + s["skip"] * dy, ddt=ddt, dB=dB, dC=dC)
    got = {k: v.transpose(0, 1).to(s["x"].dtype) for k, v in got.items()}
    return {"y": out, "dA": dA, "dskip": (dy * x).sum((0, 1)), "ddt_bias": ddt.sum((0, 1)), **got}


def _plain_norm(s):
    case, x = s["case"], s["x"]
    G, on = case["G"], case["act"]
    N, S, C = x.shape
    w, b = s["weight"], s["bias"]
    v = x.float().view(N, S, G, C // G)
    mean = v.mean((1, 3), keepdim=True)
    c = v - mean
    rstd = 1 / torch.sqrt((c * c).mean((1, 3), keepdim=True) + EPS)
    xh = (c * rstd).view(N, S, C)
    u = xh * w + b
    z = s["gate"].float() if s["gate"] is not None else None
    y = _act(u, on) if z is None else u * _act(z, on)
    if case["kind"] == "fwd":
        return {"y": y.to(x.dtype)}
    dy = s["d_y"].float()
    out = {"y": y.to(x.dtype)}
    if z is None:
        du = dy * _act_grad(u, on)
    else:
        out["dgate"] = (dy * u * _act_grad(z, on)).to(x.dtype)
        du = dy * _act(z, on)
    g = (du * w).view(N, S, G, C // G)
    xg = xh.view(N, S, G, C // G)
    dx = rstd * (g - g.mean((1, 3), keepdim=True) - xg * (g * xg).mean((1, 3), keepdim=True))
    out.update(dx=dx.view(N, S, C).to(x.dtype), dweight=(du * xh).sum((0, 1)), dbias=du.sum((0, 1)))
    return out


_OWN = {"conv": _own_conv, "scan": _own_scan, "norm": _own_norm}
_PLAIN = {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------ the floor

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    train, step = case["kind"] == "train", case["kind"] == "step"
    if case["op"] == "norm":
        n = case["N"] * case["S"] * case["C"]
        tensors = 2 + case["gate"] + (train and 2 + 2 * case["gate"])
        # x, the gate and y; for the gradients d_y, dx and the gate's besides (x and the gate once)
        return {"bytes": n * e * tensors + case["C"] * 4 * (4 if train else 2), "flops": n * (30 if train else 12)}
    n = case["B"] * case["T"] * case["D"]
    if case["op"] == "conv":
        W = case["W"]
        state = 0 if train else 2 * case["B"] * (W - 1) * case["D"] * e
        params = case["D"] * (W + 1) * 4 * (2 if train else 1)
        return {"bytes": n * e * (4 if train else 2) + state + params,
                "flops": n * ((6 * W + 12) if train else (2 * W + 4))}
    N, gate = case["N"], case["gate"]
    rows = case["B"] * case["T"] * 2 * N * e  # B and C
    tensors = 3 + gate + (train and 3 + gate)
    state = 0 if train else 2 * case["B"] * case["D"] * N * 4
    params = case["D"] * (N + 2) * 4 * (2 if train else 1)
    # a state and token: the rate's product, exp, the input's product, the state's and the output's sums;
    # the gradients: the state again, its gradient, and the sums for x, dt, A, B, C
    flops = n * N * (24 if train else 7) + n * (40 if train else 20)
    return {"bytes": n * e * tensors + rows * (2 if train else 1) + state + params, "flops": flops}


# ------------------------------------------------------------------------------------ 64 bits

def _exact_conv(case, s):
    d = torch.float64
    x, w, b = s["x"].to(d), s["weight"].to(d), s["bias"].to(d)
    W, kind = case["W"], case["kind"]
    x = x[:, None] if kind == "step" else x
    nb, T, D = x.shape
    first = s["initial"].to(d) if s["initial"] is not None else None
    n = s["lengths"].tolist() if s["lengths"] is not None else [T] * nb
    act = (lambda v: v * torch.sigmoid(v)) if case["act"] else (lambda v: v)
    y, state = torch.zeros_like(x), torch.zeros((nb, W - 1, D), dtype=d, device="cuda")
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(b)
    for i in range(nb):
        seq = torch.zeros((W - 1 + n[i], D), dtype=d, device="cuda")
        if first is not None:
            seq[:W - 1] = first[i]
        seq[W - 1:] = x[i, :n[i]]
        state[i] = seq[n[i]:]
        if n[i] == 0:
            continue
        win = seq.unfold(0, W, 1)  # [tokens, D, W]
        v = (win * w).sum(-1) + b
        y[i, :n[i]] = act(v)
        if kind == "train":
            p = torch.sigmoid(v)
            dv = s["d_y"][i, :n[i]].to(d) * (p + v * p * (1 - p) if case["act"] else 1.0)
            dw += (dv[..., None] * win).sum(0)
            db += dv.sum(0)
            pad = torch.cat([dv, dv.new_zeros((W - 1, D))])
            dx[i, :n[i]] = (pad.unfold(0, W, 1) * w.flip(1)).sum(-1)
    if kind == "train":
        return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
    return {"y": y[:, 0] if kind == "step" else y, "state": state}


def _exact_scan(case, s):
    d = torch.float64
    kind = case["kind"]
    get = (lambda k: s[k][:, None].to(d)) if kind == "step" else (lambda k: s[k].to(d))
    x, dt, Bm, Cm = (get(k) for k in ("x", "dt", "B", "C"))
    nb, T, D = x.shape
    A, skip, bias = s["A"].to(d), s["skip"].to(d), s["dt_bias"].to(d)
    dead = torch.zeros((nb, T, 1), dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        dead = torch.arange(T, device="cuda").view(1, T, 1) >= s["lengths"].view(-1, 1, 1)
    x, Bm, Cm = (v.masked_fill(dead, 0) for v in (x, Bm, Cm))
    pre = dt + bias
    delta = torch.where(pre > 30, pre, torch.log1p(torch.exp(pre.clamp(max=30)))).masked_fill(dead, 0)
    h = s["initial"].to(d) if s["initial"] is not None else torch.zeros((nb, D, A.shape[1]), dtype=d, device="cuda")
    hs = torch.empty((T + 1, *h.shape), dtype=d, device="cuda") if kind == "train" else None
    if kind == "train":
        hs[0] = h
    y = torch.empty_like(x)
    xd = x * delta
    for t in range(T):
        h = torch.addcmul(xd[:, t, :, None] * Bm[:, t, None], torch.exp(delta[:, t, :, None] * A), h)
        y[:, t] = (h * Cm[:, t, None]).sum(-1)
        if kind == "train":
            hs[t + 1] = h
    inner = y + skip * x
    z = get("z").masked_fill(dead, 0) if s["z"] is not None else None
    out = (inner * z * torch.sigmoid(z) if z is not None else inner).masked_fill(dead, 0)
    if kind != "train":
        return {"y": out[:, 0] if kind == "step" else out, "state": h}
    dy = s["d_y"].to(d).masked_fill(dead, 0)
    got = {}
    if z is not None:
        p = torch.sigmoid(z)
        got["dz"] = dy * inner * (p + z * p * (1 - p))
        dy = dy * z * p
    dx, dd = torch.empty_like(x), torch.empty_like(x)
    dB, dC, dA = torch.empty_like(Bm), torch.empty_like(Cm), torch.zeros_like(A)
    g = torch.zeros_like(h)
    for t in range(T - 1, -1, -1):
        g = g + dy[:, t, :, None] * Cm[:, t, None]
        dC[:, t] = (dy[:, t, :, None] * hs[t + 1]).sum(1)
        dB[:, t] = (g * xd[:, t, :, None]).sum(1)
        along = (g * Bm[:, t, None]).sum(-1)
        dx[:, t] = along * delta[:, t]
        g = g * torch.exp(delta[:, t, :, None] * A)
        gh = g * hs[t]
        dd[:, t] = along * x[:, t] + (gh * A).sum(-1)
        dA += (gh * delta[:, t, :, None]).sum(0)
    ddt = (dd * torch.sigmoid(pre)).masked_fill(dead, 0)
    return {"y": out, "dx": dx + skip * dy, "ddt": ddt, "dA": dA, "dB": dB, "dC": dC,
            "dskip": (dy * x).sum((0, 1)), "ddt_bias": ddt.sum((0, 1)), **got}


def _exact_norm(case, s):
    d = torch.float64
    x = s["x"].to(d)
    N, S, C = x.shape
    G = case["G"]
    v = x.reshape(N, S, G, C // G)
    var, mean = torch.var_mean(v, (1, 3), correction=0, keepdim=True)
    inv = (var + EPS) ** -0.5
    xh = (v - mean) * inv
    wg, bg = s["weight"].to(d).view(G, -1), s["bias"].to(d).view(G, -1)
    u = xh * wg + bg
    f = (lambda v: v * torch.sigmoid(v)) if case["act"] else (lambda v: v)

    def df(v):
        p = torch.sigmoid(v)
        return p + v * p * (1 - p) if case["act"] else torch.ones_like(v)

    z = s["gate"].to(d).reshape(v.shape) if s["gate"] is not None else None
    y = f(u) if z is None else u * f(z)
    out = {"y": y.reshape(N, S, C)}
    if case["kind"] == "train":
        dy = s["d_y"].to(d).view(v.shape)
        if z is None:
            du = dy * df(u)
        else:
            out["dgate"] = (dy * u * df(z)).reshape(N, S, C)
            du = dy * f(z)
        out["dweight"], out["dbias"] = (du * xh).sum((0, 1)).reshape(C), du.sum((0, 1)).reshape(C)
        # x enters through its own centred value, the mean and the variance
        dxh = du * wg
        M = S * (C // G)
        dvar = (-0.5 * inv ** 3 * (dxh * (v - mean)).sum((1, 3), keepdim=True))
        dmean = -(dxh * inv).sum((1, 3), keepdim=True)
        out["dx"] = (dxh * inv + dvar * 2 * (v - mean) / M + dmean / M).reshape(N, S, C)
    return out


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm}[case["op"]](case, s)
