"""A block around a mixer whose heads forget at a fixed rate, as cases to be timed and checked: linear attention with a
decay for each head, and the projections of such a block: matrix products with bias, activation and residual.

Each case is one pass through one operator, as a layer's prompt, training step or single decoded token makes it.  Tensors
have the shapes and strides that a layer leaves: q, k and v are columns of one projection's rows, and so may the rows be
that a projection takes.

`run` computes the operator in plain torch (32 bits, rounded once at the end), or, with `own` set, through the entry
points of paper_2506_04761_amd.  `exact` computes it in 64 bits from the definitions alone, the attention token by token.

Definitions, with t a token, h a head, g_h = exp(log_decay_h), n a sequence's length:
  decay attention  S_t = g S_(t-1) + k_t v_t^T,  o_t = scale S_t^T q_t,  from an initial state to a final one;
                   heads share queries and keys in groups: head h of H reads head h / (H / H_qk) of those
  projection       u = x W^T + b,  y = act(u) + r,  act(v) = v sigmoid(v) or v
A sequence shorter than its batch's longest ends at its length: outputs after it are zero.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------ the cases

def _attn(name, kind, B, T, H, dk, dv, Hqk=None, dtype="bf16", ragged=False):
    c = {"op": "attn", "kind": kind, "dtype": dtype, "B": B, "T": T, "H": H, "Hqk": Hqk or H, "dk": dk, "dv": dv,
         "ragged": ragged}
    return {"name": name, **c} if name else c


def _proj(name, kind, M, K, N, dtype="bf16", bias=True, act=False, residual=False, wide=False):
    c = {"op": "proj", "kind": kind, "dtype": dtype, "M": M, "K": K, "N": N, "bias": bias, "act": act,
         "residual": residual, "wide": wide}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one short prompt through one small layer: latency and launches
        _attn("attn_short", "fwd", 1, 320, 8, 64, 64),
        # a layer's prompts at full batch, continued from a cache
        _attn("attn_8k", "fwd", 4, 8192, 32, 128, 64),
        # one long context
        _attn("attn_64k", "fwd", 1, 65536, 16, 128, 128),
        # float32, sequences of different lengths, odd head sizes, queries and keys shared by three heads each
        _attn("attn_f32", "fwd", 3, 1984, 12, 40, 72, Hqk=4, dtype="f32", ragged=True),
        # the training step of a padded batch at an odd length
        _attn("attn_train", "train", 4, 4032, 16, 128, 128, ragged=True),
        # one token for 64 sequences
        _attn("attn_step", "step", 64, 1, 16, 128, 128),
        # prompts into a mixer: input and gate of 2048 channels each from 1024
        _proj("proj_prompt", "fwd", 32768, 1024, 4096),
        # the training step of the projection back into the residual stream
        _proj("proj_train", "train", 8064, 2048, 1024, residual=True),
        # the training step of a layer with an activation
        _proj("proj_train_act", "train", 4096, 1024, 2816, act=True),
        # float32 at odd sizes, rows that are columns of wider ones
        _proj("proj_f32", "fwd", 1001, 1000, 1501, dtype="f32", act=True, residual=True, wide=True),
        # one token for 64 sequences
        _proj("proj_step", "fwd", 64, 1024, 4096, act=True),
        # one token for one sequence
        _proj("proj_step1", "fwd", 1, 2048, 1024, residual=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """Channel counts: multiples of 64 mostly, some odd."""
    d = _log_int(rng, lo, hi)
    return d if rng.random() < 0.3 else max(64, d // 64 * 64)


def draw(rng):
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if rng.random() < 0.5:
        kind = rng.choice(["fwd", "fwd", "train"])
        K, N = _width(rng, 48, 8192), _width(rng, 48, 8192)
        # products of the whole batch, up to the work of the largest listed case
        most = (1 << 37) // (K * N) // (4 if kind == "train" else 1) // (8 if dtype == "f32" else 1)
        most = min(most, (1 << 27) // max(K, N))
        M = _log_int(rng, 1, max(1, min(65536, most)))
        return _proj(None, kind, M, K, N, dtype, bias=rng.random() < 0.7, act=rng.random() < 0.5,
                     residual=rng.random() < 0.4, wide=rng.random() < 0.3)
    kind = rng.choice(["fwd", "fwd", "train", "step"])
    dk, dv = (rng.choice([16, 32, 64, 64, 128, 128, 256]) if rng.random() < 0.7 else rng.randint(8, 200) for _ in "kv")
    Hqk = rng.choice([1, 2, 4, 8, 16])
    H = Hqk * rng.choice([1, 1, 2, 3, 6])
    if kind == "step":
        return _attn(None, kind, _log_int(rng, 1, max(1, min(256, (1 << 24) // (H * dk * dv)))), 1, H, dk, dv, Hqk, dtype)
    # tokens of the whole batch, up to the work of the largest listed cases
    most = (1 << 28) // (H * (dk + dv)) // (4 if kind == "train" else 1) // (2 if dtype == "f32" else 1)
    T = _log_int(rng, 1, max(1, min(65536, most)))
    B = _log_int(rng, 1, max(1, min(32, most // T, (1 << 24) // (H * dk * dv))))
    return _attn(None, kind, B, T, H, dk, dv, Hqk, dtype, ragged=rng.random() < 0.4)


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


def _attn_inputs(case, seed):
    B, T, H, Hqk, dk, dv, dt = (case[n] for n in ("B", "T", "H", "Hqk", "dk", "dv", "dtype"))
    dt = DTYPES[dt]
    g = _gen(seed)
    s = {"case": case, "lengths": _lengths(case, seed), "scale": 1 / math.sqrt(dk)}
    rows = _blank(_normal(g, (B, T, 2 * Hqk * dk + H * dv), dt), s["lengths"])
    s["q"] = rows[..., :Hqk * dk].unflatten(-1, (Hqk, dk))
    s["k"] = rows[..., Hqk * dk:2 * Hqk * dk].unflatten(-1, (Hqk, dk))
    s["v"] = rows[..., 2 * Hqk * dk:].unflatten(-1, (H, dv))
    # heads remember some 30 to 4000 tokens
    spread = torch.arange(H, device="cuda") / max(1, H - 1)
    s["log_decay"] = torch.log1p(-torch.exp2(-5 - 7 * spread - 0.5 * torch.rand(H, generator=g, device="cuda")))
    s["initial"] = _normal(g, (B, H, dk, dv))
    if case["kind"] == "step":
        s.update({n: s[n][:, 0] for n in "qkv"})
    if case["kind"] == "train":
        s["initial"] = None
        s["d_o"] = _blank(_normal(g, (B, T, H, dv), dt), s["lengths"])
    return s


def _proj_inputs(case, seed):
    M, K, N, dt = case["M"], case["K"], case["N"], DTYPES[case["dtype"]]
    g = _gen(seed)
    s = {"case": case}
    s["x"] = _normal(g, (M, 2 * K if case["wide"] else K), dt)[:, :K]
    s["weight"] = _normal(g, (N, K), dt, 1 / math.sqrt(K))
    s["bias"] = _normal(g, (N,), scale=0.1) if case["bias"] else None
    s["residual"] = _normal(g, (M, N), dt) if case["residual"] else None
    if case["kind"] == "train":
        s["d_y"] = _normal(g, (M, N), dt)
    return s


_INPUTS = {"attn": _attn_inputs, "proj": _proj_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    if own:
        _prepare_own(s)
    return s


# ------------------------------------------------------------------------------------ through the library

def _prepare_own(s):
    """The buffers that a program keeps from call to call: outputs, states and workspaces."""
    from paper_2506_04761_amd import block as ll
    case = s["case"]
    kind, s["ll"] = case["kind"], ll
    if case["op"] == "attn":
        s["out"] = torch.empty(s["v"].shape, dtype=s["v"].dtype, device="cuda")
        s["final"] = torch.empty_like(s["initial"]) if s["initial"] is not None else None
        if kind != "step":
            s["ws"] = ll.ll_decay_attention_workspace(s["q"], s["v"], backward=kind == "train")
        if kind == "train":
            s["states"] = ll.ll_decay_attention_states(s["q"], s["v"])
    else:
        s["act"] = ll.LL_ACT_SILU if case["act"] else ll.LL_ACT_NONE
        s["out"] = s["x"].new_empty((case["M"], case["N"]))
        s["ws"] = ll.ll_projection_workspace(s["x"], s["weight"], s["act"], backward=kind == "train")
        s["pre"] = None
        if kind == "train" and case["act"]:
            s["pre"] = torch.empty((case["M"], case["N"]), device="cuda")


def _own_attn(s):
    ll, kind = s["ll"], s["case"]["kind"]
    a = (s["q"], s["k"], s["v"], s["log_decay"])
    if kind == "step":
        o = ll.ll_decay_attention_step(*a, s["initial"], scale=s["scale"], new_state=s["final"], out=s["out"])
        return {"o": o, "state": s["final"]}
    if kind == "fwd":
        o = ll.ll_decay_attention_fwd(*a, scale=s["scale"], initial_state=s["initial"], final_state=s["final"],
                                      lengths=s["lengths"], out=s["out"], workspace=s["ws"])
        return {"o": o, "state": s["final"]}
    o = ll.ll_decay_attention_fwd(*a, scale=s["scale"], lengths=s["lengths"], states=s["states"], out=s["out"],
                                  workspace=s["ws"])
    g = ll.ll_decay_attention_bwd(*a, s["states"], s["d_o"], scale=s["scale"], lengths=s["lengths"], workspace=s["ws"])
    return {"o": o, "dq": g.q, "dk": g.k, "dv": g.v}


def _own_proj(s):
    ll = s["ll"]
    a = (s["x"], s["weight"], s["bias"])
    y = ll.ll_projection_fwd(*a, residual=s["residual"], act=s["act"], pre=s["pre"], out=s["out"], workspace=s["ws"])
    if s["case"]["kind"] == "fwd":
        return {"y": y}
    g = ll.ll_projection_bwd(*a, s["d_y"], act=s["act"], pre=s["pre"], workspace=s["ws"])
    return _grads(s, y, g.x, g.weight, g.bias)


def _grads(s, y, dx, dw, db):
    out = {"y": y, "dx": dx, "dweight": dw}
    if s["bias"] is not None:
        out["dbias"] = db
    return out


# ------------------------------------------------------------------------------------ the plain form

CHUNK = 128  # tokens that the plain attention takes as one matrix


def _only(x, lengths):
    """[B, T, ..] in 32 bits, zeros after each sequence's end."""
    x = x.float()
    if lengths is None:
        return x
    live = torch.arange(x.shape[1], device=x.device)[None, :] < lengths[:, None]
    return torch.where(live.view(*live.shape, *([1] * (x.dim() - 2))), x, torch.zeros((), device=x.device))


def _power(log_decay, n):
    """g^n of each head over whole numbers n: [H, *n.shape]."""
    return torch.exp(log_decay.view(-1, *([1] * n.dim())) * n)


def _chunked(q, k, v, log_decay, first=None):
    """sum_{s <= t} g^(t-s) (q_t . k_s) v_s, and g^(t+1) q_t first: [B, H, T, d], T a multiple of CHUNK."""
    B, H, T, dk = q.shape
    C, dv = CHUNK, v.shape[-1]
    N = T // C
    q, k, v = (x.view(B, H, N, C, -1) for x in (q, k, v))
    i = torch.arange(C, device=q.device)
    gap = i[:, None] - i[None, :]
    inside = torch.where(gap >= 0, _power(log_decay, gap.clamp(min=0)), torch.zeros((), device=q.device))
    o = (q @ k.transpose(-1, -2) * inside[:, None]) @ v
    # a chunk's own part of the state, then every chunk's start as the sum over the chunks before it
    u = (k * _power(log_decay, C - 1 - i)[:, None, :, None]).transpose(-1, -2) @ v
    n = torch.arange(N, device=q.device)
    gap = n[:, None] - 1 - n[None, :]
    across = torch.where(gap >= 0, _power(log_decay, gap.clamp(min=0) * C), torch.zeros((), device=q.device))
    start = (across @ u.permute(1, 2, 0, 3, 4).reshape(H, N, B * dk * dv)).view(H, N, B, dk, dv).permute(2, 0, 1, 3, 4)
    if first is not None:
        start = start + first[:, :, None] * _power(log_decay, n * C)[:, :, None, None]
    o = o + (q @ start) * _power(log_decay, i + 1)[:, None, :, None]
    return o.reshape(B, H, T, dv)


def _heads(x, H, T):
    """[B, H, T', d] of [B, T, H', d], T' the whole chunks that hold T tokens."""
    x = x.transpose(1, 2)
    x = x.repeat_interleave(H // x.shape[1], 1) if x.shape[1] != H else x
    return torch.nn.functional.pad(x, (0, 0, 0, -T % CHUNK)).contiguous()


def _tokens(x, T, heads):
    """[B, T, heads, d] of [B, H, T', d]: heads of a group are added."""
    x = x[:, :, :T]
    return x.unflatten(1, (heads, -1)).sum(2).transpose(1, 2)


def _plain_attn(s):
    case = s["case"]
    H, T, kind, dt = case["H"], case["T"], case["kind"], s["v"].dtype
    ld, scale = s["log_decay"], s["scale"]
    if kind == "step":
        q, k, v = (s[n].float() for n in "qkv")
        q, k = (x.repeat_interleave(H // x.shape[1], 1) for x in (q, k))
        state = s["initial"] * torch.exp(ld)[:, None, None] + k[..., None] * v[..., None, :]
        return {"o": (scale * (q[..., None] * state).sum(-2)).to(dt), "state": state}
    ln = s["lengths"]
    q, k, v = (_heads(_only(s[n], ln), H, T) for n in "qkv")
    # rows after an end are zero in q, k, v and d, and so in what comes of them
    o = _tokens(scale * _chunked(q, k, v, ld, s["initial"]), T, H).contiguous().to(dt)
    if kind == "fwd":
        # the state at each sequence's end, as one weighted product
        end = torch.full((case["B"],), T, device="cuda") if ln is None else ln.long()
        after = end[:, None] - 1 - torch.arange(q.shape[2], device="cuda")
        w = torch.exp(ld[None, :, None] * after[:, None].clamp(min=0)) * (after[:, None] >= 0)
        state = (k * w[..., None]).transpose(-1, -2) @ v
        state = state + s["initial"] * torch.exp(ld[None, :] * end[:, None])[..., None, None]
        return {"o": o, "state": state}
    d = _heads(_only(s["d_o"], ln), H, T)
    back = [x.flip(2) for x in (q, k, v, d)]
    dq = scale * _chunked(d, v, k, ld)
    dk = scale * _chunked(back[2], back[3], back[0], ld).flip(2)
    dv = scale * _chunked(back[1], back[0], back[3], ld).flip(2)
    g = {"dq": _tokens(dq, T, case["Hqk"]), "dk": _tokens(dk, T, case["Hqk"]), "dv": _tokens(dv, T, H)}
    return {"o": o, **{n: x.contiguous().to(dt) for n, x in g.items()}}


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _plain_proj(s):
    case, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["weight"].float()
    u = x @ w.t()
    if s["bias"] is not None:
        u = u + s["bias"]
    y = u * _sigmoid(u) if case["act"] else u
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(dt)
    if case["kind"] == "fwd":
        return {"y": y}
    du = s["d_y"].float()
    if case["act"]:
        p = _sigmoid(u)
        du = du * (p * (1 + u * (1 - p)))
    return _grads(s, y, (du @ w).to(dt), (du.t() @ x).to(dt), du.sum(0))


def run(s):
    if own:
        return _own_attn(s) if s["case"]["op"] == "attn" else _own_proj(s)
    return _plain_attn(s) if s["case"]["op"] == "attn" else _plain_proj(s)


# ------------------------------------------------------------------------------------ work

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    train = case["kind"] == "train"
    if case["op"] == "proj":
        M, K, N = case["M"], case["K"], case["N"]
        b = e * (M * K + N * K + M * N * (2 if case["residual"] else 1)) + (4 * N if case["bias"] else 0)
        if train:  # dy in, dx, dW and db out
            b += e * (M * N + M * K + N * K) + (4 * N if case["bias"] else 0)
        return {"bytes": b, "flops": (6 if train else 2) * M * N * K}
    B, T, H, Hqk, dk, dv = (case[n] for n in ("B", "T", "H", "Hqk", "dk", "dv"))
    # sequences that end early are half the batch's length on average
    n = T * (1 + 0.5 * (B - 1)) if case["ragged"] else B * T
    b = e * (2 * Hqk * dk + H * dv) * n + e * H * dv * B * T + 4 * H
    if train:  # d_o in, dq, dk and dv out
        return {"bytes": b + e * H * dv * n + e * (2 * Hqk * dk + H * dv) * B * T, "flops": 12 * n * H * dk * dv}
    return {"bytes": b + 8 * B * H * dk * dv, "flops": 4 * n * H * dk * dv}


# ------------------------------------------------------------------------------------ 64 bits

def _exact_attn(s):
    """Token by token: the state forward in time, its gradient backward."""
    case = s["case"]
    B, T, H, kind = case["B"], case["T"], case["H"], case["kind"]
    group = H // case["Hqk"]
    q, k, v = ((s[n][:, None] if kind == "step" else s[n]).double() for n in "qkv")
    q, k = q.repeat_interleave(group, 2), k.repeat_interleave(group, 2)
    g = torch.exp(s["log_decay"].double())[:, None, None]
    ends = torch.full((B,), T) if s["lengths"] is None else s["lengths"].cpu()
    live = (torch.arange(T)[:, None] < ends).cuda()
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    every = bool(live.all())
    q, k, v = (x if every else torch.where(live.t()[..., None, None], x, zero) for x in (q, k, v))
    d = None
    if kind == "train":
        d = s["d_o"].double()
        d = d if every else torch.where(live.t()[..., None, None], d, zero)
    S = torch.zeros((B, H, case["dk"], case["dv"]), dtype=torch.float64, device="cuda")
    if s["initial"] is not None:
        S += s["initial"].double()
    o, dq = torch.zeros_like(v), torch.zeros_like(q)
    for t in range(T):
        new = g * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        S = new if every else torch.where(live[t, :, None, None, None], new, S)
        o[:, t] = (q[:, t, :, None, :] @ S)[:, :, 0]
        if d is not None:
            dq[:, t] = (S @ d[:, t, :, :, None])[..., 0]
    scale = s["scale"]
    if kind != "train":
        return {"o": scale * (o[:, 0] if kind == "step" else o), "state": S}
    D = torch.zeros_like(S)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    for t in reversed(range(T)):
        D = g * D + q[:, t, :, :, None] * d[:, t, :, None, :]
        dk[:, t] = (D @ v[:, t, :, :, None])[..., 0]
        dv[:, t] = (k[:, t, :, None, :] @ D)[:, :, 0]
    dq, dk = (x.unflatten(2, (-1, group)).sum(3) for x in (dq, dk))
    return {"o": scale * o, "dq": scale * dq, "dk": scale * dk, "dv": scale * dv}


def _exact_proj(s):
    case = s["case"]
    x, w = s["x"].double(), s["weight"].double()
    u = torch.addmm(s["bias"].double(), x, w.t()) if s["bias"] is not None else x @ w.t()
    p = torch.sigmoid(u) if case["act"] else torch.ones_like(u)
    y = u * p
    if s["residual"] is not None:
        y += s["residual"].double()
    if case["kind"] == "fwd":
        return {"y": y}
    du = s["d_y"].double() * (p + u * p * (1 - p) if case["act"] else p)
    return _grads(s, y, du @ w, du.t() @ x, du.sum(0))


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    return _exact_attn(s) if case["op"] == "attn" else _exact_proj(s)
