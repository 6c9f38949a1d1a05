"""ctypes binding of what makes a block around a mixer (include/libloglinear.h): the linear attention with a
decay for each head, and the projections in front of and behind a mixer, with their backward passes and, for
the attention, its form for one token; and both as functions that can be differentiated once.

    from paper_2506_04761_amd import block

As in the rest of the binding, the wrappers check and pass arguments and every step of the computation runs
in the library's HIP kernels.  q, k, v, and the rows that a projection takes, may be columns of wider rows
(channels adjacent); everything else is contiguous.  Work is enqueued on `stream` (default: torch's current
stream) and is not synchronised; outputs, gradients and workspaces that a call allocates are memory of that
stream.
"""

import ctypes
from collections import namedtuple

import torch

from ._layer import (LL_ACT_NONE, LL_ACT_SILU, _buffer, _channels_last, _declare, _dense, _dims, _lengths, _ok, _opt,  # noqa: F401
                     _rows, _sized)
from ._lib import LLError, _check, _dtype_code, _i32, _i64, _once, _ptr, _results, _stream, _sz, _vp, lib  # noqa: F401

DecayGrads = namedtuple("DecayGrads", "q k v initial_state")
ProjectionGrads = namedtuple("ProjectionGrads", "x weight bias")


class _DecayInputs(ctypes.Structure):
    # ll_decay_inputs; its pairs of strides are single fields here, for one constructor call
    _fields_ = ([(n, _vp) for n in "qkv"] + [(n + "_" + axis, _i64) for n in "qkv" for axis in ("batch", "token")]
                + [("log_decay", _vp), ("lengths", _vp)]
                + [(n, _i64) for n in ("batch", "T", "heads", "qk_heads", "d_k", "d_v")]
                + [("scale", ctypes.c_float), ("dtype", _i32)])


_decay = ctypes.POINTER(_DecayInputs)
_declare("ll_decay_attention_workspace_size", [_i64] * 6 + [_i32], _sz)
_declare("ll_decay_attention_states_bytes", [_i64] * 5, _sz)
_declare("ll_decay_attention_fwd", [_decay] + [_vp] * 5 + [_sz, _vp])
_declare("ll_decay_attention_step", [_decay] + [_vp] * 4)
_declare("ll_decay_attention_bwd", [_decay] + [_vp] * 8 + [_sz, _vp])
_declare("ll_projection_workspace_size", [_i32] + [_i64] * 3 + [_i32, _i32], _sz)
_declare("ll_projection_fwd", [_vp, _i64] + [_vp] * 3 + [_i64] + [_vp] * 2 + [_i64] * 3 + [_i32, _i32, _vp, _sz, _vp])
_declare("ll_projection_bwd", [_vp, _i64] + [_vp] * 6 + [_i64] * 3 + [_i32, _i32, _vp, _sz, _vp])


# ------------------------------------------------------------------------------------ decay attention

def _heads(t, name, dtype, shape):
    """Checks [.., heads, d] whose heads are adjacent, any strides of the axes before, which it returns."""
    strides = _rows(t, name, dtype, shape)
    if shape[-2] != 1 and strides[-2] != shape[-1]:
        raise ValueError(f"{name} must have adjacent heads")
    return strides


def _decay_sizes(q, v, n=4):
    """B, T, H, H_qk, d_k, d_v of q [B, T, H_qk, d_k] and v [B, T, H, d_v]."""
    shape, (H, dv) = _dims(q, "q", n), _dims(v, "v", n)[-2:]
    return shape[0], shape[1] if n == 4 else 1, H, shape[-2], shape[-1], dv


def _decay_inputs(q, k, v, log_decay, scale, lengths, step):
    """The checked inputs of a call.  With `step`, tensors of one token ([B, heads, d])."""
    B, T, H, Hqk, dk, dv = _decay_sizes(q, v, 3 if step else 4)
    dtype, lead = q.dtype, q.shape[:-2]
    qs = _heads(q, "q", dtype, q.shape)
    ks = _heads(k, "k", dtype, q.shape)
    vs = _heads(v, "v", dtype, (*lead, H, dv))
    _check(log_decay, "log_decay", torch.float32, (H,))
    _lengths(lengths, B)
    if T == 1:  # the stride of an only token is whatever the tensor came by, and not used
        qs, ks, vs = (qs[0], 0), (ks[0], 0), (vs[0], 0)
    return _DecayInputs(q.data_ptr(), k.data_ptr(), v.data_ptr(), qs[0], qs[1], ks[0], ks[1], vs[0], vs[1],
                        log_decay.data_ptr(), _ptr(lengths), B, T, H, Hqk, dk, dv, scale, _dtype_code(q))


def ll_decay_attention_workspace(q, v, backward=False):
    """A workspace for the forward (or backward, which serves both) of q [B, T, H_qk, d_k] with v [B, T, H, d_v]."""
    return _buffer(lib.ll_decay_attention_workspace_size(*_decay_sizes(q, v), int(backward)), q.device)


def ll_decay_attention_states(q, v):
    """The buffer in which a forward leaves its states for the backward."""
    B, T, H, _, dk, dv = _decay_sizes(q, v)
    return _buffer(lib.ll_decay_attention_states_bytes(B, T, H, dk, dv), q.device)


def _check_decay_states(states, s):
    _check(states, "states", torch.uint8)
    if states.numel() < lib.ll_decay_attention_states_bytes(s.batch, s.T, s.heads, s.d_k, s.d_v):
        raise ValueError("states is smaller than ll_decay_attention_states gives")


def _decay_need(s, backward):
    return lib.ll_decay_attention_workspace_size(s.batch, s.T, s.heads, s.qk_heads, s.d_k, s.d_v, backward)


def ll_decay_attention_fwd(q, k, v, log_decay, scale=1.0, initial_state=None, final_state=None, lengths=None,
                           states=None, out=None, workspace=None, stream=None):
    """Linear attention with a decay for each head: S_t = exp(log_decay) S_(t-1) + k_t v_t^T, o_t = scale S_t^T q_t, of
    q, k [B, T, H_qk, d_k], v [B, T, H, d_v] and log_decay [H]; returns o [B, T, H, d_v].  `initial_state`
    [B, H, d_k, d_v] float32 is continued from (None: zeros), `final_state` receives the state at each sequence's end (it
    may be the same tensor).  `states` (see ll_decay_attention_states) keeps what ll_decay_attention_bwd needs."""
    s = _decay_inputs(q, k, v, log_decay, scale, lengths, False)
    shape = (s.batch, s.heads, s.d_k, s.d_v)
    _opt(initial_state, "initial_state", torch.float32, shape)
    _opt(final_state, "final_state", torch.float32, shape)
    if states is not None:
        _check_decay_states(states, s)
    if out is None:
        out = _results(lambda: v.new_empty(v.shape), stream)
    else:
        _check(out, "out", v.dtype, v.shape)
    ws = _sized(workspace, lambda: 0 if states is not None else _decay_need(s, 0), q.device, stream)
    _ok(lib.ll_decay_attention_fwd(s, _ptr(initial_state), out.data_ptr(), _ptr(final_state), _ptr(states), _ptr(ws),
                                   ws.numel(), _stream(stream)))
    return out


def ll_decay_attention_step(q, k, v, log_decay, state, scale=1.0, new_state=None, out=None, stream=None):
    """One token: q, k [B, H_qk, d_k], v [B, H, d_v]; returns o [B, H, d_v].  `state` [B, H, d_k, d_v] is read,
    `new_state` written (None: in place)."""
    s = _decay_inputs(q, k, v, log_decay, scale, None, True)
    shape = (s.batch, s.heads, s.d_k, s.d_v)
    _check(state, "state", torch.float32, shape)
    _opt(new_state, "new_state", torch.float32, shape)
    if out is None:
        out = _results(lambda: v.new_empty(v.shape), stream)
    else:
        _check(out, "out", v.dtype, v.shape)
    _ok(lib.ll_decay_attention_step(s, state.data_ptr(), (state if new_state is None else new_state).data_ptr(),
                                    out.data_ptr(), _stream(stream)))
    return out


def ll_decay_attention_bwd(q, k, v, log_decay, states, d_o, scale=1.0, lengths=None, d_final_state=None,
                           initial_state_grad=False, grads=None, workspace=None, stream=None):
    """Gradients of the ll_decay_attention_fwd that left `states`, on the same inputs: a DecayGrads (q, k, v,
    initial_state) of new tensors, or `grads` filled in; that of the initial state is None unless `initial_state_grad`.
    Those of shared query/key heads are sums over their group.  The decays are constants."""
    s = _decay_inputs(q, k, v, log_decay, scale, lengths, False)
    shape = (s.batch, s.heads, s.d_k, s.d_v)
    _check_decay_states(states, s)
    _check(d_o, "d_o", v.dtype, v.shape)
    _opt(d_final_state, "d_final_state", torch.float32, shape)
    if grads is None:
        grads = _results(lambda: DecayGrads(q.new_empty(q.shape), q.new_empty(q.shape), q.new_empty(v.shape),
                                            log_decay.new_empty(shape) if initial_state_grad else None), stream)
    g = DecayGrads(*grads)
    _check(g.q, "grads.q", q.dtype, q.shape)
    _check(g.k, "grads.k", q.dtype, q.shape)
    _check(g.v, "grads.v", q.dtype, v.shape)
    _opt(g.initial_state, "grads.initial_state", torch.float32, shape)
    ws = _sized(workspace, lambda: _decay_need(s, 1), q.device, stream)
    _ok(lib.ll_decay_attention_bwd(s, states.data_ptr(), d_o.data_ptr(), _ptr(d_final_state), g.q.data_ptr(),
                                   g.k.data_ptr(), g.v.data_ptr(), _ptr(g.initial_state), _ptr(ws), ws.numel(),
                                   _stream(stream)))
    return grads


# ------------------------------------------------------------------------------------ projection

def _projection_args(x, weight, bias):
    """M, K, N and the stride of x's rows (that of an only row is not used) of checked arguments."""
    M, K = _dims(x, "x", 2)
    N = _dims(weight, "weight", 2)[0]
    stride = _rows(x, "x", x.dtype, x.shape)[0]
    _check(weight, "weight", x.dtype, (N, K))
    _opt(bias, "bias", torch.float32, (N,))
    return M, K, N, stride if M != 1 else 0


def _projection_need(x, weight, act, backward):
    return lib.ll_projection_workspace_size(_dtype_code(x), *x.shape, weight.shape[0], act, int(backward))


def ll_projection_workspace(x, weight, act=LL_ACT_NONE, backward=False):
    """A workspace for the forward (or backward, which serves both) projection of x [M, K] with weight [N, K]."""
    _dims(x, "x", 2), _dims(weight, "weight", 2)
    return _buffer(_projection_need(x, weight, act, backward), x.device)


def ll_projection_fwd(x, weight, bias=None, residual=None, act=LL_ACT_NONE, pre=None, out=None, workspace=None,
                      stream=None):
    """y = act(u) + residual, u = x [M, K] @ weight [N, K].T + bias; returns y [M, N].  x and residual may be columns of
    wider rows.  `pre` (float32 [M, N]) receives u, for ll_projection_bwd of an activation."""
    M, K, N, stride = _projection_args(x, weight, bias)
    dtype = x.dtype
    code = _dtype_code(x)
    res_stride = 0 if residual is None else _rows(residual, "residual", dtype, (M, N))[0]
    _opt(pre, "pre", torch.float32, (M, N))
    if out is None:
        out = _results(lambda: x.new_empty((M, N)), stream)
    else:
        _check(out, "out", dtype, (M, N))
    ws = _sized(workspace, lambda: lib.ll_projection_workspace_size(code, M, K, N, act, 0), x.device, stream)
    _ok(lib.ll_projection_fwd(x.data_ptr(), stride, weight.data_ptr(), _ptr(bias), _ptr(residual),
                              res_stride if M != 1 else 0, out.data_ptr(), _ptr(pre), M, K, N, act, code, _ptr(ws), ws.numel(), _stream(stream)))
    return out


def ll_projection_bwd(x, weight, bias, d_y, act=LL_ACT_NONE, pre=None, grads=None, workspace=None, stream=None):
    """Gradients of ll_projection_fwd on the same inputs (that of a residual is d_y): a ProjectionGrads (x, weight,
    bias) of new tensors, or `grads` filled in, of which each may be None: not wanted.  That of a bias that is None is
    None.  With an activation `pre` is what the forward left."""
    M, K, N, stride = _projection_args(x, weight, bias)
    _check(d_y, "d_y", x.dtype, (M, N))
    _opt(pre, "pre", torch.float32, (M, N))
    code = _dtype_code(x)
    if grads is None:
        grads = _results(lambda: ProjectionGrads(x.new_empty((M, K)), torch.empty_like(weight),
                                                 None if bias is None else torch.empty_like(bias)), stream)
    g = ProjectionGrads(*grads)
    _opt(g.x, "grads.x", x.dtype, (M, K))
    _opt(g.weight, "grads.weight", x.dtype, (N, K))
    _opt(g.bias, "grads.bias", torch.float32, (N,))
    ws = _sized(workspace, lambda: lib.ll_projection_workspace_size(code, M, K, N, act, 1), x.device, stream)
    _ok(lib.ll_projection_bwd(x.data_ptr(), stride, weight.data_ptr(), _ptr(pre), d_y.data_ptr(), _ptr(g.x),
                              _ptr(g.weight), _ptr(g.bias), M, K, N, act, code, _ptr(ws), ws.numel(),
                              _stream(stream)))
    return grads


# ------------------------------------------------------------------------------------ autograd

def _heads_last(t):
    """`t` as it is where its heads and their elements are adjacent, else a copy."""
    return t if t.stride(-1) == 1 and (t.shape[-2] == 1 or t.stride(-2) == t.shape[-1]) else t.contiguous()


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, initial_state, lengths, scale, want_state):
        for t, name in ((q, "q"), (k, "k"), (v, "v")):
            _dims(t, name, 4)
        q, k, v = _heads_last(q), _heads_last(k), _heads_last(v)
        log_decay, initial_state = log_decay.contiguous(), _dense(initial_state)
        shape = (v.shape[0], v.shape[2], q.shape[3], v.shape[3])
        final = torch.empty(shape, dtype=torch.float32, device=v.device) if want_state else None
        states = ll_decay_attention_states(q, v) if any(ctx.needs_input_grad) else None
        o = ll_decay_attention_fwd(q, k, v, log_decay, scale, initial_state, final, lengths, states)
        ctx.save_for_backward(q, k, v, log_decay, lengths, states)
        ctx.scale, ctx.from_state = scale, ctx.needs_input_grad[4]
        ctx.set_materialize_grads(False)
        return o, final

    @staticmethod
    def backward(ctx, d_o, d_final):
        q, k, v, log_decay, lengths, states = ctx.saved_tensors
        d_o = v.new_zeros(v.shape) if d_o is None else d_o.contiguous()
        g = ll_decay_attention_bwd(q, k, v, log_decay, states, d_o, ctx.scale, lengths, _dense(d_final), ctx.from_state)
        dq, dk, dv, di = _once(g)
        return dq, dk, dv, None, di, None, None, None


class _Projection(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act):
        lead = x.shape[:-1]
        x, weight, bias = _channels_last(x.reshape(-1, x.shape[-1])), weight.contiguous(), _dense(bias)
        if residual is not None:
            if residual.shape != (*lead, weight.shape[0]):
                raise ValueError(f"residual has shape {tuple(residual.shape)}, expected {(*lead, weight.shape[0])}")
            residual = _channels_last(residual.reshape(-1, residual.shape[-1]))
        keep = act != LL_ACT_NONE and any(ctx.needs_input_grad[:3])
        pre = weight.new_empty((x.shape[0], weight.shape[0]), dtype=torch.float32) if keep else None
        y = ll_projection_fwd(x, weight, bias, residual, act, pre)
        ctx.save_for_backward(x, weight, bias, pre)
        ctx.act, ctx.lead = act, lead
        return y.view(*lead, -1)

    @staticmethod
    def backward(ctx, d_y):
        x, weight, bias, pre = ctx.saved_tensors
        wants = ctx.needs_input_grad
        dx = dw = db = None
        if any(wants[:3]):
            dy = d_y.reshape(x.shape[0], -1).contiguous()
            want = ProjectionGrads(x.new_empty(x.shape) if wants[0] else None,
                                   torch.empty_like(weight) if wants[1] else None,
                                   torch.empty_like(bias) if wants[2] else None)
            # the residual's gradient is d_y, which may be differentiated again; what the kernels give may not
            dx, dw, db = _once(ll_projection_bwd(x, weight, bias, dy, ctx.act, pre, want))
            dx = None if dx is None else dx.view(*ctx.lead, -1)
        return dx, dw, db, d_y if wants[3] else None, None


def decay_attention(q, k, v, log_decay, scale=1.0, initial_state=None, lengths=None, return_final_state=False):
    """Differentiable ll_decay_attention_fwd: o, or (o, final state); gradients flow to q, k, v and the states.  Memory
    held until the graph is freed: the inputs and ll_decay_attention_states_bytes(...) bytes."""
    if log_decay.requires_grad and torch.is_grad_enabled():
        raise ValueError("log_decay must not require a gradient: the decays are constants")
    o, final = _DecayAttention.apply(q, k, v, log_decay, initial_state, lengths, scale, return_final_state)
    return (o, final) if return_final_state else o


def projection(x, weight, bias=None, residual=None, act=LL_ACT_NONE):
    """Differentiable ll_projection_fwd of x [.., K] with weight [N, K], for any leading axes: act(x @ weight.T + bias) +
    residual [.., N]; gradients flow to x, weight, bias and residual."""
    return _Projection.apply(x, weight, bias, residual, act)
