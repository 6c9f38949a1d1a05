"""ctypes binding of the operators around a token mixer (include/libloglinear.h): the short causal
convolution, the selective state space scan and the group norm, with their backward passes and their forms
for one token; and the three as functions that can be differentiated once.

As in the rest of the binding, the wrappers check and pass arguments and every step of the computation runs
in the library's HIP kernels.  x, dt, z, gate, B and C may be columns of wider rows (channels adjacent);
everything else is contiguous.  Work is enqueued on `stream` (default: torch's current stream) and is not
synchronised; outputs, gradients and workspaces that a call allocates are memory of that stream.
"""

import ctypes
from collections import namedtuple

import torch

from ._lib import (LL_OK, LLError, _check, _dtype_code, _i32, _i64, _once, _ptr, _results, _scratch, _stream, _sz,
                   _vp, lib)

LL_ACT_NONE, LL_ACT_SILU = 0, 1

ConvGrads = namedtuple("ConvGrads", "x weight bias initial_state")
ScanGrads = namedtuple("ScanGrads", "x dt A B C D z dt_bias initial_state")
NormGrads = namedtuple("NormGrads", "x weight bias gate")


class _ScanInputs(ctypes.Structure):
    # ll_scan_inputs; its pairs of strides are single fields here, for one constructor call
    _fields_ = ([(n, _vp) for n in ("x", "dt", "z", "B", "C")]
                + [(n + "_" + axis, _i64) for n in ("x", "dt", "z", "B", "C") for axis in ("batch", "token")]
                + [(n, _vp) for n in ("A", "D", "dt_bias", "lengths")]
                + [(n, _i64) for n in ("batch", "T", "channels", "N", "groups")]
                + [("delta_softplus", _i32), ("dtype", _i32)])


def _declare(name, args, restype=_i32):
    fn = getattr(lib, name)
    fn.argtypes, fn.restype = args, restype


_f32 = ctypes.c_float
_inputs = ctypes.POINTER(_ScanInputs)
_declare("ll_causal_conv_fwd", [_vp, _i64, _i64] + [_vp] * 6 + [_i64] * 4 + [_i32, _i32, _vp])
_declare("ll_causal_conv_step", [_vp, _i64] + [_vp] * 5 + [_i64] * 3 + [_i32, _i32, _vp])
_declare("ll_causal_conv_bwd", [_vp, _i64, _i64] + [_vp] * 10 + [_i64] * 4 + [_i32, _i32, _vp, _sz, _vp])
_declare("ll_causal_conv_bwd_workspace_size", [_i32] + [_i64] * 4, _sz)
_declare("ll_selective_scan_workspace_size", [_i64] * 5 + [_i32], _sz)
_declare("ll_selective_scan_states_bytes", [_i64] * 4, _sz)
_declare("ll_selective_scan_fwd", [_inputs, _vp, _vp, _vp, _vp, _vp, _sz, _vp])
_declare("ll_selective_scan_step", [_inputs, _vp, _vp, _vp, _vp])
_declare("ll_selective_scan_bwd", [_inputs] + [_vp] * 13 + [_sz, _vp])
_declare("ll_group_norm_workspace_size", [_i32] + [_i64] * 4 + [_i32], _sz)
_declare("ll_group_norm_fwd", [_vp, _i64, _i64] * 2 + [_vp] * 4 + [_i64] * 4 + [_f32, _i32, _i32, _vp, _sz, _vp])
_declare("ll_group_norm_bwd", [_vp, _i64, _i64] * 2 + [_vp] * 8 + [_i64] * 4 + [_i32, _i32, _vp, _sz, _vp])


# ------------------------------------------------------------------------------------ checks

def _rows(t, name, dtype, shape):
    """Checks columns of wider rows: adjacent channels, any strides of the other axes, which it returns."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"{name} must have adjacent channels (a last stride of 1)")
    return strides


def _token_stride(t):
    """The stride of a token of [B, T, channels]; that of an only token is whatever the tensor came by, and not used."""
    return t.stride(1) if t.shape[1] != 1 else 0


def _opt(t, name, dtype, shape):
    if t is not None:
        _check(t, name, dtype, shape)


def _lengths(t, B):
    if t is not None:
        _check(t, "lengths", torch.int32, (B,))


def _dims(x, name, n):
    if not isinstance(x, torch.Tensor) or x.dim() != n:
        raise ValueError(f"{name} must be a tensor of {n} axes")
    return x.shape


def _ok(st):
    if st != LL_OK:
        raise LLError(st)


def _buffer(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _sized(workspace, need, device, stream):
    """A call's workspace: the caller's, or a new one."""
    if workspace is None:
        workspace = _scratch(lambda: _buffer(need(), device), stream)
    _check(workspace, "workspace", torch.uint8)
    return workspace


# ------------------------------------------------------------------------------------ convolution

def ll_causal_conv_fwd(x, weight, bias=None, act=LL_ACT_SILU, initial_state=None, final_state=None, lengths=None,
                       out=None, stream=None):
    """y = act(causal convolution of x [B, T, D] with weight [D, W]); `initial_state` [B, W - 1, D] holds the
    tokens before the first (None: zeros), `final_state` receives those before the end (it may be the same
    tensor).  `lengths` (int32 [B]) ends sequences early; outputs after an end are zero.  Returns y."""
    B, T, D = _dims(x, "x", 3)
    W = _dims(weight, "weight", 2)[1]
    _rows(x, "x", x.dtype, x.shape)
    _check(weight, "weight", torch.float32, (D, W))
    _opt(bias, "bias", torch.float32, (D,))
    _opt(initial_state, "initial_state", x.dtype, (B, W - 1, D))
    _opt(final_state, "final_state", x.dtype, (B, W - 1, D))
    _lengths(lengths, B)
    code = _dtype_code(x)
    if out is None:
        out = _results(lambda: x.new_empty((B, T, D)), stream)
    else:
        _check(out, "out", x.dtype, (B, T, D))
    _ok(lib.ll_causal_conv_fwd(x.data_ptr(), x.stride(0), _token_stride(x), weight.data_ptr(), _ptr(bias),
                               _ptr(initial_state), _ptr(final_state), _ptr(lengths), out.data_ptr(), B, T, D, W,
                               act, code, _stream(stream)))
    return out


def ll_causal_conv_step(x, weight, bias, state, act=LL_ACT_SILU, new_state=None, out=None, stream=None):
    """One token x [B, D]: returns y [B, D].  `state` [B, W - 1, D] is read, `new_state` written (None: in
    place)."""
    B, D = _dims(x, "x", 2)
    W = _dims(weight, "weight", 2)[1]
    _rows(x, "x", x.dtype, x.shape)
    _check(weight, "weight", torch.float32, (D, W))
    _opt(bias, "bias", torch.float32, (D,))
    _check(state, "state", x.dtype, (B, W - 1, D))
    _opt(new_state, "new_state", x.dtype, (B, W - 1, D))
    code = _dtype_code(x)
    if out is None:
        out = _results(lambda: x.new_empty((B, D)), stream)
    else:
        _check(out, "out", x.dtype, (B, D))
    _ok(lib.ll_causal_conv_step(x.data_ptr(), x.stride(0), weight.data_ptr(), _ptr(bias), state.data_ptr(),
                                (state if new_state is None else new_state).data_ptr(), out.data_ptr(), B, D, W,
                                act, code, _stream(stream)))
    return out


def ll_causal_conv_bwd_workspace(x, weight):
    """A workspace for ll_causal_conv_bwd of x [B, T, D] with weight [D, W]."""
    B, T, D = _dims(x, "x", 3)
    W = _dims(weight, "weight", 2)[1]
    return _buffer(lib.ll_causal_conv_bwd_workspace_size(_dtype_code(x), B, T, D, W), x.device)


def ll_causal_conv_bwd(x, weight, bias, d_y, act=LL_ACT_SILU, initial_state=None, lengths=None, d_final_state=None,
                       grads=None, workspace=None, stream=None):
    """Gradients of ll_causal_conv_fwd on the same inputs: a ConvGrads (x, weight, bias, initial_state) of new
    tensors, or `grads` filled in; those of a bias or initial state that is None are None."""
    B, T, D = _dims(x, "x", 3)
    W = _dims(weight, "weight", 2)[1]
    _rows(x, "x", x.dtype, x.shape)
    _check(weight, "weight", torch.float32, (D, W))
    _opt(bias, "bias", torch.float32, (D,))
    _opt(initial_state, "initial_state", x.dtype, (B, W - 1, D))
    _check(d_y, "d_y", x.dtype, (B, T, D))
    _opt(d_final_state, "d_final_state", x.dtype, (B, W - 1, D))
    _lengths(lengths, B)
    code = _dtype_code(x)
    if grads is None:
        grads = _results(lambda: ConvGrads(x.new_empty((B, T, D)), torch.empty_like(weight),
                                           None if bias is None else torch.empty_like(bias),
                                           None if initial_state is None else torch.empty_like(initial_state)), stream)
    dx, dw, db, di = grads
    _check(dx, "grads.x", x.dtype, (B, T, D))
    _check(dw, "grads.weight", torch.float32, (D, W))
    _opt(db, "grads.bias", torch.float32, (D,))
    _opt(di, "grads.initial_state", x.dtype, (B, W - 1, D))
    ws = _sized(workspace, lambda: lib.ll_causal_conv_bwd_workspace_size(code, B, T, D, W), x.device, stream)
    _ok(lib.ll_causal_conv_bwd(x.data_ptr(), x.stride(0), _token_stride(x), weight.data_ptr(), _ptr(bias),
                               _ptr(initial_state), _ptr(lengths), d_y.data_ptr(), _ptr(d_final_state),
                               dx.data_ptr(), dw.data_ptr(), _ptr(db), _ptr(di), B, T, D, W, act, code,
                               _ptr(ws), ws.numel(), _stream(stream)))
    return grads


# ------------------------------------------------------------------------------------ selective scan

def _groups(t, name, n):
    """The groups of B or C: [.., N], of `n` axes, for one, [.., groups, N] for several."""
    if not isinstance(t, torch.Tensor) or not n <= t.dim() <= n + 1:
        raise ValueError(f"{name} must be a tensor of {n} axes, or of {n + 1} with groups")
    return 1 if t.dim() == n else t.shape[-2]


def _scan_inputs(x, dt, A, Bm, Cm, D, z, dt_bias, delta_softplus, lengths, step):
    """The checked inputs of a scan call.  With `step`, tensors of one token ([B, ...])."""
    lead = _dims(x, "x", 2 if step else 3)
    nb, ch = lead[0], lead[-1]
    N = _dims(A, "A", 2)[1]
    dtype = x.dtype
    xs, ds = _rows(x, "x", dtype, lead), _rows(dt, "dt", dtype, lead)
    zs = (0, 0, 1) if z is None else _rows(z, "z", dtype, lead)
    _check(A, "A", torch.float32, (ch, N))
    groups = _groups(Bm, "B", len(lead))
    shape = (*lead[:-1], N) if Bm.dim() == len(lead) else (*lead[:-1], groups, N)
    bs, cs = _rows(Bm, "B", dtype, shape), _rows(Cm, "C", dtype, shape)
    if groups > 1 and (bs[-2] != N or cs[-2] != N):
        raise ValueError("B and C must have adjacent groups")
    if D is not None:
        _check(D, "D", torch.float32, (ch,))
    if dt_bias is not None:
        _check(dt_bias, "dt_bias", torch.float32, (ch,))
    if lengths is not None:
        _lengths(lengths, nb)
    T = 1 if step else lead[1]
    if T == 1 and not step:  # see _token_stride
        xs, ds, zs, bs, cs = ((v[0], 0) for v in (xs, ds, zs, bs, cs))
    return _ScanInputs(x.data_ptr(), dt.data_ptr(), _ptr(z), Bm.data_ptr(), Cm.data_ptr(), xs[0], xs[1], ds[0], ds[1],
                       zs[0], zs[1], bs[0], bs[1], cs[0], cs[1], A.data_ptr(), _ptr(D), _ptr(dt_bias), _ptr(lengths), nb,
                       T, ch, N, groups, 1 if delta_softplus else 0, _dtype_code(x))


def ll_selective_scan_workspace(x, B, backward=False):
    """A workspace for the forward (or backward) scan of x [B, T, D] with B [B, T, N] or [B, T, groups, N]."""
    nb, T, ch = _dims(x, "x", 3)
    groups = _groups(B, "B", 3)
    need = lib.ll_selective_scan_workspace_size(nb, T, ch, B.shape[-1], groups, int(backward))
    return _buffer(need, x.device)


def ll_selective_scan_states(x, B):
    """The buffer in which a forward scan of x [B, T, D] leaves its states for the backward."""
    nb, T, ch = _dims(x, "x", 3)
    _groups(B, "B", 3)
    return _buffer(lib.ll_selective_scan_states_bytes(nb, T, ch, B.shape[-1]), x.device)


def _check_states(states, s):
    _check(states, "states", torch.uint8)
    if states.numel() < lib.ll_selective_scan_states_bytes(s.batch, s.T, s.channels, s.N):
        raise ValueError("states is smaller than ll_selective_scan_states gives")


def ll_selective_scan_fwd(x, dt, A, B, C, D=None, z=None, dt_bias=None, delta_softplus=True, initial_state=None,
                          final_state=None, lengths=None, states=None, out=None, workspace=None, stream=None):
    """Selective scan of x, dt [B, T, D] (gate z or None) with A [D, N] and B, C [B, T, N] (or [B, T, groups, N]);
    returns y [B, T, D].  `initial_state` [B, D, N] float32 is continued from (None: zeros), `final_state`
    receives the state at each sequence's end (it may be the same tensor).  `states` (see
    ll_selective_scan_states) keeps what ll_selective_scan_bwd needs."""
    s = _scan_inputs(x, dt, A, B, C, D, z, dt_bias, delta_softplus, lengths, False)
    shape = (s.batch, s.channels, s.N)
    _opt(initial_state, "initial_state", torch.float32, shape)
    _opt(final_state, "final_state", torch.float32, shape)
    if states is not None:
        _check_states(states, s)
    if out is None:
        out = _results(lambda: x.new_empty(x.shape), stream)
    else:
        _check(out, "out", x.dtype, x.shape)
    ws = _sized(workspace, lambda: lib.ll_selective_scan_workspace_size(s.batch, s.T, s.channels, s.N, s.groups, 0), x.device, stream)
    _ok(lib.ll_selective_scan_fwd(s, _ptr(initial_state), out.data_ptr(), _ptr(final_state), _ptr(states),
                                  _ptr(ws), ws.numel(), _stream(stream)))
    return out


def ll_selective_scan_step(x, dt, A, B, C, state, D=None, z=None, dt_bias=None, delta_softplus=True, new_state=None,
                           out=None, stream=None):
    """One token: x, dt, z [B, D], B, C [B, N] (or [B, groups, N]); returns y [B, D].  `state` [B, D, N] is read,
    `new_state` written (None: in place)."""
    s = _scan_inputs(x, dt, A, B, C, D, z, dt_bias, delta_softplus, None, True)
    shape = (s.batch, s.channels, s.N)
    _check(state, "state", torch.float32, shape)
    _opt(new_state, "new_state", torch.float32, shape)
    if out is None:
        out = _results(lambda: x.new_empty(x.shape), stream)
    else:
        _check(out, "out", x.dtype, x.shape)
    _ok(lib.ll_selective_scan_step(s, state.data_ptr(), (state if new_state is None else new_state).data_ptr(),
                                   out.data_ptr(), _stream(stream)))
    return out


def ll_selective_scan_bwd(x, dt, A, B, C, states, d_y, D=None, z=None, dt_bias=None, delta_softplus=True, lengths=None,
                          d_final_state=None, initial_state_grad=False, grads=None, workspace=None, stream=None):
    """Gradients of the ll_selective_scan_fwd that left `states`, on the same inputs: a ScanGrads (x, dt, A, B, C,
    D, z, dt_bias, initial_state) of new tensors, or `grads` filled in; those of inputs that are None are None, that
    of the initial state unless `initial_state_grad`."""
    s = _scan_inputs(x, dt, A, B, C, D, z, dt_bias, delta_softplus, lengths, False)
    shape = (s.batch, s.channels, s.N)
    _check_states(states, s)
    _check(d_y, "d_y", x.dtype, x.shape)
    _opt(d_final_state, "d_final_state", torch.float32, shape)
    if grads is None:
        new = x.new_empty
        grads = _results(lambda: ScanGrads(new(x.shape), new(x.shape), torch.empty_like(A), new(B.shape), new(C.shape),
                                           None if D is None else torch.empty_like(D),
                                           None if z is None else new(x.shape),
                                           None if dt_bias is None else torch.empty_like(dt_bias),
                                           A.new_empty(shape) if initial_state_grad else None), stream)
    g = ScanGrads(*grads)
    _check(g.x, "grads.x", x.dtype, x.shape)
    _check(g.dt, "grads.dt", x.dtype, x.shape)
    _check(g.A, "grads.A", torch.float32, A.shape)
    _check(g.B, "grads.B", x.dtype, B.shape)
    _check(g.C, "grads.C", x.dtype, C.shape)
    _opt(g.D, "grads.D", torch.float32, (s.channels,))
    _opt(g.z, "grads.z", x.dtype, x.shape)
    _opt(g.dt_bias, "grads.dt_bias", torch.float32, (s.channels,))
    _opt(g.initial_state, "grads.initial_state", torch.float32, shape)
    ws = _sized(workspace, lambda: lib.ll_selective_scan_workspace_size(s.batch, s.T, s.channels, s.N, s.groups, 1), x.device, stream)
    _ok(lib.ll_selective_scan_bwd(s, states.data_ptr(), d_y.data_ptr(), _ptr(d_final_state), g.x.data_ptr(),
                                  g.dt.data_ptr(), _ptr(g.z), g.A.data_ptr(), g.B.data_ptr(), g.C.data_ptr(),
                                  _ptr(g.D), _ptr(g.dt_bias), _ptr(g.initial_state), _ptr(ws), ws.numel(),
                                  _stream(stream)))
    return grads


# ------------------------------------------------------------------------------------ group norm

def _norm_args(x, groups, weight, bias, gate):
    N, S, C = _dims(x, "x", 3)
    _rows(x, "x", x.dtype, x.shape)
    if gate is not None:
        _rows(gate, "gate", x.dtype, x.shape)
    _opt(weight, "weight", torch.float32, (C,))
    _opt(bias, "bias", torch.float32, (C,))
    rows = (x.data_ptr(), x.stride(0), _token_stride(x))
    return rows + ((None, 0, 0) if gate is None else (gate.data_ptr(), gate.stride(0), _token_stride(gate)))


def _norm_need(x, groups, backward):
    N, S, C = x.shape
    return lib.ll_group_norm_workspace_size(_dtype_code(x), N, S, C, groups, int(backward))


def ll_group_norm_workspace(x, groups, backward=False):
    """A workspace for the forward (or backward) group norm of x [N, S, C]."""
    _dims(x, "x", 3)
    return _buffer(_norm_need(x, groups, backward), x.device)


def ll_group_norm_stats(x, groups):
    """The [N, groups, 2] float32 tensor in which a forward leaves its statistics for the backward."""
    return torch.empty((_dims(x, "x", 3)[0], groups, 2), dtype=torch.float32, device=x.device)


def ll_group_norm_fwd(x, groups, weight=None, bias=None, gate=None, eps=1e-5, act=LL_ACT_SILU, stats=None, out=None,
                      workspace=None, stream=None):
    """Group norm of x [N, S, C] over its S tokens and each group's channels: u = normalised * weight + bias;
    returns act(u), or u * act(gate).  To normalise every token of [B, T, C] by itself pass x.view(B * T, 1, C)."""
    rows = _norm_args(x, groups, weight, bias, gate)
    N, S, C = x.shape
    _opt(stats, "stats", torch.float32, (N, groups, 2))
    code = _dtype_code(x)
    if out is None:
        out = _results(lambda: x.new_empty(x.shape), stream)
    else:
        _check(out, "out", x.dtype, x.shape)
    ws = _sized(workspace, lambda: _norm_need(x, groups, False), x.device, stream)
    _ok(lib.ll_group_norm_fwd(*rows, _ptr(weight), _ptr(bias), out.data_ptr(), _ptr(stats), N, S, C, groups, eps, act,
                              code, _ptr(ws), ws.numel(), _stream(stream)))
    return out


def ll_group_norm_bwd(x, groups, weight, bias, stats, d_y, gate=None, act=LL_ACT_SILU, grads=None, workspace=None,
                      stream=None):
    """Gradients of the ll_group_norm_fwd that left `stats`: a NormGrads (x, weight, bias, gate) of new tensors, or
    `grads` filled in; those of inputs that are None are None."""
    rows = _norm_args(x, groups, weight, bias, gate)
    N, S, C = x.shape
    _check(stats, "stats", torch.float32, (N, groups, 2))
    _check(d_y, "d_y", x.dtype, x.shape)
    code = _dtype_code(x)
    if grads is None:
        grads = _results(lambda: NormGrads(x.new_empty(x.shape), None if weight is None else torch.empty_like(weight),
                                           None if bias is None else torch.empty_like(bias),
                                           None if gate is None else x.new_empty(x.shape)), stream)
    g = NormGrads(*grads)
    _check(g.x, "grads.x", x.dtype, x.shape)
    _opt(g.weight, "grads.weight", torch.float32, (C,))
    _opt(g.bias, "grads.bias", torch.float32, (C,))
    _opt(g.gate, "grads.gate", x.dtype, x.shape)
    ws = _sized(workspace, lambda: _norm_need(x, groups, True), x.device, stream)
    _ok(lib.ll_group_norm_bwd(*rows, _ptr(weight), _ptr(bias), stats.data_ptr(), d_y.data_ptr(), g.x.data_ptr(),
                              _ptr(g.gate), _ptr(g.weight), _ptr(g.bias), N, S, C, groups, act, code, _ptr(ws),
                              ws.numel(), _stream(stream)))
    return grads


# ------------------------------------------------------------------------------------ autograd

def _dense(t):
    return None if t is None else t.contiguous()


def _channels_last(t):
    """`t` as it is where its channels are adjacent, else a copy (a gradient's strides are not the caller's choice)."""
    return t if t is None or t.stride(-1) == 1 else t.contiguous()


class _CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, initial_state, lengths, act, want_state):
        x, weight, bias = _channels_last(x), weight.contiguous(), _dense(bias)
        initial_state = _dense(initial_state)
        final = x.new_empty((x.shape[0], weight.shape[1] - 1, x.shape[2])) if want_state else None
        y = ll_causal_conv_fwd(x, weight, bias, act, initial_state, final, lengths)
        ctx.save_for_backward(x, weight, bias, initial_state, lengths)
        ctx.act = act
        ctx.set_materialize_grads(False)
        return y, final

    @staticmethod
    def backward(ctx, d_y, d_final):
        x, weight, bias, initial_state, lengths = ctx.saved_tensors
        d_y = x.new_zeros(x.shape) if d_y is None else d_y.contiguous()
        g = ll_causal_conv_bwd(x, weight, bias, d_y, ctx.act, initial_state, lengths, _dense(d_final))
        return (*_once(g), None, None, None)


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, A, B, C, D, z, dt_bias, initial_state, lengths, delta_softplus, want_state):
        _groups(B, "B", 3), _groups(C, "C", 3)
        x, dt, z, B, C = (_channels_last(t) for t in (x, dt, z, B, C))
        if B.dim() == C.dim() == 4:  # groups of a token adjacent
            B, C = (t if t.stride(2) == t.shape[3] else t.contiguous() for t in (B, C))
        A, D, dt_bias, initial_state = (_dense(t) for t in (A, D, dt_bias, initial_state))
        final = A.new_empty((x.shape[0], *A.shape)) if want_state else None
        states = ll_selective_scan_states(x, B) if any(ctx.needs_input_grad) else None
        y = ll_selective_scan_fwd(x, dt, A, B, C, D, z, dt_bias, delta_softplus, initial_state, final, lengths, states)
        ctx.save_for_backward(x, dt, A, B, C, D, z, dt_bias, lengths, states)
        ctx.delta_softplus, ctx.from_state = delta_softplus, initial_state is not None
        ctx.set_materialize_grads(False)
        return y, final

    @staticmethod
    def backward(ctx, d_y, d_final):
        x, dt, A, B, C, D, z, dt_bias, lengths, states = ctx.saved_tensors
        d_y = x.new_zeros(x.shape) if d_y is None else d_y.contiguous()
        g = ll_selective_scan_bwd(x, dt, A, B, C, states, d_y, D, z, dt_bias, ctx.delta_softplus, lengths,
                                  _dense(d_final), ctx.from_state)
        return (*_once(g), None, None, None)


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, gate, groups, eps, act):
        x, gate, weight, bias = _channels_last(x), _channels_last(gate), _dense(weight), _dense(bias)
        stats = ll_group_norm_stats(x, groups)
        y = ll_group_norm_fwd(x, groups, weight, bias, gate, eps, act, stats)
        ctx.save_for_backward(x, weight, bias, gate, stats)
        ctx.groups, ctx.act = groups, act
        return y

    @staticmethod
    def backward(ctx, d_y):
        x, weight, bias, gate, stats = ctx.saved_tensors
        g = ll_group_norm_bwd(x, ctx.groups, weight, bias, stats, d_y.contiguous(), gate, ctx.act)
        return (*_once(g), None, None, None)


def causal_conv(x, weight, bias=None, act=LL_ACT_SILU, initial_state=None, lengths=None, return_final_state=False):
    """Differentiable ll_causal_conv_fwd: y, or (y, final state); gradients flow to x, weight, bias and the states."""
    y, final = _CausalConv.apply(x, weight, bias, initial_state, lengths, act, return_final_state)
    return (y, final) if return_final_state else y


def selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, delta_softplus=True, initial_state=None, lengths=None,
                   return_final_state=False):
    """Differentiable ll_selective_scan_fwd: y, or (y, final state); gradients flow to every tensor but lengths.
    Memory held until the graph is freed: the inputs and ll_selective_scan_states_bytes(...) bytes."""
    y, final = _SelectiveScan.apply(x, dt, A, B, C, D, z, dt_bias, initial_state, lengths, delta_softplus,
                                    return_final_state)
    return (y, final) if return_final_state else y


def group_norm(x, groups, weight=None, bias=None, gate=None, eps=1e-5, act=LL_ACT_SILU):
    """Differentiable ll_group_norm_fwd; gradients flow to x, weight, bias and gate."""
    return _GroupNorm.apply(x, weight, bias, gate, groups, eps, act)
