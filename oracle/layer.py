"""Float64 oracle of the operators around a token mixer: the short causal convolution, the selective state
space scan, the group norm, the linear attention with a decay for each head and the projections, each with its gradients.  Token by token and group by group, from the formulas;
`lengths` ends the sequences of a batch early."""

import numpy as np


def _f64(*xs):
    return [None if x is None else np.asarray(x, dtype=np.float64) for x in xs]


def sigmoid(v):
    return 1.0 / (1.0 + np.exp(-v))


def act(v, on):
    return v * sigmoid(v) if on else v


def act_grad(v, on):
    s = sigmoid(v)
    return s * (1 + v * (1 - s)) if on else np.ones_like(v)


def _ends(lengths, B, T):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


# ------------------------------------------------------------------------------------ convolution

def conv(x, w, bias=None, silu=True, initial=None, lengths=None):
    """(y, final state): y_t = act(bias + sum_j w_j e_(t+j)), e = the W - 1 tokens before the first, then x."""
    x, w, bias, initial = _f64(x, w, bias, initial)
    B, T, D = x.shape
    W = w.shape[1]
    y, final = np.zeros((B, T, D)), np.zeros((B, W - 1, D))
    for b, n in enumerate(_ends(lengths, B, T)):
        e = np.concatenate([np.zeros((W - 1, D)) if initial is None else initial[b], x[b, :n]])
        for t in range(n):
            y[b, t] = act((0.0 if bias is None else bias) + sum(w[:, j] * e[t + j] for j in range(W)), silu)
        final[b] = e[n:]
    return y, final


def conv_grad(x, w, d_y, bias=None, silu=True, initial=None, lengths=None, d_final=None):
    """Gradients of sum(y d_y) + sum(final d_final): (dx, dw, dbias, dinitial)."""
    x, w, d_y, bias, initial, d_final = _f64(x, w, d_y, bias, initial, d_final)
    B, T, D = x.shape
    W = w.shape[1]
    dx, dw, db, di = np.zeros((B, T, D)), np.zeros((D, W)), np.zeros(D), np.zeros((B, W - 1, D))
    for b, n in enumerate(_ends(lengths, B, T)):
        e = np.concatenate([np.zeros((W - 1, D)) if initial is None else initial[b], x[b, :n]])
        de = np.zeros_like(e)
        if d_final is not None:
            de[n:] += d_final[b]
        for t in range(n):
            v = (0.0 if bias is None else bias) + sum(w[:, j] * e[t + j] for j in range(W))
            dv = d_y[b, t] * act_grad(v, silu)
            db += dv
            for j in range(W):
                dw[:, j] += dv * e[t + j]
                de[t + j] += dv * w[:, j]
        di[b], dx[b, :n] = de[:W - 1], de[W - 1:]
    return dx, dw, db, di


# ------------------------------------------------------------------------------------ selective scan

def softplus(v):
    return np.logaddexp(0.0, v)


def _scan_states(x, dt, A, Bm, dt_bias, with_softplus, h0, n):
    """Step sizes and the states h_0 (before the first token), h_1, .. of one sequence of n tokens."""
    pre = dt[:n] + (0.0 if dt_bias is None else dt_bias)
    delta = softplus(pre) if with_softplus else pre
    D, N = A.shape
    per = D // Bm.shape[1]
    h = [np.zeros((D, N)) if h0 is None else h0]
    for t in range(n):
        Bt = np.repeat(Bm[t], per, axis=0)  # [D, N]
        h.append(np.exp(delta[t][:, None] * A) * h[-1] + (delta[t] * x[t])[:, None] * Bt)
    return pre, delta, h


def scan(x, dt, A, Bm, Cm, skip=None, z=None, dt_bias=None, with_softplus=True, initial=None, lengths=None):
    """(y, final state) with Bm, Cm [B, T, G, N]."""
    x, dt, A, Bm, Cm, skip, z, dt_bias, initial = _f64(x, dt, A, Bm, Cm, skip, z, dt_bias, initial)
    B, T, D = x.shape
    per = D // Bm.shape[2]
    y, final = np.zeros((B, T, D)), np.zeros((B, *A.shape))
    for b, n in enumerate(_ends(lengths, B, T)):
        _, _, h = _scan_states(x[b], dt[b], A, Bm[b], dt_bias, with_softplus, None if initial is None else initial[b], n)
        for t in range(n):
            o = (np.repeat(Cm[b, t], per, axis=0) * h[t + 1]).sum(1)
            if skip is not None:
                o = o + skip * x[b, t]
            y[b, t] = o if z is None else o * act(z[b, t], True)
        final[b] = h[-1]
    return y, final


def scan_grad(x, dt, A, Bm, Cm, d_y, skip=None, z=None, dt_bias=None, with_softplus=True, initial=None, lengths=None,
              d_final=None):
    """Gradients of sum(y d_y) + sum(final d_final), as a dict."""
    x, dt, A, Bm, Cm, d_y, skip, z, dt_bias, initial, d_final = _f64(x, dt, A, Bm, Cm, d_y, skip, z, dt_bias, initial,
                                                                     d_final)
    B, T, D = x.shape
    G, N = Bm.shape[2:]
    per = D // G
    g = {"x": np.zeros((B, T, D)), "dt": np.zeros((B, T, D)), "A": np.zeros((D, N)), "B": np.zeros((B, T, G, N)),
         "C": np.zeros((B, T, G, N)), "D": np.zeros(D), "z": np.zeros((B, T, D)), "dt_bias": np.zeros(D),
         "initial": np.zeros((B, D, N))}
    for b, n in enumerate(_ends(lengths, B, T)):
        pre, delta, h = _scan_states(x[b], dt[b], A, Bm[b], dt_bias, with_softplus,
                                     None if initial is None else initial[b], n)
        gh = np.zeros((D, N)) if d_final is None else d_final[b].copy()
        for t in range(n - 1, -1, -1):
            Bt, Ct = np.repeat(Bm[b, t], per, axis=0), np.repeat(Cm[b, t], per, axis=0)
            do = d_y[b, t]
            if z is not None:
                o = (Ct * h[t + 1]).sum(1) + (0.0 if skip is None else skip * x[b, t])
                g["z"][b, t] = do * o * act_grad(z[b, t], True)
                do = do * act(z[b, t], True)
            gh = gh + Ct * do[:, None]
            g["C"][b, t] = (h[t + 1] * do[:, None]).reshape(G, per, N).sum(1)
            g["B"][b, t] = (gh * (delta[t] * x[b, t])[:, None]).reshape(G, per, N).sum(1)
            a = np.exp(delta[t][:, None] * A)
            along = (gh * Bt).sum(1)
            g["x"][b, t] = delta[t] * along + (0.0 if skip is None else skip * do)
            g["D"] += do * x[b, t]
            q = a * h[t] * gh
            g["A"] += q * delta[t][:, None]
            dd = x[b, t] * along + (q * A).sum(1)
            g["dt"][b, t] = dd * sigmoid(pre[t]) if with_softplus else dd
            g["dt_bias"] += g["dt"][b, t]
            gh = a * gh
        g["initial"][b] = gh
    return g


# ------------------------------------------------------------------------------------ group norm

def norm(x, G, w=None, b=None, z=None, eps=1e-5, silu=True):
    x, w, b, z = _f64(x, w, b, z)
    N, S, C = x.shape
    v = x.reshape(N, S, G, C // G)
    mean = v.mean((1, 3), keepdims=True)
    xh = ((v - mean) / np.sqrt(((v - mean) ** 2).mean((1, 3), keepdims=True) + eps)).reshape(N, S, C)
    u = xh * (1.0 if w is None else w) + (0.0 if b is None else b)
    return act(u, silu) if z is None else u * act(z, silu)


def norm_grad(x, G, d_y, w=None, b=None, z=None, eps=1e-5, silu=True):
    """(dx, dw, db, dz)."""
    x, d_y, w, b, z = _f64(x, d_y, w, b, z)
    N, S, C = x.shape
    v = x.reshape(N, S, G, C // G)
    mean = v.mean((1, 3), keepdims=True)
    r = 1.0 / np.sqrt(((v - mean) ** 2).mean((1, 3), keepdims=True) + eps)
    xh = ((v - mean) * r).reshape(N, S, C)
    w1 = np.ones(C) if w is None else w
    u = xh * w1 + (0.0 if b is None else b)
    if z is None:
        du, dz = d_y * act_grad(u, silu), None
    else:
        du, dz = d_y * act(z, silu), d_y * u * act_grad(z, silu)
    g = (du * w1).reshape(v.shape)
    xg = xh.reshape(v.shape)
    dx = r * (g - g.mean((1, 3), keepdims=True) - xg * (g * xg).mean((1, 3), keepdims=True))
    return dx.reshape(N, S, C), (du * xh).sum((0, 1)), du.sum((0, 1)), dz


# ------------------------------------------------------------------------------------ decay attention

def _shared(x, H):
    return np.repeat(x, H // x.shape[2], axis=2)


def decay_attention(q, k, v, log_decay, scale=1.0, initial=None, lengths=None):
    """(o, final state): S_t = g S_(t-1) + k_t v_t^T, o_t = scale S_t^T q_t; heads share q and k in groups."""
    q, k, v, log_decay, initial = _f64(q, k, v, log_decay, initial)
    B, T, H, dv = v.shape
    q, k, g = _shared(q, H), _shared(k, H), np.exp(log_decay)[:, None, None]
    o, final = np.zeros((B, T, H, dv)), np.zeros((B, H, q.shape[-1], dv))
    for b, n in enumerate(_ends(lengths, B, T)):
        S = final[b].copy() if initial is None else initial[b]
        for t in range(n):
            S = g * S + k[b, t, :, :, None] * v[b, t, :, None, :]
            o[b, t] = scale * (q[b, t, :, :, None] * S).sum(1)
        final[b] = S
    return o, final


def decay_attention_grad(q, k, v, log_decay, d_o, scale=1.0, initial=None, lengths=None, d_final=None):
    """Gradients of sum(o d_o) + sum(final d_final): (dq, dk, dv, dinitial)."""
    q, k, v, log_decay, d_o, initial, d_final = _f64(q, k, v, log_decay, d_o, initial, d_final)
    B, T, H, dv = v.shape
    heads, group = q.shape[2], H // q.shape[2]
    q, k, g = _shared(q, H), _shared(k, H), np.exp(log_decay)[:, None, None]
    dq, dk, dv_, di = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros((B, H, q.shape[-1], dv))
    for b, n in enumerate(_ends(lengths, B, T)):
        S = np.zeros_like(di[b]) if initial is None else initial[b]
        for t in range(n):
            S = g * S + k[b, t, :, :, None] * v[b, t, :, None, :]
            dq[b, t] = scale * (S * d_o[b, t, :, None, :]).sum(2)
        D = np.zeros_like(di[b]) if d_final is None else d_final[b].copy()
        for t in reversed(range(n)):
            D = D + scale * q[b, t, :, :, None] * d_o[b, t, :, None, :]
            dk[b, t] = (D * v[b, t, :, None, :]).sum(2)
            dv_[b, t] = (D * k[b, t, :, :, None]).sum(1)
            D = g * D
        di[b] = D
    dq, dk = (x.reshape(B, T, heads, group, -1).sum(3) for x in (dq, dk))
    return dq, dk, dv_, di


# ------------------------------------------------------------------------------------ projection

def projection(x, w, bias=None, residual=None, silu=False):
    """(y, u): u = x w^T + bias, y = act(u) + residual."""
    x, w, bias, residual = _f64(x, w, bias, residual)
    u = x @ w.T + (0.0 if bias is None else bias)
    return act(u, silu) + (0.0 if residual is None else residual), u


def projection_grad(x, w, d_y, bias=None, silu=False):
    """Gradients of sum(y d_y): (dx, dw, dbias)."""
    x, w, d_y = _f64(x, w, d_y)
    du = d_y * act_grad(projection(x, w, bias)[1], silu)
    return du @ w, du.T @ x, du.sum(0)
