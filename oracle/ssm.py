"""Selective state space scan, causal convolution and RMS norm in fp64, and their gradients (test infrastructure).

  scan:  d_t = softplus(dt_t + bias);  h_t[c,n] = exp(d_t A[c,n]) h_{t-1}[c,n] + d_t x_t B_t[n];  y_t = sum_n C_t[n] h_t[c,n] + D x_t;
         out = y silu(z)
  conv:  out_t = act(bias + sum_k w[:, k] x_{t-K+1+k})
  norm:  s = x + residual;  out = s / sqrt(mean s^2 + eps) weight

Arrays: x, dt, z [B,L,C]; Bt, Ct [B,L,G,N]; A [C,N]; D, bias [C]; scan states [B,C,N]; conv states [B,K-1,C], oldest token first.
"""
import numpy as np


def _sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1 / (1 + e), e / (1 + e))


def _softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def _channels(rows, C):
    """[B, G, N] of one token -> [B, C, N]"""
    return np.repeat(rows, C // rows.shape[1], axis=1)


def _groups(per_channel, G):
    B, C, N = per_channel.shape
    return per_channel.reshape(B, G, C // G, N).sum(2)


def _order(L, reverse):
    return range(L - 1, -1, -1) if reverse else range(L)


def ssm_fwd(x, dt, A, Bt, Ct, D=None, z=None, bias=None, state=None, softplus=True, reverse=False, keep=None):
    """out and the last state; keep (a list) receives (t, state in front of the token) in walking order."""
    B, L, C = x.shape
    v = dt + (0.0 if bias is None else bias)
    d = _softplus(v) if softplus else v
    h = np.zeros((B, C, A.shape[1])) if state is None else np.array(state, dtype=np.float64)
    y = np.zeros(x.shape)
    for t in _order(L, reverse):
        if keep is not None:
            keep.append((t, h))
        h = np.exp(d[:, t, :, None] * A) * h + (d[:, t] * x[:, t])[..., None] * _channels(Bt[:, t], C)
        y[:, t] = (h * _channels(Ct[:, t], C)).sum(-1)
    if D is not None:
        y = y + D * x
    return y if z is None else y * z * _sigmoid(z), h


def ssm_bwd(x, dt, A, Bt, Ct, d_out, D=None, z=None, bias=None, state=None, d_state=None, softplus=True, reverse=False):
    """dict of dx, ddt, dA, dB, dC, dD, dz, dbias and d_state (of the initial state)."""
    B, L, C = x.shape
    G = Bt.shape[2]
    walk = []
    ssm_fwd(x, dt, A, Bt, Ct, state=state, bias=bias, softplus=softplus, reverse=reverse, keep=walk)
    v = dt + (0.0 if bias is None else bias)
    d, slope = (_softplus(v), _sigmoid(v)) if softplus else (v, np.ones_like(v))
    skip = np.zeros(C) if D is None else D
    s = None if z is None else _sigmoid(z)
    dy = d_out if z is None else d_out * z * s
    r = {"dx": skip * dy, "ddt": np.zeros(x.shape), "dA": np.zeros(A.shape), "dB": np.zeros(Bt.shape), "dC": np.zeros(Ct.shape),
         "dD": (dy * x).sum((0, 1)), "dz": np.zeros(x.shape)}
    g = np.zeros((B, C, A.shape[1])) if d_state is None else np.array(d_state, dtype=np.float64)
    for t, before in reversed(walk):
        b, c = _channels(Bt[:, t], C), _channels(Ct[:, t], C)
        a = np.exp(d[:, t, :, None] * A)
        h = a * before + (d[:, t] * x[:, t])[..., None] * b
        g = g + c * dy[:, t, :, None]
        r["dC"][:, t] = _groups(h * dy[:, t, :, None], G)
        r["dB"][:, t] = _groups(g * (d[:, t] * x[:, t])[..., None], G)
        into, through = (g * b).sum(-1), g * a * before
        r["dx"][:, t] += d[:, t] * into
        r["ddt"][:, t] = ((through * A).sum(-1) + x[:, t] * into) * slope[:, t]
        r["dA"] += (through * d[:, t, :, None]).sum(0)
        if z is not None:
            r["dz"][:, t] = d_out[:, t] * ((h * c).sum(-1) + skip * x[:, t]) * s[:, t] * (1 + z[:, t] * (1 - s[:, t]))
        g = g * a
    r["dbias"], r["d_state"] = r["ddt"].sum((0, 1)), g
    return r


def _line(x, state, K, reverse):
    B, L, C = x.shape
    past = np.zeros((B, K - 1, C)) if state is None else state
    return np.concatenate([past, x[:, ::-1] if reverse else x], 1)


def _conv_pre(line, w, bias, L):
    K = w.shape[1]
    v = sum(line[:, k:k + L] * w[:, k] for k in range(K))
    return v if bias is None else v + bias


def causal_conv(x, w, bias=None, act="silu", state=None, reverse=False):
    """out and the state behind the last token."""
    L = x.shape[1]
    line = _line(x, state, w.shape[1], reverse)
    v = _conv_pre(line, w, bias, L)
    out = v * _sigmoid(v) if act == "silu" else v
    return out[:, ::-1] if reverse else out, line[:, L:]


def causal_conv_bwd(x, w, bias, d_out, act="silu", state=None, d_state=None, reverse=False):
    """dx, dw, dbias and the gradient of the window in front."""
    L, K = x.shape[1], w.shape[1]
    line = _line(x, state, K, reverse)
    v = _conv_pre(line, w, bias, L)
    g = d_out[:, ::-1] if reverse else d_out
    if act == "silu":
        s = _sigmoid(v)
        g = g * s * (1 + v * (1 - s))
    dl = np.zeros(line.shape)
    dw = np.zeros(w.shape)
    for k in range(K):
        dl[:, k:k + L] += g * w[:, k]
        dw[:, k] = (g * line[:, k:k + L]).sum((0, 1))
    if d_state is not None:
        dl[:, L:] += d_state
    dx = dl[:, K - 1:]
    return dx[:, ::-1] if reverse else dx, dw, g.sum((0, 1)), dl[:, :K - 1]


def rms_norm(x, weight, residual=None, eps=1e-5):
    """out, the sum, 1 / sqrt(mean s^2 + eps)."""
    s = x if residual is None else x + residual
    rstd = 1 / np.sqrt((s * s).mean(-1) + eps)
    return s * rstd[..., None] * weight, s, rstd


def rms_norm_bwd(s, weight, rstd, d_out, d_sum=None):
    """dx, dweight."""
    xhat = s * rstd[..., None]
    gw = d_out * weight
    dx = rstd[..., None] * (gw - xhat * (gw * xhat).mean(-1, keepdims=True))
    return dx if d_sum is None else dx + d_sum, (d_out * xhat).reshape(-1, s.shape[-1]).sum(0)
