"""Gated delta rule in fp64, token by token, and the adjoint of that walk (test infrastructure).

  S~_t = alpha_t S_{t-1};  w_t = v_t - S~_t^T k_t;  S_t = S~_t + beta_t k_t w_t^T;  out_t = S_t^T q_t

Arrays: q, k [B,H,L,dk]; v [B,H,L,dv]; log_alpha, beta [B,H,L]; states [B,H,dk,dv].
"""
import numpy as np


def gdr_fwd(q, k, v, log_alpha, beta, state=None, reverse=False, keep=None):
    """out and the last state; keep (a list) receives (t, S~_t, w_t) of every token in walking order."""
    B, H, L, dk = q.shape
    S = np.zeros((B, H, dk, v.shape[3])) if state is None else np.array(state, dtype=np.float64)
    out = np.zeros(v.shape)
    for t in range(L - 1, -1, -1) if reverse else range(L):
        S = S * np.exp(log_alpha[:, :, t])[..., None, None]
        w = v[:, :, t] - np.matmul(k[:, :, t, None, :], S)[:, :, 0]
        if keep is not None:
            keep.append((t, S, w))
        S = S + (beta[:, :, t, None] * k[:, :, t])[..., None] * w[:, :, None, :]
        out[:, :, t] = np.matmul(q[:, :, t, None, :], S)[:, :, 0]
    return out, S


def gdr_bwd(q, k, v, log_alpha, beta, d_out, state=None, d_state=None, reverse=False):
    """dq, dk, dv, dlog_alpha, dbeta and the gradient with respect to the initial state."""
    walk = []
    _, last = gdr_fwd(q, k, v, log_alpha, beta, state, reverse, walk)
    D = np.zeros(last.shape) if d_state is None else np.array(d_state, dtype=np.float64)
    dq, dk, dv, dl, db = (np.zeros(x.shape) for x in (q, k, v, log_alpha, beta))
    row = lambda x, S: np.matmul(x[:, :, None, :], S)[:, :, 0]             # x^T S
    col = lambda S, x: np.matmul(S, x[..., None])[..., 0]                  # S x
    for t, decayed, w in reversed(walk):
        b, kt, g = beta[:, :, t, None], k[:, :, t], d_out[:, :, t]
        S = decayed + (b * kt)[..., None] * w[:, :, None, :]
        dq[:, :, t] = col(S, g)
        D = D + q[:, :, t][..., None] * g[:, :, None, :]
        # S_t = decayed + k u^T with u = beta w, w = v - decayed^T k
        du = row(kt, D)
        dw = b * du
        db[:, :, t] = (du * w).sum(-1)
        dv[:, :, t] = dw
        dk[:, :, t] = col(D, b * w) - col(decayed, dw)
        D = D - kt[..., None] * dw[:, :, None, :]
        dl[:, :, t] = (D * decayed).sum((-1, -2))
        D = D * np.exp(log_alpha[:, :, t])[..., None, None]
    return dq, dk, dv, dl, db, D
