"""The oracles of the gated delta rule and of the group norm against closed forms, other formulas and finite differences (CPU)."""
import numpy as np
import pytest

import oracle

RNG = np.random.default_rng(11)


def _inputs(B=1, H=2, L=7, dk=4, dv=3, states=True):
    n = RNG.standard_normal
    k = n((B, H, L, dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    x = [n((B, H, L, dk)), k, n((B, H, L, dv)), -np.abs(n((B, H, L))) / 4, 1 / (1 + np.exp(-n((B, H, L))))]
    return x, (n((B, H, dk, dv)) if states else None)


def test_triangular_system_of_the_whole_sequence():
    """u solves (1 + tril(beta k k^T decay, -1)) u = beta (v - decay k S_0)."""
    (q, k, v, la, be), S0 = _inputs()
    out, last = oracle.gdr_fwd(q, k, v, la, be, S0)
    b = np.cumsum(la, -1)
    decay = np.tril(np.exp(b[..., :, None] - b[..., None, :]))
    M = np.eye(7) + np.tril(be[..., None] * (k @ np.swapaxes(k, -1, -2)) * decay, -1)
    u = np.linalg.solve(M, be[..., None] * (v - np.exp(b)[..., None] * (k @ S0)))
    want = np.exp(b)[..., None] * (q @ S0) + ((q @ np.swapaxes(k, -1, -2)) * decay) @ u
    assert np.allclose(out, want, rtol=0, atol=1e-12)
    end = np.exp(b[..., -1])[..., None, None] * S0 + np.swapaxes(k * np.exp(b[..., -1:] - b)[..., None], -1, -2) @ u
    assert np.allclose(last, end, rtol=0, atol=1e-12)


def test_orthonormal_keys_store_and_overwrite():
    """beta = 1, no decay: after (e1, a), (e2, b), (e1, c) the state holds c at e1 and b at e2."""
    k = np.zeros((1, 1, 3, 2))
    k[0, 0, 0, 0] = k[0, 0, 1, 1] = k[0, 0, 2, 0] = 1
    v = RNG.standard_normal((1, 1, 3, 5))
    out, S = oracle.gdr_fwd(k, k, v, np.zeros((1, 1, 3)), np.ones((1, 1, 3)))
    assert np.allclose(S[0, 0], v[0, 0, [2, 1]]) and np.allclose(out, v)


def test_beta_zero_only_decays_and_minus_infinity_forgets():
    (q, k, v, la, be), S0 = _inputs()
    out, last = oracle.gdr_fwd(q, k, v, la, 0 * be, S0)
    assert np.allclose(last, S0 * np.exp(la.sum(-1))[..., None, None])
    la[:, :, 3] = -np.inf
    a, _ = oracle.gdr_fwd(q, k, v, la, be, S0)
    b, _ = oracle.gdr_fwd(q[:, :, 3:], k[:, :, 3:], v[:, :, 3:], la[:, :, 3:], be[:, :, 3:])
    assert np.allclose(a[:, :, 3:], b)


def test_reverse_is_the_flipped_sequence_and_cuts_join():
    (q, k, v, la, be), S0 = _inputs()
    f = lambda a: np.flip(a, 2)
    a, la_ = oracle.gdr_fwd(q, k, v, la, be, S0, reverse=True)
    b, lb_ = oracle.gdr_fwd(f(q), f(k), f(v), f(la), f(be), S0)
    assert np.array_equal(a, f(b)) and np.array_equal(la_, lb_)
    o, S = oracle.gdr_fwd(q, k, v, la, be, S0)
    x = [t[:, :, :4] for t in (q, k, v, la, be)], [t[:, :, 4:] for t in (q, k, v, la, be)]
    o1, S1 = oracle.gdr_fwd(*x[0], S0)
    o2, S2 = oracle.gdr_fwd(*x[1], S1)
    assert np.allclose(np.concatenate((o1, o2), 2), o, atol=1e-13) and np.allclose(S, S2, atol=1e-13)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("states", [False, True])
def test_gradient_against_differences(reverse, states):
    x, S0 = _inputs(L=5, states=states)
    do, dS = RNG.standard_normal(x[2].shape), RNG.standard_normal((1, 2, 4, 3)) if states else None
    args = x + ([S0] if states else [])
    grads = oracle.gdr_bwd(*x, do, S0, dS, reverse)

    def loss():
        o, S = oracle.gdr_fwd(*args, reverse=reverse)
        return (o * do).sum() + ((S * dS).sum() if states else 0.0)

    for a, g in zip(args, grads):
        for i in range(a.size):
            at, h = np.unravel_index(i, a.shape), 1e-6
            old = a[at]
            a[at] = old + h
            up = loss()
            a[at] = old - h
            down = loss()
            a[at] = old
            # central differences: h^2 / 6 times a third derivative, and rounding 2^-53 |loss| / h
            assert abs((up - down) / (2 * h) - g[at]) <= 1e-8 * max(1.0, abs(g[at]))


def test_gate_gradient_as_running_sums():
    """dlog_alpha_t = sum_{s >= t} (q . dq - v . dv) + <S_L, dS_L>."""
    x, S0 = _inputs(L=9)
    do, dS = RNG.standard_normal(x[2].shape), RNG.standard_normal(S0.shape)
    _, last = oracle.gdr_fwd(*x, S0)
    dq, dk, dv, dl, db, _ = oracle.gdr_bwd(*x, do, S0, dS)
    E = (x[0] * dq).sum(-1) - (x[2] * dv).sum(-1)
    want = np.flip(np.cumsum(np.flip(E, -1), -1), -1) + (last * dS).sum((-1, -2))[..., None]
    assert np.allclose(dl, want, atol=1e-12)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_group_norm_gradient_against_differences(act):
    x, w, b = RNG.standard_normal((2, 2, 3, 6)) + 0.5, RNG.standard_normal(6), RNG.standard_normal(6)
    do = RNG.standard_normal(x.shape)
    out, mean, rstd = oracle.group_norm(x, w, b, 2, 1e-5, act)
    if act == "none":
        y = ((out - b) / w).reshape(2, 6, 2, 3)
        assert np.allclose(y.mean((1, 3)), 0, atol=1e-12) and np.allclose(y.var((1, 3)), 1, atol=1e-4)
    grads = oracle.group_norm_bwd(x, w, b, 2, 1e-5, act, do)
    for a, g in zip((x, w, b), grads):
        for i in range(a.size):
            at, h = np.unravel_index(i, a.shape), 1e-6
            old = a[at]
            a[at] = old + h
            up = (oracle.group_norm(x, w, b, 2, 1e-5, act)[0] * do).sum()
            a[at] = old - h
            down = (oracle.group_norm(x, w, b, 2, 1e-5, act)[0] * do).sum()
            a[at] = old
            assert abs((up - down) / (2 * h) - g[at]) <= 1e-7 * max(1.0, abs(g[at]))


def test_activations_where_known():
    z = np.array([-40.0, -1.0, 0.0, 1.0, 40.0]).reshape(1, 1, 5, 1)
    from oracle.group_norm import _act

    s, ds = _act(z, "silu")
    assert np.allclose(s.ravel(), [0, -0.2689414213699951, 0, 0.7310585786300049, 40], atol=1e-15) and np.allclose(ds.ravel()[[0, 2, 4]], [0, 0.5, 1], atol=1e-12)
    g, dg = _act(z, "gelu")
    assert np.allclose(g.ravel(), [0, -0.15865525393145707, 0, 0.8413447460685429, 40], atol=1e-15) and np.allclose(dg.ravel()[[0, 2, 4]], [0, 0.5, 1])
