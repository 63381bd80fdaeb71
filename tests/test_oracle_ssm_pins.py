"""The oracles of the selective scan, the causal convolution and the RMS norm against other ways to the same numbers (CPU)."""
import numpy as np
import pytest

import oracle

N = np.random.default_rng(0).standard_normal


def _scan(B=2, L=7, C=6, G=2, n=3):
    return dict(x=N((B, L, C)), dt=N((B, L, C)), A=-np.abs(N((C, n))), Bt=N((B, L, G, n)), Ct=N((B, L, G, n)), D=N(C), z=N((B, L, C)), bias=N(C))


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("softplus", [False, True])
def test_scan_is_the_sum_over_pairs_of_tokens(reverse, softplus):
    a = _scan()
    B, L, C = a["x"].shape
    state = N((B, C, 3))
    out, last = oracle.ssm_fwd(**a, state=state, softplus=softplus, reverse=reverse)
    flip = (lambda t: t[:, ::-1]) if reverse else (lambda t: t)
    x, dt, z, Bt, Ct = (flip(a[n]) for n in ("x", "dt", "z", "Bt", "Ct"))
    Bt, Ct = (np.repeat(t, C // 2, 2) for t in (Bt, Ct))
    d = dt + a["bias"]
    d = np.log(1 + np.exp(d)) if softplus else d
    run = np.cumsum(d, 1)
    h = np.exp(run[..., None] * a["A"]) * state[:, None]
    for t in range(L):
        for s in range(t + 1):
            h[:, t] += np.exp((run[:, t] - run[:, s])[..., None] * a["A"]) * (d[:, s] * x[:, s])[..., None] * Bt[:, s]
    y = ((h * Ct).sum(-1) + a["D"] * x) * z / (1 + np.exp(-z))
    assert np.allclose(out, flip(y), atol=1e-12) and np.allclose(last, h[:, -1], atol=1e-12)


def _differences(f, args, grads, h=1e-6):
    for name, g in grads.items():
        way = N(args[name].shape)
        slope = (f({**args, name: args[name] + h * way}) - f({**args, name: args[name] - h * way})) / (2 * h)
        assert abs(slope - (g * way).sum()) < 1e-6 * max(1, abs(slope)), name


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("softplus", [False, True])
def test_scan_gradient_by_differences(reverse, softplus):
    a = {**_scan(), "state": N((2, 6, 3))}
    do, ds = N(a["x"].shape), N((2, 6, 3))

    def loss(v):
        out, last = oracle.ssm_fwd(**v, softplus=softplus, reverse=reverse)
        return (out * do).sum() + (last * ds).sum()

    g = oracle.ssm_bwd(a["x"], a["dt"], a["A"], a["Bt"], a["Ct"], do, a["D"], a["z"], a["bias"], a["state"], ds, softplus, reverse)
    _differences(loss, a, {"x": g["dx"], "dt": g["ddt"], "A": g["dA"], "Bt": g["dB"], "Ct": g["dC"], "D": g["dD"], "z": g["dz"], "bias": g["dbias"], "state": g["d_state"]})


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("L", [1, 2, 9])
def test_convolution(L, reverse, act):
    a = dict(x=N((2, L, 3)), w=N((3, 4)), bias=N(3), state=N((2, 3, 3)))
    out, last = oracle.causal_conv(**a, act=act, reverse=reverse)
    line = np.concatenate([a["state"], a["x"][:, ::-1] if reverse else a["x"]], 1)
    for t in range(L):
        v = (line[:, t:t + 4] * a["w"].T).sum(1) + a["bias"]
        want = v / (1 + np.exp(-v)) if act == "silu" else v
        assert np.allclose(out[:, L - 1 - t if reverse else t], want)
    assert np.array_equal(last, line[:, L:])
    do, ds = N(out.shape), N(last.shape)

    def loss(v):
        o, s = oracle.causal_conv(**v, act=act, reverse=reverse)
        return (o * do).sum() + (s * ds).sum()

    dx, dw, db, d0 = oracle.causal_conv_bwd(a["x"], a["w"], a["bias"], do, act, a["state"], ds, reverse)
    _differences(loss, a, {"x": dx, "w": dw, "bias": db, "state": d0})


def test_norm():
    a = dict(x=N((3, 8)), weight=N(8), residual=N((3, 8)))
    out, s, rstd = oracle.rms_norm(**a, eps=0.1)
    assert np.allclose((s / np.linalg.norm(s, axis=1, keepdims=True)) * np.sqrt(8), oracle.rms_norm(s, np.ones(8), eps=0.0)[0])
    do, ds = N(out.shape), N(out.shape)

    def loss(v):
        o, total, _ = oracle.rms_norm(**v, eps=0.1)
        return (o * do).sum() + (total * ds).sum()

    dx, dw = oracle.rms_norm_bwd(s, a["weight"], rstd, do, ds)
    _differences(loss, a, {"x": dx, "residual": dx, "weight": dw})
