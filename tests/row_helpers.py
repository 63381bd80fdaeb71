"""Inputs, calls, oracle and bounds shared by the tests of the selective scan, the causal convolution and the RMS norm."""
import numpy as np
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import T, f64

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative to the value


def put(a, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(T[dtype])


def side_by_side(*parts, dtype):
    """The parts as slices of one tensor's last dimension, as a projection writes them."""
    whole = put(np.concatenate([p.reshape(*p.shape[:2], -1) for p in parts], -1), dtype)
    got, at = [], 0
    for p in parts:
        n = int(np.prod(p.shape[2:]))
        got.append(whole[..., at:at + n] if p.ndim == 3 else whole[..., at:at + n].unflatten(2, p.shape[2:]))
        at += n
    return got


def ssm_inputs(B, L, C, N, dtype, G=1, seed=0, states=False, D=True, z=True, bias=True, sliced=False):
    """Step sizes softplus(N(-1, 1)): a state is forgotten to e^-6 within 64 tokens (A <= -0.5, mean step 0.3)."""
    n = np.random.default_rng(seed).standard_normal
    x, dt, zz, do, Bt, Ct = n((B, L, C)), n((B, L, C)) * 0.7, n((B, L, C)), n((B, L, C)), n((B, L, G, N)), n((B, L, G, N))
    d = {"A": put(-(0.5 + np.abs(n((C, N))) * 2)), "D": put(n(C)) if D else None, "dt_bias": put(n(C) * 0.7 - 1) if bias else None}
    if sliced:
        d["x"], d["z"] = side_by_side(x, zz, dtype=dtype)
        _, d["Bt"], d["Ct"] = side_by_side(n((B, L, 3)), Bt, Ct, dtype=dtype)   # (rows that begin anywhere)
    else:
        d.update(x=put(x, dtype), z=put(zz, dtype), Bt=put(Bt, dtype), Ct=put(Ct, dtype))
    if not z:
        d["z"] = None
    d["dt"], d["d_out"] = put(dt, dtype), put(do, dtype)
    d["state"], d["d_state"] = (put(n((B, C, N))) if states else None for _ in range(2))
    return d


def _nan(t, dtype=None):
    return torch.full(t.shape, float("nan"), device="cuda", dtype=dtype or t.dtype)


def ssm_forward(d, reverse=False, softplus=True, state_out=True, stream=None):
    out = _nan(d["x"])
    last = torch.full((d["x"].shape[0], *d["A"].shape), float("nan"), device="cuda") if state_out else None
    vig.vig_ssm_fwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct")), out, D=d["D"], z=d["z"], dt_bias=d["dt_bias"], state_in=d["state"], state_out=last,
                    softplus=softplus, reverse=reverse, stream=stream)
    return {"out": out} if last is None else {"out": out, "state_out": last}


def ssm_gradient(d, reverse=False, softplus=True, stream=None):
    g = {"d" + n: _nan(d[n]) for n in ("x", "dt", "A")}
    g["dB"], g["dC"] = _nan(d["Bt"]), _nan(d["Ct"])
    for n, of in (("dD", "D"), ("dz", "z"), ("dbias", "dt_bias"), ("d_state", "state")):
        if d[of] is not None:
            g[n] = _nan(d[of])
    vig.vig_ssm_bwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct")), d["d_out"], *(g[n] for n in ("dx", "ddt", "dA", "dB", "dC")), D=d["D"], z=d["z"],
                    dt_bias=d["dt_bias"], dD=g.get("dD"), dz=g.get("dz"), d_dt_bias=g.get("dbias"), state_in=d["state"], d_state_out=d["d_state"],
                    d_state_in=g.get("d_state"), softplus=softplus, reverse=reverse, stream=stream)
    return g


def _args(d):
    return [f64(d[n]) for n in ("x", "dt", "A", "Bt", "Ct")]


def ssm_oracle(d, reverse=False, softplus=True):
    out, last = oracle.ssm_fwd(*_args(d), f64(d["D"]), f64(d["z"]), f64(d["dt_bias"]), f64(d["state"]), softplus, reverse)
    return {"out": out, "state_out": last}


def ssm_oracle_gradient(d, reverse=False, softplus=True):
    return oracle.ssm_bwd(*_args(d), f64(d["d_out"]), f64(d["D"]), f64(d["z"]), f64(d["dt_bias"]), f64(d["state"]), f64(d["d_state"]), softplus, reverse)


def ssm_bound(name, t, d):
    """2-norm of the difference over the 2-norm of the result.

    fp32: a state is a product of decays, each off by 2^-22 (the exponential) and half a step for its argument, of which at most 64 are
    remembered, and there and in the sums some sixteen roundings of half a step; terms of either sign cancel to a quarter of their size:
    4 (64 2^-22 + 16 2^-24).  Sums over the tokens (dA, dD, dbias) add partial sums of n values: half a step times sqrt(n), likewise.
    bf16: half a step, and for dB and dC as much as 2^-11, the rounding of the products, times two as they cancel."""
    B, L, C = d["x"].shape
    tol = 4 * (64 * 2.0 ** -22 + 16 * 2.0 ** -24)
    if name in ("dA", "dD", "dbias", "dB", "dC"):
        tol += 4 * 2.0 ** -24 * (B * L * C) ** 0.5
    if t.dtype == torch.bfloat16:
        tol += HALF[t.dtype] + (2.0 ** -10 if name in ("dB", "dC") else 0.0)
    return tol


def compare(got, ref, bound):
    for name, t in got.items():
        a, r = f64(t), np.asarray(ref[name])
        assert a.shape == r.shape and np.isfinite(a).all(), name
        norm = np.linalg.norm(r)
        err = np.linalg.norm(a - r) / norm if norm else float(np.abs(a).max(initial=0.0))
        tol = bound(name, t)
        print(f"  {name}: {err:.2e} (at most {tol:.2e})")
        assert err <= tol, (name, err, tol)
