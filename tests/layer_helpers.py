"""Inputs, oracle and bounds shared by the GPU tests of the gated delta rule and the group norm."""
import numpy as np
import torch

import oracle
import paper_2405_18425_b200 as vig

T = {"bf16": torch.bfloat16, "f32": torch.float32}
NAMES = ("q", "k", "v", "log_alpha", "beta")


def gdr_inputs(B, H, L, dk, dv, dtype, seed=0, gate_mean=0.0, states=False):
    """Stored tensors on the GPU: unit-length keys and queries, log gates logsigmoid(g) / 16, step sizes in (0, 1)."""
    n = np.random.default_rng(seed).standard_normal
    unit = lambda x: x / np.maximum(np.linalg.norm(x, axis=-1, keepdims=True), 1e-20)
    x = {"q": unit(n((B, H, L, dk))), "k": unit(n((B, H, L, dk))), "v": n((B, H, L, dv)),
         "log_alpha": -np.log1p(np.exp(-(n((B, H, L)) + gate_mean))) / 16, "beta": 1 / (1 + np.exp(-n((B, H, L)))), "d_out": n((B, H, L, dv))}
    d = {k: torch.from_numpy(a).cuda().to(T[dtype]) for k, a in x.items()}
    for k in ("state", "d_state"):
        d[k] = torch.from_numpy(n((B, H, dk, dv)) * 0.5).cuda().float() if states else None
    return d


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def gdr_forward(d, reverse=False, state_out=True, stream=None):
    out = torch.full_like(d["v"], float("nan"))
    last = torch.full((*d["q"].shape[:2], d["q"].shape[3], d["v"].shape[3]), float("nan"), device="cuda") if state_out else None
    vig.vig_gdr_fwd(*(d[n] for n in NAMES), out, state_in=d["state"], state_out=last, reverse=reverse, stream=stream)
    return out, last


def gdr_gradient(d, reverse=False, stream=None):
    """dq, dk, dv, dlog_alpha, dbeta, and the initial state's where there is one."""
    g = [torch.full_like(d[n], float("nan")) for n in NAMES]
    ds = None if d["state"] is None else torch.full_like(d["state"], float("nan"))
    vig.vig_gdr_bwd(*(d[n] for n in NAMES), d["d_out"], *g, state_in=d["state"], d_state_out=d["d_state"], d_state_in=ds, reverse=reverse, stream=stream)
    return g + ([] if ds is None else [ds])


def gdr_oracle(d, reverse=False):
    return oracle.gdr_fwd(*(f64(d[n]) for n in NAMES), f64(d["state"]), reverse)


def gdr_oracle_gradient(d, reverse=False):
    g = oracle.gdr_bwd(*(f64(d[n]) for n in NAMES), f64(d["d_out"]), f64(d["state"]), f64(d["d_state"]), reverse)
    return list(g[:5]) + ([] if d["state"] is None else [g[5]])


def bound(t, terms):
    """How far a stored result may be from the definition, in 2-norm over 2-norm.

    fp32: every value is a chain of sums of `terms` products; each of their roundings is at most half a step, 2^-24, of the partial sum it
    is made in, and independent ones add up as the square root of their number: 2^-24 sqrt(terms), times 8 for partial sums that are
    larger than the result (states of either sign that cancel).
    bf16: half a step of the result, 2^-8, and as much again for operands that a tensor-core path may round once."""
    return 2.0 ** -7 if t.dtype == torch.bfloat16 else 8 * 2.0 ** -24 * terms ** 0.5


def off(t, ref):
    a, r = f64(t), np.asarray(ref)
    assert np.isfinite(a).all()
    norm = np.linalg.norm(r)
    return np.linalg.norm(a - r) / norm if norm else float(np.abs(a).max(initial=0.0))


def check(pairs, terms, state_of_bf16=False):
    """state_of_bf16: fp32 states of bf16 calls may come from operands of sixteen significant bits: 2^-16 an operand, two of them."""
    for name, t, ref in pairs:
        tol = bound(t, terms)
        if state_of_bf16 and t.dtype == torch.float32:
            tol = max(tol, 2.0 ** -15)
        err = off(t, ref)
        print(f"  {name}: {err:.2e} (at most {tol:.2e})")
        assert err <= tol, (name, err, tol)
