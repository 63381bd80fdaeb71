"""Gated delta rule under strong gates: decays behind gates that forget, and the gates' own gradient, which is proportional to exp(log_alpha)."""
import pytest
import torch

from layer_helpers import bound, gdr_forward, gdr_gradient, gdr_inputs, gdr_oracle, gdr_oracle_gradient, off

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gate", [float("-inf"), -1e4, -90.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_states_behind_gates_that_forget(dtype, gate):
    """Masked left padding, packed sequences: n gates of a chunk forget, ordinary ones follow.  Unit by unit; states of bf16 calls: 2^-15."""
    resets = (0, 1, 8, 24, 40, 56)
    for L in (64, 200):
        d = gdr_inputs(1, len(resets), L, 32, 48, dtype, seed=51, states=True)
        for u, n in enumerate(resets):
            d["log_alpha"][0, u, L % 64:L % 64 + n] = gate
            d["log_alpha"][0, u, :n] = gate
        for reverse in (False, True):
            out, last = gdr_forward(d, reverse)
            ref, ref_last = gdr_oracle(d, reverse)
            got, want = gdr_gradient(d, reverse), gdr_oracle_gradient(d, reverse)
            for u in range(len(resets)):
                for name, a, b in [("out", out, ref), ("state", last, ref_last)] + list(zip(("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state"), got, want)):
                    if not b[0, u].any():   # (what a gate of -inf left nothing of)
                        assert (a[0, u] == 0).all(), (name, u)
                        continue
                    tol = bound(a, L + 32 + 48)
                    if dtype == "bf16" and a.dtype == torch.float32:
                        tol = 2.0 ** -15
                    if name == "d_state" and gate == -90.0:   # (e^-90 each: below fp32's normal numbers from the second on, zero from the third)
                        continue
                    assert off(a[0, u], b[0, u]) <= tol, (name, L, reverse, u, off(a[0, u], b[0, u]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", [-0.3, -2.0, -5.0, -8.0, -12.0, -30.0])
def test_gradient_of_strong_gates(dtype, gate):
    """All gates around one value.  fp32: the gradient is a sum of some L + dk + dv products, and of both states' roundings: twice the bound of
    one chain."""
    for size in ((2, 2, 196, 32, 64), (2, 2, 100, 24, 48), (1, 3, 70, 100, 128)):
        for states in (False, True):
            d = gdr_inputs(*size, dtype, seed=52, states=states)
            d["log_alpha"] = (gate * (0.8 + 0.4 * torch.rand(d["log_alpha"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)))).to(d["v"].dtype)
            g, w = gdr_gradient(d, reverse=states)[3], gdr_oracle_gradient(d, reverse=states)[3]
            assert off(g, w) <= 2 * bound(g, sum(size[2:])) / (2 if dtype == "bf16" else 1), (size, states, off(g, w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", [-5.0, -12.0])
def test_gradient_of_one_strong_gate_among_slow_ones(dtype, gate):
    """Every token's gate gradient by itself, over sixteen units: the strong one's is e^gate of its neighbours'."""
    for at in (1, 5, 15, 16, 40, 63, 64, 90, 129):
        d = gdr_inputs(4, 4, 130, 32, 64, dtype, seed=53, gate_mean=2.0, states=True)
        d["log_alpha"][:, :, at] = gate
        g, w = gdr_gradient(d)[3], gdr_oracle_gradient(d)[3]
        for t in {at - 1, at, min(at + 1, 129)}:
            assert off(g[:, :, t], w[:, :, t]) <= 2 * bound(g, 130 + 32 + 64), (at, t, off(g[:, :, t], w[:, :, t]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["small before large", "large, forgotten", "large in steps of zero"])
def test_gate_gradient_beside_large_values(dtype, kind):
    """Values many powers of two apart in one run of 64 tokens: what a gate's gradient does not contain leaves no rounding in it."""
    for at in (3, 16, 30, 50, 80):
        d = gdr_inputs(2, 4, 140, 32, 64, dtype, seed=54, gate_mean=1.0)
        parts = [slice(1, at), slice(at + 1, None)]
        if kind == "small before large":
            d["v"][:, :, :at] *= 1e-9
            d["v"][:, :, at:] *= 1e9
        elif kind == "large, forgotten":
            d["v"][:, :, :at] *= 1e9
            d["log_alpha"][:, :, at] = float("-inf")
        else:
            d["v"][:, :, at] = 1e20
            d["beta"][:, :, at] = 0
        g, w = gdr_gradient(d)[3], gdr_oracle_gradient(d)[3]
        for part in parts:
            assert off(g[:, :, part], w[:, :, part]) <= 2 * bound(g, 140 + 32 + 64), (at, part)
        if kind == "large, forgotten":
            assert (g[:, :, at] == 0).all()
