"""Gated delta rule under strong gates: what is decayed in front of and behind gates that forget."""
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
