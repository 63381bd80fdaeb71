"""Selective scan on the GPU with an infinite row of Ct: it meets the last state alone, also where that one comes from the initial state only."""
import numpy as np
import pytest
import torch

from layer_helpers import f64
from row_helpers import ssm_forward, ssm_inputs, ssm_oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 3, 5, 8, 12, 16, 17, 31, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [3, 40, 300])
def test_last_state(L, dtype, N):
    """x of zeros: the states are the initial ones, decaying slowly, none of them zero at any token."""
    d = ssm_inputs(2, L, 72, N, dtype, seed=2, states=True)
    d["x"].zero_()
    d["A"] = d["A"] * 2.0 ** -8
    d["Ct"][1, L // 2, 0, N - 1] = float("inf")
    d["Ct"][0, L - 1, 0, N - 1] = -float("inf")
    got, ref = ssm_forward(d), ssm_oracle(d)
    a, bad = f64(got["out"]), ~np.isfinite(ref["out"])
    assert bad.sum() == 2 * 72 and np.isinf(ref["out"][bad]).all()
    assert np.array_equal(a[bad], ref["out"][bad]) and np.isfinite(a[~bad]).all() and torch.isfinite(got["state_out"]).all()
