"""Selective scan on the GPU with an infinite x: infinities where the definition has them, for any number of states, not NaN."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import ssm_forward, ssm_inputs, ssm_oracle

pytestmark = pytest.mark.gpu


def _inputs(L, N, dtype):
    """Rows of one sign, so that the sum over the states is an infinity; a skip of the same sign; decays that stay above zero."""
    d = ssm_inputs(2, L, 72, N, dtype, seed=1, states=True)
    for n in ("Bt", "Ct", "D", "z"):
        d[n] = d[n].abs() + 0.125
    d["A"] = d["A"].clamp(min=-1.0)
    d["x"][1, L // 2, 5] = float("inf")
    d["x"][0, L // 3, 33] = -float("inf")
    return d


def _same_kind(t, ref):
    a = f64(t)
    bad = ~np.isfinite(ref)
    assert bad.any() and np.isfinite(a[~bad]).all() and np.array_equal(a[bad], ref[bad])
    return a, bad


@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 12, 16, 17, 30, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [1, 13, 40, 300])
def test_sequences(L, dtype, N):
    d = _inputs(L, N, dtype)
    got, ref = ssm_forward(d), ssm_oracle(d)
    plain = {**d, "x": torch.where(torch.isinf(d["x"]), torch.zeros_like(d["x"]), d["x"])}
    beside = ssm_forward(plain)
    for n in ref:
        _, bad = _same_kind(got[n], ref[n])
        keep = torch.from_numpy(~bad).cuda()
        assert torch.equal(got[n][keep], beside[n][keep]), n      # (channels of their own: nothing else moves)


@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 16, 30, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token(dtype, N):
    d = _inputs(1, N, dtype)
    one = [d[n][:, 0].contiguous() for n in ("x", "dt", "Bt", "Ct", "z")]
    state, out = d["state"].clone(), torch.empty_like(one[0])
    vig.vig_ssm_step(one[0], one[1], d["A"], one[2], one[3], state, out, D=d["D"], z=one[4], dt_bias=d["dt_bias"])
    ref, last = oracle.ssm_fwd(*(f64(d[n]) for n in ("x", "dt", "A", "Bt", "Ct")), f64(d["D"]), f64(d["z"]), f64(d["dt_bias"]), f64(d["state"]))
    _same_kind(out, ref[:, 0])
    _same_kind(state, last)
