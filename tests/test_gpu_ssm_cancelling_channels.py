"""Gradient of the selective scan's rows (dB, dC) on the GPU where two channels of a group nearly cancel."""
import numpy as np
import pytest
import torch

import oracle
from layer_helpers import f64
from row_helpers import HALF, ssm_gradient, ssm_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [4, 16, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pair", [(0, 2), (1, 40), (6, 63)])
def test_sums_over_channels_that_cancel(pair, dtype, N):
    """Channel j is channel i with d_out -(1 + 2^-6) times as large, no others have any: sums of two terms that are 2^-6 of them.

    Beside half a step of the result, with S the sum of the terms' sizes: a term enters its sum with sixteen bits or more, 2^-17 S; it is a
    product of a step size and a state or adjoint that at most four tokens made, 2^-22 for each decay, softplus and reciprocal and 2^-24 for each
    of some four products a token: 9 2^-22 + 16 2^-24 = 13 2^-22 S.  Together less than 2^-16 S."""
    i, j = pair
    d = ssm_inputs(2, 4, 64, N, dtype, seed=4, z=False)
    for n in ("x", "dt"):
        d[n][..., j] = d[n][..., i]
    for n in ("A", "D", "dt_bias"):
        d[n][j] = d[n][i]
    g = d["d_out"][..., i].float()
    g = torch.round(g.clamp(-1.5, 1.5) * 2) / 2       # (so that 65 / 64 of it is a bf16 number)
    d["d_out"].zero_()
    d["d_out"][..., i] = g.to(d["d_out"].dtype)
    d["d_out"][..., j] = (-g * (1 + 2.0 ** -6)).to(d["d_out"].dtype)
    assert torch.equal(d["d_out"][..., j].float(), -g * (1 + 2.0 ** -6))
    got = ssm_gradient(d)
    args = [f64(d[n]) for n in ("x", "dt", "A", "Bt", "Ct")]
    ref = oracle.ssm_bwd(*args, f64(d["d_out"]), f64(d["D"]), None, f64(d["dt_bias"]))
    sizes = {"dB": 0.0, "dC": 0.0}
    for c in pair:
        alone = np.zeros(d["d_out"].shape)
        alone[..., c] = f64(d["d_out"])[..., c]
        r = oracle.ssm_bwd(*args, alone, f64(d["D"]), None, f64(d["dt_bias"]))
        for n in sizes:
            sizes[n] = sizes[n] + np.abs(r[n])
    for n, S in sizes.items():
        err = np.abs(f64(got[n]) - ref[n])
        tol = HALF[got[n].dtype] * np.abs(ref[n]) + 2.0 ** -16 * S
        print(n, "beyond half a step, over S: 2 ^", np.log2(max(((err - HALF[got[n].dtype] * np.abs(ref[n]))[S > 0] / S[S > 0]).max(), 2.0 ** -30)))
        assert (err <= tol).all(), n
