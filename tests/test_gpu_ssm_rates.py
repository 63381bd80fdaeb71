"""Selective scan on the GPU with rates beyond every bound: the state is forgotten at each token, at any length, and a step size of zero keeps it."""
import pytest
import torch

import paper_2405_18425_b200 as vig
from row_helpers import ssm_forward, ssm_gradient, ssm_inputs

pytestmark = pytest.mark.gpu

RATES = [-float("inf"), -3.4e38, -1e37]


def _both(d, reverse):
    return {**ssm_forward(d, reverse), **ssm_gradient(d, reverse)}


@pytest.mark.parametrize("reverse", [False, True], ids=["forward", "reverse"])
@pytest.mark.parametrize("rate", RATES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [1, 2, 3, 5, 41, 64, 303])
def test_forgets(L, dtype, rate, reverse):
    """Bit for bit what a rate of -1e6 gives, whose decays (step sizes of 1e-3 and more) are zero too; the other channels' bits stay."""
    d = ssm_inputs(2, L, 72, 16, dtype, seed=1, states=True)
    assert (torch.nn.functional.softplus(d["dt"].float() + d["dt_bias"]) > 1e-3).all()
    d["A"][9] = -1e6
    d["A"][20, 5] = -1e6
    want = _both(d, reverse)
    A = d["A"].clone()
    A[9] = rate
    A[20, 5] = rate
    got = _both({**d, "A": A}, reverse)
    for n in want:
        assert torch.isfinite(got[n]).all() and torch.equal(got[n], want[n]), n
    assert (got["dA"][9] == 0).all() and (got["dA"][20, 5] == 0).all()


@pytest.mark.parametrize("rate", RATES + [3.4e38])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [1, 3, 16, 303])
def test_a_step_size_of_zero_keeps_the_state(L, dtype, rate):
    """All gradients are finite but that of the channel's step sizes: its sum over the states of (what passes through) times A, sixteen terms of
    order one times 3e38, leaves fp32 by its definition, and the slope of softplus beside it is zero."""
    d = ssm_inputs(2, L, 72, 16, dtype, seed=2, states=True)
    d["dt"].fill_(-200)
    d["A"][9] = rate
    got, g = ssm_forward(d), ssm_gradient(d)
    assert torch.equal(got["state_out"], d["state"]) and torch.isfinite(got["out"]).all()
    for n in ("ddt", "dbias"):
        g[n] = torch.cat((g[n][..., :9], g[n][..., 10:]), -1)
    assert all(torch.isfinite(t).all() for t in g.values())
    state, out = d["state"].clone(), torch.empty_like(d["x"][:, 0])
    one = [d[n][:, 0].contiguous() for n in ("x", "dt", "Bt", "Ct", "z")]
    vig.vig_ssm_step(one[0], one[1], d["A"], one[2], one[3], state, out, D=d["D"], z=one[4], dt_bias=d["dt_bias"])
    assert torch.equal(state, d["state"]) and torch.isfinite(out).all()


@pytest.mark.parametrize("rate", RATES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 16])
def test_a_token_forgets(N, dtype, rate):
    d = ssm_inputs(5, 1, 40, N, dtype, seed=3, states=True)
    one = [d[n][:, 0].contiguous() for n in ("x", "dt", "Bt", "Ct")]
    got = []
    for a in (-1e6, rate):
        A = d["A"].clone()
        A[9] = a
        state, out = d["state"].clone(), torch.empty_like(one[0])
        vig.vig_ssm_step(one[0], one[1], A, one[2], one[3], state, out, D=d["D"], dt_bias=d["dt_bias"])
        got.append((state, out))
    assert all(torch.isfinite(b).all() and torch.equal(a, b) for a, b in zip(*got))
