"""Decays of the selective scan's fp32 calls on the GPU, one at a time, wherever they are computed: whole sequences, between segments, a single token."""
import numpy as np
import pytest
import torch

import paper_2405_18425_b200 as vig

pytestmark = pytest.mark.gpu

C, N = 1024, 16


def _case(most):
    """Exponents delta A in [-most, 0], delta a power of two that a channel has for itself."""
    rng = np.random.default_rng(5)
    delta = 2.0 ** rng.integers(-6, 1, C)
    v = -rng.uniform(0, most, (C, N))
    A = torch.from_numpy((v / delta[:, None]).astype(np.float32)).cuda()
    exact = np.exp(A.double().cpu().numpy() * delta[:, None])
    return torch.from_numpy(delta.astype(np.float32)).cuda(), A, exact


def _bound(form, most):
    """log2 e is off by 2^-26, its product with A by 2^-24 (that with delta is exact), and the decay by |v| times their sum; reducing the exponent is
    exact; the polynomial is off by 2^-28, its last step by half a step of a number from 0.7 to 1.42, 2^-24, the steps before by a quarter
    of that; the products with one and zero are exact.  A single token's are the special-function unit's, 2^-22."""
    return most * 1.25 * 2.0 ** -24 + (2.0 ** -22 if form == "token" else (1.25 + 0.0625) * 2.0 ** -24)


def _run(form, delta, A):
    x = torch.zeros(1, 1, C, device="cuda")
    state = torch.ones(1, C, N, device="cuda")
    rows = torch.ones(1, 1, 1, N, device="cuda")
    if form == "token":
        vig.vig_ssm_step(x[:, 0], delta[None], A, rows[:, 0], rows[:, 0], state, torch.empty_like(x[:, 0]), softplus=False)
        return state
    L = 1 if form == "sequence" else 1024
    x, rows = x.expand(1, L, C).contiguous(), rows.expand(1, L, 1, N).contiguous()
    dt = torch.zeros_like(x)
    dt[0, 0] = delta                         # (the other tokens' decays are one)
    last = torch.empty_like(state)
    vig.vig_ssm_fwd(x, dt, A, rows, rows, torch.empty_like(x), state_in=state, state_out=last, softplus=False)
    return last


@pytest.mark.parametrize("most", [0.25, 4.0])
@pytest.mark.parametrize("form", ["sequence", "segments", "token"])
def test_a_decay(form, most):
    """Of sequences and between segments 2^v as arithmetic, closer than the special-function unit's."""
    delta, A, exact = _case(most)
    got = _run(form, delta, A)[0].double().cpu().numpy()
    off = np.abs(got / exact - 1).max()
    print(form, most, "2 ^", np.log2(off), "at most 2 ^", np.log2(_bound(form, most)))
    assert off <= _bound(form, most)
