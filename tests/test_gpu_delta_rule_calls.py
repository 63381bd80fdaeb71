"""Calls of the gated delta rule with some of the states, and of one unit instead of many."""
import itertools

import pytest
import torch

import paper_2405_18425_b200 as vig
from layer_helpers import NAMES, bound, check, f64, gdr_forward, gdr_gradient, gdr_inputs, gdr_oracle, off

import oracle

pytestmark = pytest.mark.gpu
GRADS = ("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 2, 70, 24, 48), (1, 2, 64, 128, 128), (1, 3, 3, 16, 32), (1, 2, 800, 16, 40), (1, 1, 90, 32, 200), (1, 2, 33, 17, 20)], ids=str)
def test_states_given_in_every_combination(size, dtype):
    """state_in, d_state_out and d_state_in, each or not, in either direction."""
    d = gdr_inputs(*size, dtype, seed=61, gate_mean=1.0, states=True)
    terms = sum(size[2:])
    for first, last, want_first, reverse in itertools.product((False, True), repeat=4):
        e = {**d, "state": d["state"] if first else None, "d_state": d["d_state"] if last else None}
        ref = oracle.gdr_bwd(*(f64(e[n]) for n in NAMES), f64(e["d_out"]), f64(e["state"]), f64(e["d_state"]), reverse)
        g = [torch.full_like(e[n], float("nan")) for n in NAMES]
        ds = torch.full_like(d["state"], float("nan")) if want_first else None
        vig.vig_gdr_bwd(*(e[n] for n in NAMES), e["d_out"], *g, state_in=e["state"], d_state_out=e["d_state"], d_state_in=ds, reverse=reverse)
        for name, t, w in zip(GRADS, g + [ds], ref):
            if t is None:
                continue
            tol = 2.0 ** -15 if dtype == "bf16" and t.dtype == torch.float32 else (2 if name == "dlog_alpha" else 1) * bound(t, terms)
            assert off(t, w) <= tol, (name, first, last, want_first, reverse, off(t, w), tol)
        out, _ = gdr_forward(e, reverse, state_out=last)
        check([("out", out, gdr_oracle(e, reverse)[0])], terms)


def _unit(d, b, h):
    return {n: None if t is None else t[b:b + 1, h:h + 1].clone() for n, t in d.items()}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size, same", [((3, 4, 196, 32, 64), True), ((2, 2, 130, 100, 24), True), ((10, 12, 70, 20, 17), True), ((50, 4, 900, 16, 24), False), ((200, 4, 2, 16, 24), False)], ids=str)
def test_one_unit_by_itself(size, same, dtype):
    """Nothing of one unit depends on the others.  The form may depend on their number (segments of long sequences, walks of a handful of tokens): the
    same bits where it is the same one, else both forms within their bounds."""
    d = gdr_inputs(*size, dtype, seed=62, gate_mean=1.0, states=True)
    many = gdr_forward(d) + tuple(gdr_gradient(d))
    for b, h in ((0, 0), (size[0] - 1, size[1] - 1), (size[0] // 2, 1)):
        one = _unit(d, b, h)
        for i, (x, y) in enumerate(zip(gdr_forward(one) + tuple(gdr_gradient(one)), many)):
            y = y[b:b + 1, h:h + 1]
            if same or dtype == "f32":
                assert torch.equal(x, y), i
            else:
                tol = 2.0 ** -15 if x.dtype == torch.float32 else 2.0 ** -7
                assert off(x, f64(y)) <= 2 * tol, i


@pytest.mark.parametrize("size", [(2, 2, 65, 128, 128), (1, 3, 130, 20, 17), (1, 2, 196, 32, 64), (1, 1, 1100, 24, 48), (2, 1, 515, 64, 64), (1, 2, 1000, 96, 40)], ids=str)
def test_states_of_bf16_calls_hold_the_bound_of_fp32_calls(size):
    """Operands of 24 bits and fp32 sums: the roundings that the bound of fp32 calls counts, and the decays' exponentials, 2^-22 each, once a chunk."""
    d = gdr_inputs(*size, "bf16", seed=63, gate_mean=1.0, states=True)
    tol = 8 * 2.0 ** -24 * sum(size[2:]) ** 0.5 + 2.0 ** -22 * (size[2] // 64 + 1) ** 0.5
    for reverse in (False, True):
        last, ref = gdr_forward(d, reverse)[1], gdr_oracle(d, reverse)[1]
        assert off(last, ref) <= tol
        got = gdr_gradient(d, reverse)[5]
        want = oracle.gdr_bwd(*(f64(d[n]) for n in NAMES), f64(d["d_out"]), f64(d["state"]), f64(d["d_state"]), reverse)[5]
        assert off(got, want) <= tol
