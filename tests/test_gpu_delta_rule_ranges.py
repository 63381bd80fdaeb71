"""Gated delta rule where one call's values differ by many powers of two: what is small beside something that it never meets keeps its digits.

bf16 results: half a step, 2^-8, and as much for the kernels' own roundings, as everywhere; here of every token (or column) by itself."""
import numpy as np
import pytest
import torch

from layer_helpers import bound, gdr_forward, gdr_gradient, gdr_inputs, gdr_oracle, gdr_oracle_gradient, off

pytestmark = pytest.mark.gpu
GRADS = ("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state")


def _gradients_off(d, reverse=False):
    return [(n, g, w) for n, g, w in zip(GRADS, gdr_gradient(d, reverse), gdr_oracle_gradient(d, reverse))]


def _limit(t):
    return 2.0 ** -15 if t.dtype == torch.float32 else bound(t, 0)   # (states of bf16 calls)


@pytest.mark.parametrize("scale", [1e-8, 1e-4, 1e8])
@pytest.mark.parametrize("size", [(2, 2, 196, 32, 64), (2, 2, 192, 32, 64), (1, 3, 68, 24, 48), (1, 2, 7, 64, 128), (1, 2, 900, 16, 40)], ids=str)
def test_gradient_of_losses_of_other_magnitudes(size, scale):
    """Everything is linear in d_out and d_state_out: d_out of a mean-reduced loss is 1e-8."""
    for states in (False, True):
        d = gdr_inputs(*size, "bf16", seed=41, gate_mean=1.0, states=states)
        d["d_out"] = d["d_out"] * scale
        if states:
            d["d_state"] = d["d_state"] * scale
        for name, g, w in _gradients_off(d):
            assert off(g, w) <= _limit(g), (name, states)


@pytest.mark.parametrize("scale", [1.0, 1e-8])
def test_gradient_with_rows_of_zeros(scale):
    """Tokens that the loss does not see, and queries and keys of zero."""
    d = gdr_inputs(2, 2, 150, 32, 64, "bf16", seed=42, gate_mean=1.0)
    d["d_out"] = d["d_out"] * scale
    d["d_out"][:, :, 3::5] = 0
    d["q"][:, :, 4::7] = 0
    d["k"][:, :, 6::9] = 0
    d["d_out"][1, 1] = 0
    d["d_out"][1, 1, 100] = scale
    for name, g, w in _gradients_off(d):
        for u in ((0, 0), (0, 1), (1, 0), (1, 1)):
            assert off(g[u], w[u]) <= bound(g, 0), (name, u)


def test_gradient_with_columns_of_opposite_magnitudes():
    """Columns of v times 2^s and of d_out times 2^-s: each contributes alike to dq and dk, dv has the columns' own sizes."""
    for spread in (8, 30):
        d = gdr_inputs(1, 4, 140, 32, 64, "bf16", seed=43, gate_mean=1.0)
        s = torch.from_numpy(2.0 ** np.random.default_rng(1).integers(-spread, spread + 1, 64)).cuda()
        d["v"], d["d_out"] = (d["v"] * s).bfloat16(), (d["d_out"] / s).bfloat16()
        for name, g, w in _gradients_off(d):
            assert off(g, w) <= bound(g, 0), (name, spread)
            if name == "dv":
                for j in range(64):
                    assert off(g[..., j], w[..., j]) <= bound(g, 0), (name, spread, j)


def _jump(d, kind, at):
    """Values of one column and chunk that never meet, many powers of two apart."""
    la, v, be = d["log_alpha"], d["v"], d["beta"]
    if kind == "large, forgotten":
        v[:, :, :at] *= 1e7
        la[:, :, at] = float("-inf")
    elif kind == "larger, forgotten, smaller":
        v[:, :, :at] *= 1e9
        la[:, :, at] = float("-inf")
        v[:, :, at:] *= 1e-9
    elif kind == "small before large":
        v[:, :, :at] *= 1e-9
        v[:, :, at:] *= 1e9
    elif kind == "steps of zero on large values":
        v[:, :, 2::3] = 1e20
        be[:, :, 2::3] = 0
    elif kind == "strong last gate":
        la[:, :, -1] = -14
        be[:, :, -1] = 0


@pytest.mark.parametrize("size", [(1, 4, 64, 16, 32), (1, 4, 200, 32, 64), (1, 4, 50, 64, 24)], ids=str)
@pytest.mark.parametrize("kind", ["large, forgotten", "larger, forgotten, smaller", "small before large", "steps of zero on large values", "strong last gate"])
def test_jumps_inside_a_chunk(kind, size):
    for at in (5, 16, 32, 45):
        d = gdr_inputs(*size, "bf16", seed=44, gate_mean=1.0)
        _jump(d, kind, at)
        ref, ref_last = gdr_oracle(d)
        for state_out in (False, True):
            out, last = gdr_forward(d, state_out=state_out)
            for t in range(size[2]):
                assert off(out[:, :, t], ref[:, :, t]) <= 2.0 ** -7, (at, t, state_out)
        for u in range(4):
            assert off(last[0, u], ref_last[0, u]) <= 2.0 ** -15, (at, u)
        for name, g, w in _gradients_off(d):
            if name == "dlog_alpha":   # (a difference of other terms)
                continue
            if name == "dbeta" and kind == "steps of zero on large values":
                parts = [slice(2, None, 3), slice(0, None, 3), slice(1, None, 3)]   # (1e20 there)
            else:
                parts = [slice(0, at), slice(at, None)]
            for part in parts:
                assert off(g[:, :, part], w[:, :, part]) <= 2.0 ** -7, (name, at, part)


@pytest.mark.parametrize("size", [(1, 3, 60, 16, 32), (1, 2, 130, 48, 64)], ids=str)
def test_rows_of_the_state_of_very_different_size(size):
    """Keys and queries along the axes: rows of the state hold values of 1e-9 to 1e9, and a query reads one of them."""
    d = gdr_inputs(*size, "bf16", seed=45, gate_mean=3.0)
    dk = size[3]
    axis = torch.arange(size[2], device="cuda") * 7 % dk
    d["k"] = torch.nn.functional.one_hot(axis, dk).bfloat16().expand_as(d["k"]).contiguous()
    d["q"] = torch.nn.functional.one_hot((axis + 3 * 7) % dk, dk).bfloat16().expand_as(d["q"]).contiguous()
    d["v"] = (d["v"].double() * 10.0 ** (axis % 19 - 9).double()[:, None]).bfloat16()
    out, last = gdr_forward(d)
    ref, ref_last = gdr_oracle(d)
    for t in range(size[2]):
        assert off(out[:, :, t], ref[:, :, t]) <= 2.0 ** -7, t
    again, _ = gdr_forward(d, state_out=False)
    for t in range(size[2]):
        assert off(again[:, :, t], ref[:, :, t]) <= 2.0 ** -7, t
    for i in range(dk):
        assert off(last[:, :, i], ref_last[:, :, i]) <= 2.0 ** -15, i
    got, want = gdr_gradient(d), gdr_oracle_gradient(d)
    for t in range(size[2]):
        for name, g, w in zip(GRADS[:3], got, want):
            assert off(g[:, :, t], w[:, :, t]) <= 2.0 ** -7, (name, t)


@pytest.mark.parametrize("n", [4, 6, 8, 9])
@pytest.mark.parametrize("size", [(1, 3, 40, 16, 32), (1, 2, 100, 48, 64), (1, 2, 900, 16, 40)], ids=str)
def test_growth_that_is_undone(size, n):
    """n steps with beta |k|^2 = 4 along an axis (a row of the state times -3 each), then one of beta = |k| = 1 that replaces the row by its value exactly: up to
    2e4 is taken off again.  What the steps leave in fp32 is 2^-24 of that, 1e-3 of the value, and as much for the results' own rounding: 2^-7 as everywhere."""
    for at in (5, 20):
        d = gdr_inputs(*size, "bf16", seed=46, gate_mean=4.0, states=True)
        run = slice(at, at + n + 1)
        d["k"][:, :, run] = 0
        d["k"][:, :, run, 0] = 2
        d["k"][:, :, at + n, 0] = 1
        d["beta"][:, :, run] = 1
        d["log_alpha"][:, :, run] = 0
        d["q"][:, :, at + n:at + n + 4] = 0
        d["q"][:, :, at + n:at + n + 4, 0] = 1
        ref, ref_last = gdr_oracle(d)
        for state_out in (False, True):
            out, last = gdr_forward(d, state_out=state_out)
            for t in range(size[2]):
                assert off(out[:, :, t], ref[:, :, t]) <= 2.0 ** -7, (at, t, state_out, off(out[:, :, t], ref[:, :, t]))
        got, want = gdr_gradient(d), gdr_oracle_gradient(d)
        for name, g, w in zip(GRADS, got, want):
            assert off(g, w) <= 2.0 ** -7, (name, at)
