"""Gated delta rule on the GPU against the fp64 oracle: whole sequences, gradient, single tokens."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import (NAMES, T, bound, check, f64, gdr_forward, gdr_gradient, gdr_inputs, gdr_oracle, gdr_oracle_gradient, off)

pytestmark = pytest.mark.gpu

# B, H, L, dk, dv: one token, lengths around 16, 64 and 128, heads of this library and larger ones, odd ones, several blocks of columns
SIZES = [(1, 1, 1, 16, 32), (2, 3, 2, 24, 48), (3, 1, 16, 8, 8), (2, 3, 17, 24, 48), (1, 2, 64, 32, 64), (2, 2, 65, 128, 128), (1, 3, 130, 20, 17),
         (1, 1, 300, 64, 256), (1, 2, 196, 32, 64), (1, 1, 5, 1, 1), (1, 2, 33, 96, 40), (2, 1, 127, 128, 24), (1, 2, 128, 48, 96), (1, 1, 77, 100, 100),
         (1, 1, 1100, 24, 48), (2, 1, 515, 64, 64), (1, 2, 2049, 16, 40), (1, 1, 1990, 64, 128), (1, 2, 40, 70, 70), (1, 1, 50, 12, 130)]


def _terms(L, dk, dv):
    return L + dk + dv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("reverse", [False, True])
def test_forward(size, dtype, reverse):
    d = gdr_inputs(*size, dtype, seed=1, gate_mean=1.0, states=reverse)
    out, last = gdr_forward(d, reverse)
    ref, ref_last = gdr_oracle(d, reverse)
    check([("out", out, ref), ("state", last, ref_last)], _terms(*size[2:]), dtype == "bf16")
    again, _ = gdr_forward(d, reverse, state_out=False)
    check([("out without a final state", again, ref)], _terms(*size[2:]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("states", [False, True])
def test_gradient(size, dtype, states):
    d = gdr_inputs(*size, dtype, seed=2, gate_mean=1.0, states=states)
    got = gdr_gradient(d, reverse=states)
    ref = gdr_oracle_gradient(d, reverse=states)
    check(list(zip(("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state"), got, ref)), _terms(*size[2:]), dtype == "bf16")


@pytest.mark.parametrize("preference", [vig.VIG_TEST_KERNEL_SIMT, vig.VIG_TEST_KERNEL_WARP_TILES], ids=["walks", "tiles"])
@pytest.mark.parametrize("size", [(2, 3, 1, 24, 48), (1, 2, 3, 17, 33), (2, 1, 5, 128, 128), (1, 2, 8, 64, 16), (1, 1, 12, 9, 100), (3, 1, 70, 40, 72), (1, 2, 131, 33, 65)], ids=str)
@pytest.mark.parametrize("states", [False, True])
def test_either_form_of_bf16(size, states, preference):
    """Sizes of either side of the line between walks and tiles, by the form that the library would not choose as well."""
    d = gdr_inputs(*size, "bf16", seed=21, gate_mean=1.0, states=states)
    vig.vig_test_set_kernel_preference(preference)
    try:
        out, last = gdr_forward(d, reverse=states)
        got = gdr_gradient(d, reverse=states)
    finally:
        vig.vig_test_set_kernel_preference(vig.VIG_TEST_KERNEL_AUTO)
    ref, ref_last = gdr_oracle(d, reverse=states)
    check([("out", out, ref), ("state", last, ref_last)], _terms(*size[2:]), True)
    check(list(zip(("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state"), got, gdr_oracle_gradient(d, reverse=states))), _terms(*size[2:]), True)


def test_gradient_against_differences():
    """Of the GPU's own fp32 forward call along random directions.  Central differences: third derivatives h^2 / 6 and rounding
    2^-24 sqrt(values) / h; h = 2^-6 and a loss of ~700 values leave 1e-4 of either."""
    d = gdr_inputs(1, 2, 45, 24, 16, "f32", seed=3, states=True)
    grads = gdr_gradient(d)
    rng = torch.Generator(device="cuda").manual_seed(1)

    def loss(e):
        out, last = gdr_forward(e)
        return float((out.double() * d["d_out"].double()).sum() + (last.double() * d["d_state"].double()).sum())

    for name, g in zip((*NAMES, "state"), grads):
        way = torch.randn(d[name].shape, generator=rng, device="cuda")
        if name == "log_alpha":
            way = way * d[name].abs()   # stays <= 0
        h = 2.0 ** -6
        up, down = (loss({**d, name: d[name] + s * h * way}) for s in (1, -1))
        want = float((g.double() * way.double()).sum())
        assert abs((up - down) / (2 * h) - want) <= 2e-3 * max(abs(want), float(g.double().norm() * way.double().norm()) * 0.1), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [40, 200])
def test_gates_and_steps_at_their_limits(dtype, L):
    """Gates that forget everything (-inf, -1e4, the type's lowest value), that keep everything (0), steps of 0, 1 and 2."""
    d = gdr_inputs(2, 2, L, 32, 48, dtype, seed=4, states=True)
    la, be = d["log_alpha"], d["beta"]
    la[0, 0, 3::7] = float("-inf")
    la[0, 1, 5::11] = -1e4
    la[0, 1, 20] = torch.finfo(la.dtype).min
    la[1, 0] = 0
    be[1, 0, ::3] = 0
    be[1, 0, 1::3] = 1
    be[1, 1] = 2
    la[1, 1, 17:] = -3
    for reverse in (False, True):
        out, last = gdr_forward(d, reverse)
        ref, ref_last = gdr_oracle(d, reverse)
        check([("out", out, ref), ("state", last, ref_last)], _terms(L, 32, 48), dtype == "bf16")
        got, want = gdr_gradient(d, reverse), gdr_oracle_gradient(d, reverse)
        check(list(zip(("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state"), got, want)), _terms(L, 32, 48), dtype == "bf16")
        assert (got[3][0, 0, 3::7] == 0).all()   # exp(-inf) does not move


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_first_gate_without_a_state_has_no_gradient(dtype):
    for L in (1, 70):
        for reverse in (False, True):
            d = gdr_inputs(2, 2, L, 24, 32, dtype, seed=5)
            assert (gdr_gradient(d, reverse)[3][:, :, L - 1 if reverse else 0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-6, 1e6])
def test_values_of_other_magnitudes(dtype, scale):
    """Everything is linear in v and the state: no range inside but the type's own."""
    d = gdr_inputs(1, 2, 150, 32, 64, dtype, seed=6, gate_mean=2.0, states=True)
    d["v"], d["state"] = d["v"] * scale, d["state"] * scale
    out, last = gdr_forward(d)
    ref, ref_last = gdr_oracle(d)
    check([("out", out, ref), ("state", last, ref_last)], _terms(150, 32, 64), dtype == "bf16")


@pytest.mark.parametrize("parallel", [False, True])
@pytest.mark.parametrize("size", [(1, 2, 12, 16, 32), (2, 2, 20, 24, 48), (1, 1, 10, 64, 128)], ids=str)
def test_keys_beyond_unit_length(size, parallel):
    """beta |k|^2 around 8.  Parallel keys: the state grows about seven times a token, 10^9 and more in all, beyond what fp16 tiles hold; those
    units are redone in fp32 walks.  Errors grow with the state and stay relative to it; the comparison is token by token (bf16: 2^-7, as
    everywhere)."""
    d = gdr_inputs(*size, "bf16", seed=15, states=True)
    if parallel:
        d["k"] = torch.nn.functional.normalize(d["k"].float() * 0.1 + d["k"][:, :, :1].float(), dim=-1)
        d["beta"].fill_(0.5)   # (steps drawn near 1 / 16 would cancel the state instead)
    d["k"] = (d["k"].float() * 4).bfloat16()
    torch.cuda.synchronize()
    vig.vig_test_take_fallback_count()
    out, last = gdr_forward(d)
    ref, ref_last = gdr_oracle(d)
    for t in range(size[2]):
        assert off(out[:, :, t], ref[:, :, t]) <= 2.0 ** -7, t
    assert off(last, ref_last) <= 2.0 ** -15
    taken = vig.vig_test_take_fallback_count()
    got, want = gdr_gradient(d), gdr_oracle_gradient(d)
    for name, g, w in zip(("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state"), got, want):
        assert off(g, w) <= 2.0 ** -7, name
    if parallel:
        assert taken > 0 and vig.vig_test_take_fallback_count() > 0


def test_one_unit_of_a_long_call_beyond_the_range():
    """Segments side by side: a dozen parallel keys beyond unit length in the middle of one unit (10^9), forgotten soon after; that unit is redone
    whole, the others are not."""
    for size in ((1, 2, 1100, 24, 48), (2, 1, 400, 32, 64)):
        d = gdr_inputs(*size, "bf16", seed=18, gate_mean=1.0, states=True)
        mid = size[2] // 2
        d["k"][0, 0, mid:mid + 12] = d["k"][0, 0, mid] * 4
        d["beta"][0, 0, mid:mid + 12] = 0.5
        d["log_alpha"][0, 0, mid + 15] = float("-inf")
        torch.cuda.synchronize()
        vig.vig_test_take_fallback_count()
        out, last = gdr_forward(d)
        taken = vig.vig_test_take_fallback_count()
        ref, ref_last = gdr_oracle(d)
        for u in range(size[0] * size[1]):
            for part in (slice(0, mid), slice(mid, mid + 15), slice(mid + 15, None)):
                assert off(out.flatten(0, 1)[u, part], ref.reshape(-1, *ref.shape[2:])[u, part]) <= 2.0 ** -7
        check([("state", last, ref_last)], sum(size[2:]), True)
        got, want = gdr_gradient(d), gdr_oracle_gradient(d)
        assert taken > 0 and vig.vig_test_take_fallback_count() == 1
        for name, g, w in zip(("dq", "dk", "dv", "dlog_alpha", "dbeta", "d_state"), got, want):
            for u in range(size[0] * size[1]):
                assert off(g.flatten(0, 1)[u], w.reshape(-1, *w.shape[2:])[u]) <= 2.0 ** -7, (name, u)


def test_in_range_inputs_stay_on_the_tiles():
    torch.cuda.synchronize()
    vig.vig_test_take_fallback_count()
    for size in SIZES:
        d = gdr_inputs(*size, "bf16", seed=16, gate_mean=2.0, states=True)
        gdr_forward(d)
        gdr_gradient(d)
    assert vig.vig_test_take_fallback_count() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_stay_in_their_columns_and_behind_their_tokens(dtype):
    """A value that is not finite reaches its column from its token on, a key, gate or step the whole unit from its token on (and the
    token's own read-out), nothing before and no other unit."""
    for name, at, column in (("v", (0, 0, 37, 5), 5), ("v", (0, 1, 3, 0), 0), ("k", (0, 0, 70, 2), None), ("log_alpha", (0, 1, 20), None), ("beta", (0, 0, 18), None)):
        for bad in (float("nan"), float("inf")):
            if name == "log_alpha" and bad > 0:
                continue
            d = gdr_inputs(1, 3, 100, 16, 32, dtype, seed=17, gate_mean=2.0)
            clean, _ = gdr_forward(d)
            d[name][at] = bad
            out, _ = gdr_forward(d)
            same = torch.ones_like(out, dtype=torch.bool)
            u, t = at[1], at[2]
            if column is None:
                same[0, u, t:] = False
            else:
                same[0, u, t:, column] = False
            assert torch.allclose(out[same].float(), clean[same].float(), rtol=2.0 ** -6, atol=2.0 ** -6 * float(clean.float().abs().max())), (name, at, bad)
            assert not torch.isfinite(out[~same]).any(), (name, at, bad)


def test_correlated_keys():
    """Keys that are nearly one another: the triangular systems of a chunk are as ill-conditioned as unit keys make them."""
    for dtype in ("bf16", "f32"):
        d = gdr_inputs(1, 2, 200, 32, 64, dtype, seed=7, gate_mean=6.0)
        k = torch.nn.functional.normalize(d["k"].float() * 0.2 + d["k"][:, :, :1].float(), dim=-1)
        d["k"] = k.to(T[dtype])
        out, last = gdr_forward(d)
        ref, ref_last = gdr_oracle(d)
        # corrections of up to all earlier tokens instead of a few independent ones: partial sums of the size of L terms
        check([("out", out, ref), ("state", last, ref_last)], 200 ** 2, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (1, 4, 24, 48), (3, 2, 128, 128), (2, 2, 33, 70), (5, 1, 128, 256), (2, 3, 16, 36)], ids=str)
def test_single_tokens(size, dtype):
    """Step by step from a state: the walk over the sequence, and the state in place.

    Outputs are compared over all tokens at once.  out = alpha q.S + (q.k) beta (v - alpha k.S): its roundings are relative to the terms, and
    with one value a head a token's terms may cancel to any smaller sum (1 x 1: out = alpha S (1 - beta) + beta v with terms of
    0.3 and a result of 0.02), so a lone token's own norm says nothing; the terms are bounded by the states and values of the run."""
    B, H, dk, dv = size
    d = gdr_inputs(B, H, 6, dk, dv, dtype, seed=8, states=True)
    ref, ref_last = gdr_oracle(d)
    state = d["state"].clone()
    out = torch.full((6, B, H, dv), float("nan"), device="cuda", dtype=T[dtype])
    for t in range(6):
        x = [d[n][:, :, t].clone() for n in NAMES]
        one = torch.empty(B, H, dv, device="cuda", dtype=T[dtype])
        vig.vig_gdr_step(*x, state, one)
        out[t] = one
    check([("out", out, np.moveaxis(ref, 2, 0))], 6 + dk)
    check([("state", state, ref_last)], 6 + dk)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_then_single_tokens(dtype):
    """A sequence cut into a prefix (chunked, final state into the caller's buffer, which was its initial one too) and single tokens."""
    d = gdr_inputs(2, 3, 90, 32, 64, dtype, seed=9, states=True)
    ref, ref_last = gdr_oracle(d)
    state, cut = d["state"].clone(), 83
    x = [d[n][:, :, :cut].contiguous() for n in NAMES]
    out = torch.empty_like(x[2])
    vig.vig_gdr_fwd(*x, out, state_in=state, state_out=state)
    check([("prefix", out, ref[:, :, :cut])], 90 + 32, dtype == "bf16")
    one = torch.empty(2, 3, 64, device="cuda", dtype=T[dtype])
    for t in range(cut, 90):
        vig.vig_gdr_step(*(d[n][:, :, t].clone() for n in NAMES), state, one)
        check([("token", one, ref[:, :, t])], 90 + 32, dtype == "bf16")
    check([("state", state, ref_last)], 90 + 32, dtype == "bf16")


def test_no_tokens_pass_the_state_on():
    d = gdr_inputs(2, 2, 0, 16, 32, "f32", states=True)
    out, last = gdr_forward(d)
    assert torch.equal(last, d["state"])
    assert torch.equal(gdr_gradient(d)[5], d["d_state"])
    d["state"] = None
    assert (gdr_forward(d)[1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 2, 70, 24, 48), (1, 3, 33, 17, 20), (1, 2, 65, 128, 128)], ids=str)
def test_nothing_is_written_beyond_the_outputs(size, dtype):
    """Outputs inside larger buffers whose other values stay as they were, and inputs stay what they were."""
    d = gdr_inputs(*size, dtype, seed=10, states=True)
    before = {n: t.clone() for n, t in d.items()}
    buffers = []

    def inside(t):
        pad = 256
        b = torch.full((t.numel() + 2 * pad,), 7.0, device="cuda", dtype=t.dtype)
        buffers.append((b, pad, t.numel()))
        return b[pad:pad + t.numel()].view(t.shape)

    out, last = inside(d["v"]), inside(d["state"])
    vig.vig_gdr_fwd(*(d[n] for n in NAMES), out, state_in=d["state"], state_out=last)
    grads = [inside(d[n]) for n in NAMES]
    vig.vig_gdr_bwd(*(d[n] for n in NAMES), d["d_out"], *grads, state_in=d["state"], d_state_out=d["d_state"], d_state_in=inside(d["state"]))
    torch.cuda.synchronize()
    for b, pad, n in buffers:
        assert (b[:pad] == 7).all() and (b[pad + n:] == 7).all()
    for n, t in before.items():
        assert torch.equal(t, d[n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_again_and_alone(dtype):
    """Twice the same call, and a unit by itself: the same bits (no atomics, no dependence on other units)."""
    d = gdr_inputs(3, 4, 196, 32, 64, dtype, seed=11, states=True)
    a, b = gdr_forward(d) + tuple(gdr_gradient(d)), gdr_forward(d) + tuple(gdr_gradient(d))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 2, 140, 32, 64), (1, 2, 900, 24, 48), (2, 2, 50, 20, 30)], ids=str)
def test_states_in_place(size, dtype):
    """The final state over the initial one, the initial state's gradient over the final one's, and a call whose units are redone."""
    for beyond in (False, True):
        d = gdr_inputs(*size, dtype, seed=19, states=True)
        if beyond:
            d["k"][0, 0, 20:30] = d["k"][0, 0, 20] * 4
            d["beta"][0, 0, 20:30] = 0.5
            d["log_alpha"][0, 0, 33] = float("-inf")
        want, want_last = gdr_forward(d)
        want_grads = gdr_gradient(d)
        state, d_state = d["state"].clone(), d["d_state"].clone()
        out = torch.empty_like(want)
        vig.vig_gdr_fwd(*(d[n] for n in NAMES), out, state_in=state, state_out=state)
        assert torch.equal(out, want) and torch.equal(state, want_last)
        grads = [torch.empty_like(g) for g in want_grads[:5]]
        vig.vig_gdr_bwd(*(d[n] for n in NAMES), d["d_out"], *grads, state_in=d["state"], d_state_out=d_state, d_state_in=d_state)
        for a, b in zip(grads + [d_state], want_grads):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_state_after_values_of_very_different_size(dtype):
    """A chunk of values of 1e9, forgotten, then nothing at all, then values of 1e-9: scales of the columns jump both ways."""
    d = gdr_inputs(1, 2, 260, 16, 32, dtype, seed=20)
    d["v"][:, :, :64] *= 1e9
    d["log_alpha"][:, :, 64] = float("-inf")
    d["v"][:, :, 64:128] = 0
    d["v"][:, :, 128:] *= 1e-9
    torch.cuda.synchronize()
    vig.vig_test_take_fallback_count()
    out, last = gdr_forward(d)
    ref, ref_last = gdr_oracle(d)
    for part in (slice(0, 64), slice(128, None)):
        assert off(out[:, :, part], ref[:, :, part]) <= bound(out, 300)
    assert (out[:, :, 64:128] == 0).all() and off(last, ref_last) <= 2.0 ** -15
    assert vig.vig_test_take_fallback_count() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 2, 140, 32, 64), (1, 2, 1100, 24, 48)], ids=str)
def test_other_stream_and_captured_graphs(size, dtype):
    """On a side stream; captured twice, replayed in turn on new inputs beside a call outside any graph."""
    sets = [gdr_inputs(*size, dtype, seed=s, states=True) for s in (12, 13, 14)]
    want = [gdr_forward(d) + tuple(gdr_gradient(d)) for d in sets]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gdr_forward(sets[0], stream=side) + tuple(gdr_gradient(sets[0], stream=side))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))
    held, graphs = [], []
    for d in sets[:2]:
        g = torch.cuda.CUDAGraph()
        buf = {n: (None if t is None else t.clone()) for n, t in d.items()}
        with torch.cuda.graph(g):
            res = gdr_forward(buf) + tuple(gdr_gradient(buf))
        held.append((buf, res))
        graphs.append(g)
    for n, t in sets[2].items():   # the second graph on the third inputs
        held[1][0][n].copy_(t)
    for _ in range(2):
        graphs[0].replay()
        graphs[1].replay()
        eager = gdr_forward(sets[1]) + tuple(gdr_gradient(sets[1]))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held[0][1], want[0]))
        assert all(torch.equal(x, y) for x, y in zip(held[1][1], want[2]))
        assert all(torch.equal(x, y) for x, y in zip(eager, want[1]))


def test_binding_refusals_on_the_gpu():
    d = gdr_inputs(1, 2, 5, 16, 32, "f32", states=True)
    out = torch.empty_like(d["v"])
    x = [d[n] for n in NAMES]
    with pytest.raises(ValueError, match="contiguous"):
        vig.vig_gdr_fwd(x[0].transpose(1, 2), *x[1:], out)
    with pytest.raises(ValueError, match="dtype"):
        vig.vig_gdr_fwd(x[0], x[1].bfloat16(), *x[2:], out)
    with pytest.raises(ValueError, match="shape"):
        vig.vig_gdr_fwd(x[0], x[1][:, :1].contiguous(), *x[2:], out)
    with pytest.raises(ValueError, match="shape"):
        vig.vig_gdr_fwd(*x, out, state_in=d["state"].transpose(2, 3).contiguous())
    with pytest.raises(ValueError, match="dtype"):
        vig.vig_gdr_fwd(*x, out, state_in=d["state"].bfloat16())
    with pytest.raises(ValueError, match="shape"):
        vig.vig_gdr_fwd(*x[:3], x[3][..., None].contiguous(), x[4], out)
    wide = torch.zeros(1, 1, 4, 136, device="cuda")
    gate = torch.zeros(1, 1, 4, device="cuda")
    with pytest.raises(vig.VigError) as e:
        vig.vig_gdr_fwd(wide, wide, wide, gate, gate, wide)
    assert e.value.status == -3
    odd = torch.zeros(4 * 2 * 5 * 16 + 1, device="cuda")[1:161].view(1, 2, 5, 16)
    with pytest.raises(vig.VigError) as e:
        vig.vig_gdr_fwd(odd, *x[1:], out)
    assert e.value.status == -4
