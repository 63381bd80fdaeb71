"""Selective scan on the GPU against the fp64 oracle: forward, gradient, single tokens."""
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import compare, put, ssm_bound, ssm_forward, ssm_gradient, ssm_inputs, ssm_oracle, ssm_oracle_gradient

pytestmark = pytest.mark.gpu

# B, L, C, N, G: one token, lengths around the tiles of 4, 8 and 16 tokens, channels that end inside a block, states that end inside a
# lane's quarter, groups; few channels and many tokens (segments), many channels (whole sequences)
SIZES = [(1, 1, 8, 1, 1), (2, 1, 64, 16, 1), (2, 2, 72, 16, 1), (1, 3, 24, 3, 1), (3, 5, 40, 5, 1), (2, 7, 64, 8, 2), (2, 8, 128, 16, 2), (1, 9, 200, 17, 1),
         (2, 15, 16, 32, 2), (2, 16, 64, 16, 1), (1, 17, 80, 31, 1), (2, 33, 48, 13, 2), (2, 49, 192, 16, 1), (1, 65, 64, 4, 1), (2, 196, 384, 16, 1), (1, 777, 72, 16, 1),
         (1, 2050, 24, 7, 1), (300, 19, 64, 16, 1), (2, 130, 4800, 2, 2), (1, 1024, 64, 32, 1)]


def _both(d, reverse, softplus=True):
    bound = lambda name, t: ssm_bound(name, t, d)
    compare(ssm_forward(d, reverse, softplus), ssm_oracle(d, reverse, softplus), bound)
    compare(ssm_gradient(d, reverse, softplus), ssm_oracle_gradient(d, reverse, softplus), bound)


@pytest.mark.parametrize("reverse", [False, True], ids=["forward", "reverse"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_gradient(size, dtype, reverse):
    B, L, C, N, G = size
    _both(ssm_inputs(B, L, C, N, dtype, G, seed=1, states=True, sliced=reverse), reverse)


@pytest.mark.parametrize("size", [(2, 37, 72, 16, 1), (1, 777, 72, 16, 1)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left_out", ["D", "z", "bias", "state", "all"])
def test_parts_left_out(left_out, dtype, size):
    B, L, C, N, G = size
    have = {n: left_out not in (n, "all") for n in ("D", "z", "bias")}
    _both(ssm_inputs(B, L, C, N, dtype, G, seed=2, states=left_out not in ("state", "all"), **have), False)


@pytest.mark.parametrize("L", [5, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_step_sizes_as_they_come(dtype, L):
    """Without softplus, step sizes of either sign: the inputs are kept small so that states stay bounded."""
    d = ssm_inputs(2, L, 64, 16, dtype, seed=3, states=True)
    d["dt"] = (d["dt"].float().abs() * 0.3).to(d["dt"].dtype)
    d["dt_bias"] = d["dt_bias"].abs() * 0.1
    _both(d, False, softplus=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_step_sizes(dtype):
    """softplus of +-80: steps of zero keep the state as it is, large ones forget it whole; z of +-100: gate z or zero."""
    d = ssm_inputs(2, 70, 64, 16, dtype, seed=4, states=True)
    d["dt_bias"] = torch.zeros_like(d["dt_bias"])
    d["dt"][:, ::3] = -80
    d["dt"][:, 1::9] = 80
    d["z"][:, ::5] = 100
    d["z"][:, 1::5] = -100
    _both(d, False)
    d["dt"].fill_(-200)                       # nothing happens: the state is handed on, bit for bit
    r = ssm_forward(d)
    assert torch.equal(r["state_out"], d["state"])


@pytest.mark.parametrize("N", [1, 3, 8, 16, 30, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [6, 384])
def test_steps_continue_a_sequence(C, dtype, N):
    """Token by token from the state of a prefix: the outputs and states of the whole sequence."""
    G = 2
    d = ssm_inputs(3, 6, C, N, dtype, G, seed=5, states=True, sliced=True)
    state, out = d["state"].clone(), torch.empty_like(d["x"])
    for t in range(6):
        vig.vig_ssm_step(d["x"][:, t], d["dt"][:, t], d["A"], d["Bt"][:, t], d["Ct"][:, t], state, out[:, t], D=d["D"], z=d["z"][:, t], dt_bias=d["dt_bias"])
    compare({"out": out, "state_out": state}, ssm_oracle(d), lambda name, t: ssm_bound(name, t, d))


@pytest.mark.parametrize("reverse", [False, True], ids=["forward", "reverse"])
@pytest.mark.parametrize("cut", [1, 16, 100])
def test_a_prefix_and_its_continuation(cut, reverse):
    d = ssm_inputs(2, 150, 72, 16, "f32", seed=6, states=True)
    want = ssm_oracle(d, reverse)
    parts = [slice(0, cut), slice(cut, 150)]
    state, out = d["state"].clone(), torch.empty_like(d["x"])
    for p in reversed(parts) if reverse else parts:
        take = lambda t: t[:, p].contiguous()
        o = torch.empty_like(take(d["x"]))
        vig.vig_ssm_fwd(take(d["x"]), take(d["dt"]), d["A"], take(d["Bt"]), take(d["Ct"]), o, D=d["D"], z=take(d["z"]), dt_bias=d["dt_bias"], state_in=state,
                        state_out=state, reverse=reverse)
        out[:, p] = o
    compare({"out": out, "state_out": state}, want, lambda name, t: ssm_bound(name, t, d))


@pytest.mark.parametrize("size", [(2, 196, 384, 16, 1), (1, 777, 72, 16, 1)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_streams_graphs_and_bits(dtype, size):
    B, L, C, N, G = size
    d = ssm_inputs(B, L, C, N, dtype, G, seed=7, states=True)
    want, grads = ssm_forward(d), ssm_gradient(d)
    for over in ("x", "dt", "z"):              # out over one of its inputs
        e = {**d, over: d[over].clone()}
        vig.vig_ssm_fwd(*(e[n] for n in ("x", "dt", "A", "Bt", "Ct")), e[over], D=e["D"], z=e["z"], dt_bias=e["dt_bias"], state_in=e["state"])
        assert torch.equal(e[over], want["out"])
    state = d["state"].clone()
    vig.vig_ssm_fwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct")), torch.empty_like(d["x"]), D=d["D"], z=d["z"], dt_bias=d["dt_bias"], state_in=state, state_out=state)
    assert torch.equal(state, want["state_out"])
    ds = d["d_state"].clone()
    outs = [torch.empty_like(grads[n]) for n in ("dx", "ddt", "dA", "dB", "dC")]
    vig.vig_ssm_bwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct")), d["d_out"], *outs, D=d["D"], z=d["z"], dt_bias=d["dt_bias"], state_in=d["state"], d_state_out=ds,
                    d_state_in=ds)
    assert torch.equal(ds, grads["d_state"]) and all(torch.equal(o, grads[n]) for o, n in zip(outs, ("dx", "ddt", "dA", "dB", "dC")))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [(ssm_forward(d, stream=side), ssm_gradient(d, stream=side))]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            got.append((ssm_forward(d), ssm_gradient(d)))
    for _ in range(2):
        for g in graphs:
            g.replay()
        got.append((ssm_forward(d), ssm_gradient(d)))
        torch.cuda.synchronize()
        for f, b in got:
            assert all(torch.equal(f[n], want[n]) for n in want) and all(torch.equal(b[n], grads[n]) for n in grads)


def test_rows_beside_the_outputs_stay():
    """Outputs that are slices: what lies between their rows is left as it was."""
    d = ssm_inputs(2, 37, 72, 5, "bf16", seed=8, sliced=True)
    whole = torch.full((2, 37, 160), 7.0, device="cuda", dtype=torch.bfloat16)
    dxz, dbc = torch.full_like(whole, 7.0), torch.full((2, 37, 13), 7.0, device="cuda", dtype=torch.bfloat16)
    vig.vig_ssm_fwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct")), whole[..., 8:80], D=d["D"], z=d["z"], dt_bias=d["dt_bias"])
    assert torch.equal(whole[..., 8:80], ssm_forward(d)["out"]) and (whole[..., :8] == 7).all() and (whole[..., 80:] == 7).all()
    want = ssm_gradient(d)
    dB, dC = dbc[..., 1:6].unflatten(2, (1, 5)), dbc[..., 6:11].unflatten(2, (1, 5))
    vig.vig_ssm_bwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct")), d["d_out"], dxz[..., :72], torch.empty_like(d["dt"]), torch.empty_like(d["A"]), dB, dC, D=d["D"], z=d["z"],
                    dt_bias=d["dt_bias"], dz=dxz[..., 80:152])
    assert torch.equal(dxz[..., :72], want["dx"]) and torch.equal(dxz[..., 80:152], want["dz"]) and torch.equal(dB, want["dB"]) and torch.equal(dC, want["dC"])
    assert (dxz[..., 72:80] == 7).all() and (dxz[..., 152:] == 7).all() and (dbc[..., 0] == 7).all() and (dbc[..., 11:] == 7).all()


def test_empty_calls():
    d = ssm_inputs(2, 4, 64, 16, "bf16", seed=9, states=True)
    none = {**d, **{n: d[n][:, :0].contiguous() for n in ("x", "dt", "z", "Bt", "Ct", "d_out")}}
    assert torch.equal(ssm_forward(none)["state_out"], d["state"])
    g = ssm_gradient(none)
    assert torch.equal(g["d_state"], d["d_state"]) and (g["dA"] == 0).all() and (g["dD"] == 0).all() and (g["dbias"] == 0).all()
    none["state"] = None
    assert (ssm_forward(none)["state_out"] == 0).all()


def test_gradient_against_differences():
    """The kernels' own forward pass in fp32, moved a little along a random direction of every input."""
    d = ssm_inputs(1, 20, 8, 4, "f32", seed=10, states=True)
    g = ssm_gradient(d)
    total = lambda e: float((f64(ssm_forward(e)["out"]) * f64(d["d_out"])).sum() + (f64(ssm_forward(e)["state_out"]) * f64(d["d_state"])).sum())
    gen = torch.Generator(device="cuda").manual_seed(0)
    for name, of in (("dx", "x"), ("ddt", "dt"), ("dA", "A"), ("dB", "Bt"), ("dC", "Ct"), ("dD", "D"), ("dz", "z"), ("dbias", "dt_bias"), ("d_state", "state")):
        way = torch.randn(d[of].shape, generator=gen, device="cuda")
        h = 2.0 ** -7
        slope = (total({**d, of: d[of] + h * way}) - total({**d, of: d[of] - h * way})) / (2 * h)
        want = float((f64(g[name]) * f64(way)).sum())
        # the central difference's own error is of h^2 = 2^-14 beside the gradient's size; roundings 2^-22 / h
        size = float((f64(g[name]) ** 2).sum() ** 0.5 * (f64(way) ** 2).sum() ** 0.5)
        assert abs(slope - want) <= 2.0 ** -9 * max(size, 1.0), name


def test_refusals_on_the_gpu():
    d = ssm_inputs(2, 8, 64, 16, "bf16", seed=11, states=True)
    a = {n: d[n] for n in ("x", "dt", "A", "Bt", "Ct")}
    out = torch.empty_like(d["x"])
    for bad in (dict(x=d["x"].transpose(0, 1)), dict(dt=d["dt"].float()), dict(A=d["A"].to(torch.bfloat16)), dict(Ct=d["Ct"][..., :8]), dict(Bt=d["Bt"][..., ::2]),
                dict(x=d["x"][:, :, ::2]), dict(dt=d["dt"][:, :4])):
        with pytest.raises(ValueError):
            vig.vig_ssm_fwd(*{**a, **bad}.values(), out)
    with pytest.raises(ValueError):
        vig.vig_ssm_fwd(*a.values(), out, state_in=d["state"][:, :, :8].contiguous())
    wide = put(torch.zeros(2, 8, 68).numpy(), "bf16")
    with pytest.raises(vig.VigError) as e:         # rows that do not begin at 16 bytes
        vig.vig_ssm_fwd(wide[..., :64], *list(a.values())[1:], out)
    assert e.value.status == -4
    z = torch.zeros(1, 4, 12, device="cuda", dtype=torch.bfloat16)
    r = torch.zeros(1, 4, 1, 4, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(vig.VigError) as e:         # twelve channels
        vig.vig_ssm_fwd(z, z, torch.zeros(12, 4, device="cuda"), r, r, z)
    assert e.value.status == -3


def test_oracle_is_the_definition_on_the_gpu_inputs():
    """A second way to the same numbers: the sum over all pairs of tokens."""
    d = ssm_inputs(1, 12, 8, 3, "f32", seed=12)
    x, dt, A, Bt, Ct = (f64(d[n]) for n in ("x", "dt", "A", "Bt", "Ct"))
    import numpy as np
    step = np.log1p(np.exp(dt + f64(d["dt_bias"])))
    run = np.cumsum(step, 1)
    y = np.zeros(x.shape)
    for t in range(12):
        for s in range(t + 1):
            y[:, t] += (np.exp((run[:, t] - run[:, s])[..., None] * A) * (Ct[:, t, 0] * Bt[:, s, 0])[:, None]).sum(-1) * step[:, s] * x[:, s]
    y = y + f64(d["D"]) * x
    z = f64(d["z"])
    assert abs(oracle.ssm_fwd(x, dt, A, Bt, Ct, f64(d["D"]), z, f64(d["dt_bias"]))[0] - y * z / (1 + np.exp(-z))).max() < 1e-12


@pytest.mark.parametrize("L", [40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_stay_where_they_belong(dtype, L):
    """A NaN in x: its channel from its token on, in its sequence; a NaN in A: its channel; neighbours, other sequences and earlier tokens
    keep their bits."""
    d = ssm_inputs(2, L, 72, 16, dtype, seed=13, states=True)
    want = ssm_forward(d)
    x = d["x"].clone()
    x[1, 21, 5] = float("nan")
    got = ssm_forward({**d, "x": x})
    bad = torch.zeros_like(got["out"], dtype=torch.bool)
    bad[1, 21:, 5] = True
    assert torch.isnan(got["out"][bad]).all() and torch.equal(got["out"][~bad], want["out"][~bad])
    A = d["A"].clone()
    A[7, 3] = float("nan")
    got = ssm_forward({**d, "A": A})
    bad = torch.zeros_like(bad)
    bad[:, :, 7] = True
    assert torch.isnan(got["out"][bad]).all() and torch.equal(got["out"][~bad], want["out"][~bad])
    # the decay of a rate without end: the state is forgotten at every token (a step size of zero aside)
    A = d["A"].clone()
    A[9] = -float("inf")
    got = ssm_forward({**d, "A": A})
    assert torch.isfinite(got["out"]).all() and torch.equal(got["out"][:, :, 10:], want["out"][:, :, 10:])
    alone = d["dt"].float()[:, -1, 9] + d["dt_bias"][9]
    h = torch.nn.functional.softplus(alone)[:, None] * d["x"].float()[:, -1, 9, None] * d["Bt"].float()[:, -1, 0]
    assert torch.allclose(got["state_out"][:, 9], h, rtol=1e-5, atol=1e-6)
