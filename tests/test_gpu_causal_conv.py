"""Causal convolution on the GPU against the fp64 oracle: forward, gradient, single tokens."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import HALF, compare, put, side_by_side

pytestmark = pytest.mark.gpu

# B, L, C, K: sequences shorter than the window, around a piece's tokens, long ones of few channels, many sequences
SIZES = [(1, 1, 8, 4), (2, 1, 16, 2), (1, 2, 8, 4), (3, 3, 24, 4), (2, 4, 8, 3), (1, 5, 40, 4), (2, 8, 64, 2), (2, 9, 64, 4), (1, 17, 200, 3), (2, 63, 8, 4), (1, 64, 72, 4),
         (1, 65, 72, 4), (2, 196, 384, 4), (1, 3001, 16, 4), (150, 31, 1032, 4)]


def _inputs(B, L, C, K, dtype, seed, states=True, bias=True, sliced=False):
    n = np.random.default_rng(seed).standard_normal
    d = {"x": side_by_side(n((B, L, C)), n((B, L, 8)), dtype=dtype)[0] if sliced else put(n((B, L, C)), dtype), "w": put(n((C, K)) * 0.5, dtype),
         "bias": put(n(C) * 0.3, dtype) if bias else None, "d_out": put(n((B, L, C)), dtype)}
    d["state"], d["d_state"] = (put(n((B, K - 1, C)), dtype) if states else None for _ in range(2))
    return d


def _run(d, act, reverse, stream=None):
    nan = lambda t: torch.full(t.shape, float("nan"), device="cuda", dtype=t.dtype)
    B, C, K = d["x"].shape[0], *d["w"].shape
    g = {"out": nan(d["x"]), "state_out": torch.full((B, K - 1, C), float("nan"), device="cuda", dtype=d["x"].dtype), "dx": nan(d["x"]), "dw": nan(d["w"])}
    if d["bias"] is not None:
        g["dbias"] = nan(d["bias"])
    if d["state"] is not None:
        g["d_state"] = nan(d["state"])
    vig.vig_causal_conv(d["x"], d["w"], d["bias"], g["out"], act=act, state_in=d["state"], state_out=g["state_out"], reverse=reverse, stream=stream)
    vig.vig_causal_conv_bwd(d["x"], d["w"], d["bias"], d["d_out"], g["dx"], g["dw"], g.get("dbias"), act=act, state_in=d["state"], d_state_out=d["d_state"],
                            d_state_in=g.get("d_state"), reverse=reverse, stream=stream)
    return g


def _check(d, act, reverse):
    """Five products and sums and a sigmoid, half a step each, terms that cancel to a quarter: 4 * 16 2^-24; the gradient's sums over n
    tokens sqrt(n) of them; results of bf16 half a step of their own (state_out is a copy)."""
    g = _run(d, act, reverse)
    out, last = oracle.causal_conv(f64(d["x"]), f64(d["w"]), f64(d["bias"]), act, f64(d["state"]), reverse)
    dx, dw, db, ds = oracle.causal_conv_bwd(f64(d["x"]), f64(d["w"]), f64(d["bias"]), f64(d["d_out"]), act, f64(d["state"]), f64(d["d_state"]), reverse)
    n = d["x"].shape[0] * d["x"].shape[1]

    def bound(name, t):
        if name == "state_out":
            return 0.0
        tol = 64 * 2.0 ** -24 * (n ** 0.5 if name in ("dw", "dbias") else 1)
        return tol + (HALF[t.dtype] if t.dtype == torch.bfloat16 else 0)

    compare(g, {"out": out, "state_out": last, "dx": dx, "dw": dw, "dbias": db, "d_state": ds}, bound)


@pytest.mark.parametrize("reverse", [False, True], ids=["forward", "reverse"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_gradient(size, dtype, act, reverse):
    _check(_inputs(*size, dtype, seed=1, sliced=reverse), act, reverse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("states,bias", [(False, True), (True, False), (False, False)])
def test_parts_left_out(states, bias, dtype):
    for size in ((2, 2, 16, 4), (2, 70, 24, 4)):
        _check(_inputs(*size, dtype, seed=2, states=states, bias=bias), "silu", False)


@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_are_the_sequence_bit_for_bit(dtype, K):
    d = _inputs(3, 9, 40, K, dtype, seed=3, sliced=True)
    want = _run(d, "silu", False)
    state, out = d["state"].clone(), torch.empty_like(d["x"])
    for t in range(9):
        vig.vig_causal_conv_step(d["x"][:, t], d["w"], d["bias"], state, out[:, t])
    assert torch.equal(out, want["out"]) and torch.equal(state, want["state_out"])


@pytest.mark.parametrize("cut", [1, 2, 30])
def test_a_prefix_and_its_continuation_in_place(cut):
    d = _inputs(2, 70, 24, 4, "bf16", seed=4)
    want = _run(d, "silu", False)
    state = d["state"].clone()
    outs = []
    for p in (slice(0, cut), slice(cut, 70)):
        x = d["x"][:, p].contiguous()
        outs.append(torch.empty_like(x))
        vig.vig_causal_conv(x, d["w"], d["bias"], outs[-1], state_in=state, state_out=state)
    assert torch.equal(torch.cat(outs, 1), want["out"]) and torch.equal(state, want["state_out"])


def test_streams_graphs_and_bits():
    d = _inputs(2, 196, 384, 4, "bf16", seed=5)
    want = _run(d, "silu", False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [_run(d, "silu", False, stream=side)]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(_run(d, "silu", False))
    for _ in range(2):
        for g in graphs:
            g.replay()
        got.append(_run(d, "silu", False))
        torch.cuda.synchronize()
        assert all(torch.equal(r[n], want[n]) for r in got for n in want)


def test_far_values_and_empty_calls():
    """Pre-activations of +-1000: x or zero, and slopes of one and zero; no tokens: the window is handed on."""
    x = torch.tensor([1000.0, -1000.0], device="cuda").repeat(16).view(1, 4, 8).contiguous()
    w, g = torch.zeros(8, 4, device="cuda"), torch.ones(1, 4, 8, device="cuda")
    w[:, 3] = 1
    out, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    vig.vig_causal_conv(x, w, None, out)
    vig.vig_causal_conv_bwd(x, w, None, g, dx, dw, None)
    assert torch.equal(out, x.clamp(min=0)) and torch.equal(dx, (x > 0).float()) and torch.isfinite(dw).all()
    s, ds = torch.randn(1, 3, 8, device="cuda"), torch.randn(1, 3, 8, device="cuda")
    so, do, db = torch.empty_like(s), torch.empty_like(s), torch.ones(8, device="cuda")
    e = x[:, :0].contiguous()
    vig.vig_causal_conv(e, w, None, e, state_in=s, state_out=so)
    vig.vig_causal_conv_bwd(e, w, None, e, e, dw, db, state_in=s, d_state_out=ds, d_state_in=do)
    assert torch.equal(so, s) and torch.equal(do, ds) and (dw == 0).all() and (db == 0).all()


def test_refusals_on_the_gpu():
    d = _inputs(2, 8, 16, 4, "bf16", seed=6)
    out = torch.empty_like(d["x"])
    for bad in (dict(x=d["x"][:, :, ::2]), dict(w=d["w"].float()), dict(w=d["w"][:, ::2]), dict(bias=d["bias"][:8].contiguous())):
        a = {**d, **bad}
        with pytest.raises(ValueError):
            vig.vig_causal_conv(a["x"], a["w"], a["bias"], out)
    with pytest.raises(vig.VigError) as e:
        vig.vig_causal_conv(d["x"], d["w"], d["bias"], out, act="gelu")
    assert e.value.status == -3
    w = torch.zeros(16, 5, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(vig.VigError) as e:
        vig.vig_causal_conv(d["x"], w, None, out)
    assert e.value.status == -3
