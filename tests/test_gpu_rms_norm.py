"""RMS norm with the residual's addition on the GPU against the fp64 oracle: forward, 8-bit results, gradient."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import HALF, compare, put

pytestmark = pytest.mark.gpu

# rows, C: one vector, rows of a warp with and without idle lanes, of 128 to 1024 threads, more rows than a gradient's blocks
SIZES = [(1, 8), (3, 24), (7, 128), (5, 136), (9, 192), (2, 256), (196, 768), (33, 1000), (3, 1032), (2, 2056), (17, 4096), (2, 4104), (2, 8200), (1, 12296), (3, 16384),
         (5000, 64), (1300, 1536)]


def _inputs(rows, C, dtype, seed, residual=True):
    n = np.random.default_rng(seed).standard_normal
    return {"x": put(n((rows, C)), dtype), "residual": put(n((rows, C)) * 2, dtype) if residual else None, "weight": put(n(C) * 0.3 + 1, dtype),
            "d_out": put(n((rows, C)), dtype), "d_sum": put(n((rows, C)), dtype) if residual else None}


def _run(d, eps=1e-5, stream=None):
    nan = lambda t: torch.full_like(t, float("nan"))
    g = {"out": nan(d["x"]), "rstd": torch.full(d["x"].shape[:-1], float("nan"), device="cuda"), "dx": nan(d["x"]), "dweight": nan(d["weight"])}
    if d["residual"] is not None:
        g["sum"] = nan(d["x"])
    vig.vig_rms_norm(d["x"], d["weight"], g["out"], residual=d["residual"], sum_out=g.get("sum"), rstd=g["rstd"], eps=eps, stream=stream)
    vig.vig_rms_norm_bwd(g.get("sum", d["x"]), d["weight"], g["rstd"], d["d_out"], g["dx"], g["dweight"], d_sum=d["d_sum"], stream=stream)
    return g


def _check(d, eps=1e-5):
    """A sum of C squares in runs of at most 32, then pairwise, the root and four products: 16 half steps; dx is a difference whose terms
    are at most four times it; dweight a sum over the rows, sqrt of their number of half steps more."""
    g = _run(d, eps)
    out, s, rstd = oracle.rms_norm(f64(d["x"]), f64(d["weight"]), f64(d["residual"]), eps)
    kept = f64(g["sum"]) if "sum" in g else s
    dx, dw = oracle.rms_norm_bwd(kept, f64(d["weight"]), f64(g["rstd"]), f64(d["d_out"]), f64(d["d_sum"]))
    rows = d["x"].shape[0]

    def bound(name, t):
        tol = 16 * 2.0 ** -24 * {"dx": 4, "dweight": 1 + rows ** 0.5 / 4}.get(name, 1)
        return tol + (HALF[t.dtype] if t.dtype == torch.bfloat16 else 0)

    compare(g, {"out": out, "sum": s, "rstd": rstd, "dx": dx, "dweight": dw}, bound)


@pytest.mark.parametrize("residual", [True, False], ids=["residual", "alone"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_gradient(size, dtype, residual):
    _check(_inputs(*size, dtype, seed=1, residual=residual))


def _dequantised(d, block, eps=1e-5):
    rows, C = d["x"].shape
    q = torch.empty(rows, C, device="cuda", dtype=torch.float8_e4m3fn)
    scales = torch.full((rows, -(-C // 128) if block else 1), float("nan"), device="cuda")
    s = torch.empty_like(d["x"]) if d["residual"] is not None else None
    vig.vig_rms_norm_e4m3(d["x"], d["weight"], q, scales, residual=d["residual"], sum_out=s, eps=eps)
    return q, scales, s


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_eight_bits(size, dtype, block):
    """Every code is the nearest one to the oracle's value over the scale: at most half a step, 2^-4 of the value (2^-10 below the smallest
    normal number, 2^-6), and 2^-20 for the value's own roundings; the scale is max / 448 to 16 half steps."""
    d = _inputs(*size, dtype, seed=2)
    q, scales, s = _dequantised(d, block)
    out, total, _ = oracle.rms_norm(f64(d["x"]), f64(d["weight"]), f64(d["residual"]))
    rows, C = size
    n = scales.shape[1]
    width = -(-C // n) if n == 1 else 128
    pad = np.zeros((rows, n * width))
    pad[:, :C] = np.abs(out)
    want = pad.reshape(rows, n, width).max(-1) / 448
    assert np.allclose(f64(scales), want, rtol=16 * 2.0 ** -24, atol=0)
    over = out / np.repeat(want, width, 1)[:, :C]
    off = np.abs(f64(q.float()) - over)
    assert (off <= np.maximum(np.abs(over) * 2.0 ** -4, 2.0 ** -10) + 448 * 2.0 ** -20).all()
    assert np.abs(f64(q.float())).max() == 448
    compare({"sum": s}, {"sum": total}, lambda name, t: HALF[t.dtype] * 2)


def test_eight_bits_of_zeros_nan_and_tiny_rows():
    d = _inputs(4, 256, "f32", seed=3, residual=False)
    d["x"][0] = 0
    d["x"][1, 130] = float("nan")
    d["weight"][:128] = 0
    q, scales, _ = _dequantised(d, 128)
    f = q.float()
    assert (f[:, :128][[0, 2, 3]] == 0).all() and (scales[[0, 2, 3], 0] == 2.0 ** -126).all() and (f[0] == 0).all()
    assert torch.isnan(f[1]).all() and torch.isnan(scales[1]).all()
    assert torch.isfinite(f[2:]).all() and (f[2:, 128:].abs().amax(1) == 448).all()
    d["x"][3] = 0
    d["x"][3, 200] = float("inf")
    q, scales, _ = _dequantised(d, 128)
    assert torch.isnan(scales[3, 1]) and torch.isnan(q.float()[3, 128:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [64, 2048, 16384])
@pytest.mark.parametrize("size", [1e25, 3e38, 1e-25, 1e-38])
def test_rows_whose_squares_leave_the_range(size, C, dtype):
    """No eps beside small rows; with one that is far above them, out is x / sqrt(eps)."""
    n = np.random.default_rng(4).standard_normal
    x = n((3, C))
    x = x / np.abs(x).max() * size
    x[1] = n(C)                                # (a row of ordinary values beside them)
    x, w = put(x, dtype), put(n(C) * 0.3 + 1, dtype)
    for eps in (0.0, 1e-5):
        out, rstd = torch.empty_like(x), torch.empty(3, device="cuda")
        vig.vig_rms_norm(x, w, out, rstd=rstd, eps=eps)
        ref, _, r = oracle.rms_norm(f64(x), f64(w), None, eps)
        # subnormal inputs may count as zero: 2^-126 beside values of `size`
        tol = 32 * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0) + (2.0 ** -126 / size * C ** 0.5 if eps == 0 else 0)
        rows = [0, 1, 2] if eps == 0 or size > 1 else [1]
        for i in rows:
            if np.isfinite(r[i]) and r[i] < 3e38:
                assert np.linalg.norm(f64(out)[i] - ref[i]) <= tol * np.linalg.norm(ref[i]), (i, eps)


def test_zero_rows_and_rows_that_are_not_finite():
    d = _inputs(4, 64, "f32", seed=5, residual=False)
    d["x"][0] = 0
    d["x"][1, 3] = float("nan")
    d["x"][2, 3] = float("inf")
    out = torch.empty_like(d["x"])
    vig.vig_rms_norm(d["x"], d["weight"], out)
    assert (out[0] == 0).all() and torch.isnan(out[1]).all() and torch.isnan(out[2, 3]) and torch.isfinite(out[3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_streams_graphs_and_bits(dtype):
    d = _inputs(300, 768, dtype, seed=6)
    want = _run(d)
    res = d["residual"].clone()
    out = torch.empty_like(d["x"])
    vig.vig_rms_norm(d["x"], d["weight"], out, residual=res, sum_out=res)
    assert torch.equal(out, want["out"]) and torch.equal(res, want["sum"])
    x = d["x"].clone()
    vig.vig_rms_norm(x, d["weight"], x, residual=d["residual"])
    assert torch.equal(x, want["out"])
    for over in ("d_sum", "d_out"):
        e = {**d, over: d[over].clone()}
        dw = torch.empty_like(d["weight"])
        vig.vig_rms_norm_bwd(want["sum"], d["weight"], want["rstd"], e["d_out"], e[over], dw, d_sum=e["d_sum"])
        assert torch.equal(e[over], want["dx"]) and torch.equal(dw, want["dweight"])
    vig.vig_rms_norm_bwd(want["sum"], d["weight"], want["rstd"], d["d_out"], x, None, d_sum=d["d_sum"])
    assert torch.equal(x, want["dx"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [_run(d, stream=side)]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(_run(d))
    for _ in range(2):
        for g in graphs:
            g.replay()
        got.append(_run(d))
        torch.cuda.synchronize()
        assert all(torch.equal(r[n], want[n]) for r in got for n in want)


def test_shapes_empty_calls_and_refusals():
    d = _inputs(12, 64, "bf16", seed=7)
    want = _run(d)
    shaped = {n: t.view(2, 3, 2, 64) if t is not None and t.dim() == 2 else t for n, t in d.items()}
    got = _run(shaped)
    assert all(torch.equal(got[n].reshape(want[n].shape), want[n]) for n in want)
    e, r = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), torch.empty(0, device="cuda")
    vig.vig_rms_norm(e, d["weight"], e, rstd=r)
    dw = torch.ones_like(d["weight"])
    vig.vig_rms_norm_bwd(e, d["weight"], r, e, e, dw)
    assert (dw == 0).all()
    out = torch.empty_like(d["x"])
    for bad in (dict(x=d["x"][:, ::2]), dict(weight=d["weight"].float()), dict(residual=d["residual"][:6]), dict(x=d["x"].half())):
        a = {**d, **bad}
        with pytest.raises(ValueError):
            vig.vig_rms_norm(a["x"], a["weight"], out, residual=a["residual"])
    q = torch.empty(12, 64, device="cuda", dtype=torch.float8_e4m3fn)
    for scales in (torch.empty(12, 2, device="cuda"), torch.empty(12, device="cuda"), torch.empty(12, 1, device="cuda", dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            vig.vig_rms_norm_e4m3(d["x"], d["weight"], q, scales)
    with pytest.raises(vig.VigError) as err:
        vig.vig_rms_norm(d["x"], d["weight"], out, eps=-1.0)
    assert err.value.status == -2
    odd = torch.zeros(2, 12, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(vig.VigError) as err:
        vig.vig_rms_norm(odd, odd[0].clone(), torch.empty_like(odd))
    assert err.value.status == -3
