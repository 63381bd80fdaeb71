"""A layer with the selective scan as it is used, on the GPU: norm with the residual, a projection that writes x and z side by side,
causal convolution and scan in both directions over the patch sequence, and the way back; then single tokens behind a prefix."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import T, f64, off
from row_helpers import put

pytestmark = pytest.mark.gpu


def _layer(dtype, B=2, L=77, W=64, C=96, n=16, G=1, K=4):
    rng = np.random.default_rng(1).standard_normal
    d = {"x": put(rng((B, L, W)), dtype), "residual": put(rng((B, L, W)), dtype), "norm": put(rng(W) * 0.2 + 1, dtype), "w_in": put(rng((W, 2 * C)) / 8, dtype),
         "w_x": put(rng((C, 2 * G * n + 4)) / 10, dtype), "w_dt": put(rng((4, C)) / 2, dtype), "conv": put(rng((C, K)) / 2, dtype), "conv_b": put(rng(C) / 5, dtype),
         "A": put(-(1 + np.arange(n)) * np.exp(0.1 * rng((C, n)))), "D": put(rng(C)), "dt_bias": put(rng(C) * 0.5 - 2), "d_out": put(rng((B, L, C)), dtype)}
    return d, (B, L, C, n, G)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_both_directions_and_the_way_back(dtype):
    """Every call on the outputs of the one before, nothing waited for in between, against the oracles run on the stored tensors that entered
    each call.  Bounds: half a step of bf16 and as much again for sums that cancel; fp32 as each operator's own tests have it."""
    d, (B, L, C, n, G) = _layer(dtype)
    y, s = torch.empty_like(d["x"]), torch.empty_like(d["x"])
    rstd = torch.empty(B, L, device="cuda")
    vig.vig_rms_norm(d["x"], d["norm"], y, residual=d["residual"], sum_out=s, rstd=rstd)
    xz = y @ d["w_in"]
    x, z = xz[..., :C], xz[..., C:]
    dxz = torch.zeros_like(xz)
    steps = []
    for r in (False, True):
        u = torch.empty(B, L, C, device="cuda", dtype=xz.dtype)
        vig.vig_causal_conv(x, d["conv"], d["conv_b"], u, reverse=r)
        rows = u @ d["w_x"]
        dt = rows[..., :4] @ d["w_dt"]
        Bt, Ct = (rows[..., 4 + i * G * n:4 + (i + 1) * G * n].unflatten(2, (G, n)) for i in range(2))
        out = torch.empty_like(u)
        vig.vig_ssm_fwd(u, dt, d["A"], Bt, Ct, out, D=d["D"], z=z, dt_bias=d["dt_bias"], reverse=r)
        du, ddt, dA = torch.empty_like(u), torch.empty_like(u), torch.empty_like(d["A"])
        drows = torch.zeros_like(rows)
        dB, dC = (drows[..., 4 + i * G * n:4 + (i + 1) * G * n].unflatten(2, (G, n)) for i in range(2))
        dz = torch.empty_like(u)
        vig.vig_ssm_bwd(u, dt, d["A"], Bt, Ct, d["d_out"], du, ddt, dA, dB, dC, D=d["D"], z=z, dt_bias=d["dt_bias"], dz=dz, reverse=r)
        du2 = du + ddt @ d["w_dt"].t() @ d["w_x"][:, :4].t() + drows[..., 4:] @ d["w_x"][:, 4:].t()
        dx, dw, db = torch.empty_like(u), torch.empty_like(d["conv"]), torch.empty_like(d["conv_b"])
        vig.vig_causal_conv_bwd(x, d["conv"], d["conv_b"], du2, dx, dw, db, reverse=r)
        dxz[..., :C] += dx
        dxz[..., C:] += dz
        steps.append(dict(u=u, dt=dt, Bt=Bt, Ct=Ct, out=out, du=du, ddt=ddt, dA=dA, dB=dB, dC=dC, dz=dz, du2=du2, dx=dx, dw=dw, db=db))
    dy = dxz @ d["w_in"].t()
    d_in, d_norm = torch.empty_like(s), torch.empty_like(d["norm"])
    vig.vig_rms_norm_bwd(s, d["norm"], rstd, dy, d_in, d_norm, d_sum=d["residual"])
    torch.cuda.synchronize()
    tol = 2.0 ** -7 if dtype == "bf16" else 2e-4
    out, total, r64 = oracle.rms_norm(f64(d["x"]), f64(d["norm"]), f64(d["residual"]))
    assert off(y, out) <= tol and off(s, total) <= tol and off(rstd, r64) <= tol
    for p, r in zip(steps, (False, True)):
        assert off(p["u"], oracle.causal_conv(f64(x), f64(d["conv"]), f64(d["conv_b"]), "silu", None, r)[0]) <= tol
        a = [f64(p["u"]), f64(p["dt"]), f64(d["A"]), f64(p["Bt"]), f64(p["Ct"])]
        assert off(p["out"], oracle.ssm_fwd(*a, f64(d["D"]), f64(z), f64(d["dt_bias"]), reverse=r)[0]) <= tol
        g = oracle.ssm_bwd(*a, f64(d["d_out"]), f64(d["D"]), f64(z), f64(d["dt_bias"]), reverse=r)
        for name, ref in (("du", "dx"), ("ddt", "ddt"), ("dA", "dA"), ("dB", "dB"), ("dC", "dC"), ("dz", "dz")):
            assert off(p[name], g[ref]) <= tol, name
        dx, dw, db, _ = oracle.causal_conv_bwd(f64(x), f64(d["conv"]), f64(d["conv_b"]), f64(p["du2"]), "silu", None, None, r)
        for name, ref in (("dx", dx), ("dw", dw), ("db", db)):
            assert off(p[name], ref) <= tol, name
    dx, dw = oracle.rms_norm_bwd(f64(s), f64(d["norm"]), f64(rstd), f64(dy), f64(d["residual"]))
    assert off(d_in, dx) <= tol and off(d_norm, dw) <= tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_behind_a_prefix_captured(dtype):
    """A prefix by whole sequences, then one captured step (norm, convolution, scan) replayed for every further token: bit for bit the
    convolution and norm of the whole sequence, and its scan within the roundings."""
    d, (B, L, C, n, G) = _layer(dtype)
    P = 60
    u_all = torch.empty(B, L, C, device="cuda", dtype=T[dtype])
    x = (d["x"] @ d["w_in"])[..., :C].contiguous()
    vig.vig_causal_conv(x, d["conv"], d["conv_b"], u_all)
    rows = u_all @ d["w_x"]
    dt = (rows[..., :4] @ d["w_dt"]).contiguous()
    Bt, Ct = (rows[..., 4 + i * n:4 + (i + 1) * n].unflatten(2, (1, n)).contiguous() for i in range(2))
    whole, last = torch.empty_like(u_all), torch.empty(B, C, n, device="cuda")
    vig.vig_ssm_fwd(u_all, dt, d["A"], Bt, Ct, whole, D=d["D"], dt_bias=d["dt_bias"], state_out=last)
    window, state = torch.empty(B, 3, C, device="cuda", dtype=T[dtype]), torch.empty_like(last)
    first = lambda t: t[:, :P].contiguous()
    vig.vig_causal_conv(first(x), d["conv"], d["conv_b"], torch.empty_like(first(x)), state_out=window)
    vig.vig_ssm_fwd(first(u_all), first(dt), d["A"], first(Bt), first(Ct), torch.empty_like(first(x)), D=d["D"], dt_bias=d["dt_bias"], state_out=state)
    one = {"x": x[:, 0].clone(), "dt": dt[:, 0].clone(), "Bt": Bt[:, 0].clone(), "Ct": Ct[:, 0].clone()}
    u, out = torch.empty_like(one["x"]), torch.empty_like(one["x"])
    kept = window.clone(), state.clone()

    def step():
        vig.vig_causal_conv_step(one["x"], d["conv"], d["conv_b"], window, u)
        vig.vig_ssm_step(u, one["dt"], d["A"], one["Bt"], one["Ct"], state, out, D=d["D"], dt_bias=d["dt_bias"])

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    window.copy_(kept[0])
    state.copy_(kept[1])
    for t in range(P, L):
        for name, src in (("x", x), ("dt", dt), ("Bt", Bt), ("Ct", Ct)):
            one[name].copy_(src[:, t])
        graph.replay()
        assert torch.equal(u, u_all[:, t])
        assert off(out, f64(whole[:, t])) <= (2.0 ** -7 if dtype == "bf16" else 1e-4)
    assert off(state, f64(last)) <= 1e-4
