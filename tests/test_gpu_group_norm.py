"""Channels-last group norm with an activation on the GPU against the fp64 oracle, and the layer that it belongs to."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import NAMES, T, f64, gdr_inputs, off

pytestmark = pytest.mark.gpu

# B, Hh, Ww, C, groups: one pixel, odd images, groups of 1, 3, 5 and all channels, blocks of a cluster with and without rows left for the
# last, images that stay on chip and images that do not
SIZES = [(1, 1, 1, 32, 2), (3, 7, 5, 96, 32), (2, 14, 14, 768, 32), (1, 64, 64, 192, 8), (2, 9, 11, 40, 8), (2, 56, 56, 96, 32), (1, 3, 3, 64, 64),
         (2, 13, 17, 256, 1), (1, 112, 112, 64, 16), (1, 160, 200, 48, 3), (2, 31, 33, 2304, 1), (300, 4, 4, 16, 2), (1, 1, 200, 8, 1), (1, 230, 230, 8, 2),
         (2, 3, 5, 2008, 2008), (1, 5, 5, 2008, 8), (2, 20, 20, 1048, 131), (1, 9, 9, 4096, 4096), (1, 6, 6, 2056, 8),
         (1, 192, 256, 8, 2), (1, 1, 49153, 8, 2), (1, 96, 256, 8, 2), (1, 1, 24577, 8, 2)]


def _inputs(B, Hh, Ww, C, dtype, seed, mean=0.3):
    n = np.random.default_rng(seed).standard_normal
    put = lambda a: torch.from_numpy(a).cuda().to(T[dtype])
    return put(n((B, Hh, Ww, C)) + mean), put(n(C) * 0.3 + 1), put(n(C) * 0.3), put(n((B, Hh, Ww, C)))


def _run(x, w, b, do, groups, act, eps=1e-5, stream=None):
    out, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((x.shape[0], groups), float("nan"), device="cuda") for _ in range(2))
    dw, db = (torch.full((x.shape[3],), float("nan"), device="cuda", dtype=x.dtype) for _ in range(2))
    vig.vig_group_norm(x, w, b, out, groups, eps, act, mean=mean, rstd=rstd, stream=stream)
    vig.vig_group_norm_bwd(x, w, b, mean, rstd, do, dx, dw, db, groups, act, stream=stream)
    return out, mean, rstd, dx, dw, db


def _check(got, x, w, b, do, groups, act, eps=1e-5, spread=1.0):
    """Bounds in 2-norm.  bf16: half a step, 2^-8.  fp32 values: a dozen roundings of 2^-24 each, and a mean whose own rounding is
    2^-24 of its size, `spread` standard deviations: 16 (1 + spread) 2^-24.  Sums over n values (the parameters' gradients): partial
    sums of either sign, 2^-24 sqrt(n) more at most, as their blocks are summed in runs."""
    out, mean, rstd = oracle.group_norm(f64(x), f64(w), f64(b), groups, eps, act)
    dx, dw, db = oracle.group_norm_bwd(f64(x), f64(w), f64(b), groups, eps, act, f64(do))
    n = x.shape[0] * x.shape[1] * x.shape[2]
    for name, t, ref in zip(("out", "mean", "rstd", "dx", "dweight", "dbias"), got, (out, mean, rstd, dx, dw, db)):
        tol = 16 * (1 + spread) * 2.0 ** -24 * (1 + (n ** 0.5 / 8 if name[:2] == "dw" or name[:2] == "db" else 0))
        if t.dtype == torch.bfloat16:
            tol += 2.0 ** -8
        err = off(t, ref)
        print(f"  {name}: {err:.2e} (at most {tol:.2e})")
        assert err <= tol, (name, err, tol)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_gradient(size, dtype, act):
    *shape, groups = size
    x, w, b, do = _inputs(*shape, dtype, seed=1)
    # groups of a few values: their gradient is what is left of terms that cancel
    few = shape[1] * shape[2] * shape[3] // groups
    _check(_run(x, w, b, do, groups, act), x, w, b, do, groups, act, spread=1.0 if few > 64 else 8.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 14, 14, 96, 8), (1, 230, 230, 16, 2)], ids=str)
def test_mean_far_from_zero_and_first_pixel_far_from_the_rest(size, dtype):
    *shape, groups = size
    x, w, b, do = _inputs(*shape, dtype, seed=2, mean=100.0)
    x[:, 0, 0] = -400
    std = float(x.double().std())
    _check(_run(x, w, b, do, groups, "silu"), x, w, b, do, groups, "silu", spread=100.0 / std + 4)


@pytest.mark.parametrize("size", [(2, 6, 6, 32, 4), (1, 230, 230, 8, 2)], ids=str)
def test_constant_images_and_large_values(size):
    """A group without variance: out = act(bias), and 1 / sqrt(eps) as the scale; values of 1e15."""
    *shape, groups = size
    x, w, b, do = _inputs(*shape, "f32", seed=3)
    out = torch.empty_like(x)
    vig.vig_group_norm(torch.full_like(x, 0.5), w, b, out, groups, act="silu")
    want = torch.nn.functional.silu(b.double())
    assert torch.allclose(out.double(), want.expand_as(out), rtol=1e-6, atol=1e-7)
    big = x * 1e15
    _check(_run(big, w, b, do, groups, "none")[:1], big, w, b, do, groups, "none")


def test_activations_far_out():
    """Pre-activations of +-1e4: silu and gelu are z or zero there, and so are their slopes."""
    x = torch.tensor([-1.0, 1.0], device="cuda").repeat(32).view(1, 4, 2, 8).contiguous()
    w = torch.full((8,), 1e4, device="cuda")
    for dtype in ("f32", "bf16"):
        for act in ("silu", "gelu"):
            y, ww = x.to(T[dtype]), w.to(T[dtype])
            out, mean, rstd, dx, dw, db = _run(y, ww, None, torch.ones_like(y), 1, act)
            assert torch.allclose(out.double(), (x * w).clamp(min=0).double(), rtol=1e-2 if dtype == "bf16" else 1e-5, atol=1e-6)
            assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
            assert torch.equal(db, torch.tensor([0.0, 8.0], device="cuda").repeat(4).to(T[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 14, 14, 96, 8), (1, 230, 230, 16, 2)], ids=str)
def test_parameters_left_out_and_in_place(size, dtype):
    *shape, groups = size
    x, w, b, do = _inputs(*shape, dtype, seed=4)
    ones, zeros = torch.ones_like(w), torch.zeros_like(b)
    want = _run(x, ones, zeros, do, groups, "gelu")
    y, dy = x.clone(), do.clone()
    mean, rstd = (torch.empty(x.shape[0], groups, device="cuda") for _ in range(2))
    out = torch.empty_like(x)
    vig.vig_group_norm(x, None, None, out, groups, act="gelu")
    assert torch.equal(out, want[0])
    vig.vig_group_norm(x, None, None, out, groups, act="gelu", mean=mean, rstd=rstd)
    assert torch.equal(out, want[0]) and torch.equal(mean, want[1]) and torch.equal(rstd, want[2])
    vig.vig_group_norm(y, None, None, y, groups, act="gelu")
    assert torch.equal(y, want[0])
    vig.vig_group_norm_bwd(x, None, None, mean, rstd, dy, dy, None, None, groups, act="gelu")
    assert torch.equal(dy, want[3])
    dw = torch.empty_like(w)
    vig.vig_group_norm_bwd(x, None, None, mean, rstd, do, out, dw, None, groups, act="gelu")
    assert torch.equal(dw, want[4])


def test_empty_gradient_clears_the_parameters():
    w = torch.full((16,), 3.0, device="cuda")
    x, s = torch.empty(0, 4, 4, 16, device="cuda"), torch.empty(0, 2, device="cuda")
    vig.vig_group_norm(x, w, w, x, 2)
    dw, db = w.clone(), w.clone()
    vig.vig_group_norm_bwd(x, w, w, s, s, x, x, dw, db, 2)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("size", [(2, 14, 14, 96, 8), (1, 230, 230, 16, 2), (1, 64, 64, 192, 8)], ids=str)
def test_stream_graphs_bits_and_edges(size):
    *shape, groups = size
    x, w, b, do = _inputs(*shape, "bf16", seed=5)
    want = _run(x, w, b, do, groups, "silu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _run(x, w, b, do, groups, "silu", stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graphs, res = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            res.append(_run(x, w, b, do, groups, "silu"))
    for _ in range(2):
        for g in graphs:
            g.replay()
        eager = _run(x, w, b, do, groups, "silu")
        torch.cuda.synchronize()
        for r in res + [eager]:
            assert all(torch.equal(p, q) for p, q in zip(r, want))
    buf = torch.full((x.numel() + 512,), 7.0, device="cuda", dtype=x.dtype)
    out = buf[256:256 + x.numel()].view(x.shape)
    vig.vig_group_norm(x, w, b, out, groups, act="silu")
    assert torch.equal(out, want[0]) and (buf[:256] == 7).all() and (buf[256 + x.numel():] == 7).all()


def test_binding_refusals_on_the_gpu():
    x, w, b, do = _inputs(2, 4, 4, 32, "bf16", seed=6)
    out, s = torch.empty_like(x), torch.empty(2, 4, device="cuda")
    for bad in (dict(x=x[:, :, ::2]), dict(out=out.float()), dict(weight=w.float()), dict(bias=b[:8].contiguous())):
        a = {**dict(x=x, weight=w, bias=b, out=out), **bad}
        with pytest.raises(ValueError):
            vig.vig_group_norm(a["x"], a["weight"], a["bias"], a["out"], 4)
    with pytest.raises(ValueError):
        vig.vig_group_norm(x, w, b, out, 8, mean=s)   # another number of groups
    with pytest.raises(vig.VigError) as e:
        vig.vig_group_norm(x, w, b, out, 5)
    assert e.value.status == -3
    with pytest.raises(vig.VigError) as e:
        vig.vig_group_norm(x, w, b, out, 0)
    assert e.value.status == -2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_of_convolution_norm_and_mixer(dtype):
    """image -> depth-wise convolution -> group norm + SiLU -> delta rule over the patch sequence in both directions, averaged; then the
    way back through mixer and norm: every call on the outputs of the one before, nothing waited for in between, against the oracles
    run on the stored tensors that entered each call."""
    B, Hh, Ww, C, H = 2, 10, 13, 96, 2
    L, dv, dk = Hh * Ww, C // H, 24
    rng = np.random.default_rng(7)
    put = lambda a: torch.from_numpy(a).cuda().to(T[dtype])
    x, cw, cb = put(rng.standard_normal((B, Hh, Ww, C))), put(rng.standard_normal((C, 3, 3)) * 0.3), put(rng.standard_normal(C))
    w, b = put(rng.standard_normal(C) * 0.2 + 1), put(rng.standard_normal(C) * 0.2)
    d = gdr_inputs(B, H, L, dk, dv, dtype, seed=8)
    conv, y = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(B, 8, device="cuda") for _ in range(2))
    vig.vig_dwconv3x3(x, cw, cb, conv)
    vig.vig_group_norm(conv, w, b, y, 8, act="silu", mean=mean, rstd=rstd)
    v = y.view(B, L, H, dv).transpose(1, 2).contiguous()
    args = [d["q"], d["k"], v, d["log_alpha"], d["beta"]]
    outs = [torch.empty_like(v) for _ in range(2)]
    for r in range(2):
        vig.vig_gdr_fwd(*args, outs[r], reverse=bool(r))
    out = (outs[0].float() + outs[1].float()) / 2
    grads = [[torch.empty_like(a) for a in args] for _ in range(2)]
    for r in range(2):
        vig.vig_gdr_bwd(*args, d["d_out"], *grads[r], reverse=bool(r))
    dy = ((grads[0][2].float() + grads[1][2].float()) / 2).to(T[dtype]).transpose(1, 2).contiguous().view(B, Hh, Ww, C)
    dconv, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    vig.vig_group_norm_bwd(conv, w, b, mean, rstd, dy, dconv, dw, db, 8, act="silu")
    torch.cuda.synchronize()
    tol = 2.0 ** -7 if dtype == "bf16" else 2e-5
    assert off(conv, oracle.dwconv3x3(f64(x), f64(cw), f64(cb))) <= tol
    assert off(y, oracle.group_norm(f64(conv), f64(w), f64(b), 8, 1e-5, "silu")[0]) <= tol
    a64 = [f64(a) for a in args]
    both = [oracle.gdr_fwd(*a64, None, bool(r))[0] for r in range(2)]
    assert off(out, (both[0] + both[1]) / 2) <= tol
    for r in range(2):
        for g, ref in zip(grads[r], oracle.gdr_bwd(*a64, f64(d["d_out"]), None, None, bool(r))):
            assert off(g, ref) <= tol
    for g, ref in zip((dconv, dw, db), oracle.group_norm_bwd(f64(conv), f64(w), f64(b), 8, 1e-5, "silu", f64(dy))):
        assert off(g, ref) <= tol
