"""RMS norm of rows of small values on the GPU, with and without an eps beside them: results, 1 / sqrt(mean s^2 + eps), 8 bits, gradient."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import HALF, put

pytestmark = pytest.mark.gpu

SIZES = [1e-13, 1e-21, 2e-22, 1e-22, 1e-25, 1e-30, 1e-37]


def _rows(size, C, dtype, rows=3, seed=0):
    n = np.random.default_rng(seed).standard_normal
    x = n((rows, C))
    return put(x / np.abs(x).max(1, keepdims=True) * size, dtype), put(n(C) * 0.3 + 1, dtype), put(n((rows, C)), dtype)


def _close(t, ref, tol):
    """2-norm over 2-norm; what lies below the type's normal numbers is off by half of its smallest step, 2^-149 or 2^-133, at most."""
    a = f64(t)
    least = {torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[t.dtype]
    tol += HALF[t.dtype] if t.dtype == torch.bfloat16 else 0.0
    err = np.linalg.norm(a - ref)
    assert np.isfinite(a).all() and err <= tol * np.linalg.norm(ref) + least * ref.size ** 0.5, (err / np.linalg.norm(ref), tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [64, 2048, 16384])
@pytest.mark.parametrize("eps", [1e-5, 1e-20, 1e-30, 1e-42, 0.0])
@pytest.mark.parametrize("size", SIZES)
def test_result_and_gradient(size, eps, C, dtype):
    """Rounding as beside ordinary rows (sixteen half steps for rstd, as many for out; dx four times that, dweight the root of three rows more).
    eps is what fp32 holds of it."""
    x, w, g = _rows(size, C, dtype)
    out, rstd, dx, dw = torch.empty_like(x), torch.full((3,), float("nan"), device="cuda"), torch.empty_like(x), torch.empty_like(w)
    vig.vig_rms_norm(x, w, out, rstd=rstd, eps=eps)
    want, s, r = oracle.rms_norm(f64(x), f64(w), None, float(np.float32(eps)))
    tol = 16 * 2.0 ** -24
    assert np.abs(f64(rstd) / r - 1).max() <= tol, (f64(rstd), r)
    _close(out, want, 2 * tol)
    vig.vig_rms_norm_bwd(x, w, rstd, g, dx, dw)
    d, dwant = oracle.rms_norm_bwd(s, f64(w), r, f64(g))
    if np.abs(d).max() < 3e38:
        _close(dx, d, 5 * tol)
    _close(dw, dwant, 4 * tol)


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES)
def test_eight_bits(size, dtype, block):
    """Codes over their whole range: half a step, 2^-4 of a value (2^-10 below 2^-6), and the value's own roundings."""
    x, w, _ = _rows(size, 768, dtype, seed=1)
    q, scales = torch.empty(3, 768, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(3, 6 if block else 1, device="cuda")
    vig.vig_rms_norm_e4m3(x, w, q, scales)
    out = oracle.rms_norm(f64(x), f64(w), None, float(np.float32(1e-5)))[0].reshape(3, scales.shape[1], -1)
    want = np.maximum(np.abs(out).max(-1) / 448, 2.0 ** -126)
    assert np.abs(f64(scales) / want - 1).max() <= 16 * 2.0 ** -24
    over = out / want[..., None]
    off = np.abs(f64(q.float()).reshape(out.shape) - over)
    assert (off <= np.maximum(np.abs(over) * 2.0 ** -4, 2.0 ** -10) + 448 * 2.0 ** -20).all()


def test_zeros_and_small_values_meet():
    """Rows of ever smaller values come ever nearer to a row of zeros: rstd is 1 / sqrt(eps) for all of them."""
    x = torch.zeros(6, 64, device="cuda")
    for i, size in enumerate((0.0, 1e-45, 1e-38, 1e-30, 1e-25, 1e-20)):
        x[i] = size
    w, out, rstd = torch.ones(64, device="cuda"), torch.empty_like(x), torch.empty(6, device="cuda")
    vig.vig_rms_norm(x, w, out, rstd=rstd)
    assert (rstd == rstd[0]).all() and torch.equal(out, x * rstd[0])
