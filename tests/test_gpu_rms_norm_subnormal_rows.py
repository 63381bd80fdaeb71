"""RMS norm without an eps of rows whose largest value is subnormal, on the GPU: their rstd leaves the range of fp32, their result does not."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import HALF, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [64, 2048, 16384])
@pytest.mark.parametrize("size", [1e-38, 1e-39, 3e-40])
def test_result(size, C, dtype):
    """As stored they are exact, so the result is off by its own roundings only: 32 half steps, and half a step of the type."""
    n = np.random.default_rng(2).standard_normal
    x = n((3, C))
    x[:, 0] = 8.0
    x, w = put(x / 8 * size, dtype), put(n(C) * 0.3 + 1, dtype)
    assert (f64(x)[:, 0] > 0.9 * size).all()
    out, rstd = torch.empty_like(x), torch.empty(3, device="cuda")
    vig.vig_rms_norm(x, w, out, rstd=rstd, eps=0.0)
    want, _, r = oracle.rms_norm(f64(x), f64(w), None, 0.0)
    tol = 32 * 2.0 ** -24 + (HALF[x.dtype] if dtype == "bf16" else 0.0)
    assert np.linalg.norm(f64(out) - want) <= tol * np.linalg.norm(want)
    top = float(np.finfo(np.float32).max)
    got = f64(rstd)
    assert (np.abs(got / r - 1) <= 16 * 2.0 ** -24)[r < top * (1 - 2.0 ** -16)].all() and np.isinf(got[r > top * (1 + 2.0 ** -16)]).all()
    q, scales = torch.empty(3, C, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(3, 1, device="cuda")
    vig.vig_rms_norm_e4m3(x, w, q, scales, eps=0.0)
    scale = np.abs(want).max(1, keepdims=True) / 448
    assert np.abs(f64(scales) / scale - 1).max() <= 32 * 2.0 ** -24
    off = np.abs(f64(q.float()) - want / scale)
    assert (off <= np.maximum(np.abs(want / scale) * 2.0 ** -4, 2.0 ** -10) + 448 * 2.0 ** -20).all()
