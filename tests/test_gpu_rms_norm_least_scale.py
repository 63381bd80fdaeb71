"""RMS norm in 8 bits on the GPU where the scale is the smallest normal number, not max / 448: codes are out over that."""
import numpy as np
import pytest
import torch

import oracle
import paper_2405_18425_b200 as vig
from layer_helpers import f64
from row_helpers import put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -124, 2.0 ** -122, 2.0 ** -119, 2.0 ** -117])
def test_codes(size, dtype, block):
    """Weights of `size`, as many above it as below.  A code is off by half a step, 2^-4 of its value (2^-10 below 2^-6), and the value's own
    roundings, 2^-20 of the largest code."""
    n = np.random.default_rng(7).standard_normal
    x, w = put(n((5, 768)), dtype), put(2.0 ** n(768) * size, dtype)
    q, scales = torch.empty(5, 768, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(5, 6 if block else 1, device="cuda")
    vig.vig_rms_norm_e4m3(x, w, q, scales)
    out = oracle.rms_norm(f64(x), f64(w), None, float(np.float32(1e-5)))[0].reshape(5, scales.shape[1], -1)
    scale = np.maximum(np.abs(out).max(-1) / 448, 2.0 ** -126)
    assert (scale == 2.0 ** -126).any() or size > 2.0 ** -120
    assert np.abs(f64(scales) / scale - 1).max() <= 2.0 ** -20
    over = out / scale[..., None]
    off = np.abs(f64(q.float()).reshape(out.shape) - over)
    assert (off <= np.maximum(np.abs(over) * 2.0 ** -4, 2.0 ** -10) + 448 * 2.0 ** -20).all()
