"""RMS norm in 8 bits on the GPU: every code the nearest one, the even one of two that are as near."""
import pytest
import torch

import paper_2405_18425_b200 as vig

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("residual", [False, True], ids=["alone", "residual"])
@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(12544, 768), (4000, 200), (600, 16384)], ids=str)
def test_codes(size, dtype, block, residual):
    """out / scale is s w over its largest value, times 448: 1 / sqrt(mean s^2 + eps) cancels.

    bf16: s w has 24 bits at most where s has sixteen (the sum of two numbers within a factor of 2^8), and the quotient is off by half a step, 2^-24: a
    code is the other neighbour only that near to a middle, and not at the middle itself.  Where s has more bits s w and the largest
    one are rounded: 3 2^-24, as in fp32 calls, whose quotient is a rounded reciprocal's product: 4 2^-24 with a sum's rounding in both, 6 2^-24."""
    rows, C = size
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, C, generator=gen, device="cuda").to(dtype)
    r = (2 * torch.randn(rows, C, generator=gen, device="cuda")).to(dtype) if residual else None
    w = (1 + 0.2 * torch.randn(C, generator=gen, device="cuda")).to(dtype)
    q = torch.empty(rows, C, device="cuda", dtype=torch.float8_e4m3fn)
    scales = torch.empty(rows, -(-C // 128) if block else 1, device="cuda")
    vig.vig_rms_norm_e4m3(x, w, q, scales, residual=r)
    n = scales.shape[1]
    width = 128 if n > 1 else C
    s = x.double() if r is None else x.double() + r.double()
    t = torch.nn.functional.pad(s * w.double(), (0, n * width - C)).view(rows, n, width)
    over = (t * 448 / t.abs().amax(-1, keepdim=True)).view(rows, -1)[:, :C]
    step = torch.exp2(torch.floor(torch.log2(over.abs().clamp(min=2.0 ** -6))) - 3)   # between the codes around a value
    place = over.abs() / step
    middle = (place - place.floor() - 0.5).abs() / place.clamp(min=2.0 ** -10)
    wrong = q.double() != torch.copysign(torch.round(place) * step, over)
    few = (s.float().view(torch.int32) & 0xff) == 0 if dtype == torch.bfloat16 else torch.zeros_like(wrong)
    print("middles:", int((middle == 0).sum()), "codes beside the nearest:", int(wrong.sum()))
    assert not (wrong & few & ((middle == 0) | (middle > 2.0 ** -24))).any()
    assert not (wrong & (middle > 6 * 2.0 ** -24)).any()
    if dtype == torch.bfloat16 and rows > 4000:
        assert (few & (middle == 0)).sum() > 10
