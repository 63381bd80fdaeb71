"""Group norm of values that are not finite, or too large to be squared."""
import pytest
import torch

import paper_2405_18425_b200 as vig
from layer_helpers import T

pytestmark = pytest.mark.gpu

SIZES = [(2, 6, 6, 32, 4), (2, 14, 14, 96, 8), (3, 30, 30, 48, 16), (1, 230, 230, 16, 2), (2, 13, 17, 256, 1)]


def _run(x, groups, act="silu"):
    out, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(x.shape[0], groups, device="cuda") for _ in range(2))
    vig.vig_group_norm(x, None, None, out, groups, act=act, mean=mean, rstd=rstd)
    vig.vig_group_norm_bwd(x, None, None, mean, rstd, torch.ones_like(x), dx, None, None, groups, act=act)
    return out, dx, mean, rstd


def _image(size, dtype, seed=71):
    *shape, groups = size
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(T[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_what_is_not_finite_stays_in_its_group(size, bad, dtype):
    """One value: its group's statistics and results are not a number, all others are what they were."""
    *shape, groups = size
    x, per = _image(size, dtype), size[3] // groups
    clean = _run(x, groups)
    for place in ((0, 0, 0, 0), (shape[0] - 1, shape[1] - 1, shape[2] - 1, shape[3] - 1), (0, shape[1] // 2, shape[2] // 3, shape[3] // 2)):
        y = x.clone()
        y[place] = bad
        got = _run(y, groups)
        b, g = place[0], place[3] // per
        hit = torch.zeros(shape[0], groups, dtype=torch.bool, device="cuda")
        hit[b, g] = True
        wide = hit.repeat_interleave(per, 1)[:, None, None].expand(shape)
        for i, (a, c) in enumerate(zip(got, clean)):
            where = wide if a.dim() == 4 else hit
            assert torch.equal(a[~where], c[~where]), (i, place)
            if i == 2 and abs(bad) == float("inf"):
                assert not torch.isfinite(a[where]).any()
            else:
                assert torch.isnan(a[where]).all(), (i, place)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e17, 3e18, 1e19, 3e19, 1e21, 1e30])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_values_too_large_to_be_squared_are_never_half_counted(size, scale, dtype):
    """Sums of squares beyond fp32: the results are right or not a number (or, with a variance of infinity, zero), never some of the variance."""
    groups = size[-1]
    x = (_image(size, dtype).float() * scale).to(T[dtype])
    out, _, _, rstd = _run(x, groups, act="none")
    y = x.double().reshape(x.shape[0], -1, groups, x.shape[3] // groups)
    var = y.var((1, 3), correction=0)
    want = var.rsqrt()
    right = (rstd.double() - want).abs() <= 1e-4 * want
    assert (right | torch.isnan(rstd) | (rstd == 0)).all(), (rstd.double() / want).tolist()
    if y[0, :, 0].numel() * scale ** 2 < 1e37:   # (n values of N(0, 1) times scale: the sum of squares, about a value of up to five, is below 26 n scale^2 < 3.4e38)
        assert right.all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [1e17, 1e18, 5e18, 1e19, 1e20])
def test_a_first_pixel_far_beyond_the_rest(value, dtype):
    """One value whose square is within fp32, all others are zero: its variance is right or not a number."""
    for size in SIZES + [(1, 64, 64, 192, 8), (40, 56, 56, 96, 32)]:
        *shape, groups = size
        x = torch.zeros(shape, device="cuda", dtype=T[dtype])
        x[:, 0, 0] = value
        rstd = _run(x, groups, act="none")[3]
        n = shape[1] * shape[2]
        want = (float(x[0, 0, 0, 0]) ** 2 * (1 / n - 1 / n ** 2)) ** -0.5
        right = (rstd.double() - want).abs() <= 1e-4 * want
        assert (right | torch.isnan(rstd) | (rstd == 0)).all(), (size, (rstd.double() / want).tolist())
        if n * shape[3] // groups * value ** 2 < 3e38:
            assert right.all(), size
