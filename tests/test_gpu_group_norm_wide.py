"""Group norm of images that do not stay on chip in groups of many channels: thousands of partial sums a group."""
import pytest
import torch

from test_gpu_group_norm import _check, _inputs, _run

pytestmark = pytest.mark.gpu

# B, Hh, Ww, C, groups: around the number of partial sums that a warp takes, and up to 300000
SIZES = [(1, 56, 56, 768, 1), (2, 31, 33, 2304, 1), (8, 56, 56, 256, 1), (1, 112, 112, 96, 1), (2, 80, 80, 320, 4), (1, 170, 230, 24, 3), (3, 130, 190, 16, 1), (1, 120, 130, 1032, 3)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_gradient(size, dtype):
    *shape, groups = size
    x, w, b, do = _inputs(*shape, dtype, seed=81)
    _check(_run(x, w, b, do, groups, "silu"), x, w, b, do, groups, "silu")


@pytest.mark.parametrize("size", SIZES[:3], ids=str)
def test_channels_of_different_means(size):
    """Channels' means of up to a hundred, the first one's a thousand: squares are taken about the group's own mean."""
    *shape, groups = size
    x, w, b, do = _inputs(*shape, "f32", seed=82)
    x += torch.randn(shape[3], generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 30
    x[..., 0] += 1000
    _check(_run(x, w, b, do, groups, "none"), x, w, b, do, groups, "none", spread=float(x.double().mean().abs() / x.double().std()) + 1)
