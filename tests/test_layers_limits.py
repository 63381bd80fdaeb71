"""Sizes at the end of 32 bits, on the host: counts of tokens and pixels whose next multiple of a tile no longer fits are refused (no kernel is launched)."""
import pytest

import paper_2405_18425_b200 as vig
from paper_2405_18425_b200 import build as vig_build

A = 0x10000  # fake, 16-byte aligned, never dereferenced: validation fails before any CUDA call
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    vig_build.build()
    return vig.load()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_tokens(lib, t):
    before = vig.vig_kernel_launch_count()
    for L in (MOST, MOST - 1, MOST - 62, MOST - 4000):
        assert getattr(lib, f"vig_gdr_fwd_{t}")(*([A] * 8 + [1, 1, L, 8, 8, 0, None])) == -3
        assert getattr(lib, f"vig_gdr_bwd_{t}")(*([A] * 14 + [1, 1, L, 8, 8, 0, None])) == -3
    assert vig.vig_kernel_launch_count() == before


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_pixels(lib, t):
    before = vig.vig_kernel_launch_count()
    for Hh, Ww in ((1, MOST), (MOST, 1), (1, MOST - 7), (1, MOST - 40000), (2, 2 ** 30 - 1)):
        assert getattr(lib, f"vig_group_norm_{t}")(*([A] * 6 + [1, Hh, Ww, 8, 1, 1e-5, 0, None])) == -3
        assert getattr(lib, f"vig_group_norm_bwd_{t}")(*([A] * 9 + [1, Hh, Ww, 8, 1, 0, None])) == -3
    assert vig.vig_kernel_launch_count() == before
