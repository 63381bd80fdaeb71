"""Scratch of the selective scan's gradient: bounded by its own outputs and a constant, whatever the length (no GPU)."""
import ctypes

import pytest

import paper_2405_18425_b200 as vig
from paper_2405_18425_b200 import build as vig_build


@pytest.fixture(scope="module")
def scratch():
    vig_build.build()
    f = vig.load().vig_test_ssm_bwd_scratch
    f.argtypes, f.restype = [ctypes.c_int] * 5, ctypes.c_size_t
    return f


def _padded(N):
    return 8 if N <= 8 else 16 if N <= 16 else 32


@pytest.mark.parametrize("N", [1, 8, 16, 32])
@pytest.mark.parametrize("B,C,G", [(1, 64, 1), (1, 8192, 1), (1, 37888, 1), (8, 2432, 1), (32, 1152, 1), (64, 1152, 2), (512, 1152, 1)])
@pytest.mark.parametrize("L", [1, 17, 196, 4096, 16384, 30000, 65536, 300000, 1 << 20, 1 << 24])
def test_bounded(scratch, L, B, C, G, N):
    """Beside the sums over blocks of 64 channels (two padded rows a token and block) and what a segment of 64 tokens or more leaves (three
    padded rows and three values a channel), 16 GiB of kept states, and what rounding segments to sixteen tokens adds."""
    P = _padded(N)
    blocks = G * -(-C // G // 64)
    sums = blocks * B * L * 2 * P * 4
    segments = B * C * (3 * P + 3) * 4 * (L // 64 + 1)
    assert scratch(B, L, C, G, N) <= sums + segments + (16 << 30) * 1.01 + 2048


def test_usual_lengths_stay_whole(scratch):
    """Sequences that fill a round of blocks are not cut, so nothing is computed twice for them: states of every fourth token of 576 blocks."""
    for L in (196, 4096, 16384):
        kept = 576 * (-(-L // 16) * 4) * 64 * 16 * 4
        sums, each = 18 * 32 * L * 2 * 16 * 4, 32 * 1152 * (16 + 2) * 4
        assert kept + sums + each <= scratch(32, L, 1152, 1, 16) <= kept + sums + each + 2048
