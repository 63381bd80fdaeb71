"""Refusals of the gated delta rule and the group norm, on the host (no kernel is launched, no GPU is needed)."""
import os

import pytest
import torch

import paper_2405_18425_b200 as vig
from paper_2405_18425_b200 import build as vig_build

A = 0x10000  # fake, 16-byte aligned, never dereferenced: validation fails before any CUDA call


@pytest.fixture(scope="module")
def lib():
    vig_build.build()
    return vig.load()


def _walk(f, ok, pointers, optional, refusals, unsupported=()):
    before = vig.vig_kernel_launch_count()
    for i in range(pointers):
        bad = list(ok)
        if i not in optional:
            bad[i] = None
            assert f(*bad) == -1, i
        bad[i] = A + 8
        assert f(*bad) == -4, i
    for at, value in refusals:
        bad = list(ok)
        bad[at] = value
        assert f(*bad) == -2, (at, value)
    for change in unsupported:
        bad = list(ok)
        for at, value in change.items():
            bad[at] = value
        assert f(*bad) == -3, change
    assert vig.vig_kernel_launch_count() == before


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_delta_rule_arguments(lib, t):
    ok = [A] * 8 + [2, 3, 5, 16, 32, 0, None]
    _walk(getattr(lib, f"vig_gdr_fwd_{t}"), ok, 8, (5, 7), [(8, -1), (9, -1), (10, -1), (11, 0), (12, 0)],
          [{11: 129}, {12: 257}, {8: 1 << 16, 9: 1 << 15, 10: 1}, {8: 1 << 20, 9: 64, 10: 4096}])
    ok = [A] * 14 + [2, 3, 5, 16, 32, 0, None]
    _walk(getattr(lib, f"vig_gdr_bwd_{t}"), ok, 14, (5, 7, 13), [(14, -1), (15, -1), (16, -1), (17, 0), (18, 0)], [{17: 129}, {18: 257}])
    ok = [A] * 7 + [2, 3, 16, 32, None]
    _walk(getattr(lib, f"vig_gdr_step_{t}"), ok, 7, (), [(7, -1), (8, -1), (9, 0), (10, 0)], [{9: 129}, {10: 257}])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_group_norm_arguments(lib, t):
    ok = [A] * 6 + [2, 4, 4, 32, 8, 1e-5, 1, None]
    _walk(getattr(lib, f"vig_group_norm_{t}"), ok, 6, (1, 2, 4, 5), [(6, -1), (7, -1), (8, -1), (9, 0), (10, 0), (11, -1e-5), (11, float("nan")), (11, float("inf"))],
          [{9: 34}, {10: 7}, {10: 64}, {9: (1 << 20) + 8, 10: 1}, {12: 3}, {12: -1}, {7: 1 << 16, 8: 1 << 15}])
    ok = [A] * 9 + [2, 4, 4, 32, 8, 1, None]
    _walk(getattr(lib, f"vig_group_norm_bwd_{t}"), ok, 9, (1, 2, 7, 8), [(9, -1), (10, -1), (11, -1), (12, 0), (13, 0)],
          [{12: 34}, {13: 7}, {14: 3}, {10: 1 << 16, 11: 1 << 15}])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_empty_calls_launch_nothing(lib, t):
    before = vig.vig_kernel_launch_count()
    for at in (8, 9):
        args = [A] * 8 + [2, 3, 5, 16, 32, 0, None]
        args[at] = 0
        assert getattr(lib, f"vig_gdr_fwd_{t}")(*args) == 0
    args = [A] * 7 + [A] + [2, 3, 0, 16, 32, 0, None]   # no tokens, state_out given and the same as state_in
    assert getattr(lib, f"vig_gdr_fwd_{t}")(*(args[:5] + [A, A, A] + args[8:])) == 0
    for at in (14, 15):
        args = [A] * 14 + [2, 3, 5, 16, 32, 0, None]
        args[at] = 0
        assert getattr(lib, f"vig_gdr_bwd_{t}")(*args) == 0
    assert getattr(lib, f"vig_gdr_step_{t}")(*([A] * 7 + [0, 3, 16, 32, None])) == 0
    assert getattr(lib, f"vig_group_norm_{t}")(*([A] * 6 + [2, 0, 4, 32, 8, 1e-5, 1, None])) == 0
    assert getattr(lib, f"vig_group_norm_bwd_{t}")(*([A] * 7 + [None, None] + [0, 4, 4, 32, 8, 1, None])) == 0
    assert vig.vig_kernel_launch_count() == before


def test_binding_refuses_host_tensors_and_wrong_arguments(lib):
    x = torch.zeros(1, 2, 3, 16)
    g = torch.zeros(1, 2, 3)
    with pytest.raises(ValueError, match="contiguous CUDA"):
        vig.vig_gdr_fwd(x, x, x, g, g, x)
    with pytest.raises(ValueError, match="contiguous CUDA"):
        vig.vig_gdr_bwd(x, x, x, g, g, x, x, x, x, g, g)
    with pytest.raises(ValueError, match="contiguous CUDA"):
        vig.vig_gdr_step(x[0], x[0], x[0], g[0], g[0], x, x[0])
    with pytest.raises(ValueError, match="contiguous CUDA"):
        vig.vig_group_norm(x, None, None, x, 2)
    with pytest.raises(ValueError, match="contiguous CUDA"):
        vig.vig_group_norm_bwd(x, None, None, x, x, x, x, None, None, 2)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        vig.vig_gdr_fwd(x.half(), x, x, g, g, x)
    with pytest.raises(ValueError, match="4 dimensions"):
        vig.vig_gdr_fwd(x[0], x, x, g, g, x)
    with pytest.raises(TypeError):
        vig.vig_gdr_fwd(None, x, x, g, g, x)
    with pytest.raises(ValueError, match="activation"):
        vig.vig_group_norm(x, None, None, x, 2, act="tanh")
