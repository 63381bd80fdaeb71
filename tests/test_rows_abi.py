"""Refusals of the selective scan, the causal convolution and the RMS norm, on the host (no kernel is launched, no GPU is needed)."""
import ctypes

import pytest
import torch

import paper_2405_18425_b200 as vig
from paper_2405_18425_b200 import build as vig_build

A = 0x10000  # fake, 16-byte aligned, never dereferenced: validation fails before any CUDA call
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    vig_build.build()
    return vig.load()


def _walk(f, ok, pointers, optional, aligned, refusals, unsupported):
    """aligned: by how many bytes each pointer has to be aligned, (pointer, offset that is refused)."""
    before = vig.vig_kernel_launch_count()
    for i in range(pointers):
        bad = list(ok)
        if i not in optional:
            bad[i] = None
            assert f(*bad) == -1, i
        bad[i] = A + aligned.get(i, 8)
        assert f(*bad) == -4, i
    for want, cases in ((-2, refusals), (-3, unsupported)):
        for change in cases:
            bad = list(ok)
            for at, value in change.items():
                bad[at] = value
            assert f(*bad) == want, change
    assert vig.vig_kernel_launch_count() == before


def _pitches(*v):
    return (ctypes.c_longlong * len(v))(*v)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_scan_arguments(lib, t):
    e = 2 if t == "bf16" else 4
    # x dt A Bt Ct D z dt_bias state_in out state_out | B L C G N ld softplus reverse stream
    ok = [A] * 11 + [2, 5, 64, 2, 16, None, 1, 0, None]
    f = getattr(lib, f"vig_ssm_fwd_{t}")
    sizes = [{11: -1}, {12: -1}, {13: 0}, {14: 0}, {15: 0}]
    most = [{15: 33}, {13: 60}, {13: 66}, {13: (1 << 20) + 32}, {12: MOST}, {12: MOST - 4000}, {11: 1 << 20, 12: 1 << 20}]
    half = {i: e // 2 for i in (3, 4)}
    words = {i: 2 for i in (2, 5, 7, 8, 10)}
    _walk(f, ok, 11, (5, 6, 7, 8, 10), {**half, **words}, sizes, most)
    dense = [64, 64, 64, 64, 32, 32]
    for i in range(6):
        ld = list(dense)
        ld[i] -= 16                                    # rows that overlap
        assert f(*ok[:16], _pitches(*ld), *ok[17:]) == -2, i
        ld[i] = 1 << 41
        assert f(*ok[:16], _pitches(*ld), *ok[17:]) == -2, i
    for i in range(4):
        ld = list(dense)
        ld[i] += 8 // e                                # rows that do not begin at 16 bytes
        assert f(*ok[:16], _pitches(*ld), *ok[17:]) == -4, i
    # x dt A Bt Ct D z dt_bias state_in d_out d_state_out dx ddt dA dB dC dD dz d_dt_bias d_state_in | ...
    ok = [A] * 20 + [2, 5, 64, 2, 16, None, 1, 0, None]
    f = getattr(lib, f"vig_ssm_bwd_{t}")
    up = lambda cases: [{at + 9: v for at, v in c.items()} for c in cases]
    half = {i: e // 2 for i in (3, 4, 14, 15)}
    words = {i: 2 for i in (2, 5, 7, 8, 10, 13, 16, 18, 19)}
    _walk(f, ok, 20, (5, 6, 7, 8, 10, 16, 17, 18, 19), {**half, **words}, up(sizes), up(most))
    bad = list(ok)
    bad[6] = None                                      # the gate's gradient without a gate
    assert f(*bad) == -1
    dense = [64, 64, 64, 64, 32, 32, 64, 64, 64, 32, 32]
    for i in range(11):
        ld = list(dense)
        ld[i] -= 16
        assert f(*ok[:25], _pitches(*ld), *ok[26:]) == -2, i
    # x dt A Bt Ct D z dt_bias state out | B C G N ld softplus stream
    ok = [A] * 10 + [2, 64, 2, 16, None, 1, None]
    own = {i: e // 2 for i in (0, 1, 3, 4, 6, 9)}
    _walk(getattr(lib, f"vig_ssm_step_{t}"), ok, 10, (5, 6, 7), {**own, 2: 2, 5: 2, 7: 2}, [{10: -1}, {11: 0}, {12: 0}, {13: 0}],
          [{13: 33}, {11: 63}, {11: (1 << 20) + 2}, {10: MOST, 11: 64}])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_convolution_arguments(lib, t):
    # x w bias state_in out state_out | B L C K ld act reverse stream
    ok = [A] * 6 + [2, 5, 64, 4, None, 1, 0, None]
    sizes = [{6: -1}, {7: -1}, {8: 0}, {9: 0}]
    most = [{9: 1}, {9: 5}, {8: 66}, {8: (1 << 20) + 8}, {11: 2}, {11: -1}, {7: MOST}, {6: 1 << 20, 7: 1 << 20}]
    _walk(getattr(lib, f"vig_causal_conv_{t}"), ok, 6, (2, 3, 5), {}, sizes, most)
    assert getattr(lib, f"vig_causal_conv_{t}")(*ok[:10], _pitches(56, 64), *ok[11:]) == -2
    assert getattr(lib, f"vig_causal_conv_{t}")(*ok[:10], _pitches(64, 66), *ok[11:]) == -4
    ok = [A] * 10 + [2, 5, 64, 4, None, 1, 0, None]
    up = lambda cases: [{at + 4: v for at, v in c.items()} for c in cases]
    _walk(getattr(lib, f"vig_causal_conv_bwd_{t}"), ok, 10, (2, 3, 5, 7, 8, 9), {}, up(sizes), up(most))
    ok = [A] * 5 + [2, 64, 4, None, 1, None]
    _walk(getattr(lib, f"vig_causal_conv_step_{t}"), ok, 5, (2,), {}, [{5: -1}, {6: 0}, {7: 0}], [{7: 1}, {7: 5}, {6: 66}, {9: 2}])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_norm_arguments(lib, t):
    nan, inf = float("nan"), float("inf")
    # x residual weight out sum_out rstd | rows C eps stream
    ok = [A] * 6 + [3, 64, 1e-5, None]
    _walk(getattr(lib, f"vig_rms_norm_{t}"), ok, 6, (1, 4, 5), {5: 2}, [{6: -1}, {7: 0}, {8: -1e-5}, {8: nan}, {8: inf}], [{7: 66}, {7: 16392}, {6: 1 << 31}])
    # x residual weight out scales sum_out | rows C block eps stream
    ok = [A] * 6 + [3, 64, 128, 1e-5, None]
    _walk(getattr(lib, f"vig_rms_norm_e4m3_{t}"), ok, 6, (1, 5), {3: 4, 4: 2}, [{6: -1}, {7: 0}, {9: nan}], [{7: 66}, {7: 16392}, {8: 64}, {8: -1}])
    ok = [A] * 7 + [3, 64, None]
    _walk(getattr(lib, f"vig_rms_norm_bwd_{t}"), ok, 7, (4, 6), {2: 2}, [{7: -1}, {8: 0}], [{8: 66}, {8: 16392}, {7: 1 << 31}])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_empty_calls_launch_nothing(lib, t):
    before = vig.vig_kernel_launch_count()
    assert getattr(lib, f"vig_ssm_fwd_{t}")(*([A] * 11 + [0, 5, 64, 2, 16, None, 1, 0, None])) == 0
    assert getattr(lib, f"vig_ssm_fwd_{t}")(*([A] * 8 + [A, A, A] + [2, 0, 64, 2, 16, None, 1, 0, None])) == 0   # state_out is state_in
    assert getattr(lib, f"vig_ssm_step_{t}")(*([A] * 10 + [0, 64, 2, 16, None, 1, None])) == 0
    assert getattr(lib, f"vig_causal_conv_{t}")(*([A] * 6 + [0, 5, 64, 4, None, 1, 0, None])) == 0
    assert getattr(lib, f"vig_causal_conv_step_{t}")(*([A] * 5 + [0, 64, 4, None, 1, None])) == 0
    assert getattr(lib, f"vig_rms_norm_{t}")(*([A] * 6 + [0, 64, 1e-5, None])) == 0
    assert getattr(lib, f"vig_rms_norm_e4m3_{t}")(*([A] * 6 + [0, 64, 0, 1e-5, None])) == 0
    assert getattr(lib, f"vig_rms_norm_bwd_{t}")(*([A] * 6 + [None, 0, 64, None])) == 0
    assert vig.vig_kernel_launch_count() == before


def test_binding_refuses_host_tensors_and_wrong_arguments(lib):
    x, r, f = torch.zeros(1, 2, 16), torch.zeros(1, 2, 1, 4), torch.zeros(16, 4)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_ssm_fwd(x, x, f, r, r, x)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_ssm_bwd(x, x, f, r, r, x, x, x, f, r, r)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_ssm_step(x[0], x[0], f, r[0], r[0], x, x[0])
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_causal_conv(x, f, None, x)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_causal_conv_bwd(x, f, None, x, x, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_causal_conv_step(x[0], f, None, x, x[0])
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_rms_norm(x, x[0, 0], x)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_rms_norm_e4m3(x, x[0, 0], x, x)
    with pytest.raises(ValueError, match="CUDA"):
        vig.vig_rms_norm_bwd(x, x[0, 0], x[..., 0], x, x, None)
    with pytest.raises(ValueError, match="3 dimensions"):
        vig.vig_ssm_fwd(x[0], x, f, r, r, x)
    with pytest.raises(ValueError, match="4 dimensions"):
        vig.vig_ssm_fwd(x, x, f, r[0], r, x)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        vig.vig_rms_norm(x.half(), x, x)
    with pytest.raises(TypeError):
        vig.vig_causal_conv(x, None, None, x)
    with pytest.raises(ValueError, match="activation"):
        vig.vig_causal_conv(x, f, None, x, act="tanh")
