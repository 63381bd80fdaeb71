"""Gradient of the selective scan over sequences too long to keep their states whole, on the GPU."""
import pytest
import torch

import paper_2405_18425_b200 as vig

pytestmark = pytest.mark.gpu


def _gradient(d):
    g = {"d" + n: torch.full_like(d[n], float("nan")) for n in ("x", "dt", "A", "Bt", "Ct", "D", "z", "dt_bias", "state")}
    vig.vig_ssm_bwd(*(d[n] for n in ("x", "dt", "A", "Bt", "Ct", "d_out")), *(g["d" + n] for n in ("x", "dt", "A", "Bt", "Ct")), D=d["D"], z=d["z"],
                    dt_bias=d["dt_bias"], dD=g["dD"], dz=g["dz"], d_dt_bias=g["ddt_bias"], state_in=d["state"], d_state_out=d["d_state"],
                    d_state_in=g["dstate"])
    return g


@pytest.mark.parametrize("L", [28336, 28400])
def test_channels_are_those_of_a_call_of_their_own(L):
    """296 blocks of 64 channels, a sequence that is kept whole and one that is cut; the first and last channels by themselves are cut into many
    segments.  Both are as far from the definition as half a step of bf16 (2^-8) and the fp32 sums' 2^-13 (64 decays of 2^-22, cancelling to
    a quarter), those over all tokens another 4 2^-24 sqrt(L)."""
    C, N = 64 * 296, 32
    gen = torch.Generator(device="cuda").manual_seed(6)
    half = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.bfloat16)
    full = lambda *s: torch.randn(s, generator=gen, device="cuda")
    d = {n: half(1, L, C) for n in ("x", "z", "d_out")}
    d.update(dt=half(1, L, C) * 0.7, Bt=half(1, L, 1, N), Ct=half(1, L, 1, N), A=-(0.5 + full(C, N).abs() * 2), D=full(C), dt_bias=full(C) * 0.7 - 1,
             state=full(1, C, N), d_state=full(1, C, N))
    got = _gradient(d)
    for part in (slice(0, 64), slice(C - 64, C)):
        cut = lambda n, t: t if n in ("Bt", "Ct") else t[part].contiguous() if n in ("A", "D", "dt_bias") else t[:, part].contiguous() if "state" in n else \
            t[..., part].contiguous()
        alone = _gradient({n: cut(n, t) for n, t in d.items()})
        for n in ("x", "dt", "z", "A", "D", "dt_bias", "state"):
            a, b = cut(n, got["d" + n]).double(), alone["d" + n].double()
            tol = 2 * ((2.0 ** -8 if n in ("x", "dt", "z") else 0) + 2.0 ** -13 + (4 * 2.0 ** -24 * L ** 0.5 if n in ("A", "D", "dt_bias") else 0))
            off = float((a - b).norm() / b.norm())
            print(n, off, tol)
            assert torch.isfinite(a).all() and off <= tol, n
    assert torch.isfinite(got["dBt"]).all() and torch.isfinite(got["dCt"]).all()
