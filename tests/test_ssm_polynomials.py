"""The polynomials of the selective scan's exponential and logarithm, as their source has them, keep the errors stated beside them (no GPU)."""
import pathlib
import re

import numpy as np

import paper_2405_18425_b200 as vig

SOURCE = pathlib.Path(vig.__file__).parent / "csrc" / "ssm.cuh"


def _coefficients(name):
    """Of the Horner steps "ffma2(x, .., both(c))" of a function, the highest power first, as fp32 holds them."""
    body = re.search(r"f32x2 " + name + r"\(.*?\n}\n", SOURCE.read_text(), re.S).group(0)
    steps = [line for line in body.splitlines() if re.search(r"\bp = ffma2\(", line)]
    c = [float(v) for line in steps for v in re.findall(r"both\((-?[\d.]+)f\)", line)]
    assert len(c) == len(steps) + 1 and all(float(np.float32(v)) == v for v in c)
    return c


def test_exponential():
    c = _coefficients("exp2_arithmetic")
    f = np.linspace(-0.5, 0.5, 200001)
    assert c[-1] == 1.0 and np.abs(np.polyval(c, f) / 2.0 ** f - 1).max() <= 2.0 ** -28


def test_logarithm():
    """The error is relative at small step sizes too: the constant is one."""
    c = _coefficients("softplus2")
    u = np.linspace(2.0 ** -20, 1, 200001)
    assert c[-1] == 1.0 and np.abs(np.polyval(c, u) * u / np.log1p(u) - 1).max() <= 2.0 ** -24.8
