"""Rotations at the farthest positions, against angles that are reduced in exact arithmetic.

Tolerance per element as in the other tests of the rows: a rounding to fp32 of the value and 8 roundings to 32 bits, 4.8e-7, of
|a| + |b|. An angle near 2^31 whose products are rounded to 64 bits is off by up to 7e-7, twice that where a frequency is 2."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paged_util import i32

pytestmark = pytest.mark.gpu
TWO_PI = 2 * Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862089986280, 10**85)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("theta", [1e4, 0.5])
def test_far_positions(layout, theta):
    import paper_2604_17397_amd as P
    rng = np.random.default_rng(5)
    pos = np.concatenate([[-2**31, 2**31 - 1, 2**30 + 1, -2**30 - 3, 0, 1, -1], rng.integers(2**29, 2**31 - 1, 60), -rng.integers(2**20, 2**31, 30)])
    freqs, _ = P.rope_frequencies(32, theta=theta)
    torch.manual_seed(1)
    x = torch.randn((len(pos), 3, 128), device="cuda")
    got = P.rope_positions(x, i32(pos), freqs, layout=layout).double().cpu().numpy()
    # the angle is the exact product of the two numbers; what is left of it below one turn is exact to 2^-52
    ang = np.array([[float(Fraction(int(p)) * Fraction(float(w)) % TWO_PI) for w in freqs.cpu()] for p in pos])[:, None]
    c, s = np.cos(ang), np.sin(ang)
    i, j = (slice(0, 16), slice(16, 32)) if layout == "half" else (slice(0, 32, 2), slice(1, 32, 2))
    y = x.double().cpu().numpy()
    a, b = y[..., i].copy(), y[..., j].copy()
    size = np.abs(a) + np.abs(b)
    for part, want in ((i, a * c - b * s), (j, a * s + b * c)):
        excess = np.abs(got[..., part] - want) - (2.0**-24 * np.abs(want) + 8 * 2.0**-24 * size)
        assert excess.max() <= 0, excess.max()
    assert np.array_equal(got[..., 32:], y[..., 32:]) and math.isclose(float(TWO_PI), 2 * math.pi)
