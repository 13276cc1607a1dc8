"""The rational exponent that the epilogue's GELU of bf16 results takes for erfc
(masq_epilogue.h): its coefficients from their definition, and the formula's error
in fp32, emulated (each operation rounded once)."""
import math
import os
import re

import numpy as np
from scipy.special import erfc, erfcx

from paper_2603_04800_amd import build

f32 = np.float32


def _coefficients():
    with open(os.path.join(build.CSRC, "masq_epilogue.h")) as f:
        text = re.search(r"kQ\[10\] = \{([^}]*)\}", f.read()).group(1)
    return [float(v.strip().rstrip("f")) for v in text.split(",")]


def _target(t):
    """log2(erfc(x) e^(x^2) / t) at t = 1 / (1 + x / 2)."""
    return np.log2(erfcx(2 * (1 / t - 1)) / t)


def test_coefficients_are_the_chebyshev_interpolant():
    lo, hi, n = 1 / 6, 1.0, 10                              # x in [0, 10]
    t = (lo + hi) / 2 + (hi - lo) / 2 * np.cos((2 * np.arange(n) + 1) * math.pi / (2 * n))
    want = np.polynomial.polynomial.polyfit(t, _target(t), n - 1)
    # fp32 coefficients: half a step of the largest is 2^-24 (1.72)
    assert np.abs(np.array(_coefficients()) - want).max() < 2 * 2.0 ** -24
    t = np.linspace(lo, hi, 100001)
    off = np.polynomial.polynomial.polyval(t, _coefficients()) - _target(t)
    assert np.abs(np.exp2(off) - 1).max() < 1.2e-7


def _fma(a, b, c):
    return (np.float64(a) * np.float64(b) + np.float64(c)).astype(f32)


def _gelu(z):
    x = np.abs(z) * f32(0.70710678118654752)
    t = (1 / np.float64(_fma(f32(0.5), x, f32(1)))).astype(f32)
    q = np.full_like(t, f32(_coefficients()[9]))
    for c in _coefficients()[8::-1]:
        q = _fma(q, t, f32(c))
    e = t * np.exp2(np.float64(_fma(x * f32(-1.44269504), x, q))).astype(f32)
    return f32(0.5) * z * np.where(z > 0, f32(2) - e, e)


def test_error_of_the_formula():
    """Relative to the value, with u = 2^-24: the interpolant 2 u, t 2 u and as much
    through Q, Horner's steps (terms up to 1.8 in an exponent of 2) 6 u, the
    exponential, its product with t and those with z 4 u: 16 u.  The exponent's
    part x^2 log2 e, x^2 = z^2 / 2: x is off by 1.5 u (its constant and product),
    so x^2 by 3 u, the constant and the product by 1.5 u, and the sum rounds to 1 u
    of the exponent: 6 u z^2 / 2 at most, as it is the natural exponent of e^-x^2
    that this multiplies.  4 z^2 u leaves room for second-order terms."""
    u = 2.0 ** -24
    z = np.linspace(-13, 13, 2000001).astype(f32)
    want = 0.5 * np.float64(z) * erfc(-np.float64(z) / math.sqrt(2))
    off = np.abs(_gelu(z) - want)
    keep = np.abs(want) > 2.0 ** -126
    assert (off[keep] <= (16 + 4 * np.float64(z[keep]) ** 2) * u * np.abs(want[keep])).all()
    # in absolute terms: z^2 |h| <= 0.23 and |h| <= 0.17 for z < 0
    assert off[z < 0].max() <= (16 * 0.17 + 4 * 0.23) * u
