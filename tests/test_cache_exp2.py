"""The exponential that the cache's tensor-memory kernel forms on the multiply-add pipe (hifa4_cache_attention.cu, exp2_pair): its FP32
steps, with the coefficients of the source, against 2^x in FP64.

Bound: the polynomial with these coefficients is off by 1.55e-7 at most on [-1/2, 1/2].  Horner steps: the last one rounds a result in
[1, 1.42) by 2^-24 (in [0.7, 1) by 2^-25), the ones before, of less than 1, 0.5 and 0.0625, by 2^-25, 2^-26 and 2^-29 times |f|, f^2, |f|^3
with |f| <= 1/2: 2^-26 + 2^-28 + 2^-32 + .. < 1.9e-8.  Relative to 2^f >= 1: 5.97e-8 + 1.9e-8 = 7.87e-8; to 2^f in [0.7, 1):
(2.99e-8 + 1.9e-8) / 0.7 = 6.99e-8.  Together 2.34e-7 (all FP32 numbers of the range from 2^-14 up, tried once: 2.15e-7).  n is added to
the exponent exactly."""
import os
import re

import numpy as np

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_04302_b200", "csrc", "hifa4_cache_attention.cu")


def coefficients():
    text = open(SRC).read()
    body = text[text.index("void exp2_pair"):]
    body = body[:body.index("\n}")]
    coef = [np.float32(c) for c in re.findall(r"pack2\((\d+\.\d+)f, \1f\)", body)]           # (1.5 * 2^23 has no decimals)
    assert len(coef) == 6
    return coef


def exp2_pair(x):
    coef = coefficients()
    f32 = lambda y: y.astype(np.float32)
    x = np.maximum(x, np.float32(-126))
    t = f32(x + np.float32(12582912))
    f = f32(f32(t - np.float32(12582912)).astype(np.float64) * -1.0 + x)                     # one rounding, and exact
    p = np.full_like(x, coef[0])
    for c in coef[1:]:
        p = f32(p.astype(np.float64) * f + np.float64(c))                                    # the product is exact in FP64
    return f32((p.view(np.uint32) + (t.view(np.uint32) << np.uint32(23))).view(np.float32))


def test_relative_error():
    rng = np.random.default_rng(0)
    x = np.concatenate([np.linspace(-0.5, 0.5, 400001), rng.uniform(-126, 8, 400000), np.arange(-126, 9), np.arange(-126, 9) + 0.5]).astype(np.float32)
    x = x[x >= -126]
    want = np.exp2(x.astype(np.float64))
    err = np.abs(exp2_pair(x).astype(np.float64) - want) / want
    assert err.max() <= 2.34e-7, err.max()


def test_what_lies_below_counts_as_the_least_exponent():
    x = np.float32([-126, -127, -1000, -1e30, -np.inf])
    assert (exp2_pair(x) == np.float32(2.0 ** -126) * np.float32(1.0000001192092896)).all()


def test_the_polynomial_alone():
    f = np.linspace(-0.5, 0.5, 1000001)
    p = np.polyval([float(c) for c in coefficients()], f)
    assert np.abs(p / np.exp2(f) - 1).max() <= 1.55e-7
