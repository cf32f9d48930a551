"""GELU's normal distribution: the polynomial that the kernels evaluate, with the coefficients of their source, against erfc in 64 bits."""
import math
import os
import re

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _coefficients():
    text = open(os.path.join(ROOT, "paper_2602_06183_b200", "csrc", "gated.cuh")).read()
    body = text[text.index("float normal_cdf("):]
    body = body[:body.index("\n}\n")]
    assert "fmaf(0.3f, x, 1.f)" in body
    c = re.findall(r"(?:p = |fmaf\(p, t, )(-?\d[\d.e-]*)f", body)
    assert len(c) == 9
    return [np.float32(v) for v in c]


def _ratio(x):
    """Phi(-x) e^(x^2 / 2): erfcx(x / sqrt 2) / 2, by its continued fraction where erfc and the exponential leave float64's range together."""
    if x < 12:
        return 0.5 * math.erfc(x / math.sqrt(2)) * math.exp(x * x / 2)
    f = x
    for k in range(60, 0, -1):
        f = x + k / f
    return 1 / (f * math.sqrt(2 * math.pi))


X = np.concatenate([np.linspace(0, 14.5, 5801), np.linspace(0.05, 0.15, 1001)])
REF = np.array([_ratio(float(x)) for x in X])


def test_polynomial():
    t = 1 / (1 + float(np.float32(0.3)) * X)
    p = np.zeros_like(X)
    for c in _coefficients():
        p = p * t + float(c)
    err = np.abs(p / REF - 1)
    assert err[X <= 14].max() < 1.2e-7 and err.max() < 1.7e-7


def test_in_float32():
    """Fused steps and a reciprocal that is rounded to nearest: the exact value of each step, then one rounding."""
    x = X.astype(np.float32).astype(np.float64)
    t = (1 / (x * float(np.float32(0.3)) + 1).astype(np.float32).astype(np.float64)).astype(np.float32).astype(np.float64)
    p = np.zeros_like(x)
    for c in _coefficients():
        p = (p * t + float(c)).astype(np.float32).astype(np.float64)
    ref = np.array([_ratio(float(v)) for v in x])
    assert np.abs(p / ref - 1).max() < 4e-7
