"""The normal distribution function of the feed-forward block's GELU (host only): what its comment says of the polynomial holds for the coefficients as they stand
in the source, in 64 bits, and the whole within its bound when it is evaluated in FP32."""
import os
import re

import numpy as np
import pytest

special = pytest.importorskip("scipy.special")
SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_11205_amd", "csrc", "jz_ffn_gemm.h")


@pytest.fixture(scope="module")
def text():
    with open(SOURCE) as f:
        return f.read()


def coefficients(text):
    return np.array([float(c.rstrip("f")) for c in re.search(r"P\[9\] = \{([^}]*)\}", text).group(1).split(", ")], dtype=np.float32)


def test_largest_relative_error_of_the_polynomial(text):
    figure, end = re.search(r"relative error, ([0-9.e-]+) with the coefficients rounded to FP32, up to \|v\| = (\d+)", text).groups()
    v = np.concatenate([np.linspace(0, float(end), 200001), np.linspace(0, 1, 100001)])
    t = 1 / (1 + float(np.float32(0.35)) * v)
    p = t * np.polynomial.polynomial.polyval(t, coefficients(text).astype(np.float64))
    error = np.max(np.abs(p / (special.erfcx(v / 2 ** 0.5) / 2) - 1))         # Phi(-v) exp(v^2 / 2)
    assert 0.9 * float(figure) <= error <= float(figure), error


def test_the_whole_in_fp32(text):
    """Roundings where the kernel has them (its reciprocal and exponential may be off by one more): within 10 (1 + |v|) 2^-24 of itself."""
    f, P = np.float32, coefficients(text)
    v = np.linspace(-13, 13, 200001).astype(f)

    def fma(a, b, c):
        return (a.astype(np.float64) * b.astype(np.float64) + np.float64(c)).astype(f)
    t = (f(1) / fma(np.abs(v), np.full_like(v, 0.35), f(1))).astype(f)
    p = np.full_like(v, P[8])
    for i in range(7, -1, -1):
        p = fma(p, t, P[i])
    bell = np.exp2(((v * v).astype(f) * f(-0.72134752)).astype(f).astype(np.float64)).astype(f)
    tail = ((t * p).astype(f) * bell).astype(f)
    got = np.where(v < 0, tail, (f(1) - tail).astype(f)).astype(np.float64)
    want = special.ndtr(v.astype(np.float64))
    assert np.max(np.abs(got / want - 1) / (1 + np.abs(v))) <= 10 * 2.0 ** -24
