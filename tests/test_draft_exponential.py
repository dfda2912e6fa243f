"""CPU test of the bound that the header gives for verification's exponentials: e^x, x = (logit - largest) / T, to
5e-14 + 4e-16 |x| of itself.  The kernel's steps (pp_draft.hip: 2^(k / 256) from a table, the rest by a polynomial, the argument as
one operation or as two) in 64-bit numpy with its coefficients, against 80 bits.

  polynomial                        3.5e-14
  table entry, product, Horner      4 roundings, 4.5e-16
  largest * log2(e) / T, below 256  ln 2 * 2^-46 = 9.9e-15 (where it is rounded on its own)
  log2(e), its quotient by T, the argument: 2^-53 of it each, ln 2 * 3 * 2^-53 * 1.45 |x| = 3.4e-16 |x|"""
import os
import re

import numpy as np
import pytest

from paper_2602_24082_amd import build

L = np.longdouble
SRC = open(os.path.join(build.CSRC, "pp_draft.hip")).read()


def _coefficients():
    m = re.search(r"x\.p = fma\(fma\(fma\(([\d.e-]+), f, ([\d.e-]+)\), f, ([\d.e-]+)\), f, 1\.0\);", SRC)
    return [float(c) for c in m.groups()]


def fma(a, b, c):
    """One rounding (80 bits stand in for the exact sum)."""
    return (L(a) * L(b) + L(c)).astype(np.float64)


def exp2_neg(t):
    c3, c2, c1 = _coefficients()
    shift = 1.5 * 2.0 ** 44
    u = t + shift
    f = t - (u - shift)
    k = np.rint((u - shift) * 256).astype(np.int64)
    root = np.exp2((k & 255).astype(L) / 256).astype(np.float64)
    p = fma(fma(fma(c3, f, c2), f, c1), f, 1.0)
    return np.ldexp(root * p, (k >> 8).astype(np.int64))


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("fast", [True, False])
def test_exponentials_keep_the_bound_of_the_header(fast, seed):
    rng = np.random.default_rng(seed)
    n = 400_000
    T = np.float32(rng.choice([1.0, 0.7, 1.25, 0.3, 3.0], n)).astype(np.float64)
    top = rng.uniform(-120, 120, n) * np.minimum(T, 1.0) if fast else rng.uniform(-3e4, 3e4, n)
    top = top.astype(np.float32).astype(np.float64)
    x = (top - rng.uniform(0, 1, n) ** 3 * 690 * T).astype(np.float32).astype(np.float64)
    a = 1.4426950408889634 / T
    if fast:
        b = -top * a
        keep = np.abs(b) < 256
        t = fma(x, a, b)
    else:
        keep = np.ones(n, bool)
        t = (x - top) * a
    keep &= (t > -999) & (t <= 0)
    exact = (L(x) - L(top)) / L(T)
    want = np.exp(exact)
    err = np.abs(exp2_neg(t).astype(L) / want - 1)[keep]
    size = np.abs(exact)[keep]
    assert keep.sum() > n // 2 and float((err / (5e-14 + 4e-16 * size)).max()) < 1
    assert float(err.max()) > 3e-14  # (a shorter bound would not be true)
