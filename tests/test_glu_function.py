"""The polynomial of the gated feed-forward's GELU in bf16 (csrc/glu_gemm.h), on the CPU: its coefficients, read from the source,
against the fit they come from, its error in exact arithmetic and in fp32.

The form: erfc(x) = exp(-x^2) t q(t) with t = 1 / (1 + 0.33 x), q of degree 7.  The fit is a linear program: the least e such that
|t q(t) / erfcx(x) - 1| <= e at every point, erfcx(x) = exp(x^2) erfc(x); points from 0 to 10, evenly in t."""
import os
import re

import numpy as np
import pytest

special = pytest.importorskip("scipy.special")
optimize = pytest.importorskip("scipy.optimize")

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_26430_amd", "csrc", "glu_gemm.h")


def coefficients():
    """Of t^7 to t^0, as the kernel has them."""
    text = open(SOURCE).read()
    body = text[text.index("float q = fmaf(t,"):text.index("const float half = 0.5f * t * q * e")]
    c = [float(x) for x in re.findall(r"(-?\d\.\d+)f", body)]
    assert len(c) == 8 and body.count("fmaf") == 7
    return c


def points(n):
    t = np.linspace(1.0 / 4.3, 1.0, n)
    return t, (1.0 / t - 1.0) / 0.33


def test_the_coefficients_are_the_best_fit():
    """No coefficients of this form come closer than 0.9 of the error that these have."""
    t, x = points(2001)
    u = (2 * t - (1 + t.min())) / (1 - t.min())
    a = np.polynomial.chebyshev.chebvander(u, 7) * t[:, None] / special.erfcx(x)[:, None]
    one, unit = np.ones((t.size, 1)), 1e6       # errors in millionths, so that the solver's tolerance is far below them
    lp = optimize.linprog(np.r_[np.zeros(8), 1.0], A_ub=np.r_[np.c_[a * unit, -one], np.c_[-a * unit, -one]],
                          b_ub=np.r_[np.full(t.size, unit), np.full(t.size, -unit)], bounds=[(None, None)] * 9, method="highs")
    assert lp.success
    t, x = points(100_001)
    ours = np.abs(t * np.polyval(coefficients(), t) / special.erfcx(x) - 1.0).max()
    assert ours <= 1e-7 and 0.9 * ours <= lp.fun / unit, (ours, lp.fun / unit)


def test_error_in_fp32():
    """The kernel's steps in fp32.  Bound, u = 2^-24: the fit's 1e-7; t is off by u of its denominator and a unit of the reciprocal, 3 u
    in all, and carries d log(t q) / d log t of it on; each of the fused steps adds u of its result, times t for every later one; the
    product adds u."""
    f, u = np.float32, 2.0 ** -24
    c = [f(k) for k in coefficients()]
    g = np.linspace(0.0, 14.0, 400_001).astype(f)
    exact = 1.0 / (1.0 + g.astype(np.float64) * (0.33 / np.sqrt(2.0)))
    want = special.erfcx(g.astype(np.float64) / np.sqrt(2.0))
    part, err = np.full_like(exact, float(c[0])), np.zeros_like(exact)
    for k in c[1:]:
        part = exact * part + float(k)
        err = exact * err + u * np.abs(part)
    slope = 1.0 + exact * np.polyval(np.polyder([float(k) for k in c]), exact) / part
    bound = 1.01 * (1e-7 + np.abs(slope) * 3.2 * u + err / part + u)      # (0.2 u: the rounding of 0.33 / sqrt 2)
    assert bound.max() <= 1.1e-6        # as the kernel's comment has it
    for unit in (-1, 0, 1):
        t = (1.0 / f(1.0 + g.astype(np.float64) * float(f(0.33 * 0.70710678118654752)))).astype(f)
        t = t if unit == 0 else np.nextafter(t, f(2 * unit), dtype=f)
        q = np.full_like(t, c[0])
        for k in c[1:]:
            q = (t.astype(np.float64) * q.astype(np.float64) + float(k)).astype(f)
        off = np.abs((t * q).astype(np.float64) / want - 1.0)
        assert (off <= bound).all(), (unit, float(off.max()))
