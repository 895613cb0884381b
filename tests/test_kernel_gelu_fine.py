"""The GELUs of the 8-bit products, checked on the CPU: their coefficients are
read from the kernel source, the same fp32 steps (each FMA rounded once) are
taken, and the result is compared with a Phi(a) from erfc in binary64.  The
bounds are the ones the source states: 7e-7 (results in fp32) and 8.4e-6."""
import math
import pathlib
import re

import numpy as np
import pytest

SRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2609_35587_amd" / "csrc" / "fp8_matmul.hip"
KINDS = {"gelu_fine": (5, 64.0, 7e-7), "gelu_short": (4, 5.5, 8.4e-6)}     # degree, limit of |a|, bound


def coefficients(kind):
    body, deg = SRC.read_text(), KINDS[kind][0]
    body = body[body.index(f"float {kind}(float a)"):]
    body = body[:body.index("}")]
    found = dict(re.findall(r"\b(c[0-9])\s*=\s*([-+0-9.eE]+)f", body))
    assert sorted(found) == [f"c{i}" for i in range(deg + 1)]
    assert f"fmed3f(fabsf(a), 0.0f, {KINDS[kind][1]}f)" in body
    return [np.float32(float(found[f"c{i}"])) for i in range(deg, -1, -1)]


def fma32(a, b, c):
    return (a.astype(np.float64) * b.astype(np.float64) + c.astype(np.float64)).astype(np.float32)


def kernel_gelu(a, kind):
    a = np.asarray(a, np.float32)
    c, x = coefficients(kind), np.minimum(np.abs(a), np.float32(KINDS[kind][1]))
    p = np.full_like(x, c[0])
    for ci in c[1:]:
        p = fma32(p, x, np.full_like(x, ci))
    with np.errstate(under="ignore"):
        e = np.exp2(p.astype(np.float64)).astype(np.float32)
    return fma32(-x, e, np.maximum(a, np.float32(0.0)))


@pytest.mark.parametrize("kind", KINDS)
def test_error_bound(kind):
    a = np.concatenate([np.linspace(-70, 70, 280_001), np.geomspace(1e-30, 1e30, 4001), -np.geomspace(1e-30, 1e30, 4001)])
    a = a.astype(np.float32)
    exact = np.array([v * 0.5 * math.erfc(-v / math.sqrt(2.0)) for v in a.astype(np.float64)])
    off = np.abs(kernel_gelu(a, kind) - exact)
    assert np.all(off <= KINDS[kind][2] + 2.0 ** -24 * np.abs(exact)), off.max()


@pytest.mark.parametrize("kind", KINDS)
def test_past_the_fitted_range(kind):
    a = np.array([20.0, 64.0, 1e3, 1e38, np.inf, -20.0, -64.0, -1e3, -1e38], np.float32)
    got = kernel_gelu(a, kind)
    assert np.array_equal(got[:5], a[:5]) and np.all(np.abs(got[5:]) <= 2e-7)
    assert np.isnan(kernel_gelu(np.array([np.nan], np.float32), kind))[0]
