"""The GELU of the 8-bit products, checked on the CPU: its coefficients are
read from the kernel source, the same fp32 steps (each FMA rounded once) are
taken, and the result is compared with a Phi(a) from erfc in binary64.  The
bound, 7e-7, is the one the source states."""
import math
import pathlib
import re

import numpy as np

SRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2609_35587_amd" / "csrc" / "fp8_matmul.hip"
BOUND = 7e-7


def coefficients():
    body = SRC.read_text()
    body = body[body.index("float gelu_fine(float a)"):]
    found = dict(re.findall(r"\b(c[0-9])\s*=\s*([-+0-9.eE]+)f", body[:body.index("}")]))
    assert sorted(found) == [f"c{i}" for i in range(6)]
    return [np.float32(float(found[f"c{i}"])) for i in range(5, -1, -1)]


def fma32(a, b, c):
    return (a.astype(np.float64) * b.astype(np.float64) + c.astype(np.float64)).astype(np.float32)


def kernel_gelu(a):
    a = np.asarray(a, np.float32)
    c, x = coefficients(), np.minimum(np.abs(a), np.float32(64.0))
    p = np.full_like(x, c[0])
    for ci in c[1:]:
        p = fma32(p, x, np.full_like(x, ci))
    with np.errstate(under="ignore"):
        e = np.exp2(p.astype(np.float64)).astype(np.float32)
    return fma32(-x, e, np.maximum(a, np.float32(0.0)))


def test_error_bound():
    a = np.concatenate([np.linspace(-70, 70, 280_001), np.geomspace(1e-30, 1e30, 4001), -np.geomspace(1e-30, 1e30, 4001)])
    a = a.astype(np.float32)
    exact = np.array([v * 0.5 * math.erfc(-v / math.sqrt(2.0)) for v in a.astype(np.float64)])
    off = np.abs(kernel_gelu(a) - exact)
    assert np.all(off <= BOUND + 2.0 ** -24 * np.abs(exact)), off.max()


def test_past_the_fitted_range():
    a = np.array([20.0, 64.0, 1e3, 1e38, np.inf, -20.0, -64.0, -1e3, -1e38], np.float32)
    assert np.array_equal(kernel_gelu(a), np.maximum(a, np.float32(0.0)))
    assert np.isnan(kernel_gelu(np.array([np.nan], np.float32)))[0]
