"""Cuts among many equal scores: one score that many candidates share, two of
them a rounding apart, with other scores around them or none."""
import numpy as np
import pytest
import torch

import test_gpu_sample as sample
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
# candidates of a problem: a wave's, a workgroup's of each kind, shared by workgroups
SIZES = [1000, 3000, 8192, 20_000, 60_000, 300_000]


def scores(rng, n, kind):
    s = (2.0 * rng.standard_normal(n)).astype(np.float32)
    if kind == "rounded":
        s = np.round(2 * s) / 2
    elif kind == "a third rounded":
        s = np.where(rng.random(n) < 0.3, np.round(2 * s) / 2, s)
    elif kind == "one value":
        s = np.where(rng.random(n) < 0.6, np.float32(0.25), s)
    elif kind == "two neighbours":
        a = np.float32(0.25)
        s = np.where(rng.random(n) < 0.8, np.where(rng.random(n) < 0.5, a, np.nextafter(a, np.float32(1))), s)
    elif kind == "two values":
        s = np.where(rng.random(n) < 0.5, np.float32(1.0), np.float32(-1.0))
    elif kind == "at the end":
        s[-n // 3:] = 0.5
    return s.astype(np.float32)


KINDS = ["rounded", "a third rounded", "one value", "two neighbours", "two values", "at the end"]
HOW = [dict(top_p=0.9), dict(top_p=0.5, temperature=2.0), dict(top_k=-1, top_p=0.25), dict(temperature=0.5, top_p=0.7)]


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_against_the_definition(kind, n):
    rng = np.random.default_rng(n)
    parts = [scores(rng, n - i, kind) for i in range(2)]
    for how in HOW:
        for k in (0, n // 3, n // 2, 2 * n // 3):
            sample.check(parts, sample.uniform(rng, 2, 3), **{**how, "top_k": k})
    for k in (n // 5, n // 2, n - 1):
        sample.check(parts, sample.uniform(rng, 2, 3), top_k=k)


@pytest.mark.parametrize("n", [900, 4000, 13_000, 70_000])
def test_more_problems_than_compute_units(n):
    """Against the same problems one at a time."""
    P = 300 if n < 50_000 else 20
    rng = np.random.default_rng(n)
    s = torch.from_numpy(np.concatenate([scores(rng, n, KINDS[p % len(KINDS)]) for p in range(P)])).cuda()
    u = torch.from_numpy(sample.uniform(rng, P, 6)).cuda()
    seg = torch.arange(P + 1, device="cuda") * n
    got = hwsel.hwsel_sample_per_problem(s, seg, u, top_p=0.8, top_k=n // 2)
    for p in range(0, P, 7):
        one = hwsel.hwsel_sample_per_problem(s[n * p:n * p + n], seg[:2], u[p:p + 1], top_p=0.8, top_k=n // 2)
        for a, b in zip(got, one):
            assert torch.equal(a[p:p + 1], b)


def test_the_same_draws_again():
    """The lists behind a cut fill in any order; the cut does not depend on it."""
    rng = np.random.default_rng(1)
    s = torch.from_numpy(scores(rng, 3 * 534_600, "a third rounded")).cuda()
    seg, u = torch.arange(4, device="cuda") * 534_600, torch.from_numpy(sample.uniform(rng, 3, 50)).cuda()
    first = hwsel.hwsel_sample_per_problem(s, seg, u, top_p=0.9)
    for _ in range(10):
        for a, b in zip(first, hwsel.hwsel_sample_per_problem(s, seg, u, top_p=0.9)):
            assert torch.equal(a, b)
