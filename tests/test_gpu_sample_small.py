"""Draws from problems of up to 1,024 candidates and from those around that
size, alone and among longer ones: the same draws as by the definition."""
import numpy as np
import pytest
import torch

import test_gpu_sample as sample
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


def draws(scores, seg, u, **how):
    return hwsel.hwsel_sample_per_problem(scores, torch.tensor(seg, device="cuda"), u, **how)


def check(lengths, n_draws, seed, kind, **how):
    """All problems at once against each problem beside a long one, which another kernel serves."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    seg = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    R, P = int(seg[-1]), len(lengths)
    s = 2.0 * torch.randn(R, generator=g, device="cuda")
    if kind == "equal":
        s = torch.zeros_like(s)
    elif kind == "few values":
        s = torch.round(s)
    elif kind == "odd":
        d = torch.rand(R, generator=g, device="cuda")
        s[d < 0.3], s[d > 0.8], s[(d > 0.5) & (d < 0.55)] = float("-inf"), float("nan"), -0.0
    elif kind == "wide":
        s = s * 1e30
    elif kind == "infinite":
        s[torch.rand(R, generator=g, device="cuda") < 0.01] = float("inf")
    elif kind == "near":
        s = 1.0 + s * 1e-7
    u = torch.rand(P, n_draws, generator=g, device="cuda")
    got = draws(s, seg.tolist(), u, **how)
    # the same by the kernels for long problems: behind 2.5 million candidates each mean is past every rule for short ones
    pad = torch.zeros(3_000_000, device="cuda")
    for lo in range(0, P, 16):
        hi = min(P, lo + 16)
        part = s[seg[lo]:seg[hi]]
        cut = (seg[lo:hi + 1] - seg[lo]).tolist()
        want = draws(torch.cat([part, pad]), cut + [cut[-1] + pad.numel()], torch.cat([u[lo:hi], u[:1]]), **how)
        for a, b in zip(got, want):
            assert torch.equal(a[lo:hi], b[:hi - lo]), (lo, hi)


HOW = [dict(temperature=0.7, top_k=50, top_p=0.95), dict(), dict(top_k=1), dict(temperature=0.0), dict(top_p=0.3, min_p=0.05),
       dict(temperature=3.0, top_k=700), dict(top_k=3, top_p=0.999), dict(temperature=1e-3, top_p=0.5)]
LENGTHS = [1, 2, 0, 63, 64, 65, 255, 256, 257, 511, 512, 513, 1000, 1023, 1024, 1025, 0, 300]


@pytest.mark.parametrize("how", range(len(HOW)))
@pytest.mark.parametrize("kind", ["plain", "equal", "few values", "odd", "wide", "infinite", "near"])
def test_sizes_around_the_bounds(kind, how):
    for n_draws in (1, 9):
        check(LENGTHS, n_draws, 11 * how + n_draws, kind, **HOW[how])


@pytest.mark.parametrize("n_draws", [1, 8, 70])
def test_many_short_problems_and_some_long(n_draws):
    rng = np.random.default_rng(5)
    lengths = rng.integers(0, 900, 1500)
    lengths[::97] = rng.integers(1025, 9000, len(lengths[::97]))
    check(lengths, n_draws, 3, "few values", temperature=1.5, top_k=40, top_p=0.9)


def test_most_problems_longer():
    check([1500] * 300 + [20] * 100 + [1100] * 7, 5, 4, "plain", top_k=30, top_p=0.9)


def test_a_setting_of_each_problem():
    P = 40
    g = torch.Generator(device="cuda").manual_seed(9)
    r = lambda lo, hi: lo + (hi - lo) * torch.rand(P, generator=g, device="cuda")  # noqa: E731
    how = dict(temperature=r(-0.2, 2.0), top_k=r(-5, 60).to(torch.int32), top_p=r(-0.1, 1.2), min_p=r(-0.1, 0.4))
    s, u = 2 * torch.randn(P * 700, generator=g, device="cuda"), torch.rand(P, 12, generator=g, device="cuda")
    got = draws(s, [700 * i for i in range(P + 1)], u, **how)
    for p in range(P):
        one = draws(s[700 * p:700 * p + 700], [0, 700], u[p:p + 1], **{k: float(v[p]) if k != "top_k" else int(v[p]) for k, v in how.items()})
        for a, b in zip(got, one):
            assert torch.equal(a[p:p + 1], b)


@pytest.mark.parametrize("kind", sample.KINDS)
def test_against_the_definition(kind):
    """Through the statement in whole numbers that longer problems are held to."""
    rng = np.random.default_rng(21)
    parts = [sample.make_scores(rng, n, kind) for n in LENGTHS]
    for n_draws in (3, 20):
        for how in HOW:
            sample.check(parts, sample.uniform(rng, len(parts), n_draws), **how)
