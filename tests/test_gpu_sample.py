"""Drawing candidates against the definition in whole numbers (indices and
counts equal; the probability within fp32 rounding of the quotient): settings
alone and together, ties, masked scores, infinities, lengths from 0 to beyond
the catalogue's size, ragged segments, settings per problem, edge random
numbers."""
import numpy as np
import pytest
import torch

from _fp8_util import draws64
from _gpu_util import say
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
SETTINGS = [dict(), dict(temperature=0.0), dict(top_k=1), dict(top_k=7), dict(top_p=0.3), dict(top_p=0.999),
            dict(min_p=0.2), dict(top_k=50, top_p=0.9, min_p=0.01, temperature=0.7),
            dict(top_k=400, top_p=0.5, temperature=3.0)]
SPECIAL = [dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=float("nan")), dict(min_p=1.0), dict(min_p=5.0),
           dict(min_p=float("nan")), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=1e-40),
           dict(temperature=float("inf")), dict(temperature=1e30, top_p=0.5), dict(top_k=-3), dict(top_k=2 ** 31 - 1)]


def make_scores(rng, n, kind):
    s = (2.0 * rng.standard_normal(n)).astype(np.float32)
    if kind == "ties":
        s = np.round(s * 2) / 2
    elif kind == "equal":
        s[:] = 1.25
    elif kind == "zeros":
        s = np.where(rng.random(n) < 0.5, np.float32(0.0), np.float32(-0.0)).astype(np.float32)
    elif kind == "masked":
        s[rng.random(n) < 0.6] = -np.inf
        s[rng.random(n) < 0.1] = np.nan
    elif kind == "dead":
        s[:] = np.where(rng.random(n) < 0.5, -np.inf, np.nan)
    elif kind == "lowest":
        s[rng.random(n) < 0.7] = np.finfo(np.float32).min
    elif kind == "all lowest":
        s[:] = np.finfo(np.float32).min
    elif kind == "infinite":
        s[rng.random(n) < 0.2] = np.inf
    elif kind == "wide":
        s *= 50
    elif kind == "flat":
        s *= np.float32(1e-3)
    return s.astype(np.float32)


KINDS = ["normal", "ties", "equal", "zeros", "masked", "dead", "lowest", "all lowest", "infinite", "wide", "flat"]


def run(parts, u, **how):
    seg = np.zeros(len(parts) + 1, np.int64)
    seg[1:] = np.cumsum([len(p) for p in parts])
    s = torch.from_numpy(np.concatenate(parts + [np.zeros(0, np.float32)])).cuda()
    idx, prob, kept = hwsel.hwsel_sample_per_problem(s, torch.from_numpy(seg).cuda(), torch.from_numpy(u).cuda(), **how)
    return idx.cpu().numpy(), prob.cpu().numpy(), kept.cpu().numpy()


def check(parts, u, per_problem=None, **how):
    dev = {k: torch.from_numpy(v).cuda() for k, v in (per_problem or {}).items()}
    idx, prob, kept = run(parts, u, **how, **dev)
    for p, s in enumerate(parts):
        own = {**how, **{k: v[p] for k, v in (per_problem or {}).items()}}
        i, q, n = draws64(s, u[p], **own)
        assert kept[p] == n, (p, len(s), own, kept[p], n)
        assert np.array_equal(idx[p], i), (p, len(s), own, idx[p][:8], i[:8])
        assert np.all(np.abs(prob[p] - q) <= 2.0 ** -23 * q)


def uniform(rng, P, n):
    u = rng.random((P, n), np.float32)
    u[:, 0] = 0.0
    if n > 1:
        u[:, 1] = 1.0 - 2.0 ** -24
    return u


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("how", range(len(SETTINGS) + len(SPECIAL)))
def test_settings_and_scores(kind, how):
    how = (SETTINGS + SPECIAL)[how]
    rng = np.random.default_rng([KINDS.index(kind), len(str(how))])
    parts = [make_scores(rng, n, kind) for n in (0, 1, 2, 63, 64, 65, 300, 1025)]
    check(parts, uniform(rng, len(parts), 5), **how)


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "flat", "masked"])
@pytest.mark.parametrize("n", [4095, 8192, 8193, 16_385, 65_536, 70_001])
def test_long_segments(n, kind):
    say(f"sample {n} {kind}")
    rng = np.random.default_rng([n, KINDS.index(kind)])
    parts = [make_scores(rng, n, kind)]
    u = uniform(rng, 1, 33)
    for how in (dict(), dict(top_k=900), dict(top_p=0.8), dict(top_k=n // 2, top_p=0.95, min_p=0.001, temperature=1.3)):
        check(parts, u, **how)


@pytest.mark.parametrize("P,n", [(1, 534_600), (3, 200_003), (2, 1_100_000)])
def test_very_long_segments(P, n):
    say(f"sample {P} x {n}")
    rng = np.random.default_rng([P, n])
    parts = [make_scores(rng, n - 17 * p, "ties" if p == 1 else "normal") for p in range(P)]
    u = uniform(rng, P, 4)
    check(parts, u, top_p=0.9, min_p=0.05, temperature=1.5)
    check(parts, u, top_k=1000)
    check(parts, u)


def test_ragged_with_settings_per_problem():
    rng = np.random.default_rng(5)
    P = 200
    parts = [make_scores(rng, int(rng.integers(0, 900)), KINDS[p % len(KINDS)]) for p in range(P)]
    per = dict(temperature=rng.uniform(0, 2, P).astype(np.float32), top_k=rng.integers(-2, 60, P).astype(np.int32),
               top_p=rng.uniform(-0.1, 1.1, P).astype(np.float32), min_p=rng.uniform(-0.1, 0.5, P).astype(np.float32))
    per["temperature"][::10] = 0.0
    check(parts, uniform(rng, P, 9), per)


@pytest.mark.parametrize("draws", [1, 64, 65, 2000])
def test_many_draws(draws):
    rng = np.random.default_rng(draws)
    parts = [make_scores(rng, n, "normal") for n in (100, 5000, 9000)]
    u = uniform(rng, 3, draws)
    if draws > 8:
        u[:, 2:8] = np.array([-1.0, 1.0, 2.0, np.nan, np.inf, 1e-30], np.float32)
    check(parts, u, top_p=0.97)


def test_many_problems():
    rng = np.random.default_rng(8)
    parts = [make_scores(rng, int(n), "ties") for n in rng.integers(0, 40, 3000)]
    check(parts, uniform(rng, 3000, 2), top_k=5, top_p=0.9)


def test_offsets_outside_the_scores_are_limited():
    """Offsets beyond the scores are read as their end: nothing outside is touched."""
    s = torch.randn(100, device="cuda")
    seg = torch.tensor([-5, 40, 1 << 40, 90, 200], dtype=torch.int64, device="cuda")
    u = torch.rand(4, 3, device="cuda")
    idx, _, kept = hwsel.hwsel_sample_per_problem(s, seg, u)
    assert kept.tolist() == [40, 60, 0, 10] and bool((idx[2] == -1).all()) and int(idx.max()) < 60


def test_draws_follow_the_probabilities():
    """200,000 draws over 6 candidates: the counts within 5 standard deviations of n p."""
    s = torch.tensor([0.0, 1.0, 2.0, -1.0, 2.0, float("-inf")], device="cuda")
    n = 200_000
    u = torch.rand(1, n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    idx, prob, kept = hwsel.hwsel_sample_per_problem(s, torch.tensor([0, 6], device="cuda"), u, temperature=2.0)
    p = torch.softmax(s.double() / 2.0, 0)
    got = torch.bincount(idx[0].long(), minlength=6).double()
    assert int(kept[0]) == 5
    assert bool(((got - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt() + 1e-9).all())
    assert float((prob[0].double() - p[idx[0].long()]).abs().max()) < 1e-6


def test_no_scores_at_all():
    idx, prob, kept = hwsel.hwsel_sample_per_problem(torch.empty(0, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"),
                                                     torch.rand(2, 4, device="cuda"))
    assert bool((idx == -1).all()) and bool((prob == 0).all()) and bool((kept == 0).all())
