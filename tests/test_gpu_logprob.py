"""Log probabilities, entropies, alternatives and gradients against binary64, within bounds counted from
their fp32 operations."""
import math

import numpy as np
import pytest
import torch

from _learn_util import Logprob, near
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
INF = float("inf")


def scores_of(rng, n, kind):
    s = rng.standard_normal(n).astype(np.float32) * 3
    if kind == "ties":
        s = np.round(s)
    elif kind == "equal":
        s[:] = 1.5
    elif kind == "holes":
        s[rng.random(n) < 0.3] = -INF
        s[rng.random(n) < 0.1] = np.nan
    elif kind == "none":
        s[:] = np.where(rng.random(n) < 0.5, -INF, np.nan)
    elif kind == "inf":
        s[rng.integers(0, max(n, 1), 3) % max(n, 1)] = INF
    elif kind == "peaked":
        s *= 1e-3
        s[n // 2] = 12.0
    elif kind == "wide":
        s *= 1e37
    elif kind == "zeros":
        s[:] = np.where(rng.random(n) < 0.5, 0.0, -0.0)
    return s


KINDS = ["plain", "ties", "equal", "holes", "none", "inf", "peaked", "wide", "zeros"]


def check(parts, T, n_picks=5, top=7, seed=0, d_entropy=True, lead=0, trail=0):
    """Problems (arrays of scores) one behind another; T a number or one for each."""
    rng = np.random.default_rng(seed)
    P = len(parts)
    seg = np.concatenate([[0], np.cumsum([len(s) for s in parts])]) + lead
    flat = np.concatenate([np.full(lead, 5.0, np.float32), *parts, np.full(trail, 5.0, np.float32)]).astype(np.float32)
    picks = np.stack([rng.integers(-2, max(len(s), 1) + 2, n_picks) for s in parts]).astype(np.int32) if n_picks else None
    if n_picks > 2:
        picks[:, 1] = picks[:, 0]                           # the same one twice
    d_logp = rng.standard_normal((P, n_picks)).astype(np.float32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    Ts = np.broadcast_to(np.float32(T), P)
    temp = dev(Ts.copy()) if np.ndim(T) else T
    s, o = dev(flat), dev(seg)
    pk = dev(picks) if n_picks else None
    logp, entropy, norm, top_idx, top_logp = hwsel.hwsel_logprob_per_problem(s, o, pk, temperature=temp, top=top)
    de = rng.standard_normal(P).astype(np.float32) if d_entropy else None
    grad = hwsel.hwsel_logprob_gradient(s, o, norm, pk, dev(d_logp) if n_picks else None, entropy, dev(de) if d_entropy else None, temperature=temp)
    grad = grad.cpu()
    assert not bool(grad[:lead].any()) and not bool(grad[lead + sum(map(len, parts)):].any())
    entropy, norm = entropy.cpu(), norm.cpu()
    for p, a in enumerate(parts):
        q = Logprob(a, Ts[p])
        near(norm[p, :1], torch.tensor([q.best]).double(), 0.0, f"best of {p}")
        if len(q.live):
            near(norm[p, 1:], torch.tensor([q.log_mass]).double(), getattr(q, "em", 0.0), f"log mass of {p}")
            near(entropy[p:p + 1], torch.tensor([q.entropy]).double(), getattr(q, "eentropy", 0.0), f"entropy of {p}")
        else:
            assert float(norm[p, 1]) == -INF and float(entropy[p]) == 0.0
        if n_picks:
            want = np.array([q.of(j) for j in picks[p]])
            near(logp[p], torch.from_numpy(want[:, 0]), torch.from_numpy(want[:, 1]), f"log p of {p}")
        if top:
            order = q.live[np.lexsort((q.live, -(a[q.live].astype(np.float64) + 0.0)))]
            order = [j for j in order if q.lp[j] > -INF][:top]
            assert top_idx[p].tolist() == [int(j) for j in order] + [-1] * (top - len(order)), f"alternatives of {p}"
            want = np.full(top, -INF)
            want[:len(order)] = q.lp[order]
            near(top_logp[p], torch.from_numpy(want), torch.from_numpy(np.concatenate([q.elp[order], np.zeros(top - len(order))])) if order else 0.0,
                 f"alternatives' log p of {p}")
        g, bound = q.gradient(picks[p] if n_picks else [], d_logp[p], de[p] if d_entropy else 0.0)
        near(grad[seg[p]:seg[p + 1]], torch.from_numpy(g), torch.from_numpy(bound), f"gradient of {p}")


LENGTHS = [0, 1, 2, 3, 15, 63, 64, 65, 255, 256, 257, 1000, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 8193]


@pytest.mark.parametrize("kind", KINDS)
def test_kinds_and_lengths(kind):
    rng = np.random.default_rng(KINDS.index(kind))
    check([scores_of(rng, n, kind if n else "plain") for n in LENGTHS], 0.8, lead=3, trail=5)


@pytest.mark.parametrize("T", [1.0, 1e-3, 0.05, 30.0, 1e30, INF, 0.0, -1.0, math.nan])
def test_temperatures(T):
    rng = np.random.default_rng(5)
    parts = [scores_of(rng, n, kind) for n in (1, 40, 700, 3000) for kind in ("plain", "ties", "holes", "peaked")]
    check(parts, T)


def test_a_temperature_of_each():
    rng = np.random.default_rng(6)
    parts = [scores_of(rng, int(n), KINDS[i % 4]) for i, n in enumerate(rng.integers(0, 600, 30))]
    check(parts, np.where(np.arange(30) % 5 == 0, 0.0, rng.uniform(0.1, 3.0, 30)).astype(np.float32))


@pytest.mark.parametrize("n_picks,top", [(0, 0), (0, 64), (1, 1), (1, 0), (64, 64), (300, 33), (5000, 2)])
def test_numbers_of_picks_and_alternatives(n_picks, top):
    rng = np.random.default_rng(n_picks + top)
    check([scores_of(rng, n, "ties") for n in (5, 64, 100, 1500, 9000)], 1.0, n_picks, top)


@pytest.mark.parametrize("P,n", [(3, 200_000), (1, 534_600), (2, 40_000), (40, 20_000)])
@pytest.mark.parametrize("kind", ["plain", "ties", "holes"])
def test_long_problems(P, n, kind):
    rng = np.random.default_rng(P + n)
    parts = [scores_of(rng, n - 7 * p, kind) for p in range(P)]
    check(parts, 1.2, 20, 16)
    check(parts[:2] + [parts[0][:0], parts[0][:100]], 0.0, 3, 3)


@pytest.mark.parametrize("P,n", [(5000, 20), (2000, 300), (700, 1200)])
def test_many_problems(P, n):
    rng = np.random.default_rng(P)
    parts = [scores_of(rng, int(m), "holes" if m % 2 else "ties") for m in rng.integers(0, n, P)]
    parts[P // 2] = scores_of(rng, 20_000, "ties")
    check(parts, 0.9, 3, 5)


def test_without_entropy():
    rng = np.random.default_rng(8)
    check([scores_of(rng, n, "plain") for n in (10, 2000)], 1.0, 4, 0, d_entropy=False)


def test_offsets_outside_the_scores():
    s = torch.arange(10.0, device="cuda")
    seg = torch.tensor([-5, 4, 4, 100, 3], device="cuda")
    picks = torch.tensor([[3], [0], [5], [0]], dtype=torch.int32, device="cuda")
    logp, entropy, norm, idx, lp = hwsel.hwsel_logprob_per_problem(s, seg, picks, top=2)
    for p, a in enumerate((s[0:4], s[4:4], s[4:10], s[:0])):
        q = Logprob(a.cpu().numpy())
        near(logp[p], torch.tensor([q.of(int(picks[p, 0]))[0]]).double(), q.of(int(picks[p, 0]))[1])
    assert idx.tolist() == [[3, 2], [-1, -1], [5, 4], [-1, -1]]


def test_rows_of_no_problem():
    s = torch.randn(1000, device="cuda")
    seg = torch.tensor([100, 300, 900], device="cuda")
    picks = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    logp, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks)
    out = torch.full((1000,), 7.0, device="cuda")
    d = torch.ones(2, 1, device="cuda")
    assert hwsel.hwsel_logprob_gradient(s, seg, norm, picks, d, out=out) is out
    assert not bool(out[:100].any()) and not bool(out[900:].any()) and bool((out[100:900] != 0).all())


def test_gradients_that_are_not_finite():
    rng = np.random.default_rng(9)
    s = torch.from_numpy(rng.standard_normal(90).astype(np.float32)).cuda()
    seg = torch.tensor([0, 30, 60, 90], device="cuda")
    picks = torch.tensor([[1, 2]] * 3, dtype=torch.int32, device="cuda")
    logp, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks)
    d = torch.ones(3, 2, device="cuda")
    d[1, 1] = float("nan")
    got = hwsel.hwsel_logprob_gradient(s, seg, norm, picks, d)
    assert not bool(torch.isfinite(got[30:60]).any()) and bool(torch.isfinite(got[:30]).all()) and bool(torch.isfinite(got[60:]).all())
    de = torch.tensor([INF, 0.0, 0.0], device="cuda")
    got = hwsel.hwsel_logprob_gradient(s, seg, norm, picks, torch.ones(3, 2, device="cuda"), entropy, de)
    assert not bool(torch.isfinite(got[:30]).any()) and bool(torch.isfinite(got[30:]).all())


def test_same_bits():
    """Picks added in any order, the same one many times: the same gradient."""
    g = torch.Generator(device="cuda").manual_seed(1)
    s = torch.randn(3 * 5000, generator=g, device="cuda")
    seg = torch.arange(4, device="cuda") * 5000
    picks = torch.randint(0, 40, (3, 500), generator=g, device="cuda", dtype=torch.int32)
    d = torch.randn(3, 500, generator=g, device="cuda")
    _, _, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks)
    want = hwsel.hwsel_logprob_gradient(s, seg, norm, picks, d)
    for _ in range(3):
        order = torch.randperm(500, generator=g, device="cuda")
        got = hwsel.hwsel_logprob_gradient(s, seg, norm, picks[:, order].contiguous(), d[:, order].contiguous())
        assert torch.equal(got, want)


def test_drawn_candidates_have_the_probability_they_were_drawn_with():
    """Without limits a draw's probability is its whole-number weight against their sum: weights are within 3 u of 2^32
    exp(t), u = 2^-24, and one more (of 2^-32), so a sum of 3,000 within 3 u and 3,000 2^-32; a log probability is within (4
    |t| + 8) u and the 63 u of its sum's longest chain, 3,000 / 64 + 16 additions."""
    g = torch.Generator(device="cuda").manual_seed(2)
    s = torch.randn(4 * 3000, generator=g, device="cuda")
    seg = torch.arange(5, device="cuda") * 3000
    idx, prob, _ = hwsel.hwsel_sample_per_problem(s, seg, torch.rand(4, 50, generator=g, device="cuda"), temperature=0.7)
    logp, _, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, idx, temperature=0.7)
    t = (logp + norm[:, 1:]).double()                       # (s - best) / T
    bound = (6 + 71 + 4 * t.abs() + 4) * 2.0 ** -24 + 2.0 ** -32 * (torch.exp(-t) + 3000)
    assert bool(((logp.double().exp() / prob.double() - 1).abs() <= bound).all())
