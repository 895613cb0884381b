"""Log probabilities against binary64 on each way a call can go.  Which one that is goes by the number of problems, their mean
length and whether alternatives are asked for; the lengths here are on both sides of each rule for 256 compute units (P problems):
  parts and their join    mean from 32,768 on, P <= 128
  a wave a problem        mean <= 1,024; with alternatives <= 256 where P <= 1,024; longer problems among them by workgroups of 256
  256 threads a problem   mean <= 4,096 where P <= 256, else <= 8,192
  512 threads             mean <= 8,192 where P <= 256, else all longer ones
  1,024 threads           the rest"""
import numpy as np
import pytest
import torch

from _learn_util import Logprob, near
from paper_2609_35587_amd import hwsel
from test_gpu_logprob import KINDS, check, scores_of

pytestmark = pytest.mark.gpu


def mixed(rng, lengths, kinds=("ties", "holes", "plain", "equal")):
    return [scores_of(rng, int(n), kinds[i % len(kinds)] if n else "plain") for i, n in enumerate(lengths)]


@pytest.mark.parametrize("top", [1, 8, 9, 33, 64])
@pytest.mark.parametrize("T", [0.7, 0.0])
def test_waves_with_alternatives(top, T):
    """Up to 8 alternatives a bound of the lanes' best, more a bound of all candidates; registers of 1, 4, 8 and 16 scores."""
    rng = np.random.default_rng(top)
    lengths = [0, 1, 8, 9, 63, 64, 65, 128, 255, 256, 257, 300, 511, 512, 513, 700, 1000, 1023, 1024, *rng.integers(0, 130, 40)]
    assert sum(lengths) / len(lengths) <= 256
    check(mixed(rng, lengths), T, 4, top)
    check(mixed(rng, lengths, KINDS), T, 4, top)


@pytest.mark.parametrize("top", [5, 33])
def test_waves_of_many_problems_with_alternatives(top):
    rng = np.random.default_rng(top)
    check(mixed(rng, rng.integers(500, 1025, 1100)), 0.9, 3, top)


@pytest.mark.parametrize("top", [0, 7])
def test_long_problems_among_waves(top):
    """Longer than 1,024, by the whole workgroup behind the waves' own; two of them in one workgroup."""
    rng = np.random.default_rng(top)
    lengths = [*rng.integers(0, 40, 60), 1025, 0, 3000, 5, 40, 9000, 1024]
    check(mixed(rng, lengths), 1.1, 4, top)
    check(mixed(rng, lengths), 0.0, 4, top)


@pytest.mark.parametrize("top", [0, 10, 64])
@pytest.mark.parametrize("P,n", [(20, 3000), (300, 2500), (8, 6000), (300, 9000), (6, 20_000)])
def test_a_workgroup_a_problem(P, n, top):
    """256 threads, 256, 512, 512 and 1,024."""
    rng = np.random.default_rng(n + top)
    check(mixed(rng, n + rng.integers(-40, 40, P)), 0.8, 4, top)


@pytest.mark.parametrize("P,n", [(3, 200_000), (100, 34_000)])
@pytest.mark.parametrize("top", [0, 64])
def test_parts(P, n, top):
    rng = np.random.default_rng(P + top)
    check(mixed(rng, n + rng.integers(0, 9, P), ("ties", "holes", "plain", "peaked")), 1.3, 6, top)


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("lengths", [[5, 64, 200, 700, 1000], [3000, 2500, 3500], [6000, 5000, 7000], [20_000, 9000], [120_000, 80_000, 0]])
def test_the_first_best_alone(lengths, top):
    """T <= 0, of all problems and of every second one, on each way; the best score is there many times ("ties", "equal")."""
    rng = np.random.default_rng(len(lengths) + lengths[0])
    parts = mixed(rng, lengths, ("ties", "equal", "holes"))
    check(parts, 0.0, 5, top)
    check(parts, np.where(np.arange(len(parts)) % 2 == 0, 0.0, 0.6).astype(np.float32), 5, top)
    check(parts, np.where(np.arange(len(parts)) % 2 == 0, 0.6, -1.0).astype(np.float32), 5, top)


def test_picks_of_the_first_best():
    """T <= 0: picks of the first best candidate have log probability 0, of its equals none."""
    for n in (40, 900, 3000, 6000, 20_000, 100_000):
        s = torch.zeros(2 * n, device="cuda")
        s[n // 3], s[n // 2], s[n - 1] = 2.0, 2.0, 2.0
        s[n + n - 1] = 1.0
        seg = torch.tensor([0, n, 2 * n], device="cuda")
        picks = torch.tensor([[n // 3, n // 2, n - 1, 0], [n - 1, 0, 1, -1]], dtype=torch.int32, device="cuda")
        for top in (0, 1):
            logp, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks, temperature=0.0, top=top)
            none = -float("inf")
            assert logp.tolist() == [[0.0, none, none, none], [0.0, none, none, 0.0]], n
            assert entropy.tolist() == [0.0, 0.0] and norm.tolist() == [[2.0, 0.0], [1.0, 0.0]]


def test_gradients_of_more_problems_than_one_launch_has():
    """A launch has 2^15 problems of more than 1,024 candidates."""
    P, n = 33_000, 1100
    g = torch.Generator(device="cuda").manual_seed(4)
    s = torch.randn(P * n, generator=g, device="cuda")
    seg = torch.arange(P + 1, device="cuda") * n
    picks = torch.randint(0, n, (P, 3), generator=g, device="cuda", dtype=torch.int32)
    d, de = torch.randn(P, 3, generator=g, device="cuda"), torch.randn(P, generator=g, device="cuda")
    _, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks)
    out = torch.full((P * n,), float("nan"), device="cuda")
    hwsel.hwsel_logprob_gradient(s, seg, norm, picks, d, entropy, de, out=out)
    assert bool(torch.isfinite(out).all())
    for p in (0, 1, 2 ** 15 - 1, 2 ** 15, 2 ** 15 + 1, P - 1):
        want, bound = Logprob(s[p * n:(p + 1) * n].cpu().numpy()).gradient(picks[p].tolist(), d[p].tolist(), float(de[p]))
        near(out[p * n:(p + 1) * n], torch.from_numpy(want), torch.from_numpy(bound), f"gradient of {p}")
