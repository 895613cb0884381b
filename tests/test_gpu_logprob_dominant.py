"""Gradients of log probabilities where one candidate has nearly all of the probability and nearly all of the picks."""
import numpy as np
import pytest
import torch

from _learn_util import Logprob
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("P,n", [(1, 2), (9, 60), (3, 1000), (5, 3000), (300, 5000), (2, 60_000), (1, 534_600)])
@pytest.mark.parametrize("lead", [14.0, 40.0])
def test_the_others_picks(P, n, lead):
    """Candidate j's gradient is g_j (1 - p_j) - p_j (S - g_j): of the dominant one the first part is next to nothing
    and the second is the few other picks' sum, far below a step of S and g."""
    rng = np.random.default_rng(n + int(lead))
    picks = np.empty((P, 64), np.int32)
    d = np.empty((P, 64), np.float32)
    s = rng.standard_normal((P, n)).astype(np.float32)
    for p in range(P):
        best, other = rng.permutation(n)[:2]
        s[p, best] = lead
        picks[p] = best
        picks[p, 7] = other
        d[p] = rng.uniform(30.0, 60.0, 64)
        d[p, 7] = rng.uniform(1e-4, 2e-4)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    seg = torch.arange(P + 1, device="cuda") * n
    _, _, norm, _, _ = hwsel.hwsel_logprob_per_problem(dev(s.reshape(-1)), seg, dev(picks))
    got = hwsel.hwsel_logprob_gradient(dev(s.reshape(-1)), seg, norm, dev(picks), dev(d)).cpu().numpy().astype(np.float64).reshape(P, n)
    for p in range(P):
        q = Logprob(s[p])
        best, other = int(picks[p, 0]), int(picks[p, 7])
        g = float(np.delete(d[p], 7).astype(np.float64).sum())
        lp = q.lp[best]
        rest = -np.expm1(lp)                                # 1 - p
        want = g * rest - np.exp(lp) * float(d[p, 7])
        # 1 - p is -lp times a series, lp within em: relative to it em / |lp|, and 16 steps of operations.  Fixed point's
        # unit is 2^e for gradients below 2^6 and 64 of them: e = 6 + 7 - 62, half of it for each pick.
        bound = g * (q.em + 16 * U * rest) + float(d[p, 7]) * (q.em + 8 * U) + 64 * 2.0 ** -50 + 4 * U * abs(want)
        assert abs(got[p, best] - want) <= bound, (p, got[p, best], want, bound)
        want = float(d[p, 7]) * -np.expm1(q.lp[other]) - np.exp(q.lp[other]) * g
        err = q.elp[other] + (4 * abs(q.lp[other]) + 8) * U + q.em
        bound = 20 * U * float(d[p, 7]) + np.exp(q.lp[other]) * g * (err + 8 * U) + 64 * 2.0 ** -50
        assert abs(got[p, other] - want) <= bound, (p, got[p, other], want, bound)
