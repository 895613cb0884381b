"""Joins, dropout, draws and log probabilities run together: a ranker in fp32
against autograd in binary64, and the example's rounds and gradients."""
import importlib.util
import os

import pytest
import torch

from _learn_util import mask64
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("deep_selection", os.path.join(ROOT, "examples", "deep_selection.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def norm64(a, eps=1e-5):
    return a / torch.sqrt((a * a).mean(1, keepdim=True) + torch.tensor(eps, dtype=torch.float32).double())


def join64(x, y, gate, w_branch, w_pre, kept, scale):
    """A join as the example and the test below set it."""
    v = scale * torch.sigmoid(gate) * w_branch * norm64(y) * kept
    x = x + v
    return x, norm64(x) * w_pre


def loss64(scores, seg, picks, d_logp, d_entropy):
    total = 0.0
    for p in range(len(seg) - 1):
        lp = torch.log_softmax(scores[seg[p]:seg[p + 1]], 0)
        total = total + (d_logp[p].double() * lp[picks[p].long()]).sum() - d_entropy[p].double() * (lp.exp() * lp).sum()
    return total


def test_chain_in_fp32():
    """Two joins, a dropped-out readout and the loss, no product but a row's sum: the whole gradient within 1e-5 of its norm (some
    200 fp32 operations of 2^-24, a third of them additions of terms of one size, one after another)."""
    g = torch.Generator(device="cuda").manual_seed(3)
    R, C = 700, 152
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, ys, gates = r(R, C), [r(R, C) for _ in range(2)], [r(R, C) for _ in range(2)]
    wb, wp, out = [1 + 0.1 * r(C) for _ in range(2)], [1 + 0.1 * r(C) for _ in range(2)], r(C) * C ** -0.5
    joins = [dict(post_norm=True, gate_sigmoid=True, w_branch=wb[i], w_pre=wp[i], eps=1e-5, branch_scale=0.5, p=0.2, seed=i, offset=9) for i in range(2)]
    seg = torch.tensor([0, 100, 101, 400, 700], device="cuda")
    s0, z0 = hwsel.hwsel_block_join(joins[0], x, ys[0], gates[0])
    s1, z1 = hwsel.hwsel_block_join(joins[1], s0, ys[1] * z0, gates[1])
    dropped = hwsel.hwsel_dropout(z1, 0.25, 7, 8)
    scores = (dropped * out).sum(1)
    idx, _, _ = hwsel.hwsel_sample_per_problem(scores, seg, torch.rand(4, 6, generator=g, device="cuda"))
    _, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(scores, seg, idx)
    d_logp, d_entropy = r(4, 6), r(4)
    ds = hwsel.hwsel_logprob_gradient(scores, seg, norm, idx, d_logp, entropy, d_entropy)
    dz1 = hwsel.hwsel_dropout((ds[:, None] * out).contiguous(), 0.25, 7, 8)
    dx1, dy1, dg1, dwb1, dwp1 = hwsel.hwsel_block_join_gradient(joins[1], s1, ys[1] * z0, gates[1], None, dz1)
    dx0, dy0, dg0, dwb0, dwp0 = hwsel.hwsel_block_join_gradient(joins[0], s0, ys[0], gates[0], dx1, dy1 * ys[1])
    got = [dx0, dy0, dg0, dwb0, dwp0, dy1 * z0, dg1, dwb1, dwp1]

    leaves = [t.double().requires_grad_() for t in (x, ys[0], gates[0], wb[0], wp[0], ys[1], gates[1], wb[1], wp[1])]
    X, Y0, G0, B0, P0, Y1, G1, B1, P1 = leaves
    mask = lambda p, s, o: (lambda k: k[0].double().cuda() * k[1])(mask64(R, C, p, s, o))  # noqa: E731
    S0, Z0 = join64(X, Y0, G0, B0, P0, mask(0.2, 0, 9), 0.5)
    S1, Z1 = join64(S0, Y1 * Z0, G1, B1, P1, mask(0.2, 1, 9), 0.5)
    want_scores = (Z1 * mask(0.25, 7, 8) * out.double()).sum(1)
    assert float((scores.double() - want_scores).detach().norm() / want_scores.detach().norm()) < 1e-6
    loss64(want_scores, seg.tolist(), idx, d_logp, d_entropy).backward()
    for a, leaf in zip(got, leaves):
        assert float((a.double() - leaf.grad).norm()) <= 1e-5 * float(leaf.grad.norm())


def test_rounds():
    lines = []
    regrets = example().run("tiny", rounds=3, say=lines.append)
    assert len(regrets) == 3 and len(lines) == 4 and all(0.0 <= r <= 1.0 for r in regrets)


def test_example_follows_the_gradient():
    """The example's gradients against autograd in binary64 on unquantised values.  An operand of a gradient has been
    rounded to 3 (E4M3) or 2 (E5M2) digits up to six times on its way through two blocks: 2^-4 and 2^-3 at most for one
    element of random sign, some 3 and 7 % of the norm each, 15 % together; 35 % is asked, and a cosine of 0.94."""
    ex = example()
    g = torch.Generator(device="cuda").manual_seed(6)
    net = ex.Net(96, g, "cuda", width=128, hidden=256, dropout=0.1)
    x = torch.randn(600, 96, generator=g, device="cuda")
    W = {n: w.double().clone().requires_grad_() for n, w in net.W.items()}
    v = {n: w.double().clone().requires_grad_() for n, w in net.v.items()}
    s = x.double() @ W["in"].t()
    z = norm64(s) * v["pre"]
    for b in range(net.blocks):
        kept, factor = mask64(600, 128, 0.1, b, 4)
        y = torch.nn.functional.gelu(z @ W[f"up{b}"].t() + v[f"up{b}"]) @ W[f"down{b}"].t()
        s, z = join64(s, y, z @ W[f"gate{b}"].t() + v[f"gate{b}"], v[f"branch{b}"], v[f"pre{b}"], kept.double().cuda() * factor, 0.5)
    scores = (z @ W["out"].t())[:, 0]
    d = torch.randn(600, generator=g, device="cuda") / 600
    (scores * d.double()).sum().backward()
    got, saved = net.forward(hwsel.hwsel_fp8_quantise(x), 4)
    assert float((got.double() - scores).detach().norm() / scores.detach().norm()) < 0.2
    gW, gv = net.gradients(saved, d, 4)
    assert gW.keys() == W.keys() and gv.keys() == v.keys()
    for grads, leaves in ((gW, W), (gv, v)):
        for name, a in grads.items():
            a, want = a.double().flatten(), leaves[name].grad.flatten()
            assert float((a - want).norm()) <= 0.35 * float(want.norm()), name
            assert float(a @ want) >= 0.94 * float(a.norm() * want.norm()), name
