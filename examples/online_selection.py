"""Learning which kernel to run while running it, in 8 bits: one round.

The features of every (problem, candidate) row are standardised and kept in 8
bits (a quarter of fp32); two 8-bit layers with GELU and a last product score
them; a few candidates of every problem are drawn by temperature, top-k and
top-p, to be timed; the regret of the draws is what the round is judged by.
The drawn rows' gradient of a loss on their runtimes then goes back through
the layers: from the 8-bit activations for the weights, by 8-bit products with
E5M2 gradients for the inputs.

    python examples/online_selection.py [--workload tiny] [--rounds 5]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synth  # noqa: E402
from paper_2609_35587_amd import hwsel  # noqa: E402

E5M2 = hwsel.FP8_E5M2


class Net:
    """n_features -> 512 -> 256 -> 1.  Weights live in fp32 beside their 8-bit forms."""

    def __init__(self, n_features, generator, device):
        sizes = [n_features, 512, 256, 1]
        self.W = [torch.randn(n, k, generator=generator, device=device) * (2.0 / k) ** 0.5 for k, n in zip(sizes, sizes[1:])]
        self.b = [torch.zeros(n, device=device) for n in sizes[1:]]
        self.lay_out()

    def lay_out(self):
        quantise = hwsel.hwsel_fp8_quantise
        self.w8 = [quantise(w, block_rows=128) for w in self.W]
        self.w8t = [quantise(w, block_rows=128, transpose=True) for w in self.W]

    def forward(self, x8):
        """Scores fp32 [rows], and the 8-bit input of each layer."""
        h1 = hwsel.hwsel_fp8_layer(x8, self.w8[0], bias=self.b[0], gelu=True)
        h2 = hwsel.hwsel_fp8_layer(h1, self.w8[1], bias=self.b[1], gelu=True)
        y = hwsel.hwsel_fp8_matmul(h2, self.w8[2], torch.float32, bias=self.b[2])
        return y[:, 0], [x8, h1, h2]

    def gelu_slope(self, i, x8):
        """GELU's derivative where layer i's sums were (they are made again, not kept)."""
        a = hwsel.hwsel_fp8_matmul(x8, self.w8[i], torch.float32, bias=self.b[i])
        cdf = 0.5 * (1.0 + torch.erf(a * 0.5 ** 0.5))
        return cdf + a * torch.exp(-0.5 * a * a) * (2.0 * torch.pi) ** -0.5

    def step(self, inputs, d_scores, rate):
        """One step of gradient descent; d_scores: the loss's gradient of the scores."""
        d = d_scores[:, None].contiguous()
        grads = []
        for i in (2, 1, 0):
            if i < 2:
                d = d * self.gelu_slope(i, inputs[i])
            d8t = hwsel.hwsel_fp8_quantise(d, format=E5M2, transpose=True)
            grads.append((i, hwsel.hwsel_fp8_matmul(d8t, hwsel.hwsel_fp8_transpose(inputs[i]), torch.float32), d.sum(0)))
            if i:
                d = hwsel.hwsel_fp8_matmul(hwsel.hwsel_fp8_quantise(d, format=E5M2), self.w8t[i], torch.float32)
        for i, dw, db in grads:
            self.W[i] -= rate * dw
            self.b[i] -= rate * db
        self.lay_out()


def take_rows(m, rows):
    """Rows of an 8-bit matrix whose scales are one to a row."""
    return dict(m, q=m["q"][rows], scale=m["scale"][rows], rows=rows.numel())


def run(workload="tiny", rounds=5, draws=8, device="cuda", seed=0, say=print):
    """Mean regret of each round's best draw."""
    w = synth.workload(workload)
    cfg, P = w.cfg, w.problems.shape[0]
    probs, seg = hwsel.to_device(w.problems, device), hwsel.to_device(w.seg, device)
    cands = {n: hwsel.to_device(v, device) for n, v in w.cands.items()}
    runtimes = hwsel.to_device(w.runtimes, device)
    X = hwsel.hwsel_features(w.hw, probs, seg, cands, cfg.n_features)
    clean = torch.where(torch.isfinite(X), X, 0.0)
    inv_std = 1.0 / clean.std(0).clamp(min=1e-6)
    x8 = hwsel.hwsel_fp8_quantise(X, mean=clean.mean(0), inv_std=inv_std)
    g = torch.Generator(device=device).manual_seed(seed)
    net = Net(cfg.n_features, g, device)
    # what a score should be: minus the log of the runtime against its problem's mean
    owner = torch.repeat_interleave(torch.arange(P, device=device), seg[1:] - seg[:-1])
    ran = torch.isfinite(runtimes) & (runtimes > 0)
    log_t = torch.where(ran, runtimes, 1.0).log()
    count = torch.zeros(P, device=device).index_add_(0, owner, ran.float()).clamp(min=1)
    target = (torch.zeros(P, device=device).index_add_(0, owner, log_t) / count)[owner] - log_t
    regrets = []
    for turn in range(rounds):
        scores, _ = net.forward(x8)
        u = torch.rand(P, draws, generator=g, device=device)
        idx, prob, kept = hwsel.hwsel_sample_per_problem(scores, seg, u, temperature=0.5, top_k=256, top_p=0.95)
        _, regret, _ = hwsel.hwsel_regret(runtimes, seg, idx)
        regrets.append(float(regret.mean()))
        say(f"round {turn}: mean regret of {draws} draws {regrets[-1]:.4f}, {float(kept.float().mean()):.0f} candidates kept")
        drawn = (seg[:-1, None] + idx)[idx >= 0].unique()   # each timed row once
        drawn = drawn[ran[drawn]]
        for _ in range(20):
            y, inputs = net.forward(take_rows(x8, drawn))
            net.step(inputs, (y - target[drawn]) / drawn.numel(), 0.02)
    return regrets


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--workload", choices=sorted(synth.CONFIGS), default="tiny")
    a.add_argument("--rounds", type=int, default=5)
    args = a.parse_args()
    run(args.workload, args.rounds)
