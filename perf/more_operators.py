"""The operators around an 8-bit ranker's products and draws, as cases that can be timed and checked.

A ranker deep enough to learn from its own draws is a stack of blocks on a residual stream: the
block's products run in 8 bits, and between two blocks the block's result is normed, gated, dropped
out, scaled and added to the stream, whose norm is the next block's input ("join").  Hidden layers
are regularised by dropout whose mask is made again from a counter instead of kept.  What it learns
from is the log probability of the candidates that were drawn and timed, with the entropy of every
problem's distribution, and their gradient with respect to the scores; a report names the best
alternatives of a problem with their log probabilities.

Every case is one such call, or one forward and backward pass.  `run` makes it through the
framework's binding (own) or computes it in plain torch operations.

Dropout's random numbers are a function of inputs alone: the eight columns 8 g ... 8 g + 7 of row r
are the eight 16-bit halves, low half first, of the four words of Philox4x32-10 (Salmon, Moraes,
Dror and Shaw, 2011) with the counter (g, r, offset's low word, offset's high word) and the key
(seed's low word, seed's high word).  An element is kept where its number is at least p 2^16
(rounded) and is then divided by the share that is kept.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"


# ----------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------
def listed():
    return [
        # A few problems of 512 candidates, the log probability of the one that was chosen and five alternatives: the
        # smallest call, while a caller waits.
        dict(name="logprob-small", kind="logprob", P=16, C=512, ragged=False, picks=1, top=5, temperature=1.0,
             per_problem=False, ties=0.0, train=False),
        # A report over the data set: ragged problems, 64 timed candidates and ten alternatives of each, a temperature of its own for every problem.
        dict(name="logprob-dataset", kind="logprob", P=600, C=8192, ragged=True, picks=64, top=10, temperature=1.0,
             per_problem=True, ties=0.2, train=False),
        # Few problems over the whole catalogue of 534,600 points.
        dict(name="logprob-long", kind="logprob", P=3, C=534_600, ragged=False, picks=8, top=16, temperature=1.5,
             per_problem=False, ties=0.1, train=False),
        # A training step on the data set's draws: log probabilities and entropies, then the scores' gradient.
        dict(name="logprob-train", kind="logprob", P=600, C=8192, ragged=True, picks=64, top=0, temperature=0.7,
             per_problem=False, ties=0.2, train=True),
        # The same over the whole 65,536-point grid of 256 problems.
        dict(name="logprob-train-grid", kind="logprob", P=256, C=65_536, ragged=False, picks=16, top=0, temperature=1.0,
             per_problem=True, ties=0.0, train=True),
        # One row of a hidden layer: the smallest call.
        dict(name="dropout-row", kind="dropout", R=1, C=1024, dtype="bf16", p=0.1, residual=False, pad=0, train=False),
        # A training batch: onto the residual stream, and the gradient back.
        dict(name="dropout-batch", kind="dropout", R=65_536, C=1024, dtype="bf16", p=0.1, residual=True, pad=0, train=True),
        # Odd sizes, rows at odd places, fp32.
        dict(name="dropout-odd", kind="dropout", R=4099, C=2500, dtype="fp32", p=0.3, residual=False, pad=3, train=False),
        # One row between two blocks of a scorer that answers one request at a time.
        dict(name="join-row", kind="join", R=1, C=1024, stream="bf16", block="bf16", post_norm=True, gate="none",
             sigmoid=False, p=0.0, pad=0, train=False),
        # A scoring run's rows between two blocks: fp32 stream, bf16 blocks, a gate for every element.
        dict(name="join-bulk", kind="join", R=1_048_576, C=512, stream="fp32", block="bf16", post_norm=True, gate="element",
             sigmoid=True, p=0.0, pad=0, train=False),
        # A training batch: forward and all gradients, with gate and dropout.
        dict(name="join-train", kind="join", R=65_536, C=1024, stream="bf16", block="bf16", post_norm=True, gate="element",
             sigmoid=True, p=0.1, pad=0, train=True),
        # Odd sizes in fp32, a gate for every row, rows at odd places.
        dict(name="join-train-odd", kind="join", R=4099, C=2500, stream="fp32", block="fp32", post_norm=True, gate="row",
             sigmoid=False, p=0.0, pad=3, train=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "dropout", "join", "join"])
    if kind == "logprob":
        P = _log(rng, 1, 4096)
        C = _log(rng, 1, max(1, min(534_600, 16_000_000 // P)))
        train = rng.random() < 0.5
        return dict(kind=kind, P=P, C=C, ragged=rng.random() < 0.5, picks=_log(rng, 1, 256),
                    top=0 if train else rng.choice([0, _log(rng, 1, 64)]), temperature=rng.uniform(0.2, 3.0),
                    per_problem=rng.random() < 0.5, ties=rng.choice([0.0, 0.3, 1.0]), train=train)
    if kind == "dropout":
        C = _log(rng, 1, 65_536)
        return dict(kind=kind, R=_log(rng, 1, max(1, min(1_000_000, 67_000_000 // C))), C=C, dtype=rng.choice(["bf16", "fp32"]),
                    p=rng.uniform(0.0, 0.9), residual=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 8]), train=rng.random() < 0.5)
    C = _log(rng, 8, 32_768)
    return dict(kind=kind, R=_log(rng, 1, max(1, min(1_000_000, 67_000_000 // C))), C=C, stream=rng.choice(["bf16", "fp32"]),
                block=rng.choice(["bf16", "fp32"]), post_norm=rng.random() < 0.5, gate=rng.choice(["none", "row", "element"]),
                sigmoid=rng.random() < 0.5, p=rng.choice([0.0, rng.uniform(0.05, 0.5)]), pad=rng.choice([0, 0, 1, 8]),
                train=rng.random() < 0.5)


def _size(dtype):
    return 4 if dtype == "fp32" else 2


def work(case):
    c = case
    if c["kind"] == "logprob":
        rows, P, n = sum(_lengths(c)), c["P"], c["picks"]
        b = 4 * rows + P * (8 + 8 * n + 12 + 8 * c["top"])
        return {"bytes": b + (4 * rows + P * (4 * n + 4) if c["train"] else 0), "flops": rows * (12 if c["train"] else 6)}
    n = c["R"] * c["C"]
    if c["kind"] == "dropout":
        one = n * _size(c["dtype"])
        return {"bytes": one * (2 + c["residual"] + (2 if c["train"] else 0)), "flops": 3 * n}
    s, b = _size(c["stream"]), _size(c["block"])
    gate = {"none": 0, "row": b * c["R"], "element": b * n}[c["gate"]]
    out = {"bytes": n * (2 * s + 2 * b) + gate + 8 * c["C"], "flops": 10 * n}
    if c["train"]:
        # the stream, the block's result, the gate and two gradients read; the gradients of the first three written
        out = {"bytes": out["bytes"] + n * (3 * s + 3 * b) + 2 * gate + 16 * c["C"], "flops": 30 * n}
    return out


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------
def _lengths(case):
    P, C = case["P"], case["C"]
    if not case["ragged"]:
        return [C] * P
    rng = np.random.default_rng(1_000_003 * P + C)         # shapes go by the case, values by the seed
    n = rng.integers(0, C + 1, P)
    n[rng.random(P) < 0.02] = 0                            # problems without a valid candidate
    n[rng.integers(0, P)] = C
    return [int(v) for v in n]


def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _matrix(gen, R, C, name, pad, sd=1.0):
    """Activations with a few large units, their rows `pad` elements further apart than they are long."""
    x = torch.randn(R, C + pad, generator=gen, device=DEV).mul_(sd)
    x.mul_(torch.exp(0.5 * torch.randn(1, C + pad, generator=gen, device=DEV)))
    return x.to(_type(name))[:, :C]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    c, st = case, dict(case=dict(case))
    if c["kind"] == "logprob":
        P, n = c["P"], _lengths(c)
        seg = np.zeros(P + 1, np.int64)
        seg[1:] = np.cumsum(n)
        R = int(seg[-1])
        s = 2.0 * torch.randn(max(R, 1), generator=g, device=DEV)
        tied = torch.rand(max(R, 1), generator=g, device=DEV) < c["ties"]
        s = torch.where(tied, torch.round(2.0 * s) / 2.0, s)        # sums of few tree leaves: equal scores
        dead = torch.rand(max(R, 1), generator=g, device=DEV)
        s[dead < 0.05] = float("-inf")                              # infeasible configurations
        s[dead > 0.999] = float("nan")
        seg = torch.from_numpy(seg).to(DEV)
        # drawn candidates, the same one twice now and then, fewer than asked for (-1) in some problems
        u = torch.rand(P, c["picks"], generator=g, device=DEV)
        picks = (u * (seg[1:] - seg[:-1])[:, None]).to(torch.int32)
        if c["picks"] > 1:
            picks[::7, -1] = -1
            picks[::3, -1] = picks[::3, 0]
        st.update(scores=s[:R], seg=seg, longest=max(n), rows=R, picks=picks)
        st["temperature"] = c["temperature"] * (0.5 + torch.rand(P, generator=g, device=DEV)) if c["per_problem"] else c["temperature"]
        if c["train"]:
            st["d_logp"] = torch.randn(P, c["picks"], generator=g, device=DEV) / (P * c["picks"])
            st["d_entropy"] = torch.full((P,), -0.01 / P, device=DEV)
        return st
    R, C = c["R"], c["C"]
    st["seed"], st["offset"] = int(seed) * 0x9E3779B97F4A7C15 % (1 << 63), int(seed) % 1000
    if c["kind"] == "dropout":
        st["x"] = _matrix(g, R, C, c["dtype"], c["pad"])
        st["residual"] = _matrix(g, R, C, c["dtype"], c["pad"], 3.0) if c["residual"] else None
        st["dy"] = _matrix(g, R, C, c["dtype"], c["pad"], 1e-3) if c["train"] else None
        return st
    st["x"], st["y"] = _matrix(g, R, C, c["stream"], c["pad"], 3.0), _matrix(g, R, C, c["block"], c["pad"])
    width = {"none": 0, "row": 1, "element": C}[c["gate"]]
    st["gate"] = _matrix(g, R, width, c["block"], c["pad"]) if width else None
    st["w_branch"], st["w_pre"] = (1.0 + 0.2 * torch.randn(C, generator=g, device=DEV) for _ in range(2))
    if c["train"]:
        st["d_x1"], st["d_z"] = _matrix(g, R, C, c["stream"], c["pad"], 1e-3), _matrix(g, R, C, c["block"], c["pad"], 1e-3)
    st["join"] = dict(post_norm=c["post_norm"], gate_sigmoid=c["sigmoid"], w_branch=st["w_branch"], w_pre=st["w_pre"], eps=1e-5,
                      stream_scale=1.0, branch_scale=0.5, p=c["p"], seed=st["seed"], offset=st["offset"])
    return st


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------
def run(state):
    return run_own(state) if own else run_plain(state)


def run_own(st):
    from paper_2609_35587_amd import hwsel
    c = st["case"]
    if c["kind"] == "logprob":
        logp, entropy, norm, top_idx, top_logp = hwsel.hwsel_logprob_per_problem(
            st["scores"], st["seg"], st["picks"], temperature=st["temperature"], top=c["top"])
        out = {"logp": logp, "entropy": entropy, "norm": norm}
        if c["top"]:
            out.update(top_idx=top_idx, top_logp=top_logp)
        if c["train"]:
            out["d_scores"] = hwsel.hwsel_logprob_gradient(
                st["scores"], st["seg"], norm, st["picks"], st["d_logp"], entropy, st["d_entropy"], temperature=st["temperature"])
        return out
    if c["kind"] == "dropout":
        out = {"y": hwsel.hwsel_dropout(st["x"], c["p"], st["seed"], st["offset"], residual=st["residual"])}
        if c["train"]:
            out["dx"] = hwsel.hwsel_dropout(st["dy"], c["p"], st["seed"], st["offset"])
        return out
    x1, z = hwsel.hwsel_block_join(st["join"], st["x"], st["y"], st["gate"])
    out = {"x1": x1, "z": z}
    if c["train"]:
        dx, dy, dgate, dw_branch, dw_pre = hwsel.hwsel_block_join_gradient(st["join"], x1, st["y"], st["gate"], st["d_x1"], st["d_z"])
        out.update(dx=dx, dy=dy, dw_branch=dw_branch, dw_pre=dw_pre)
        if st["gate"] is not None:
            out["dgate"] = dgate
    return out


def run_plain(st):
    kind = st["case"]["kind"]
    return plain_logprob(st) if kind == "logprob" else plain_dropout(st) if kind == "dropout" else plain_join(st)


def plain_logprob(st):
    c, seg, R, picks = st["case"], st["seg"], st["rows"], st["picks"].long()
    P, L = seg.numel() - 1, max(1, st["longest"])
    T = st["temperature"] if isinstance(st["temperature"], torch.Tensor) else torch.full((P,), st["temperature"], device=DEV)
    length = (seg[1:] - seg[:-1])[:, None]
    col = torch.arange(L, device=DEV)
    valid = col[None, :] < length
    at = (seg[:-1, None] + col).clamp(max=max(R - 1, 0))
    s = st["scores"][at] + 0.0 if R else torch.zeros(P, L, device=DEV)
    s = torch.where(valid & ~torch.isnan(s), s, float("-inf"))
    best = s.amax(1)
    alive = best > float("-inf")
    t = (s - torch.where(alive, best, 0.0)[:, None]) / T[:, None]
    e = torch.exp(t)
    mass = e.sum(1)
    log_mass = torch.log(mass)
    lp = t - torch.where(alive, log_mass, 0.0)[:, None]
    entropy = torch.where(alive, log_mass - torch.where(e > 0, e * t, 0.0).sum(1) / mass, 0.0)
    here = (picks >= 0) & (picks < length)
    logp = torch.where(here, lp.gather(1, picks.clamp(0, L - 1)), 0.0)
    out = {"logp": logp, "entropy": entropy, "norm": torch.stack([best, log_mass], 1)}
    if c["top"]:
        k = min(c["top"], L)
        order = torch.sort(s, dim=1, descending=True, stable=True)
        top_idx = torch.full((P, c["top"]), -1, dtype=torch.int32, device=DEV)
        top_logp = torch.full((P, c["top"]), float("-inf"), device=DEV)
        some = order.values[:, :k] > float("-inf")
        top_idx[:, :k] = torch.where(some, order.indices[:, :k].to(torch.int32), -1)
        top_logp[:, :k] = torch.where(some, lp.gather(1, order.indices[:, :k]), float("-inf"))
        out.update(top_idx=top_idx, top_logp=top_logp)
    if c["train"]:
        p = e / torch.where(alive, mass, 1.0)[:, None]
        d = torch.where(here & (logp > float("-inf")), st["d_logp"], 0.0)
        grad = torch.zeros_like(s).scatter_add_(1, picks.clamp(0, L - 1), d) - p * d.sum(1, keepdim=True)
        grad = grad - st["d_entropy"][:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
        out["d_scores"] = (grad / T[:, None])[valid]
    return out


M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _product(a, b):
    """High and low word of the product of the 32-bit numbers a and b (int64 tensors)."""
    high, low = a * (b >> 16), a * (b & 0xFFFF)
    return (high + (low >> 16)) >> 16, (low + ((high & 0xFFFF) << 16)) & LOW


def plain_kept(R, C, p, seed, offset):
    """Where the mask keeps, and what is kept is multiplied by."""
    G = -(-C // 8)
    full = lambda v: torch.full((R, G), v, dtype=torch.int64, device=DEV)  # noqa: E731
    c0, c1 = torch.arange(G, device=DEV).expand(R, G), torch.arange(R, device=DEV)[:, None].expand(R, G)
    c2, c3, k0, k1 = full(offset & LOW), full(offset >> 32), seed & LOW, seed >> 32
    for i in range(10):
        h0, l0 = _product(c0, M0)
        h1, l1 = _product(c2, M1)
        c0, c1, c2, c3 = h1 ^ c1 ^ ((k0 + i * W0) & LOW), l1, h0 ^ c3 ^ ((k1 + i * W1) & LOW), l0
    words = torch.stack([c0, c1, c2, c3], 2)
    halves = torch.stack([words & 0xFFFF, words >> 16], 3).view(R, 8 * G)[:, :C]
    least = _least(p)
    return halves >= least, 65536.0 / (65536 - least) if least < 65536 else 0.0


def _least(p):
    return int(np.rint(np.float32(p) * np.float32(65536.0)))


def plain_dropout(st):
    c = st["case"]
    R, C = c["R"], c["C"]
    kept, factor = plain_kept(R, C, c["p"], st["seed"], st["offset"])
    y = torch.where(kept, st["x"].float() * factor, 0.0)
    y = y if st["residual"] is None else y + st["residual"].float()
    out = {"y": y.to(_type(c["dtype"]))}
    if c["train"]:
        out["dx"] = torch.where(kept, st["dy"].float() * factor, 0.0).to(_type(c["dtype"]))
    return out


def plain_join(st):
    c, j = st["case"], st["join"]
    R, C, stream, block = c["R"], c["C"], _type(c["stream"]), _type(c["block"])
    x, y, eps = st["x"].float(), st["y"].float(), j["eps"]
    scale = torch.rsqrt(y.square().mean(1, keepdim=True) + eps) if c["post_norm"] else 1.0
    yn = y * scale
    u = yn * j["w_branch"]
    gate = 1.0 if st["gate"] is None else st["gate"].float()
    g = torch.sigmoid(gate) if c["sigmoid"] and st["gate"] is not None else gate
    kept, factor = plain_kept(R, C, c["p"], st["seed"], st["offset"]) if c["p"] > 0 else (torch.ones((), dtype=torch.bool, device=DEV), 1.0)
    v = torch.where(kept, j["branch_scale"] * factor * g * u, 0.0)
    x1 = j["stream_scale"] * x + v
    z = x1 * torch.rsqrt(x1.square().mean(1, keepdim=True) + eps) * j["w_pre"]
    out = {"x1": x1.to(stream), "z": z.to(block)}
    if not c["train"]:
        return out
    # the gradients at the stream as it is kept
    x1 = out["x1"].float()
    r = torch.rsqrt(x1.square().mean(1, keepdim=True) + eps)
    xn = x1 * r
    dz = st["d_z"].float()
    out["dw_pre"] = (dz * xn).sum(0)
    dn = dz * j["w_pre"]
    d = st["d_x1"].float() + r * (dn - xn * (dn * xn).mean(1, keepdim=True))
    out["dx"] = (j["stream_scale"] * d).to(stream)
    dv = torch.where(kept, j["branch_scale"] * factor * d, 0.0)
    if st["gate"] is not None:
        dg = dv * u
        dg = dg.sum(1, keepdim=True) if c["gate"] == "row" else dg
        out["dgate"] = (dg * g * (1.0 - g) if c["sigmoid"] else dg).to(block)
    du = dv * g
    out["dw_branch"] = (du * yn).sum(0)
    dn = du * j["w_branch"]
    out["dy"] = (scale * (dn - yn * (dn * yn).mean(1, keepdim=True)) if c["post_norm"] else dn).to(block)
    return out


# ----------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    return _logprob64(st) if kind == "logprob" else _dropout64(st) if kind == "dropout" else _join64(st)


def _logprob64(st):
    """One problem after another, gradients by differentiating the sum that the given gradients weight."""
    c = st["case"]
    seg = st["seg"].tolist()
    P, n, k = c["P"], c["picks"], c["top"]
    T = st["temperature"].double() if isinstance(st["temperature"], torch.Tensor) else torch.full((P,), np.float32(st["temperature"]), dtype=torch.float64, device=DEV)
    f8 = dict(dtype=torch.float64, device=DEV)
    out = {"logp": torch.zeros(P, n, **f8), "entropy": torch.zeros(P, **f8), "norm": torch.full((P, 2), -math.inf, **f8)}
    if k:
        out.update(top_idx=torch.full((P, k), -1, dtype=torch.int32, device=DEV), top_logp=torch.full((P, k), -math.inf, **f8))
    grad = torch.zeros(st["rows"], **f8)
    for p in range(P):
        s = st["scores"][seg[p]:seg[p + 1]]
        live = torch.nonzero(s > -math.inf)[:, 0]          # neither NaN nor -inf
        if not live.numel():
            picks = st["picks"][p].long()
            out["logp"][p] = torch.where((picks >= 0) & (picks < s.numel()), -math.inf, 0.0)
            continue
        a = s[live].double().requires_grad_(c["train"])
        lp = torch.log_softmax(a / T[p], 0)
        entropy = -(torch.exp(lp) * lp).sum()
        every = torch.full((s.numel(),), -math.inf, **f8).index_put((live,), lp)
        picks = st["picks"][p].long()
        inside = (picks >= 0) & (picks < s.numel())
        logp = torch.where(inside, every[picks.clamp(0, s.numel() - 1)], torch.zeros((), **f8))
        with torch.no_grad():
            out["logp"][p], out["entropy"][p] = logp, entropy
            out["norm"][p, 0] = a.max()
            out["norm"][p, 1] = torch.logsumexp((a - a.max()) / T[p], 0)
            if k:
                order = torch.sort(s[live], descending=True, stable=True).indices[:k]
                out["top_idx"][p, : len(order)] = live[order].to(torch.int32)
                out["top_logp"][p, : len(order)] = lp[order]
        if c["train"]:
            counts = inside & (logp > -math.inf)
            loss = (torch.where(counts, st["d_logp"][p].double(), 0.0) * torch.where(counts, logp, 0.0)).sum() + st["d_entropy"][p].double() * entropy
            grad[seg[p] + live] = torch.autograd.grad(loss, a)[0]
    if c["train"]:
        out["d_scores"] = grad
    return out


def _factor64(c, st, lo, hi):
    """What the mask multiplies rows lo to hi by, in numpy's unsigned 64-bit numbers."""
    u8 = np.uint64
    G = -(-c["C"] // 8)
    word = [np.broadcast_to(np.arange(G, dtype=u8), (hi - lo, G)), np.broadcast_to(np.arange(lo, hi, dtype=u8)[:, None], (hi - lo, G)),
            np.full((hi - lo, G), st["offset"] % 2**32, u8), np.full((hi - lo, G), st["offset"] >> 32, u8)]
    key = [st["seed"] % 2**32, st["seed"] >> 32]
    for _ in range(10):
        p0, p1 = word[0] * u8(0xD2511F53), word[2] * u8(0xCD9E8D57)
        word = [(p1 >> u8(32)) ^ word[1] ^ u8(key[0]), p1 & u8(0xFFFFFFFF), (p0 >> u8(32)) ^ word[3] ^ u8(key[1]), p0 & u8(0xFFFFFFFF)]
        key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
    number = np.stack(word, 2).astype(np.uint32).view(np.uint16).reshape(hi - lo, 8 * G)[:, : c["C"]]
    dropped = round(float(np.float32(c["p"])) * 65536.0)
    share = (65536 - dropped) / 65536
    return torch.from_numpy(number.astype(np.int32)).to(DEV).ge(dropped).double() * (1.0 / share if share else 0.0)


STEP = 1 << 24                                              # elements that are worked on at once


def _spans(c):
    rows = max(1, STEP // c["C"])
    return [(lo, min(c["R"], lo + rows)) for lo in range(0, c["R"], rows)]


def _dropout64(st):
    c = st["case"]
    out = {"y": torch.empty(c["R"], c["C"], dtype=torch.float64, device=DEV)}
    if c["train"]:
        out["dx"] = torch.empty_like(out["y"])
    for lo, hi in _spans(c):
        m = _factor64(c, st, lo, hi)
        out["y"][lo:hi] = m * st["x"][lo:hi].double()
        if st["residual"] is not None:
            out["y"][lo:hi] += st["residual"][lo:hi].double()
        if c["train"]:
            out["dx"][lo:hi] = m * st["dy"][lo:hi].double()
    return out


def _join64(st):
    """Rows in parts; gradients by differentiating the parts' weighted sums."""
    c, j = st["case"], st["join"]
    R, C = c["R"], c["C"]
    eps, branch, stream = (float(np.float32(j[n])) for n in ("eps", "branch_scale", "stream_scale"))
    f8 = dict(dtype=torch.float64, device=DEV)
    normed = lambda a: a / torch.sqrt((a * a).sum(1, keepdim=True) / C + eps)  # noqa: E731
    out = {"x1": torch.empty(R, C, **f8), "z": torch.empty(R, C, **f8)}
    if c["train"]:
        out.update(dx=torch.empty(R, C, **f8), dy=torch.empty(R, C, **f8), dw_branch=torch.zeros(C, **f8), dw_pre=torch.zeros(C, **f8))
        if st["gate"] is not None:
            out["dgate"] = torch.empty(st["gate"].shape, **f8)
    for lo, hi in _spans(c):
        m = _factor64(c, st, lo, hi) if c["p"] > 0 else torch.ones((), **f8)
        x, y, wb, wp = st["x"][lo:hi].double(), st["y"][lo:hi].double(), j["w_branch"].double(), j["w_pre"].double()
        gate = None if st["gate"] is None else st["gate"][lo:hi].double()
        leaves = [t.requires_grad_(c["train"]) for t in (y, wb, gate) if t is not None]
        v = branch * m * wb * (normed(y) if c["post_norm"] else y)
        if gate is not None:
            v = v * (1.0 / (1.0 + torch.exp(-gate)) if c["sigmoid"] else gate)
        x1 = stream * x + v
        with torch.no_grad():
            out["x1"][lo:hi], out["z"][lo:hi] = x1, normed(x1) * wp
        if not c["train"]:
            continue
        kept = x1.detach().to(_type(c["stream"])).double().requires_grad_()      # as the stream is kept
        wp.requires_grad_()
        through, dwp = torch.autograd.grad((st["d_z"][lo:hi].double() * normed(kept) * wp).sum(), (kept, wp))
        d = st["d_x1"][lo:hi].double() + through
        grads = torch.autograd.grad((d * v).sum(), leaves)
        with torch.no_grad():
            out["dx"][lo:hi], out["dy"][lo:hi] = stream * d, grads[0]
            out["dw_branch"] += grads[1]
            out["dw_pre"] += dwp
            if gate is not None:
                out["dgate"][lo:hi] = grads[2]
    return out
