"""64-bit statements of the 8-bit operators for the tests: codes by the grid's
spacing, values bit by bit, products and draws from their definitions."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2609_35587_amd import hwsel

E4M3, E5M2 = hwsel.FP8_E4M3, hwsel.FP8_E5M2
DIGITS, LOWEST, TOP = {E4M3: 3, E5M2: 2}, {E4M3: -6, E5M2: -14}, {E4M3: 448.0, E5M2: 57344.0}


def grid_values(x: torch.Tensor, fmt: int, block_rows: int = 1):
    """Values and exponents e of quantised x (any float dtype; computed in
    binary64): per block the least e >= -126 with amax <= TOP 2^e over the
    finite elements (-126 for zeros), values rounded to the grid, ties to even."""
    x = x.double()
    R, C = x.shape
    rb, kb = -(-R // block_rows), -(-C // 128)
    z = torch.zeros(rb * block_rows, kb * 128, dtype=torch.float64, device=x.device)
    z[:R, :C] = x
    z = z.view(rb, block_rows, kb, 128)
    finite = torch.isfinite(z)
    amax = torch.where(finite, z.abs(), 0.0).amax(dim=(1, 3))
    m, e = torch.frexp(amax / TOP[fmt])                     # amax / TOP = m 2^e, m in [1/2, 1)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-126)
    e = torch.where(amax == 0, -126, e)
    s = torch.exp2(e.double())[:, None, :, None]
    v = torch.where(finite, z, 0.0) / s
    _, x2 = torch.frexp(v)
    step = torch.exp2((x2 - 1).clamp(min=LOWEST[fmt]).double() - DIGITS[fmt])
    q = torch.round(v / step) * step * s
    q = torch.where(finite, q, z if fmt == E5M2 else torch.full_like(z, math.nan))
    return q.view(rb * block_rows, kb * 128)[:R, :C], e


def code_values(m: dict) -> torch.Tensor:
    """Values of an 8-bit operand in binary64, from its bits."""
    q = m["q"].to(torch.int32)
    ebits, mbits, bias = (4, 3, 7) if m["format"] == E4M3 else (5, 2, 15)
    e, f = (q >> mbits) & ((1 << ebits) - 1), (q & ((1 << mbits) - 1)).double() / (1 << mbits)
    v = torch.where(e == 0, f * 2.0 ** (1 - bias), (1.0 + f) * torch.exp2((e - bias).double()))
    top = e == (1 << ebits) - 1
    if m["format"] == E4M3:
        v = torch.where(top & (f == 7 / 8), math.nan, v)
    else:
        v = torch.where(top, torch.where(f == 0, math.inf, math.nan), v)
    v = torch.where(q >= 128, -v, v)
    dev = v.device
    rows, cols = torch.arange(m["rows"], device=dev) // m["block_rows"], torch.arange(m["cols"], device=dev) // 128
    byte = m["scale"].double()
    scale = torch.where(byte == 255, math.nan, torch.exp2(byte - 127.0))
    return v[: m["rows"], : m["cols"]] * scale[rows][:, cols]


def same_values(a: torch.Tensor, b: torch.Tensor) -> bool:
    a, b = a.double().cpu(), b.double().cpu()
    return bool(torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0)))


def random_rows(g, R, C, dev="cuda"):
    """Rows and columns of different sizes."""
    x = torch.randn(R, C, generator=g, device=dev)
    return x * torch.exp(torch.randn(R, 1, generator=g, device=dev)) * torch.exp(torch.randn(1, C, generator=g, device=dev))


def gelu64(y: torch.Tensor) -> torch.Tensor:
    return 0.5 * y * torch.erfc(-y / math.sqrt(2.0))


EXP2 = tuple(np.float32(math.log(2.0) ** i / math.factorial(i)) for i in range(7))


def draws64(scores, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One problem's draws by the definition: (idx, prob, kept)."""
    f4 = np.float32
    n_draws = len(u)
    i = np.nonzero(scores > f4("-inf"))[0]
    if not len(i):
        return np.full(n_draws, -1), np.zeros(n_draws), 0
    T, tp, mp = f4(temperature), float(f4(top_p)), float(f4(min_p))
    order = np.lexsort((i, -(scores[i].astype(np.float64))))
    i = i[order]
    if not T > 0:
        i = i[:1]
    elif top_k > 0:
        i = i[:top_k]
    s = scores[i]
    with np.errstate(all="ignore"):
        rate = f4(np.float64(1.4426950408889634) / np.float64(T)) if T > 0 else f4(1)
        t = ((s - s[0]).astype(f4) * rate).astype(f4)
    t[s == s[0]] = 0
    t[~(t > -60)] = -60
    n = np.rint(t)
    f = (t - n).astype(f4)
    p = np.full(len(t), EXP2[6], f4)
    for a in EXP2[5::-1]:
        p = ((p * f).astype(f4) + a).astype(f4)
    w = [(int(pp * f4(16777216)) << 8) >> int(-nn) for pp, nn in zip(p, n)]
    least = max(1, math.ceil(min(max(mp if mp == mp else 0.0, 0.0), 1.0) * 4294967296.0))
    need = max(1, math.ceil(float(sum(w)) * max(tp, 0.0))) if tp < 1 else None
    keep, before = {}, 0
    for at, weight in zip(i, w):
        if weight >= least and (need is None or before < need):
            keep[int(at)] = weight
        before += weight
    total = sum(keep.values())
    idx, prob = [], []
    for x in u:
        v = math.floor(min(max(float(x), 0.0), 1.0) * 16777216.0) if x == x else 0
        r = total * min(v, (1 << 24) - 1) >> 24
        run = 0
        for at in sorted(keep):
            run += keep[at]
            if run > r:
                idx.append(at)
                prob.append(keep[at] / total)
                break
    return np.array(idx), np.array(prob), len(keep)
