"""64-bit statements of log probabilities, dropout and joins for the tests, with
bounds on how far a kernel in fp32 may be from them.

u = 2^-24 is half a step of fp32: an operation's result is within u of it
relatively; the hardware's exponential, reciprocal and root within 2 u.  A sum
whose longest chain has D additions is within D u of the sum of magnitudes."""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype: torch.dtype) -> float:
    return torch.finfo(dtype).eps / 2


def philox(counter, key):
    """Philox4x32-10 of Salmon, Moraes, Dror and Shaw (2011) in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def numbers(rows, cols: int, seed: int, offset: int) -> np.ndarray:
    """The 16-bit numbers of the given rows' elements."""
    rows, G = np.asarray(rows, np.uint64), -(-cols // 8)
    one = np.ones((len(rows), G), np.uint64)
    c = [one * np.arange(G, dtype=np.uint64), one * rows[:, None], one * np.uint64(offset & 0xFFFFFFFF), one * np.uint64(offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    s, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> s) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> s) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack(c, 2)
    return np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 3).reshape(len(rows), 8 * G)[:, :cols].astype(np.int64)


def least_of(p: float) -> int:
    return int(np.rint(np.float32(p) * np.float32(65536)))


def mask64(rows: int, cols: int, p: float, seed: int = 0, offset: int = 0, first: int = 0) -> tuple[torch.Tensor, float]:
    """(kept, what kept elements are multiplied by)."""
    least = least_of(p)
    kept = numbers(range(first, first + rows), cols, seed, offset) >= least
    return torch.from_numpy(kept), 65536.0 / (65536 - least) if least < 65536 else 0.0


def chain(cols: int) -> int:
    """Longest chain of a row's sum: each of at least 16 lanes adds its columns, then the lanes and waves are added."""
    return cols // 16 + 48


class Join:
    """hwsel_block_join and its gradients in binary64 on the CPU, and bounds of their errors in fp32."""

    def __init__(self, join, x, y=None, gate=None, x1=None, d_x1=None, d_z=None):
        f = lambda t: None if t is None else t.detach().cpu().double()  # noqa: E731
        j = dict(post_norm=False, gate_sigmoid=False, w_branch=None, w_pre=None, eps=1e-6, stream_scale=1.0, branch_scale=1.0,
                 p=0.0, seed=0, offset=0)
        j.update({k: v for k, v in join.items() if k != "state"})
        if join.get("state") is not None:
            j["seed"], j["offset"] = (int(v) % 2 ** 64 for v in join["state"].tolist())
        eps, ss, bs = (float(np.float32(j[n])) for n in ("eps", "stream_scale", "branch_scale"))
        x = f(x)
        R, C = x.shape
        D = chain(C)
        one = torch.ones(C, dtype=torch.float64)
        wb = one if j["w_branch"] is None else f(j["w_branch"])
        wp = one if j["w_pre"] is None else f(j["w_pre"])
        mean = lambda a: a.mean(1, keepdim=True)  # noqa: E731
        big = lambda a: a.abs().sum(1, keepdim=True) / C  # noqa: E731
        size = lambda a: a.square().sum(1, keepdim=True).sqrt()  # noqa: E731
        tiny = 1e-37                                        # (results below the normal numbers)
        self.x1, e1 = ss * x, 2 * U * (ss * x).abs()
        if y is not None:
            y = f(y)
            r = (mean(y * y) + eps).rsqrt() if j["post_norm"] else torch.ones(R, 1, dtype=torch.float64)
            er = (D / 2 + 6) * U if j["post_norm"] else 0.0  # relative, of r
            yn = y * r
            a = None if gate is None else f(gate)
            g = one if a is None else torch.sigmoid(a) if j["gate_sigmoid"] else a
            slope = g * (1 - g) if j["gate_sigmoid"] else one
            eg = (a.abs().clamp(max=200.0) + 6) * U if a is not None and j["gate_sigmoid"] else 0.0 * U
            if j["p"] > 0:
                kept, factor = mask64(R, C, j["p"], j["seed"], j["offset"])
                m = kept.double() * factor
            else:
                m = torch.ones((), dtype=torch.float64)
            v = torch.where(m > 0, bs * m * g * wb * yn, 0.0)
            self.x1 = self.x1 + v
            e1 = e1 + v.abs() * (er + eg + 6 * U) + 2 * U * (v.abs() + (ss * x).abs())
        self.e1 = e1 + tiny
        r1 = (mean(self.x1.square()) + eps).rsqrt()
        er1 = size(self.e1) / size(self.x1).clamp(min=1e-300) + (D / 2 + 6) * U
        er1 = torch.minimum(er1, torch.full_like(er1, 1.0))
        self.z = self.x1 * r1 * wp
        self.ez = (wp * r1).abs() * (self.e1 * (1 + er1) + self.x1.abs() * er1) + 4 * U * self.z.abs() + tiny
        if d_x1 is None and d_z is None:
            return
        k = f(x1)                                           # the stream as it was written
        dx1 = torch.zeros_like(k) if d_x1 is None else f(d_x1)
        d, ed = dx1, torch.zeros_like(k)
        self.dw_pre = self.edw_pre = None
        if d_z is not None:
            dz = f(d_z)
            r1 = (mean(k * k) + eps).rsqrt()
            er1 = (D / 2 + 6) * U
            xn, dn = k * r1, dz * wp
            mm, em = mean(dn * xn), big(dn * xn) * (D + 4) * U + mean(dn * xn).abs() * (er1 + 4 * U)
            d = dx1 + r1 * (dn - xn * mm)
            part = r1 * (dn.abs() + (xn * mm).abs())
            ed = part * (2 * er1 + 8 * U) + r1 * xn.abs() * em + U * (dx1.abs() + part) * 2
            self.dw_pre = (dz * xn).sum(0)
            self.edw_pre = (dz * xn).abs().sum(0) * (er1 + 4 * U + (R + 40) * U) + tiny
        self.dx, self.edx = ss * d, abs(ss) * ed + 2 * U * (ss * d).abs() + tiny
        self.dy = self.dgate = self.dw_branch = None
        if y is None:
            return
        dv = torch.where(m > 0, bs * m * d, 0.0)
        edv = torch.where(m > 0, (bs * m).abs() * ed, 0.0) + 4 * U * dv.abs()
        if a is not None:
            u = wb * yn
            dg = dv * u * slope
            edg = (u * slope).abs() * edv + dg.abs() * (er + eg + 8 * U)
            if a.shape[1] != C or C == 1:
                edg = edg.sum(1, keepdim=True) + dg.abs().sum(1, keepdim=True) * (D + 4) * U
                dg = dg.sum(1, keepdim=True)
            self.dgate, self.edgate = dg, edg + tiny
        du = dv * g
        edu = edv * torch.as_tensor(g).abs() + du.abs() * (eg + 2 * U)
        self.dw_branch = (du * yn).sum(0)
        self.edw_branch = (edu * yn.abs() + (du * yn).abs() * (er + 4 * U)).sum(0) + (du * yn).abs().sum(0) * (R + 40) * U + tiny
        dn, edn = du * wb, edu * wb.abs() + 2 * U * (du * wb).abs()
        if j["post_norm"]:
            mm = mean(dn * yn)
            em = (edn * yn.abs()).sum(1, keepdim=True) / C + big(dn * yn) * (D + 4 + D / 2 + 6) * U
            self.dy = r * (dn - yn * mm)
            part = r * (dn.abs() + (yn * mm).abs())
            self.edy = r * edn + r * yn.abs() * em + part * (2 * er + 8 * U) + tiny
        else:
            self.dy, self.edy = dn, edn + tiny


def near(got: torch.Tensor, want: torch.Tensor, bound, what: str = "") -> None:
    """got is want within bound and half a step of got's type; NaN and infinities are where they are in want."""
    step = half_step(got.dtype)
    got = got.detach().cpu().double()
    bound = torch.as_tensor(bound).expand_as(want) * (1 + step) + step * want.abs()
    fine = torch.isfinite(want)
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: infinities"
    off = ((got - want).abs() - bound)[fine]
    assert not off.numel() or float(off.max()) <= 0.0, f"{what}: over the bound by {float(off.max()):.3g}"


class Logprob:
    """Log probabilities of one problem in binary64, and bounds."""

    def __init__(self, scores, T=1.0):
        s = np.asarray(scores, np.float32)
        T = float(np.float32(T))
        self.n, self.live = len(s), np.nonzero(s > -np.inf)[0]
        self.lp = np.full(len(s), -np.inf)
        self.elp = np.zeros(len(s))
        self.entropy, self.best, self.log_mass, self.T = 0.0, -np.inf, -np.inf, T
        if not len(self.live):
            return
        a = s[self.live].astype(np.float64)
        self.best = float(a.max())
        if not T > 0:
            self.lp[self.live[np.argmax(a)]], self.log_mass = 0.0, 0.0
            return
        with np.errstate(invalid="ignore", over="ignore"):
            t = np.where(a == self.best, 0.0, (a - self.best) / T)
        e = np.exp(t)
        k = (a == self.best).sum()
        rest = e[a != self.best].sum()
        self.log_mass = float(np.log1p((k - 1) + rest))
        # log Z moves by the error of Z over Z, and Z - 1 = (k - 1) + rest, k - 1 a count.  Each weight of the rest is within (4
        # |t| + 8) u, and their sum, whose longest chain is below n / 16 + 64, within that many u of the rest: so the error of Z
        # is the sum over the rest alone, not a share of it once more.  A weight below the normal numbers (2^-126) may be 0,
        # and so may log Z or an entropy below them.
        finite = np.isfinite(t)
        size = np.abs(np.where(finite, t, 0.0))
        others = np.where(finite & (a != self.best), e, 0.0)
        tiny = (len(a) + 1) * 2.0 ** -126
        self.em = ((others * (4 * size + 8)).sum() + (len(a) / 16 + 64) * rest) / e.sum() * U + 4 * U * self.log_mass + tiny
        with np.errstate(invalid="ignore"):
            self.lp[self.live] = t - self.log_mass
            self.elp[self.live] = np.where(finite, 3 * U * np.abs(np.where(finite, t, 0.0)) + self.em + U * np.abs(np.where(finite, self.lp[self.live], 0.0)), 0.0)
        p = np.exp(self.lp[self.live])
        with np.errstate(invalid="ignore"):
            self.entropy = float(-np.where(p > 0, p * self.lp[self.live], 0.0).sum())
        second = np.where(finite, e * np.abs(np.where(finite, t, 0.0)) * (np.abs(np.where(finite, t, 0.0)) * 4 + 12 + len(a) / 16 + 64), 0.0).sum() / e.sum()
        self.eentropy = self.em * (1 + self.entropy) + second * U + 4 * U * self.entropy + tiny * (1 + size.max() if len(a) else 1)

    def of(self, j):
        j = int(j)
        return (0.0, 0.0) if not 0 <= j < self.n else (self.lp[j], self.elp[j])

    def gradient(self, picks, d_logp, d_entropy=0.0):
        """The scores' gradient and a bound of its error."""
        out, bound = np.zeros(self.n), np.zeros(self.n)
        if not len(self.live) or not self.T > 0:
            return out, bound
        g, S, size = np.zeros(self.n), 0.0, 0.0
        for j, d in zip(picks, d_logp):
            if 0 <= j < self.n and self.lp[j] > -np.inf:
                g[j] += float(d)
                S += float(d)
                size = max(size, abs(float(d)))
        fixed = len(picks) * size * 2.0 ** -30
        p = np.where(self.lp > -np.inf, np.exp(self.lp), 0.0)
        lp = np.where(p > 0, self.lp, 0.0)
        de = float(d_entropy)
        some = self.lp > -np.inf
        out[some] = ((g - p * S - de * p * (lp + self.entropy)) / self.T)[some]
        ep = p * (self.elp + (np.abs(lp) * 4 + 8) * U + self.em)
        inner = np.abs(lp) + self.entropy
        bound = (np.abs(g) * (1 - p) * 16 * U + np.abs(g) * p * (self.elp + 4 * U) + ep * np.abs(S - g) + 8 * U * (p * np.abs(S - g)) + fixed
                 + abs(de) * (ep * inner + p * (self.elp + self.eentropy + 4 * U * inner) + 4 * U * p * inner)) / self.T
        bound = bound + 4 * U * (np.abs(g) * (1 - p) + p * np.abs(S - g) + abs(de) * p * inner) / self.T
        return out, np.where(some, bound, 0.0) + 1e-37
