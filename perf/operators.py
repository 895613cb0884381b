"""The operators of an 8-bit neural ranker and of drawing candidates, as cases that can be timed and checked.

A ranker with wider layers than the fixed 128-512-512-256-1 network runs its
products in 8-bit floating point with a power-of-two scale for each block of
128 elements, keeps its activations in that form for the backward pass, and
its scores either go to the per-problem top-k or, when a tuner decides which
candidates to measure next, to a draw with temperature, top-k, top-p and min-p.

Every case is one such call or short chain of calls.  `run` makes it through
the framework's binding (own) or computes it in plain torch operations.

8-bit operand: a dict of q (uint8 [rows][cols rounded up to 128], codes of
E4M3 or E5M2, padding 0), scale (uint8 [rows / block_rows][blocks rounded up
to 4], the exponent byte b of a block standing for 2^(b - 127)), rows, cols,
format (0 E4M3, 1 E5M2) and block_rows (1, or 128 where 128 rows share it).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
E4M3, E5M2 = 0, 1
LOG2E = 1.4426950408889634
# 2^f on [-1/2, 1/2]: the Taylor coefficients ln(2)^i / i!, i = 0..6, in fp32
EXP2 = tuple(float(np.float32(math.log(2.0) ** i / math.factorial(i))) for i in range(7))


# ----------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------
def listed():
    return [
        # The feature matrix of the whole data set (600 problems x 8,192 rows) standardised and kept
        # in 8 bits, and read back: the first layer's operand and its checkpoint.
        dict(name="keep-features", kind="keep", R=4_915_200, C=128, dtype="fp32", standardise=True, format=E4M3),
        # Two hidden layers over one problem's catalogue of 8,192 rows, while the caller waits.
        dict(name="layers-online", kind="layers", R=8192, K=1024, H=1024, N=512),
        # Two hidden layers over the whole data set: the bulk of a scoring run.
        dict(name="layers-bulk", kind="layers", R=4_915_200, K=512, H=512, N=256),
        # One row through one layer: the smallest product, where latency counts.
        dict(name="product-row", kind="product", M=1, N=1024, K=1024, out="bf16", bias=True, gelu=True),
        # Sixteen rows through a wide layer: bound by reading the weights.
        dict(name="product-few", kind="product", M=16, N=16_384, K=16_384, out="bf16", bias=False, gelu=False),
        # Odd sizes, fp32 results: a last layer whose scores are compared.
        dict(name="product-odd", kind="product", M=4099, N=1000, K=2500, out="fp32", bias=True, gelu=False),
        # A large product, where the matrix cores are what counts.
        dict(name="product-large", kind="product", M=16_384, N=16_384, K=8192, out="bf16", bias=False, gelu=False),
        # A training batch: gradients of a layer's input and weights from the 8-bit checkpoint.
        dict(name="backward-batch", kind="backward", R=65_536, K=1024, N=512),
        # A few problems of 512 candidates, one draw each: the smallest call.
        dict(name="sample-small", kind="sample", P=16, C=512, ragged=False, draws=1, top_k=50, top_p=0.95, min_p=0.0,
             temperature=0.7, per_problem=False, ties=0.0),
        # Ragged problems of the data set, 64 candidates to measure of each, settings of its own for every problem.
        dict(name="sample-dataset", kind="sample", P=600, C=8192, ragged=True, draws=64, top_k=500, top_p=0.9,
             min_p=0.02, temperature=1.0, per_problem=True, ties=0.2),
        # The whole 65,536-point grid of 256 problems, no limit on the number kept.
        dict(name="sample-grid", kind="sample", P=256, C=65_536, ragged=False, draws=4, top_k=0, top_p=0.95,
             min_p=0.0, temperature=1.0, per_problem=False, ties=0.0),
        # Few problems with very many candidates.
        dict(name="sample-long", kind="sample", P=3, C=534_600, ragged=False, draws=1, top_k=0, top_p=0.9,
             min_p=0.05, temperature=1.5, per_problem=False, ties=0.1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["keep", "layers", "product", "product", "backward", "sample", "sample"])
    if kind == "keep":
        C = _log(rng, 1, 4096)
        R = _log(rng, 1, max(1, min(4_915_200, 600_000_000 // C)))
        standardise = rng.random() < 0.5
        dtype = "fp32" if standardise else rng.choice(["fp32", "bf16"])
        return dict(kind=kind, R=R, C=C, dtype=dtype, standardise=standardise, format=rng.choice([E4M3, E5M2]))
    if kind == "layers":
        K, H, N = (_log(rng, 32, 2048) for _ in range(3))
        R = _log(rng, 1, max(1, min(2_000_000, int(3e12 / (2 * H * (K + N))))))
        return dict(kind=kind, R=R, K=K, H=H, N=N)
    if kind == "product":
        N, K = _log(rng, 1, 16_384), _log(rng, 32, 16_384)
        M = _log(rng, 1, max(1, min(100_000, int(2e12 / (2 * N * K)))))
        return dict(kind=kind, M=M, N=N, K=K, out=rng.choice(["bf16", "fp32"]), bias=rng.random() < 0.5,
                    gelu=rng.random() < 0.3)
    if kind == "backward":
        K, N = _log(rng, 32, 2048), _log(rng, 32, 2048)
        R = _log(rng, 32, max(32, min(1_000_000, int(5e11 / (4 * N * K)))))
        return dict(kind=kind, R=R, K=K, N=N)
    P = _log(rng, 1, 4096)
    C = _log(rng, 1, max(1, min(534_600, 16_000_000 // P)))
    return dict(kind=kind, P=P, C=C, ragged=rng.random() < 0.5, draws=_log(rng, 1, 256),
                top_k=rng.choice([0, 1, _log(rng, 1, 2000)]), top_p=rng.choice([1.0, rng.uniform(0.05, 1.0)]),
                min_p=rng.choice([0.0, rng.uniform(0.0, 0.3)]), temperature=rng.choice([0.0, rng.uniform(0.2, 3.0)]),
                per_problem=rng.random() < 0.5, ties=rng.choice([0.0, 0.3, 1.0]))


def work(case):
    c = case
    if c["kind"] == "keep":
        n = c["R"] * c["C"]
        return {"bytes": n * ((4 if c["dtype"] == "fp32" else 2) + 1 + 1 + 2) + 2 * c["R"] * -(-c["C"] // 128), "flops": 3 * n}
    if c["kind"] == "layers":
        R, K, H, N = c["R"], c["K"], c["H"], c["N"]
        return {"bytes": R * (K + 2 * H + 2 * N) + H * K + N * H, "flops": 2 * R * H * (K + N)}
    if c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": M * K + N * K + M * N * (4 if c["out"] == "fp32" else 2), "flops": 2 * M * N * K}
    if c["kind"] == "backward":
        R, K, N = c["R"], c["K"], c["N"]
        # the bf16 gradient read once, its two 8-bit forms and the transposed checkpoint written and read, dX and dW
        return {"bytes": R * N * (2 + 4) + R * K * (1 + 2) + R * K * 2 + 5 * N * K, "flops": 4 * R * N * K}
    rows = sum(_lengths(c))
    return {"bytes": 4 * rows + c["P"] * (8 + 4 + 12 * c["draws"]), "flops": 20 * rows}


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


def _operand(x, block_rows=1, fmt=E4M3):
    """An fp32 matrix as a user's program has it after quantising: codes, scales, sizes."""
    q, scale = plain_quantise(x, block_rows, fmt)
    return dict(q=q, scale=scale, rows=x.shape[0], cols=x.shape[1], format=fmt, block_rows=block_rows)


def _rows(gen, R, C, sd=1.0):
    """Activations: normal, with a spread of sizes over rows and a few large units."""
    x = torch.randn(R, C, generator=gen, device=DEV).mul_(sd)
    x.mul_(torch.exp(0.5 * torch.randn(R, 1, generator=gen, device=DEV)))
    x.mul_(torch.exp(0.5 * torch.randn(1, C, generator=gen, device=DEV)))
    return x


def _weights(gen, N, K):
    return torch.randn(N, K, generator=gen, device=DEV) * (2.0 / K) ** 0.5


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    c, st = case, dict(case=dict(case))
    if c["kind"] == "keep":
        R, C = c["R"], c["C"]
        x = _rows(g, R, C)
        if c["standardise"]:
            # columns of very different sizes, some values missing
            st["mean"] = 100.0 * torch.randn(C, generator=g, device=DEV)
            sd = torch.exp(3.0 * torch.randn(C, generator=g, device=DEV))
            st["inv_std"] = 1.0 / sd
            x.mul_(sd).add_(st["mean"])
            x[:: 97, C // 3] = float("nan")
            x[5 :: 1009, C // 2] = float("inf")
        st["x"] = x if c["dtype"] == "fp32" else x.bfloat16()
    elif c["kind"] == "layers":
        R, K, H, N = c["R"], c["K"], c["H"], c["N"]
        st["x"] = _operand(_rows(g, R, K))
        st["w1"], st["w2"] = _operand(_weights(g, H, K), 128), _operand(_weights(g, N, H), 128)
        st["b1"], st["b2"] = (0.1 * torch.randn(n, generator=g, device=DEV) for n in (H, N))
    elif c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        st["a"], st["b"] = _operand(_rows(g, M, K)), _operand(_weights(g, N, K), 128)
        st["bias"] = 0.1 * torch.randn(N, generator=g, device=DEV) if c["bias"] else None
    elif c["kind"] == "backward":
        R, K, N = c["R"], c["K"], c["N"]
        st["x"] = _operand(_rows(g, R, K))                          # the forward pass's checkpoint
        st["wt"] = _operand(_weights(g, N, K).t().contiguous(), 128)  # weights, transposed: [K][N]
        st["dy"] = _rows(g, R, N, 1e-3).bfloat16()
    else:
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
        st.update(scores=s[:R], seg=torch.from_numpy(seg).to(DEV), longest=max(n), rows=R,
                  u=torch.rand(P, c["draws"], generator=g, device=DEV))
        if c["per_problem"]:
            e = torch.rand(4, P, generator=g, device=DEV)
            st["temperature"] = c["temperature"] * (0.5 + e[0])
            st["top_k"] = (c["top_k"] * (0.5 + e[1])).to(torch.int32)
            st["top_p"] = 1.0 - (1.0 - c["top_p"]) * 2.0 * e[2]
            st["min_p"] = c["min_p"] * 2.0 * e[3]
        else:
            for k in ("temperature", "top_k", "top_p", "min_p"):
                st[k] = c[k]
    return st


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------
def run(state):
    return run_own(state) if own else run_plain(state)


def run_own(st):
    from paper_2609_35587_amd import hwsel
    c = st["case"]
    if c["kind"] == "keep":
        kept = hwsel.hwsel_fp8_quantise(st["x"], format=c["format"], mean=st.get("mean"), inv_std=st.get("inv_std"))
        return {"kept": hwsel.hwsel_fp8_dequantise(kept, torch.bfloat16)}
    if c["kind"] == "layers":
        h = hwsel.hwsel_fp8_layer(st["x"], st["w1"], bias=st["b1"], gelu=True)
        return {"y": hwsel.hwsel_fp8_matmul(h, st["w2"], torch.bfloat16, bias=st["b2"], gelu=True)}
    if c["kind"] == "product":
        return {"y": hwsel.hwsel_fp8_matmul(st["a"], st["b"], torch.float32 if c["out"] == "fp32" else torch.bfloat16,
                                            bias=st["bias"], gelu=c["gelu"])}
    if c["kind"] == "backward":
        dy = hwsel.hwsel_fp8_quantise(st["dy"], format=E5M2)
        dyt = hwsel.hwsel_fp8_quantise(st["dy"], format=E5M2, transpose=True)
        xt = hwsel.hwsel_fp8_transpose(st["x"])
        return {"dx": hwsel.hwsel_fp8_matmul(dy, st["wt"], torch.bfloat16),
                "dw": hwsel.hwsel_fp8_matmul(dyt, xt, torch.float32)}
    idx, prob, kept = hwsel.hwsel_sample_per_problem(
        st["scores"], st["seg"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
        min_p=st["min_p"])
    return {"idx": idx, "prob": prob, "kept": kept}


def run_plain(st):
    c = st["case"]
    if c["kind"] == "keep":
        x = st["x"].float()
        if c["standardise"]:
            x = (torch.where(torch.isfinite(x), x, 0.0) - st["mean"]) * st["inv_std"]
        q, scale = plain_quantise(x, 1, c["format"])
        return {"kept": plain_values(q, scale, x.shape[0], x.shape[1], c["format"], 1).bfloat16()}
    if c["kind"] == "layers":
        h = plain_gelu(plain_product(st["x"], st["w1"]).add_(st["b1"]))
        return {"y": plain_gelu(plain_product(_operand(h), st["w2"]).add_(st["b2"])).bfloat16()}
    if c["kind"] == "product":
        y = plain_product(st["a"], st["b"])
        y = y if st["bias"] is None else y + st["bias"]
        y = plain_gelu(y) if c["gelu"] else y
        return {"y": y if c["out"] == "fp32" else y.bfloat16()}
    if c["kind"] == "backward":
        dy = st["dy"].float()
        xt = _operand(plain_values(**st["x"]).t().contiguous())
        return {"dx": plain_product(_operand(dy, 1, E5M2), st["wt"]).bfloat16(),
                "dw": plain_product(_operand(dy.t().contiguous(), 1, E5M2), xt)}
    return plain_sample(st)


def plain_quantise(x, block_rows, fmt):
    """Codes and exponent bytes of an fp32 matrix, a scale for each 128 columns (of block_rows rows)."""
    R, C = x.shape
    kb = -(-C // 128)
    rb = -(-R // block_rows)
    z = torch.zeros(rb * block_rows, kb * 128, dtype=torch.float32, device=x.device)
    z[:R, :C] = x
    z = z.view(rb, block_rows, kb, 128)
    a = z.abs()
    amax = torch.where(torch.isfinite(a), a, 0.0).amax(dim=(1, 3))
    m, e = torch.frexp(amax)                               # amax = m 2^e, 1/2 <= m < 1; the largest code is 7/8 2^(9 or 16)
    e = e - (9 if fmt == E4M3 else 16) + (m > 0.875).to(torch.int32)
    byte = torch.where(amax == 0.0, 1, (e + 127).clamp(1, 254)).to(torch.int32)
    z = z * ((254 - byte) << 23).view(torch.float32)[:, None, :, None]
    q = z.to(torch.float8_e4m3fn if fmt == E4M3 else torch.float8_e5m2).view(torch.uint8).view(rb * block_rows, kb * 128)
    scale = torch.zeros(rb, -(-kb // 4) * 4, dtype=torch.uint8, device=x.device)
    scale[:, :kb] = byte.to(torch.uint8)
    return q[:R].contiguous(), scale


def plain_values(q, scale, rows, cols, format, block_rows):
    kb = -(-cols // 128)
    v = q.view(torch.float8_e4m3fn if format == E4M3 else torch.float8_e5m2).float()
    s = (scale[:, :kb].to(torch.int32) << 23).view(torch.float32)
    s = s.repeat_interleave(block_rows, 0)[:rows] if block_rows > 1 else s
    return v.view(rows, kb, 128).mul_(s[:, :, None]).view(rows, kb * 128)[:, :cols].contiguous()


def plain_product(a, b):
    return plain_values(**a) @ plain_values(**b).t()


def plain_gelu(y):
    return 0.5 * y * (1.0 + torch.erf(y * 0.7071067811865476))


def _per_problem(v, P, dtype):
    return v.to(dtype) if isinstance(v, torch.Tensor) else torch.full((P,), v, dtype=dtype, device=DEV)


def plain_sample(st):
    seg, u, R = st["seg"], st["u"], st["rows"]
    P, L = seg.numel() - 1, max(1, st["longest"])
    T, k = _per_problem(st["temperature"], P, torch.float32), _per_problem(st["top_k"], P, torch.int32)
    top_p, min_p = (_per_problem(st[n], P, torch.float32).double() for n in ("top_p", "min_p"))
    col = torch.arange(L, device=DEV)
    valid = col[None, :] < (seg[1:] - seg[:-1])[:, None]
    at = (seg[:-1, None] + col).clamp(max=max(R - 1, 0))
    s = st["scores"][at] + 0.0 if R else torch.zeros(P, L, device=DEV)
    s = torch.where(valid & ~torch.isnan(s), s, float("-inf"))
    alive = s > float("-inf")
    best = s.amax(1, keepdim=True)
    # the weight of a candidate, a whole number: 2^32 exp((s - best) / T) by these fp32 steps
    cold = ~(T > 0.0)
    rate = (LOG2E / torch.where(cold, 1.0, T).double()).float()
    t = torch.where(s == best, 0.0, (s - best) * rate[:, None])
    t = torch.where(t > -60.0, t, -60.0)                    # no weight is left from -34 on
    n = torch.round(t)
    f = t - n
    p = torch.full_like(f, EXP2[6])
    for i in range(5, -1, -1):
        p = p * f
        p = p + EXP2[i]
    w = (((p * 16777216.0).to(torch.int64) << 8) >> (-n).to(torch.int64))
    w = torch.where(alive, w, 0)
    # best first: the k best, then the shortest prefix of top_p of their mass, then min_p of the best's weight
    order = torch.sort(s, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    k = torch.where(cold, 1, torch.where(k > 0, k, 1 << 30))
    keep = col[None, :] < k[:, None]
    ws = ws * keep
    mass = ws.sum(1)
    need = torch.where(top_p < 1.0, torch.ceil(mass.double() * top_p.clamp(min=0.0)).to(torch.int64).clamp(min=1), 1 << 62)
    keep &= ws.cumsum(1) - ws < need[:, None]
    least = torch.ceil(min_p.clamp(0.0, 1.0) * 4294967296.0).to(torch.int64).clamp(min=1)
    keep &= ws >= least[:, None]
    w = w * torch.zeros_like(keep).scatter_(1, order, keep)
    # a draw: the first candidate, in index order, whose running sum passes u of the whole
    run_sum = w.cumsum(1)
    total = run_sum[:, -1:]
    u24 = torch.floor(u * 16777216.0).to(torch.int64).clamp(0, (1 << 24) - 1)
    r = (total >> 24) * u24 + (((total & 0xffffff) * u24) >> 24)
    idx = torch.searchsorted(run_sum, r, right=True).clamp(max=L - 1)
    prob = (w.gather(1, idx).double() / total.clamp(min=1).double()).float()
    return {"idx": torch.where(total > 0, idx, -1).to(torch.int32), "prob": torch.where(total > 0, prob, 0.0),
            "kept": keep.sum(1).to(torch.int32)}


# ----------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["kind"] == "keep":
        x = st["x"]
        if c["standardise"]:
            # standardised values are fp32 by definition: one subtraction, one multiplication
            x = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).sub_(st["mean"]).mul_(st["inv_std"])
        y = torch.empty(x.shape, dtype=torch.float64, device=DEV)
        for lo in range(0, c["R"], 1 << 18):
            y[lo:lo + (1 << 18)] = _grid64(x[lo:lo + (1 << 18)].double(), c["format"])
        return {"kept": y}
    if c["kind"] == "layers":
        w1, w2 = _values64(st["w1"]).t(), _values64(st["w2"]).t()
        y = torch.empty(c["R"], c["N"], dtype=torch.float64, device=DEV)
        for lo in range(0, c["R"], 1 << 18):
            part = {**st["x"], "q": st["x"]["q"][lo:lo + (1 << 18)], "scale": st["x"]["scale"][lo:lo + (1 << 18)]}
            part["rows"] = part["q"].shape[0]
            h = _grid64(_gelu64(_values64(part).matmul(w1) + st["b1"].double()), E4M3)
            y[lo:lo + (1 << 18)] = _gelu64(h.matmul(w2) + st["b2"].double())
        return {"y": y}
    if c["kind"] == "product":
        y = _values64(st["a"]).matmul(_values64(st["b"]).t())
        y = y + st["bias"].double() if c["bias"] else y
        return {"y": _gelu64(y) if c["gelu"] else y}
    if c["kind"] == "backward":
        dy = st["dy"].double()
        dyt, xt = _grid64(dy.t().contiguous(), E5M2), _grid64(_values64(st["x"]).t().contiguous(), E4M3)
        return {"dx": _grid64(dy, E5M2).matmul(_values64(st["wt"]).t()), "dw": dyt.matmul(xt.t())}
    return _sample64(st)


def _grid64(x, fmt):
    """The nearest 8-bit value times its block's scale, by the grid's spacing (ties to the even neighbour)."""
    digits, lowest, top = (3, -6, 448.0) if fmt == E4M3 else (2, -14, 57344.0)
    R, C = x.shape
    out = torch.empty_like(x)
    for lo in range(0, C, 128):
        b = x[:, lo:lo + 128]
        a = b.abs().amax(1, keepdim=True)
        s = torch.exp2(torch.ceil(torch.log2((a / top).clamp(min=2.0 ** -126))))
        # log2 near a whole number may be a rounding step off: the least power of two that holds a
        s = torch.where(a > s * top, s * 2, torch.where((a <= s * (top / 2)) & (s > 2.0 ** -126), s / 2, s))
        v = b / s
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** lowest))) - digits)
        out[:, lo:lo + 128] = torch.round(v / step) * step * s
    return out


def _values64(o):
    """Values of an operand from its codes, bit by bit."""
    q = o["q"].to(torch.int32)
    ebits, mbits, bias = (4, 3, 7) if o["format"] == E4M3 else (5, 2, 15)
    e, m = (q >> mbits) & ((1 << ebits) - 1), q & ((1 << mbits) - 1)
    frac = m.double() / (1 << mbits)
    v = torch.where(e == 0, frac * 2.0 ** (1 - bias), (1.0 + frac) * torch.exp2((e - bias).double()))
    v = torch.where(q >= 128, -v, v)
    rows = torch.arange(o["rows"], device=DEV) // o["block_rows"]
    cols = torch.arange(o["cols"], device=DEV)
    return v[:, : o["cols"]] * torch.exp2(o["scale"].double() - 127.0)[rows][:, cols // 128]


def _gelu64(y):
    return 0.5 * y * torch.erfc(-y / math.sqrt(2.0))


def _sample64(st):
    """Draws by the definition: whole-number weights, one problem after another, in numpy."""
    f4 = np.float32
    scores, seg, u = st["scores"].cpu().numpy(), st["seg"].cpu().numpy(), st["u"].cpu().numpy()
    P, draws = u.shape
    setting = {n: st[n].cpu().numpy() if isinstance(st[n], torch.Tensor) else np.full(P, st[n]) for n in
               ("temperature", "top_k", "top_p", "min_p")}
    idx, prob, kept = np.full((P, draws), -1, np.int32), np.zeros((P, draws)), np.zeros(P, np.int32)
    for p in range(P):
        s = scores[seg[p]:seg[p + 1]]
        i = np.nonzero(s > f4("-inf"))[0]                   # neither NaN nor -inf
        if not len(i):
            continue
        s = s[i]
        T, k, tp, mp = (setting[n][p] for n in ("temperature", "top_k", "top_p", "min_p"))
        T, tp, mp = f4(T), float(f4(tp)), float(f4(mp))
        i = i[np.argsort(-s, kind="stable")]
        s = scores[seg[p]:seg[p + 1]][i]
        i, s = (i[:1], s[:1]) if not T > 0 else (i[:k], s[:k]) if k > 0 else (i, s)
        with np.errstate(all="ignore"):
            t = (s - s[0]) * f4(LOG2E / float(T)) if T > 0 else f4(0) * s
        t[s == s[0]] = 0
        i, t = i[t > -60], t[t > -60]
        n = np.rint(t)
        f = t - n
        w = np.full(len(t), EXP2[6], f4)
        for a in EXP2[5::-1]:
            w = w * f + f4(a)                               # two fp32 operations in numpy
        w = ((w * f4(16777216)).astype(np.int64) * 256) >> (-n).astype(np.int64)
        before = np.cumsum(w) - w
        ok = w >= max(1, math.ceil(min(max(mp, 0.0), 1.0) * 4294967296.0))
        if tp < 1:
            ok &= before < max(1, math.ceil(float(w.sum()) * max(tp, 0.0)))
        i, w = i[ok], w[ok]
        back = np.argsort(i)
        i, w = i[back], w[back]
        kept[p] = len(i)
        run_sum = np.cumsum(w)
        total = int(run_sum[-1])
        for j in range(draws):
            r = (total * min(max(math.floor(float(u[p, j]) * 16777216.0), 0), (1 << 24) - 1)) >> 24
            at = int(np.searchsorted(run_sum, r, side="right"))
            idx[p, j], prob[p, j] = i[at], int(w[at]) / total
    return {"idx": torch.from_numpy(idx), "prob": torch.from_numpy(prob), "kept": torch.from_numpy(kept)}
