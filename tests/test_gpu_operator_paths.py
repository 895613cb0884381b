"""The kernels that only large or odd calls reach, and what surrounds a call:
long strides and offsets past 2^31, streams, captured graphs, settings that
come one to a problem.  Bounds and binary64 statements are those of the
operators' own tests."""
import numpy as np
import pytest
import torch

import test_gpu_fp8_product as product
import test_gpu_sample as sample
from _fp8_util import E4M3, E5M2, code_values, grid_values, same_values
from _gpu_util import say
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
# 256 x 256 tiles: results of 160 such and more, K >= 1,024
DEEP = [(2600, 4096, 1100), (4099, 2700, 1024), (3000, 3500, 2177)]
# short sums over at least 3,072 tiles of 128 x 128, one to four blocks of K
ROWS = [(50_000, 1000, 100), (50_000, 1000, 256), (200_000, 130, 384), (50_001, 1024, 500)]


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", DEEP + ROWS)
def test_many_tiles(M, N, K, gelu):
    product.test_product(M, N, K, gelu, gelu, torch.bfloat16)
    product.test_layer(M, N, K, gelu)


@pytest.mark.parametrize("M,N,K", [DEEP[0], ROWS[3]])
def test_many_tiles_of_gradients(M, N, K):
    """E5M2 rows against blocks of E4M3, as the gradient of a layer's input takes them."""
    _, a, b = product.operands(M, N, K, E5M2)
    product.assert_within(hwsel.hwsel_fp8_matmul(a, b), *product.exact(a, b, fine=False), torch.bfloat16)


@pytest.mark.parametrize("M,N,K", [(2600, 4000, 1200), (50_000, 900, 300), (60, 9000, 3000), (700, 700, 9000)])
def test_large_products_are_exact_where_sums_are(M, N, K):
    g = product.gen(M, N, K)
    x = torch.randint(-3, 4, (M, K), generator=g, device="cuda").float()
    w = torch.randint(-2, 3, (N, K), generator=g, device="cuda").float()
    a, b = hwsel.hwsel_fp8_quantise(x), hwsel.hwsel_fp8_quantise(w, block_rows=128)
    y = x.double() @ w.double().t()
    for _ in range(3):
        assert torch.equal(hwsel.hwsel_fp8_matmul(a, b).double(), y.bfloat16().double())
        assert torch.equal(hwsel.hwsel_fp8_matmul(a, b, torch.float32).double(), y)
    assert same_values(code_values(hwsel.hwsel_fp8_layer(a, b)), grid_values(y, E4M3)[0])


@pytest.mark.parametrize("M,N,K", [(3, 40, 700), (50, 40, 700), (150, 200, 300), (300, 300, 5000), (2600, 4096, 1100),
                                   (50_000, 1000, 128)])
def test_a_scale_of_255_makes_its_block_nan(M, N, K):
    """One row's first block: that row of the result is NaN, the others are as without it."""
    _, a, b = product.operands(M, N, K)
    results = lambda: [hwsel.hwsel_fp8_matmul(a, b), hwsel.hwsel_fp8_matmul(a, b, torch.float32),  # noqa: E731
                       hwsel.hwsel_fp8_dequantise(hwsel.hwsel_fp8_layer(a, b), torch.float32)]
    want = results()
    a["scale"][1, 0] = 255
    for got, before in zip(results(), want):
        assert bool(torch.isnan(got[1]).all())
        got[1], before[1] = 0.0, 0.0
        assert torch.equal(got, before)


@pytest.mark.parametrize("M,N,K", [(300, 200, 300), (20, 300, 256), (300, 256, 1024)])
def test_rows_16_mb_apart(M, N, K):
    """Leading dimensions near their limit: offsets within a tile pass 2^31."""
    ld = (1 << 24) - 128
    say(f"16 MB apart {M}x{N}x{K}")
    _, a, b = product.operands(M, N, K)

    def apart(m):
        cols = m["q"].shape[1]
        q = torch.empty(m["rows"] * ld, dtype=torch.uint8, device="cuda").as_strided((m["rows"], cols), (ld, 1))
        q.copy_(m["q"])
        return dict(m, q=q)

    far_a, far_b = apart(a), apart(b)
    for dtype in (torch.bfloat16, torch.float32):
        want = hwsel.hwsel_fp8_matmul(a, b, dtype)
        assert torch.equal(hwsel.hwsel_fp8_matmul(far_a, b, dtype), want)
        assert torch.equal(hwsel.hwsel_fp8_matmul(a, far_b, dtype), want)
    assert torch.equal(hwsel.hwsel_fp8_dequantise(far_a, torch.float32), hwsel.hwsel_fp8_dequantise(a, torch.float32))
    t, far_t = hwsel.hwsel_fp8_transpose(a), hwsel.hwsel_fp8_transpose(far_a)
    blocks = -(-M // 128)                                   # (bytes past the blocks are not written)
    assert torch.equal(t["q"], far_t["q"]) and torch.equal(t["scale"][:, :blocks], far_t["scale"][:, :blocks])


def test_matrices_of_more_than_2_31_elements():
    """Quantised, restored, transposed and a product's result: the last rows as of those rows alone."""
    R, C, last = (1 << 20) + 77, 2100, 300
    say("2^31 elements")
    x = torch.empty(R, C, dtype=torch.bfloat16, device="cuda").normal_(generator=product.gen(31))
    m = hwsel.hwsel_fp8_quantise(x)
    tail = hwsel.hwsel_fp8_quantise(x[R - last:])
    assert torch.equal(m["q"][R - last:], tail["q"]) and torch.equal(m["scale"][R - last:, :17], tail["scale"][:, :17])
    y = hwsel.hwsel_fp8_dequantise(m)
    assert torch.equal(y[R - last:], hwsel.hwsel_fp8_dequantise(tail))
    first = R - R % 128 - 128                               # whole blocks of the transposed rows from here on
    want = hwsel.hwsel_fp8_transpose({**m, "q": m["q"][first:], "scale": m["scale"][first:], "rows": R - first})
    t = hwsel.hwsel_fp8_transpose(m)
    assert torch.equal(t["q"][:, first:R], want["q"][:, :R - first])
    del x, y, t
    N = 2200
    w = hwsel.hwsel_fp8_quantise(torch.randn(N, 100, device="cuda"), block_rows=128)
    a = hwsel.hwsel_fp8_quantise(torch.randn(R, 100, device="cuda"))
    c = hwsel.hwsel_fp8_matmul(a, w)
    end = {**a, "q": a["q"][R - last:], "scale": a["scale"][R - last:], "rows": last}
    product.assert_within(c[R - last:], *product.exact(end, w, fine=False), torch.bfloat16)


def test_draws_from_the_end_of_2_30_scores():
    """Few candidates far into the scores, by the kernels that are chosen for many."""
    R, n = 1 << 30, 1000
    s = torch.empty(R, device="cuda")
    tail = np.random.default_rng(30).standard_normal(n).astype(np.float32)
    s[R - n:] = torch.from_numpy(tail).cuda()
    u = sample.uniform(np.random.default_rng(1), 2, 7)
    seg = torch.tensor([R - n, R - 300, R], device="cuda")
    idx, _, kept = hwsel.hwsel_sample_per_problem(s, seg, torch.from_numpy(u).cuda(), top_k=200, top_p=0.9)
    for p, part in enumerate((tail[:n - 300], tail[n - 300:])):
        i, _, k = sample.draws64(part, u[p], top_k=200, top_p=0.9)
        assert int(kept[p]) == k and np.array_equal(idx[p].cpu().numpy(), i)


@pytest.mark.parametrize("lengths", [[0] * 99 + [300_000], [5, 0, 700_000], [20_000] * 40, [13_000] * 3, [30_000] * 130])
def test_lengths_far_from_their_mean(lengths):
    """Kernels are chosen by the mean length; every length is right in each."""
    say(f"sample {len(lengths)} problems, mean {sum(lengths) // len(lengths)}")
    rng = np.random.default_rng(len(lengths))
    kinds = ["normal", "ties", "masked"]
    parts = [sample.make_scores(rng, n, kinds[p % 3]) for p, n in enumerate(lengths)]
    u = sample.uniform(rng, len(lengths), 3)
    sample.check(parts, u, top_k=400, top_p=0.9)
    sample.check(parts, u, top_p=0.5, min_p=0.01)


def test_settings_per_problem_of_long_problems():
    rng = np.random.default_rng(12)
    P = 6
    parts = [sample.make_scores(rng, int(rng.integers(100_000, 200_000)), ["normal", "ties", "dead"][p % 3]) for p in range(P)]
    per = dict(temperature=np.array([1, 0, 0.5, 2, 1, 1], np.float32), top_k=np.array([0, 5, 40_000, 7, 1, -3], np.int32),
               top_p=np.array([0.9, 0.5, 1.5, -1.0, 0.99, 1.0], np.float32),
               min_p=np.array([0.0, 0.1, 0.0, 0.2, 1.5, 0.001], np.float32))
    sample.check(parts, sample.uniform(rng, P, 5), per)


@pytest.mark.parametrize("P,n", [(40, 700), (3, 20_000), (2, 150_000)])
def test_draws_on_a_stream_and_in_a_graph(P, n):
    rng = np.random.default_rng([P, n])
    s, u = (torch.from_numpy(rng.standard_normal(k, dtype=np.float32)).cuda() for k in (P * n, P * 8))
    u = (u.view(P, 8) * 0.2 + 0.5).clamp(0, 1)
    seg = torch.arange(P + 1, device="cuda") * n
    how = dict(top_k=300, top_p=0.95, temperature=0.8)
    idx, prob, kept = hwsel.hwsel_sample_per_problem(s, seg, u, **how)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = hwsel.hwsel_sample_per_problem(s, seg, u, stream=side, **how)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (idx, prob, kept)))
    ws = torch.empty(max(256, hwsel.hwsel_sample_workspace_bytes(P * n, P, 8)), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(t) for t in (idx, prob, kept)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hwsel.hwsel_sample_per_problem(s, seg, u, idx=out[0], prob=out[1], kept=out[2], workspace=ws, **how)
    for turn in range(4):
        s.copy_(torch.roll(s, 1))                           # other scores for every replay
        want = hwsel.hwsel_sample_per_problem(s, seg, u, **how)
        for t in out:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
