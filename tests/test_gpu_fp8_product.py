"""Products of 8-bit matrices against binary64 products of the same values.

Bounds, from the arithmetic.  Results in fp32: a product of two codes is exact,
so the result is off by the roundings of the running sums alone.  With |a| |b|
the product of the magnitudes, K / 128 + 8 partial sums on the longest way of
any term, and 2^-23 for each (a matrix core may truncate where fp32 rounds),
|error| <= (K / 128 + 8) 2^-23 (|a| |b|) + 2^-23 |result|.  Results in bf16 and
8 bits: the instruction keeps each product of a group of eight to 2^-13 of the
group's largest, so up to seven lose at most that much of it, 7 2^-13 of the
group's magnitudes at the very most, plus the result's rounding (2^-8 relative
in bf16, whose significand has 8 bits); over a whole matrix such errors are of either sign and the norm of
all errors is held to 2^-8 of the result's, the most bf16 rounding alone can
do.  GELU has a slope of at most 1.13 and adds 1e-6 (fp32) or 1e-5, the bounds
that the header states; the bias adds one rounding."""
import pytest
import torch

from _fp8_util import E4M3, E5M2, code_values, gelu64, grid_values, random_rows, same_values
from _gpu_util import say
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
SIZES = [(1, 1, 1), (1, 1024, 1024), (2, 7, 130), (16, 1000, 4096), (17, 128, 256), (33, 512, 16384), (64, 130, 129),
         (127, 129, 1000), (128, 256, 512), (129, 257, 640), (300, 1, 256), (513, 1000, 2500), (1024, 1024, 1024),
         (100, 200, 100_000), (4099, 384, 128), (600, 2048, 640)]


def gen(*seed):
    return torch.Generator(device="cuda").manual_seed(hash(seed) % (1 << 31))


def operands(M, N, K, fmt_a=E4M3, block_a=1, block_b=128):
    g = gen(M, N, K, fmt_a, block_a, block_b)
    a = hwsel.hwsel_fp8_quantise(random_rows(g, M, K), format=fmt_a, block_rows=block_a)
    b = hwsel.hwsel_fp8_quantise(random_rows(g, N, K) / K ** 0.5, block_rows=block_b)
    return g, a, b


def exact(a, b, bias=None, gelu=False, fine=True):
    """The result in binary64 and the bound on the error of its sums (fine: those of fp32 results)."""
    A, B = code_values(a), code_values(b)
    y, mag = A @ B.t(), A.abs() @ B.abs().t()
    err = ((a["cols"] / 128 + 8) * 2.0 ** -23 + (0.0 if fine else 7 * 2.0 ** -13)) * mag
    if bias is not None:
        y = y + bias.double()
        err = err + 2.0 ** -24 * y.abs()
    if gelu:
        y, err = gelu64(y), 1.13 * err + (1e-6 if fine else 1e-5)
    return y, err


def assert_within(got, y, err, dtype):
    bound = err + y.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) + 1e-37
    off = (got.double() - y).abs()
    assert bool((off <= bound).all()), f"worst {float((off / bound).max()):.3g} of the bound"
    if dtype == torch.bfloat16:
        assert float(off.norm()) <= 2.0 ** -8 * float(y.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bias,gelu", [(False, False), (True, True)])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(M, N, K, bias, gelu, dtype):
    say(f"product {M}x{N}x{K} bias={bias} gelu={gelu} {dtype}")
    g, a, b = operands(M, N, K)
    v = torch.randn(N, generator=g, device="cuda") if bias else None
    out = torch.full((M + 1, N), 7.0, dtype=dtype, device="cuda")
    hwsel.hwsel_fp8_matmul(a, b, bias=v, gelu=gelu, out=out[:M])
    assert_within(out[:M], *exact(a, b, v, gelu, dtype == torch.float32), dtype)
    assert bool((out[M] == 7.0).all())
    again = hwsel.hwsel_fp8_matmul(a, b, dtype, bias=v, gelu=gelu)
    assert torch.equal(again, out[:M])                     # the same bits from call to call


@pytest.mark.parametrize("fmt_a", [E4M3, E5M2])
@pytest.mark.parametrize("block_a,block_b", [(1, 1), (128, 1), (128, 128)])
@pytest.mark.parametrize("M,N,K", [(5, 300, 1111), (200, 140, 700), (513, 129, 3000)])
def test_formats_and_blocks(M, N, K, block_a, block_b, fmt_a):
    _, a, b = operands(M, N, K, fmt_a, block_a, block_b)
    assert_within(hwsel.hwsel_fp8_matmul(a, b, torch.float32), *exact(a, b), torch.float32)


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_layer(M, N, K, gelu):
    """The quantised result: each block's exponent is the least that holds its
    largest value (give or take the sums' error), each value is within half a
    step of the grid of the exact one, plus that error, and padding is 0."""
    say(f"layer {M}x{N}x{K} gelu={gelu}")
    g, a, b = operands(M, N, K)
    v = torch.randn(N, generator=g, device="cuda")
    m = hwsel.hwsel_fp8_layer(a, b, bias=v, gelu=gelu)
    blocks = -(-N // 128)
    assert int(m["q"][:, N:blocks * 128].to(torch.int32).sum()) == 0
    y, err = exact(a, b, v, gelu, False)
    pad = torch.nn.functional.pad
    per = lambda t: pad(t, (0, blocks * 128 - N)).view(M, blocks, 128).amax(2)  # noqa: E731
    top, slack = per(y.abs()), per(err)
    scale = torch.exp2(m["scale"][:, :blocks].double() - 127.0)
    assert bool((top - slack <= 448.0 * scale).all()) and bool(((top + slack > 224.0 * scale) | (scale <= 2.0 ** -126)).all())
    step = torch.maximum(y.abs() / 8, scale.repeat_interleave(128, 1)[:, :N] * 2.0 ** -9)
    off = (code_values(m) - y).abs()
    assert bool((off <= step / 2 * 1.07 + 2 * err).all())
    assert float(off.norm()) <= 2.0 ** -4 * float(y.norm())


def test_products_are_exact_where_sums_are():
    """Small whole numbers: every sum fits fp32, so the result is exact whatever the order."""
    g = gen(1)
    for M, N, K in ((3, 5, 128), (40, 300, 5000), (300, 300, 2048), (16, 16, 65536)):
        x = torch.randint(-3, 4, (M, K), generator=g, device="cuda").float()
        w = torch.randint(-2, 3, (N, K), generator=g, device="cuda").float()
        a, b = hwsel.hwsel_fp8_quantise(x), hwsel.hwsel_fp8_quantise(w, block_rows=128)
        y = x.double() @ w.double().t()
        assert torch.equal(hwsel.hwsel_fp8_matmul(a, b, torch.float32).double(), y)
        assert torch.equal(hwsel.hwsel_fp8_matmul(a, b).double(), y.bfloat16().double())
        m = hwsel.hwsel_fp8_layer(a, b)
        want, e = grid_values(y, E4M3)
        assert same_values(code_values(m), want)
        assert torch.equal(m["scale"][:, :-(-N // 128)].to(torch.int32) - 127, e.to(torch.int32))


def test_rows_keep_to_themselves():
    """NaN and infinities of one row of A reach that row of C alone."""
    g = gen(2)
    x, w = random_rows(g, 70, 500), random_rows(g, 90, 500)
    x[5, 3] = float("nan")
    x[66, 499] = float("inf")
    a, b = hwsel.hwsel_fp8_quantise(x), hwsel.hwsel_fp8_quantise(w, block_rows=128)
    y = hwsel.hwsel_fp8_matmul(a, b, torch.float32, gelu=True)
    bad = torch.isnan(y).any(1).nonzero().flatten().tolist()
    assert bad == [5, 66] and bool(torch.isnan(y[5]).all())
    clean = x.clone()
    clean[[5, 66]] = 0.0
    z = hwsel.hwsel_fp8_matmul(hwsel.hwsel_fp8_quantise(clean), b, torch.float32, gelu=True)
    rest = [r for r in range(70) if r not in bad]
    assert torch.equal(y[rest], z[rest])


def test_gelu_limits():
    """Through the product of one element: large, infinite and NaN arguments."""
    one = hwsel.hwsel_fp8_quantise(torch.ones(1, 1, device="cuda"), block_rows=128)
    a = hwsel.hwsel_fp8_quantise(torch.tensor([[1.0], [-1.0], [0.0]], device="cuda"))
    for bias, want in ((1e30, [1e30, 1e30, 1e30]), (-1e30, [0.0, 0.0, 0.0]), (float("inf"), [float("inf")] * 3)):
        y = hwsel.hwsel_fp8_matmul(a, one, torch.float32, bias=torch.tensor([bias], device="cuda"), gelu=True)
        assert torch.equal(y.flatten().cpu(), torch.tensor(want)), bias
    y = hwsel.hwsel_fp8_matmul(a, one, torch.float32, bias=torch.tensor([float("nan")], device="cuda"), gelu=True)
    assert bool(torch.isnan(y).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,ld", [(0, 300), (1, 301), (2, 308), (4, 304)])
def test_result_strides(offset, ld, dtype):
    _, a, b = operands(150, 290, 400)
    out = torch.full((150, ld), 7.0, dtype=dtype, device="cuda")
    hwsel.hwsel_fp8_matmul(a, b, out=out[:, offset:offset + 290])
    assert torch.equal(out[:, offset:offset + 290], hwsel.hwsel_fp8_matmul(a, b, dtype))
    assert bool((out[:, :offset] == 7.0).all()) and bool((out[:, offset + 290:] == 7.0).all())


@pytest.mark.parametrize("R,N,K", [(40, 30, 50), (300, 260, 140), (5000, 96, 200)])
def test_gradients(R, N, K):
    """dX and dW of L = sum(G * (X W^T)) by 8-bit products: against the formulas
    on the quantised values (bound of a product), and against central
    differences of L in binary64 along random directions: L is linear in X and
    in W, so the difference is <D, dX> up to binary64 rounding, and the 8-bit
    operands' own rounding (half a step: 2^-4 for E4M3, 2^-3 for E5M2) averages
    over the entries: 3 % of the norms at these sizes, five times that is asked."""
    g = gen(R, N, K)
    x, w, dy = (torch.randn(s, generator=g, device="cuda") for s in ((R, K), (N, K), (R, N)))
    x8, w8t = hwsel.hwsel_fp8_quantise(x), hwsel.hwsel_fp8_quantise(w, block_rows=128, transpose=True)
    g8 = hwsel.hwsel_fp8_quantise(dy, format=E5M2)
    g8t, x8t = hwsel.hwsel_fp8_quantise(dy, format=E5M2, transpose=True), hwsel.hwsel_fp8_transpose(x8)
    dx, dw = hwsel.hwsel_fp8_matmul(g8, w8t, torch.float32), hwsel.hwsel_fp8_matmul(g8t, x8t, torch.float32)
    assert_within(dx, *exact(g8, w8t), torch.float32)
    assert_within(dw, *exact(g8t, x8t), torch.float32)
    loss = lambda X, W: float((dy.double() * (X @ W.t())).sum())  # noqa: E731
    X, W = x.double(), w.double()
    for grad, at, f in ((dx, X, lambda v: loss(v, W)), (dw, W, lambda v: loss(X, v))):
        d = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64)
        diff = (f(at + 0.5 * d) - f(at - 0.5 * d))
        along = float((grad.double() * d).sum())
        assert abs(along - diff) <= 0.15 * float(grad.double().norm() * d.norm()) / at.numel() ** 0.5 * 3


def test_repeated_in_a_graph():
    """Captured and replayed with other work in between; the split sums' workspace is the caller's."""
    _, a, b = operands(40, 200, 60_000)
    _, a2, _ = operands(40, 200, 60_000, E4M3, 128)
    ws = torch.empty(max(hwsel.hwsel_fp8_matmul_workspace_bytes(a, b), 256), dtype=torch.uint8, device="cuda")
    out, m = torch.empty(40, 200, device="cuda"), hwsel.hwsel_fp8_empty(40, 200)
    call = lambda: (hwsel.hwsel_fp8_matmul(a, b, out=out, workspace=ws),  # noqa: E731
                    hwsel.hwsel_fp8_layer(a, b, out=m, workspace=ws))
    call()
    want, codes = out.clone(), m["q"].clone()
    other = hwsel.hwsel_fp8_matmul(a2, b, torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        out.fill_(3.0)
        m["q"].fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(m["q"], codes)
        assert torch.equal(hwsel.hwsel_fp8_matmul(a2, b, torch.float32), other)


def test_two_streams_at_once():
    """Calls on two streams, each with a workspace of its own."""
    cases = [operands(64, 300, 40_000)[1:], operands(70, 256, 30_000)[1:]]
    want = [hwsel.hwsel_fp8_matmul(a, b, torch.float32) for a, b in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (s, (a, b)) in enumerate(zip(streams, cases)):
            with torch.cuda.stream(s):
                got[i].append(hwsel.hwsel_fp8_matmul(a, b, torch.float32))
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for ys, w in zip(got, want) for y in ys)


@pytest.mark.parametrize("M,N,K", [(16, 300, 20_000), (100, 200, 100_000), (513, 1000, 2500), (1024, 1024, 1024),
                                   (3000, 700, 512), (700, 600, 2048)])
def test_the_same_bits_every_time(M, N, K):
    """Thirty calls on the same operands, other work in between: a stage read before all waves' loads to it have
    come shows as another result now and then."""
    _, a, b = operands(M, N, K)
    noise = torch.empty(1 << 22, device="cuda")
    for call in (lambda: hwsel.hwsel_fp8_matmul(a, b, torch.float32), lambda: hwsel.hwsel_fp8_matmul(a, b),
                 lambda: hwsel.hwsel_fp8_layer(a, b)["q"]):
        want = call().clone()
        for i in range(30):
            noise.normal_() if i % 3 == 0 else None
            assert torch.equal(call(), want)
