"""dX and dW of L = sum(G * (X W^T)) by 8-bit products against binary64 on the
values before they were rounded, tight enough that a share of a gradient that
is missing, or a factor, shows.

Bounds.  Rounding to E4M3 is off by a uniform share of a step, 2^-3 of the power
of two below a value: sd 2^-3 / 12^0.5 = 0.036 of it, 0.025 of the norm over
normal values; to E5M2 twice that, 0.05.  dX sums products of one of each: 0.056
of its norm; dW those of E5M2 and of E4M3 rounded twice (rows, then columns):
0.061.  0.08 is asked, and a cosine of 1 - 0.08^2 / 2 less a half again, 0.995.
Along the gradient itself, d = grad / |grad|, the errors average out but for
their square: <grad, d> is within 0.061^2 = 0.4 % of <true, d>; 2 % is asked of
the difference L(at + d / 2) - L(at - d / 2), which is <true, d> since L is
linear in either."""
import pytest
import torch

from _fp8_util import E5M2
from _gpu_util import say
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,N,K", [(300, 260, 140), (5000, 96, 200), (65, 512, 1000), (2000, 33, 70), (4096, 512, 512)])
def test_gradients(R, N, K, dtype):
    say(f"gradients {R} x {K} -> {N} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(R + N + K)
    x, w, dy = (torch.randn(s, generator=g, device="cuda") for s in ((R, K), (N, K), (R, N)))
    dy = dy.to(dtype)
    x8, w8t = hwsel.hwsel_fp8_quantise(x), hwsel.hwsel_fp8_quantise(w, block_rows=128, transpose=True)
    dx = hwsel.hwsel_fp8_matmul(hwsel.hwsel_fp8_quantise(dy, format=E5M2), w8t, dtype)
    dw = hwsel.hwsel_fp8_matmul(hwsel.hwsel_fp8_quantise(dy, format=E5M2, transpose=True), hwsel.hwsel_fp8_transpose(x8),
                                torch.float32)
    X, W, G = x.double(), w.double(), dy.double()
    loss = lambda X, W: float((G * (X @ W.t())).sum())  # noqa: E731
    for got, want, at, f in ((dx, G @ W, X, lambda v: loss(v, W)), (dw, G.t() @ X, W, lambda v: loss(X, v))):
        got = got.double()
        assert got.shape == want.shape
        assert float((got - want).norm()) <= 0.08 * float(want.norm())
        assert float((got * want).sum()) >= 0.995 * float(got.norm() * want.norm())
        d = got / got.norm()
        along = f(at + 0.5 * d) - f(at - 0.5 * d)
        assert abs(float(got.norm()) - along) <= 0.02 * along
