"""Few rows against so many columns that they take more than one launch: 2^22
workgroups of 32 or 64 columns cover 2^27 and 2^28.  The first columns, those
around each launch's end and the last ones are as of those columns alone."""
import pytest
import torch

from _gpu_util import say
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,span", [(17, (1 << 28) + 77, 1 << 27), (2, (1 << 29) + 133, 1 << 28)])
def test_columns_past_a_launch(M, N, span):
    say(f"product {M} x {N} x 128")
    g = torch.Generator(device="cuda").manual_seed(M)
    q = torch.empty(N, 128, dtype=torch.uint8, device="cuda").random_(0, 120, generator=g)
    scale = torch.full((-(-N // 128), 4), 120, dtype=torch.uint8, device="cuda")
    scale[:, 0] += torch.arange(scale.shape[0], device="cuda").remainder_(7).to(torch.uint8)
    b = dict(q=q, scale=scale, rows=N, cols=128, format=0, block_rows=128)
    a = hwsel.hwsel_fp8_quantise(torch.randn(M, 128, generator=g, device="cuda"))
    bias = torch.empty(N, device="cuda").normal_(generator=g)
    for dtype in (torch.bfloat16, torch.float32):
        y = hwsel.hwsel_fp8_matmul(a, b, dtype, bias=bias, gelu=True)
        for lo in sorted({0, span - 512, span, 2 * span - 512, 2 * span, (N - 600) // 128 * 128}):
            hi = min(N, lo + 1000)
            part = dict(b, q=q[lo:hi], scale=scale[lo // 128:], rows=hi - lo)
            want = hwsel.hwsel_fp8_matmul(a, part, dtype, bias=bias[lo:hi].clone(), gelu=True)
            assert torch.equal(y[:, lo:hi], want), (dtype, lo)
        del y
