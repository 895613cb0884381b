"""Views whose rows overlap, beside those whose rows only lie apart: the calls on
8-bit matrices refuse the first before anything runs and take the second."""
import pytest
import torch

from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


def base(n, dtype=torch.float32):
    return torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("step", [1, 2, 64, 127])
def test_overlapping_rows_are_not_read(step, dtype):
    x = base(1000, dtype).unfold(0, 128, step)
    assert x.shape[0] > 1 and x.stride() == (step, 1)
    ones = torch.ones(128, device="cuda")
    for kw in (dict(), dict(transpose=True), dict(block_rows=128), dict(mean=ones, inv_std=ones),
               dict(out=hwsel.hwsel_fp8_empty(*x.shape))):
        with pytest.raises(ValueError, match="overlap"):
            hwsel.hwsel_fp8_quantise(x, **kw)


@pytest.mark.parametrize("step", [0, 1, 39, 40, 49])
def test_overlapping_rows_are_not_written(step):
    """Also where the columns that would be written, 40 of 50, lie within a step."""
    a = hwsel.hwsel_fp8_quantise(base(20 * 300).view(20, 300))
    b = hwsel.hwsel_fp8_quantise(base(40 * 300).view(40, 300), block_rows=128)
    m = hwsel.hwsel_fp8_quantise(base(20 * 40).view(20, 40))
    flat = torch.full((1000,), 7.0, device="cuda")
    out = flat.as_strided((20, 50), (step, 1))
    with pytest.raises(ValueError, match="overlap"):
        hwsel.hwsel_fp8_matmul(a, b, out=out)
    with pytest.raises(ValueError, match="overlap"):
        hwsel.hwsel_fp8_dequantise(m, out=out)
    assert bool((flat == 7.0).all())


@pytest.mark.parametrize("step", [128, 129, 200])
def test_rows_that_lie_apart_are_taken(step):
    x = base(1000).unfold(0, 128, step)
    got, want = hwsel.hwsel_fp8_quantise(x), hwsel.hwsel_fp8_quantise(x.contiguous())
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["scale"][:, 0], want["scale"][:, 0])


def test_one_row_or_one_column_of_any_stride():
    x = base(300)
    row, column = x.as_strided((1, 128), (1, 1)), x.as_strided((50, 1), (6, 3))
    want = hwsel.hwsel_fp8_dequantise(hwsel.hwsel_fp8_quantise(x[:128].view(1, 128).clone()), torch.float32)
    assert torch.equal(hwsel.hwsel_fp8_dequantise(hwsel.hwsel_fp8_quantise(row), torch.float32), want)
    want = hwsel.hwsel_fp8_dequantise(hwsel.hwsel_fp8_quantise(x[::6].view(50, 1).clone()), torch.float32)
    assert torch.equal(hwsel.hwsel_fp8_dequantise(hwsel.hwsel_fp8_quantise(column), torch.float32), want)
