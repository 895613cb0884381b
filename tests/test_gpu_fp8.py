"""8-bit matrices with block scales against 64-bit statements of the same:
quantising and restoring are exact, so codes and exponents are compared bit
for bit (as values); block edges, odd sizes and strides, blocks of zeros,
subnormal and huge blocks, NaN and infinities, scalar and vector loads."""
import math

import pytest
import torch

from _fp8_util import E4M3, E5M2, code_values, grid_values, random_rows, same_values
from _gpu_util import say
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
SIZES = [(1, 1), (1, 128), (3, 27), (16, 129), (65, 256), (130, 385), (257, 512), (70, 1000), (1000, 128)]


def gen(*seed):
    return torch.Generator(device="cuda").manual_seed(hash(seed) % (1 << 31))


def check(m, want, exps, rows, cols):
    assert m["rows"] == rows and m["cols"] == cols
    assert same_values(code_values(m), want)
    blocks = -(-cols // 128)
    got = m["scale"][:, :blocks].to(torch.int32).cpu() - 127
    assert torch.equal(got, exps.to(torch.int32).cpu())
    pad = m["q"][:rows, cols:blocks * 128]
    assert int(pad.to(torch.int32).abs().sum()) == 0


def special(x):
    """Blocks of zeros, subnormals, huge values, values at the scale's limit, NaN and infinities."""
    R, C = x.shape
    x = x.clone()
    x[0] = 0.0
    if R > 2:
        x[1] *= 2.0 ** -140
        x[2] = x[2].clamp(-1, 1) * 3e38
    if R > 8:
        x[3, : min(C, 100)] = 448.0                        # exactly the largest code
        x[4, C // 2] = 448.0 * (1 + 2 ** -8)               # just above (also in bf16)
        x[5, C // 2], x[5, 0] = math.nan, math.inf
        x[6] = -math.inf
        x[7, C - 1] = 57344.0
        x[8, C - 1] = -math.nan
    return x


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", SIZES)
def test_quantise_rows_and_restore(R, C, dtype, fmt):
    say(f"quantise rows {R}x{C} {dtype} {fmt}")
    x = special(random_rows(gen(R, C, fmt), R, C)).to(dtype)
    m = hwsel.hwsel_fp8_quantise(x, format=fmt)
    want, e = grid_values(x, fmt)
    check(m, want, e, R, C)
    y32 = hwsel.hwsel_fp8_dequantise(m, torch.float32)
    assert same_values(y32, want.float())
    assert same_values(hwsel.hwsel_fp8_dequantise(m), want.float().bfloat16())


@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", SIZES)
def test_quantise_blocks_and_transposed(R, C, dtype, fmt):
    say(f"quantise blocks and transposed {R}x{C} {dtype} {fmt}")
    x = special(random_rows(gen(R, C, fmt, 1), R, C)).to(dtype)
    for block_rows in (1, 128):
        m = hwsel.hwsel_fp8_quantise(x, format=fmt, block_rows=block_rows, transpose=True)
        check(m, *grid_values(x.t(), fmt, block_rows), C, R)
    m = hwsel.hwsel_fp8_quantise(x, format=fmt, block_rows=128)
    check(m, *grid_values(x, fmt, 128), R, C)
    assert same_values(hwsel.hwsel_fp8_dequantise(m, torch.float32), grid_values(x, fmt, 128)[0].float())


@pytest.mark.parametrize("fmt_in,fmt_out", [(E4M3, E4M3), (E5M2, E4M3), (E4M3, E5M2)])
@pytest.mark.parametrize("block_in,block_out", [(1, 1), (1, 128), (128, 1)])
@pytest.mark.parametrize("R,C", SIZES)
def test_transpose_of_kept(R, C, block_in, block_out, fmt_in, fmt_out):
    say(f"transpose {R}x{C} {block_in}->{block_out} {fmt_in}->{fmt_out}")
    m = hwsel.hwsel_fp8_quantise(special(random_rows(gen(R, C, 2), R, C)), format=fmt_in, block_rows=block_in)
    t = hwsel.hwsel_fp8_transpose(m, format=fmt_out, block_rows=block_out)
    check(t, *grid_values(code_values(m).t(), fmt_out, block_out), C, R)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", SIZES)
def test_quantise_standardised(R, C, dtype):
    g = gen(R, C, 3)
    x = special(100.0 * random_rows(g, R, C) + 30.0).to(dtype)
    mean, inv = torch.randn(C, generator=g, device="cuda") * 30, torch.rand(C, generator=g, device="cuda") + 0.01
    z = x.float()
    z = (torch.where(torch.isfinite(z), z, 0.0) - mean) * inv
    m = hwsel.hwsel_fp8_quantise(x, mean=mean, inv_std=inv)
    check(m, *grid_values(z, E4M3), R, C)


@pytest.mark.parametrize("offset,extra", [(0, 0), (1, 0), (0, 3), (2, 5), (4, 4), (8, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(dtype, offset, extra):
    """A column slice of a wider matrix, from an element that is not 16-byte aligned; rows of the
    operand's buffers further apart than they are long."""
    R, C = 150, 300
    wide = random_rows(gen(offset, extra), R, C + offset + extra).to(dtype)
    x = wide[:, offset:offset + C]
    want, e = grid_values(x, E4M3)
    big = torch.full((R, 512), 77, dtype=torch.uint8, device="cuda")
    m = hwsel.hwsel_fp8_empty(R, C)
    m["q"], m["scale"] = big[:, 16:16 + 384], torch.full((R, 12), 77, dtype=torch.uint8, device="cuda")[:, 4:8]
    hwsel.hwsel_fp8_quantise(x, out=m)
    check(m, want, e, R, C)
    assert int((big[:, :16] != 77).sum()) == 0 and int((big[:, 400:] != 77).sum()) == 0
    check(hwsel.hwsel_fp8_quantise(x, transpose=True), *grid_values(x.t(), E4M3), C, R)
    check(hwsel.hwsel_fp8_quantise(x, block_rows=128), *grid_values(x, E4M3, 128), R, C)
    out = torch.full((R, C + offset + extra), 7.0, dtype=dtype, device="cuda")
    hwsel.hwsel_fp8_dequantise(m, out=out[:, offset:offset + C])
    assert same_values(out[:, offset:offset + C], want.to(dtype))
    assert bool((out[:, :offset] == 7.0).all()) and bool((out[:, offset + C:] == 7.0).all())


def test_many_rows_reach_past_32_bits():
    """2,300,000 rows of 1,000 bf16 elements: element and byte offsets beyond 2^31."""
    R, C = 2_300_000, 1000
    x = torch.empty(R, C, dtype=torch.bfloat16, device="cuda").normal_(generator=gen(9))
    m = hwsel.hwsel_fp8_quantise(x)
    y = hwsel.hwsel_fp8_dequantise(m)
    for rows in (slice(0, 300), slice(R // 2, R // 2 + 300), slice(R - 300, R)):
        assert same_values(y[rows], grid_values(x[rows], E4M3)[0].float().bfloat16())
    t = hwsel.hwsel_fp8_transpose(m)
    lo = (R - 1000) // 128 * 128
    part = {**m, "q": m["q"][lo:], "scale": m["scale"][lo:], "rows": R - lo}
    want, e = grid_values(code_values(part).t(), E4M3)
    end = {**t, "q": t["q"][:, lo:], "scale": t["scale"][:, lo // 128:], "cols": R - lo}
    assert same_values(code_values(end), want)
    del e


def test_on_another_stream():
    x = random_rows(gen(5), 500, 700)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = hwsel.hwsel_fp8_dequantise(hwsel.hwsel_fp8_quantise(x), torch.float32)
    side.synchronize()
    assert same_values(y, grid_values(x, E4M3)[0].float())
