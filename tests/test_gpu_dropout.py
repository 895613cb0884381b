"""Dropout by a mask made from a counter: every bit against the stated numbers
and two fp32 operations."""
import pytest
import torch

from _learn_util import mask64
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
F, B = torch.float32, torch.bfloat16


def some(rows, cols, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn(rows, cols + pad, generator=g, device="cuda").to(dtype)
    return wide[:, pad // 2:pad // 2 + cols]


def stated(x, p, seed=0, offset=0, residual=None, first=0):
    kept, factor = mask64(*x.shape, p, seed, offset, first)
    y = torch.where(kept, x.cpu().float() * torch.tensor(factor, dtype=F), 0.0)
    if residual is None:
        return y.to(x.dtype)
    return (y + residual.cpu().float()).to(residual.dtype)


SIZES = [(1, 1), (1, 7), (3, 8), (5, 9), (2, 100), (17, 128), (33, 257), (4, 2500), (1, 70_001), (70_001, 1), (300, 1000)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("xt,yt", [(F, F), (B, B), (F, B), (B, F)])
@pytest.mark.parametrize("pad", [0, 3])
def test_every_bit(rows, cols, xt, yt, pad):
    x, r = some(rows, cols, xt, 1, pad), some(rows, cols, yt, 2, 2 * pad)
    assert torch.equal(hwsel.hwsel_dropout(x, 0.3, 5, 6).cpu(), stated(x, 0.3, 5, 6))
    got = hwsel.hwsel_dropout(x, 0.3, 5, 6, residual=r)
    assert got.dtype == yt and torch.equal(got.cpu(), stated(x, 0.3, 5, 6, r))


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 1e-3, 0.5, 0.9, 1 - 2.0 ** -16, 1 - 2.0 ** -20, 1.0])
def test_shares(p):
    x = some(50, 300, F, 3)
    x[0, :9], x[1, :9] = float("nan"), float("inf")
    r = some(50, 300, F, 4)
    for residual in (None, r):
        got, want = hwsel.hwsel_dropout(x, p, 1, 2, residual=residual).cpu(), stated(x, p, 1, 2, residual)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))
    if p == 0.0:
        assert torch.equal(hwsel.hwsel_dropout(r, p, 1, 2), r)
    if p == 1.0:
        assert not bool(hwsel.hwsel_dropout(x, p, 1, 2).any())


@pytest.mark.parametrize("seed,offset", [(0, 0), (2 ** 32, 0), (0, 2 ** 32), (2 ** 64 - 1, 2 ** 64 - 1), (1, 2 ** 63)])
def test_all_of_seed_and_offset(seed, offset):
    x = some(9, 90, B, 5)
    want = stated(x, 0.4, seed, offset)
    assert torch.equal(hwsel.hwsel_dropout(x, 0.4, seed, offset).cpu(), want)
    signed = [v - 2 ** 64 if v >= 2 ** 63 else v for v in (seed, offset)]
    state = torch.tensor(signed, device="cuda")
    assert torch.equal(hwsel.hwsel_dropout(x, 0.4, 77, 78, state=state).cpu(), want)


def test_backward_makes_the_same_mask():
    """Whatever the types and strides of the two passes."""
    x, dy = some(40, 333, B, 6), some(40, 333, F, 7, 5)
    y = hwsel.hwsel_dropout(torch.ones_like(x), 0.25, 8, 9)
    dx = hwsel.hwsel_dropout(dy, 0.25, 8, 9)
    assert torch.equal(dx == 0, y == 0)
    # the derivative of a sum weighted by dy, by the map's linearity: a difference of one element at a time is exact
    kept, factor = mask64(40, 333, 0.25, 8, 9)
    assert torch.equal(dx.cpu(), torch.where(kept, dy.cpu() * torch.tensor(factor, dtype=F), 0.0))


def test_in_place_and_out():
    x, r = some(30, 200, B, 8), some(30, 200, B, 9)
    want, plain = stated(x, 0.5, 1, 1, r), stated(x, 0.5, 1, 1)
    for out in (x.clone(), r.clone()):
        a, b = (out, r) if torch.equal(out, x) else (x, out)
        assert hwsel.hwsel_dropout(a, 0.5, 1, 1, residual=b, out=out) is out
        assert torch.equal(out.cpu(), want)
    wide = torch.full((33, 210), 7.0, dtype=F, device="cuda")
    hwsel.hwsel_dropout(x, 0.5, 1, 1, out=wide[2:32, 3:203])
    assert torch.equal(wide[2:32, 3:203].cpu(), plain.float())
    wide[2:32, 3:203] = 7.0
    assert bool((wide == 7.0).all())


def test_rows_past_2_to_31_elements():
    """Places are not 32-bit numbers: the last rows of a matrix of 2^32 + elements."""
    rows, cols = 2 ** 21 + 3, 2048
    x = torch.ones(rows, cols, dtype=B, device="cuda")
    y = hwsel.hwsel_dropout(x, 0.5, 3, 4, out=x)
    for first in (0, 2 ** 20 - 1, rows - 2):
        assert torch.equal(y[first:first + 2].cpu(), stated(torch.ones(2, cols, dtype=B), 0.5, 3, 4, first=first))
