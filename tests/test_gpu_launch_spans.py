"""Dropout and joins of more rows than one launch has."""
import pytest
import torch

from _learn_util import mask64
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
B = torch.bfloat16


def test_dropout():
    """A launch has fewer than 2^31 groups of eight columns: rows of nine, two groups each, go in two launches."""
    rows, cols = 2 ** 30 + 100, 9
    end = (2 ** 31 - 512) // 2                              # the first launch's rows
    assert end < rows - 300
    x = torch.ones(rows, cols, dtype=B, device="cuda")
    y = hwsel.hwsel_dropout(x, 0.5, 3, 4, out=x)
    for first in (0, end - 4, end, rows - 8):
        kept, factor = mask64(8, cols, 0.5, 3, 4, first)
        assert torch.equal(y[first:first + 8].cpu(), kept.to(B) * factor), first


def test_joins_of_long_rows():
    """A launch has 2^21 rows of more columns than registers hold."""
    rows, cols = 2 ** 21 + 5, 16_392
    x = torch.ones(rows, cols, dtype=B, device="cuda")
    x[-1] = 3.0
    x1, _ = hwsel.hwsel_block_join(dict(stream_scale=2.0), x, x1=x, with_z=False)
    assert x1 is x and bool((x[-1] == 6.0).all())
    for part in x[:-1].split(2 ** 18):
        low, high = torch.aminmax(part)
        assert float(low) == 2.0 and float(high) == 2.0


def test_gradients_of_joins_of_long_rows():
    """The rows' sums have 2^21 rows a launch: the same row again and again has the same gradient."""
    rows, cols = 2 ** 21 + 5, 8200
    g = torch.Generator(device="cuda").manual_seed(6)
    one = lambda: torch.randn(1, cols, generator=g, device="cuda").to(B)  # noqa: E731
    x1, d_z = one(), one()
    want = hwsel.hwsel_block_join_gradient({}, x1, d_z=d_z)[0]
    dx = torch.zeros(rows, cols, dtype=B, device="cuda")
    x1, d_z = x1.repeat(rows, 1), d_z.repeat(rows, 1)
    assert hwsel.hwsel_block_join_gradient({}, x1, d_z=d_z, dx=dx)[0] is dx
    del x1, d_z
    assert all(bool((part == want).all()) for part in dx.split(2 ** 18))
