"""Gradients of joins where the parts of the stream's gradient nearly cancel: a row's sums over it are those of
what is left, and their errors too."""
import pytest
import torch

from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
F, B = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.mark.parametrize("cols", [1024, 8192, 16_384, 32_768])
@pytest.mark.parametrize("bt", [F, B])
@pytest.mark.parametrize("gate", ["none", "row", "element"])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_what_is_left_of_the_streams_gradient(cols, bt, gate, p):
    """x1 is 1 or -1, so 1 / sqrt(mean x1^2 + 1e-30) is 1; d_z is of whole numbers below 256, whose sum with x1's signs is below
    2^23 and its mean m a multiple of 2^-15; d_x1 = rest - (d_z - x1 m) with rest a multiple of 2^-15 below 2^-11.  All of
    these and their differences are fp32 numbers, so d = d_x1 + (d_z - x1 m) is rest without any error."""
    rows = 3
    g = torch.Generator(device="cuda").manual_seed(cols)
    rand = lambda n: torch.rand(rows, n, generator=g, device="cuda")  # noqa: E731
    x1 = torch.where(rand(cols) < 0.4, -1.0, 1.0)
    d_z = torch.floor(256.0 * rand(cols))
    m = (d_z.double() * x1.double()).mean(1, keepdim=True)
    rest = torch.floor(1.0 + 15.0 * rand(cols)).double() * 2.0 ** -15
    d_x1 = rest - (d_z.double() - x1.double() * m)
    assert torch.equal(d_x1.float().double(), d_x1) and torch.equal(d_z.to(bt).float(), d_z)
    y = (0.5 + rand(cols)).to(bt)
    a = None if gate == "none" else (0.5 + rand(1 if gate == "row" else cols)).to(bt)
    w = 0.5 + torch.rand(cols, generator=g, device="cuda")
    join = dict(post_norm=True, w_branch=w, eps=1e-30, branch_scale=1.25, p=p, seed=11, offset=3)
    dx, dy, dgate, _, _ = hwsel.hwsel_block_join_gradient(join, x1, y, a, d_x1.float(), d_z.to(bt))
    assert torch.equal(dx.double(), rest)

    keep = hwsel.hwsel_dropout(torch.ones(rows, cols, device="cuda"), p, 11, 3).double()   # the mask over the share kept
    y, w, a = y.double(), w.double(), 1.0 if a is None else a.double()
    r = (y.square().mean(1, keepdim=True) + 1e-30).rsqrt()
    yn, dv = y * r, 1.25 * keep * rest
    dn = dv * a * w
    mean = (dn * yn).mean(1, keepdim=True)
    # A sum's longest chain is of a thread's columns (128 where 512 threads have 32,768, at most; 16 in registers) and at most
    # 20 to join threads and waves; a term has 6 roundings, r half the chain's of its sum and 6 of its own.  Terms are positive.
    chain, er = 128 + 20, (128 + 20) / 2 + 6
    half = torch.finfo(bt).eps / 2
    e_mean = mean * (chain + er + 8) * U
    bound = r * (dn * (6 + 2 * er) * U + yn * (e_mean + mean * (2 * er + 8) * U)) + 4 * U * r * (dn + yn * mean)
    want = r * (dn - yn * mean)
    assert bool(((dy.double() - want).abs() <= bound * (1 + half) + half * want.abs()).all())
    if gate == "row":
        want = (dv * w * yn).sum(1, keepdim=True)
        assert bool(((dgate.double() - want).abs() <= want * (chain + er + 8) * U * (1 + half) + half * want.abs()).all())
