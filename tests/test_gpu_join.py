"""Joins of blocks to a residual stream and their gradients against binary64, within bounds counted from
their fp32 operations and the rounding of their results."""
import itertools
import math

import pytest
import torch

from _learn_util import Join, near
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
F, B = torch.float32, torch.bfloat16
TYPES = [(F, F), (B, B), (F, B), (B, F)]
SIZES = [(1, 1), (3, 2), (1, 7), (5, 8), (9, 33), (40, 128), (17, 129), (7, 250), (6, 512), (5, 513), (4, 1000), (3, 1024), (5, 1025),
         (2, 2048), (3, 2500), (3, 4096), (2, 4100), (2, 8192), (2, 8200), (2, 16_384), (3, 16_390), (2, 33_000), (1, 70_000)]
OPTIONS = list(itertools.product([False, True], ["none", "row", "element"], [False, True], [0.0, 0.2]))


def some(g, rows, cols, dtype, pad=0, sd=1.0):
    return (sd * torch.randn(rows, cols + pad, generator=g, device="cuda")).to(dtype)[:, pad // 2:pad // 2 + cols]


def made(rows, cols, st, bt, post_norm=True, gate="element", sigmoid=True, p=0.0, pad=0, seed=0, weights=True):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + rows + cols)
    d = dict(x=some(g, rows, cols, st, pad, 2.0), y=some(g, rows, cols, bt, 2 * pad), d_x1=some(g, rows, cols, st, pad), d_z=some(g, rows, cols, bt, pad))
    width = {"none": 0, "row": 1, "element": cols}[gate]
    d["gate"] = some(g, rows, width, bt, pad, 1.5) if width else None
    w = lambda: 1.0 + 0.3 * torch.randn(cols, generator=g, device="cuda")  # noqa: E731
    d["join"] = dict(post_norm=post_norm, gate_sigmoid=sigmoid, eps=1e-5, stream_scale=0.75, branch_scale=1.25, p=p, seed=2 ** 40 + seed,
                     offset=17, **(dict(w_branch=w(), w_pre=w()) if weights else {}))
    return d


def check_forward(d, x1, z):
    want = Join(d["join"], d["x"], d["y"], d["gate"])
    if x1 is not None:
        near(x1, want.x1, want.e1, "x1")
    if z is not None:
        near(z, want.z, want.ez, "z")


def check_gradient(d, x1, got):
    want = Join(d["join"], d["x"], d["y"], d["gate"], x1=x1, d_x1=d["d_x1"], d_z=d["d_z"])
    dx, dy, dgate, dw_branch, dw_pre = got
    near(dx, want.dx, want.edx, "dx")
    if d["y"] is not None:
        near(dy, want.dy, want.edy, "dy")
    else:
        assert dy is None
    if d["gate"] is not None:
        near(dgate, want.dgate, want.edgate, "dgate")
    else:
        assert dgate is None
    if d["join"].get("w_branch") is not None:
        near(dw_branch, want.dw_branch, want.edw_branch, "dw_branch")
    else:
        assert dw_branch is None
    if d["join"].get("w_pre") is not None and d["d_z"] is not None:
        near(dw_pre, want.dw_pre, want.edw_pre, "dw_pre")
    else:
        assert dw_pre is None


def both(d):
    x1, z = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"])
    assert x1.dtype == d["x"].dtype and z.dtype == d["y"].dtype
    check_forward(d, x1, z)
    check_gradient(d, x1, hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], d["d_x1"], d["d_z"]))


@pytest.mark.parametrize("i,size", enumerate(SIZES))
@pytest.mark.parametrize("st,bt", TYPES)
@pytest.mark.parametrize("turn", range(3))
def test_sizes(i, size, st, bt, turn):
    """Every size with three sets of options, every set with several sizes."""
    post_norm, gate, sigmoid, p = OPTIONS[(5 * i + 8 * turn + TYPES.index((st, bt))) % len(OPTIONS)]
    both(made(*size, st, bt, post_norm, gate, sigmoid, p, pad=(0, 1, 8)[turn]))


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("cols", [72, 1100])
def test_options(options, cols):
    both(made(6, cols, F, F, *options))


@pytest.mark.parametrize("rows,cols", [(5000, 24), (3000, 200), (1500, 640), (700, 1500), (400, 5000), (40, 20_000)])
@pytest.mark.parametrize("st,bt", [(F, F), (B, B)])
def test_many_rows(rows, cols, st, bt):
    both(made(rows, cols, st, bt, p=0.1))


@pytest.mark.parametrize("cols", [40, 700, 3000, 17_000])
def test_parts(cols):
    """Without a block, without weights, one result or one gradient alone."""
    d = made(5, cols, F, B)
    j = {k: v for k, v in d["join"].items() if k not in ("w_branch", "post_norm", "gate_sigmoid")}
    first = {**d, "join": j, "y": None, "gate": None}
    x1, z = hwsel.hwsel_block_join(j, d["x"], dtype=B)
    assert z.dtype == B
    check_forward(first, x1, z)
    check_gradient(first, x1, hwsel.hwsel_block_join_gradient(j, x1, None, None, d["d_x1"], d["d_z"]))
    bare = made(5, cols, F, B, weights=False)
    both(bare)
    x1, none = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"], with_z=False)
    assert none is None
    check_forward(d, x1, None)
    none, z = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"], with_x1=False)
    assert none is None
    check_forward(d, None, z)
    for left in ("d_x1", "d_z"):
        part = {**d, left: None}
        check_gradient(part, x1, hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], part["d_x1"], part["d_z"]))


@pytest.mark.parametrize("cols", [64, 900, 2600, 20_000])
def test_odd_values(cols):
    """Rows of zeros, very large and very small rows, infinities and NaN where dropout takes them and in rows of their own."""
    d = made(8, cols, F, F, p=0.0)
    d["y"][0], d["x"][1], d["y"][1] = 0.0, 0.0, 0.0
    d["y"][2] *= 1e15
    d["y"][3] *= 1e-15
    d["gate"][4] = 150.0
    d["gate"][5] = -150.0
    x1, z = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"])
    check_forward(d, x1, z)
    check_gradient(d, x1, hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], d["d_x1"], d["d_z"]))
    clean = [t.clone() for t in (x1, z)]
    d["x"][6, cols // 2] = float("nan")
    d["x"][7, cols // 3] = float("inf")
    x1, z = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"])
    assert torch.equal(x1[:6], clean[0][:6]) and torch.equal(z[:6], clean[1][:6])
    assert bool(torch.isnan(z[6]).all()) and int(torch.isnan(x1).sum()) == 1 and float(x1[7, cols // 3]) == float("inf")
    # all of the branch dropped: the stream alone
    d = made(4, cols, F, F, p=1.0, gate="none")
    d["y"][:, 1] = float("nan")
    d["join"]["post_norm"] = False
    x1, _ = hwsel.hwsel_block_join(d["join"], d["x"], d["y"])
    assert torch.equal(x1, 0.75 * d["x"])


@pytest.mark.parametrize("cols", [64, 900, 2600, 9000, 20_000])
@pytest.mark.parametrize("t", [F, B])
def test_in_place_and_out(cols, t):
    d = made(5, cols, t, t, p=0.3)
    x1, z = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"])
    x = d["x"].clone()
    got, z2 = hwsel.hwsel_block_join(d["join"], x, d["y"], d["gate"], x1=x)
    assert got is x and torch.equal(x, x1) and torch.equal(z, z2)
    want = hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], d["d_x1"], d["d_z"])
    wide = torch.full((9, cols + 11), 7.0, dtype=t, device="cuda")
    out = wide[2:7, 3:3 + cols]
    dx1 = d["d_x1"].clone()
    w = torch.empty(cols, device="cuda")
    got = hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], dx1, d["d_z"], dx=dx1, dy=out, dw_pre=w)
    assert got[0] is dx1 and got[1] is out and got[4] is w
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out.fill_(7.0)
    assert bool((wide == 7.0).all())
    wide = torch.full((9, cols + 11), 7.0, dtype=t, device="cuda")
    out = wide[2:7, 3:3 + cols]
    assert torch.equal(hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"], z=out)[1], z)
    out.fill_(7.0)
    assert bool((wide == 7.0).all())


def test_state_in_place_of_seed():
    d = made(6, 300, B, B, p=0.4)
    state = torch.tensor([123, 456], device="cuda")
    d["join"]["state"] = state
    both(d)
    state += 1
    both(d)


def test_same_bits():
    """Sums over rows are added in one order."""
    for cols in (100, 1024, 3000, 20_000):
        d = made(300, cols, F, B, p=0.1)
        x1, _ = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"])
        got = [hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], d["d_x1"], d["d_z"]) for _ in range(3)]
        assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_weights_of_the_longest_rows():
    """More columns than the threads of one launch can sum."""
    cols = (1 << 27) + 40
    g = torch.Generator(device="cuda").manual_seed(8)
    x1 = torch.randn(1, cols, generator=g, device="cuda")
    d_z = torch.randn(1, cols, generator=g, device="cuda")
    join = dict(w_pre=torch.ones(cols, device="cuda"))
    dw = hwsel.hwsel_block_join_gradient(join, x1, d_z=d_z)[4]
    r1 = 1.0 / math.sqrt(sum(float(p.double().square().sum()) for p in x1.split(1 << 24, 1)) / cols + 1e-6)
    # a thread adds 2^18 squares, 8 + 2 more to join threads, each rounding of a sum of positive terms within
    # 2^-24 of it; r1 has half of that; mean, root, quotient and two products here and there
    bound = (2**18 + 10) * 2.0**-24 / 2 + 10 * 2.0**-24
    want = d_z[0] * (x1[0] * r1)
    assert bool(((dw - want).abs() <= bound * want.abs() + 2.0**-126).all())
    assert bool((dw[-40:] != 0).all())


@pytest.mark.parametrize("cols", [64, 900, 2600, 9000, 20_000])
@pytest.mark.parametrize("gate", ["none", "row", "element"])
def test_gradients_that_are_dropped(cols, gate):
    """The branch has no part in what is dropped: a NaN there stays in the stream."""
    d = made(6, cols, F, B, p=0.5, gate=gate)
    x1, _ = hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"])
    kept = hwsel.hwsel_dropout(torch.ones(6, cols, device="cuda"), 0.5, d["join"]["seed"], d["join"]["offset"]) != 0
    at = (~kept[2]).nonzero()[3, 0]
    clean = hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], d["d_x1"], d["d_z"])
    d["d_x1"][2, at] = float("nan")
    got = hwsel.hwsel_block_join_gradient(d["join"], x1, d["y"], d["gate"], d["d_x1"], d["d_z"])
    assert bool(torch.isnan(got[0][2, at])) and int(torch.isnan(got[0]).sum()) == 1
    assert all(a is b or torch.equal(a, b) for a, b in zip(got[1:], clean[1:]))
