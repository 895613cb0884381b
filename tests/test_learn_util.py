"""The tests' own statements of the operators, without a GPU: the generator by
its published outputs, gradients by differences."""
import numpy as np
import pytest
import torch

from _learn_util import Join, Logprob, mask64, numbers, philox


def test_generator_gives_its_published_outputs():
    """Known answers of Philox4x32-10 (its authors' test vectors)."""
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 0xffffffff
    assert philox((ones,) * 4, (ones,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    pi = (0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)
    assert philox(*pi) == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_numbers_are_the_words_halves():
    seed, offset = 0x299f31d0a4093822, 0x0370734413198a2e
    got = numbers([5, 2 ** 31 - 1], 21, seed, offset)
    for r, row in enumerate((5, 2 ** 31 - 1)):
        for c in range(21):
            w = philox((c // 8, row, offset & 0xffffffff, offset >> 32), (seed & 0xffffffff, seed >> 32))[c % 8 // 2]
            assert got[r, c] == (w >> 16 * (c % 2)) & 0xffff


def test_share_kept():
    kept, factor = mask64(500, 400, 0.3, 7, 9)
    share = 1 / factor
    assert abs(share - 0.7) < 2.0 ** -17
    assert abs(float(kept.double().mean()) - share) < 5 * (share * (1 - share) / kept.numel()) ** 0.5


@pytest.mark.parametrize("post_norm", [False, True])
@pytest.mark.parametrize("gate_cols", [0, 1, 9])
def test_join_gradients_by_differences(post_norm, gate_cols):
    g = torch.Generator().manual_seed(3 * gate_cols + post_norm)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, y, gate = r(4, 9), r(4, 9), r(4, gate_cols) if gate_cols else None
    join = dict(post_norm=post_norm, gate_sigmoid=gate_cols != 1, w_branch=r(9), w_pre=r(9), eps=0.125, stream_scale=0.5, branch_scale=1.5,
                p=0.25, seed=11)
    dx1, dz = r(4, 9), r(4, 9)

    def value(x, y, gate, join):
        q = Join(join, x, y, gate)
        return float((dx1 * q.x1).sum() + (dz * q.z).sum())

    want = Join(join, x, y, gate, x1=Join(join, x, y, gate).x1, d_x1=dx1, d_z=dz)
    h = 1e-6
    for name, base in (("dx", x), ("dy", y), ("dgate", gate), ("dw_branch", join["w_branch"]), ("dw_pre", join["w_pre"])):
        if base is None:
            continue
        for i in range(base.numel()):
            both = []
            for s in (h, -h):
                t = base.clone()
                t.view(-1)[i] += s
                args = dict(x=x, y=y, gate=gate, join=join)
                if name in ("dw_branch", "dw_pre"):
                    args["join"] = {**join, name[1:]: t}
                else:
                    args[name[1:]] = t
                both.append(value(**args))
            got = float(getattr(want, name).reshape(-1)[i])
            assert abs((both[0] - both[1]) / (2 * h) - got) < 1e-6 * max(1.0, abs(got)), (name, i)


def test_logprob_gradient_by_differences():
    rng = np.random.default_rng(1)
    s = np.round(rng.standard_normal(12) * 64) / 64           # steps of 2^-13 are exact in fp32
    s[3] = -np.inf
    picks, dl, de, T = [5, 0, 5, 3, -1, 40], rng.standard_normal(6), 0.7, 0.5

    def value(s):
        q = Logprob(s, T)
        return sum(d * q.of(j)[0] for j, d in zip(picks, dl) if q.of(j)[0] > -np.inf) + de * q.entropy

    got, _ = Logprob(s, T).gradient(picks, dl, de)
    h = 2.0 ** -13
    for i in range(12):
        if i == 3:
            assert got[i] == 0
            continue
        a, b = s.copy(), s.copy()
        a[i] += h
        b[i] -= h
        assert abs((value(a) - value(b)) / (2 * h) - got[i]) < 1e-5, i
