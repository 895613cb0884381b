"""Results of log probabilities and of their gradient that share memory with an operand or another result: refused
on the host, so these run without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2609_35587_amd import hwsel

R, P, N, TOP = 1000, 40, 25, 8                              # (R = P N: a gradient is as long as d_logp)
IN = dict(scores=4 * R, seg=8 * (P + 1), Ts=4 * P, picks=4 * P * N)
OUT = dict(logp=4 * P * N, entropy=4 * P, norm=8 * P, top_idx=4 * P * TOP, top_logp=4 * P * TOP)
GRADIENT_IN = dict(scores=4 * R, seg=8 * (P + 1), Ts=4 * P, norm=8 * P, picks=4 * P * N, d_logp=4 * P * N, entropy=4 * P, d_entropy=4 * P)


@pytest.fixture(scope="module")
def L():
    return hwsel.lib()


def places(names):
    return {n: 0x100000 * (i + 1) for i, n in enumerate(names)}


def forward(L, n_picks=N, top=TOP, R=R, P=P, ws=None, nbytes=0, **over):
    a = places([*IN, *OUT]) | over
    st = L.hwsel_logprob_per_problem(a["scores"], R, a["seg"], P, 1.0, a["Ts"], a["picks"], n_picks, top, a["logp"], a["entropy"], a["norm"],
                                     a["top_idx"], a["top_logp"], ws, nbytes, None)
    return st, L.hwsel_last_error()


def gradient(L, n_picks=N, **over):
    a = places([*GRADIENT_IN, "out"]) | over
    st = L.hwsel_logprob_gradient(a["scores"], R, a["seg"], P, 1.0, a["Ts"], a["norm"], a["picks"], n_picks, a["d_logp"], a["entropy"],
                                  a["d_entropy"], a["out"], None)
    return st, L.hwsel_last_error()


def refused(answer, name):
    return answer[0] == 1 and (b": %s in the place of another" % name.encode()) in answer[1]


def ends(size, own):
    return 0, size - 4, 4 - own


def test_results(L):
    at = places([*IN, *OUT])
    for out, own in OUT.items():
        for other, size in IN.items():
            for by in ends(size, own):
                assert refused(forward(L, **{out: at[other] + by}), out), (out, other, by)
    names = list(OUT)
    for i, out in enumerate(names):
        for other in names[:i]:
            for by in ends(OUT[other], OUT[out]):
                assert refused(forward(L, **{out: at[other] + by}), out), (out, other, by)


def test_the_workspace(L):
    n = C.c_size_t(0)
    long = dict(R=3 * 534_600, P=3)
    assert L.hwsel_logprob_workspace_bytes(long["R"], 3, TOP, C.byref(n)) == 0
    if n.value:
        at = places([*IN, *OUT])
        for name in ("seg", "picks", "logp", "top_logp"):
            a = {**at, "scores": 1 << 40, name: (1 << 41) + n.value - 4 if name != "seg" else (1 << 41) + n.value - 8}
            assert refused(forward(L, **long, **a, ws=1 << 41, nbytes=n.value), "the workspace"), name


def test_the_gradient(L):
    at = places([*GRADIENT_IN, "out"])
    for other, size in GRADIENT_IN.items():
        for by in ends(size, 4 * R):
            st, text = gradient(L, out=at[other] + by)
            assert st == 1 and (b"overlaps the scores" if other == "scores" else b"in the place of another") in text, (other, by)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are none of a GPU's")
def test_what_lies_apart(L):
    place = b"in the place of another"
    at = places([*IN, *OUT])
    assert place not in forward(L)[1] and place not in gradient(L)[1]
    assert place not in forward(L, logp=at["scores"] + 4 * R, entropy=at["norm"] - 4 * P)[1]
    # what is none is nowhere
    assert place not in forward(L, n_picks=0, top=0, logp=at["scores"], picks=at["norm"], top_idx=at["scores"], top_logp=at["norm"])[1]
    assert place not in gradient(L, n_picks=0, picks=at["scores"], d_logp=places([*GRADIENT_IN, "out"])["out"])[1]
