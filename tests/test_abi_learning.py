"""Refusals of log probabilities, dropout and joins: checked on the host before
anything is enqueued, so they run without a GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2609_35587_amd import hwsel

FAKE = 0x1000   # never dereferenced: every call below is rejected first
F, B = 3, 0


@pytest.fixture(scope="module")
def L():
    return hwsel.lib()


def logprob(L, **over):
    a = dict(scores=FAKE, R=100, seg=FAKE, P=4, T=1.0, Ts=None, picks=FAKE, n=3, top=2, logp=FAKE, entropy=None, norm=None, idx=FAKE,
             top_logp=FAKE, ws=None, bytes=0)
    a.update(over)
    return L.hwsel_logprob_per_problem(*a.values(), None)


@pytest.mark.parametrize("over,status", [
    (dict(scores=None), 1), (dict(seg=None), 1), (dict(P=0), 1), (dict(R=-1), 1), (dict(R=(1 << 30) + 1), 2), (dict(picks=None), 1),
    (dict(logp=None), 1), (dict(n=-1), 1), (dict(top=65), 1), (dict(top=-1), 1), (dict(idx=None), 1), (dict(top_logp=None), 1)])
def test_log_probabilities_reject(L, over, status):
    assert logprob(L, **over) == status
    assert L.hwsel_last_error().startswith(b"hwsel_logprob_per_problem: ")


def test_log_probabilities_check_their_workspace(L):
    n = C.c_size_t(0)
    assert L.hwsel_logprob_workspace_bytes(100, 0, 0, C.byref(n)) == 1
    assert L.hwsel_logprob_workspace_bytes(100, 1, 65, C.byref(n)) == 1
    assert L.hwsel_logprob_workspace_bytes(100, 1, 0, None) == 1
    assert L.hwsel_logprob_workspace_bytes((1 << 30) + 1, 1, 0, C.byref(n)) == 2
    long = dict(R=3 * 534_600, P=3, top=64)
    assert L.hwsel_logprob_workspace_bytes(long["R"], 3, 64, C.byref(n)) == 0
    if n.value:
        for ws, nbytes in ((None, 0), (FAKE, n.value - 1), (FAKE + 16, n.value)):
            assert logprob(L, **long, ws=ws, bytes=nbytes) == 1
        assert L.hwsel_last_error().startswith(b"hwsel_logprob_per_problem: workspace")


@pytest.mark.parametrize("over,status", [
    (dict(scores=None), 1), (dict(seg=None), 1), (dict(P=0), 1), (dict(R=-1), 1), (dict(R=(1 << 30) + 1), 2), (dict(norm=None), 1),
    (dict(picks=None), 1), (dict(n=-1), 1), (dict(d_logp=None), 1), (dict(entropy=None), 1), (dict(d_entropy=None), 1), (dict(out=None), 1)])
def test_gradient_rejects(L, over, status):
    a = dict(scores=FAKE, R=100, seg=FAKE, P=4, T=1.0, Ts=None, norm=FAKE, picks=FAKE, n=3, d_logp=FAKE, entropy=FAKE, d_entropy=FAKE, out=FAKE)
    a.update(over)
    assert L.hwsel_logprob_gradient(*a.values(), None) == status
    assert L.hwsel_last_error().startswith(b"hwsel_logprob_gradient: ")


def mat(data=FAKE, ld=64, dtype=F):
    return hwsel.hwsel_matrix_t(data, ld, dtype)


@pytest.mark.parametrize("over,status", [
    (dict(how=None), 1), (dict(p=-0.1), 1), (dict(p=1.1), 1), (dict(p=math.nan), 1), (dict(state=FAKE + 4), 1), (dict(rows=0), 1), (dict(cols=0), 1),
    (dict(rows=1 << 31), 2), (dict(cols=1 << 31, x=mat(ld=1 << 31)), 2), (dict(x=None), 1), (dict(x=mat(None)), 1), (dict(y=None), 1),
    (dict(y=mat(None)), 1), (dict(x=mat(ld=63)), 1), (dict(x=mat(FAKE + 2)), 1), (dict(x=mat(dtype=1)), 2), (dict(y=mat(dtype=2)), 2),
    (dict(y=mat(FAKE + 1, dtype=B)), 1), (dict(r=mat(dtype=B)), 1), (dict(r=mat(ld=3)), 1), (dict(r=mat(dtype=7)), 2)])
def test_dropout_rejects(L, over, status):
    a = dict(rows=10, cols=64, x=mat(), r=mat(), y=mat(), p=0.5, state=None)
    a.update(over)
    how = hwsel.hwsel_dropout_t(1, 2, a["state"], a["p"])
    ref = lambda m: None if m is None else C.byref(m)  # noqa: E731
    how = C.byref(how) if over.get("how", 1) else None
    assert L.hwsel_dropout(how, a["rows"], a["cols"], ref(a["x"]), ref(a["r"]), ref(a["y"]), None) == status
    assert L.hwsel_last_error().startswith(b"hwsel_dropout: ")


def test_results_in_place_lie_as_their_operands(L):
    """The same address with another step or type would be read where it has been written."""
    how, m, other = hwsel.hwsel_dropout_t(1, 2, None, 0.5), mat(), 0x2000
    call = lambda x, r, y: L.hwsel_dropout(C.byref(how), 10, 64, C.byref(x), C.byref(r), C.byref(y), None)  # noqa: E731
    assert call(mat(ld=65), mat(other), m) == 1 and call(mat(dtype=B), mat(other), m) == 1 and call(mat(other), mat(ld=65), m) == 1
    assert forward(L, join(), x=mat(ld=65), y=mat(other), gate=mat(other), x1=m, z=mat(other)) == 1
    far = {n: mat(other) for n in ("x1", "y", "gate", "d_z", "dy", "dgate")}
    assert backward(L, join(), **far, d_x1=mat(ld=65), dx=m) == 1
    assert L.hwsel_last_error().startswith(b"hwsel_block_join_gradient: dx in place")


def test_results_lie_apart(L):
    place = {n: mat(0x10000 * (i + 1)) for i, n in enumerate(("x", "y", "gate", "x1", "z", "d_x1", "d_z", "dx", "dy", "dgate"))}
    for out, others in dict(x1=("y", "gate", "z"), z=("x", "y", "gate")).items():
        for n in others:
            m = {k: place[k] for k in ("x", "y", "gate", "x1", "z")} | {out: place[n]}
            assert forward(L, join(), **m) == 1 and b"in the place of another" in L.hwsel_last_error(), (out, n)
    ins = ("x1", "y", "gate", "d_z")
    for out, others in dict(dx=ins, dy=ins + ("d_x1", "dx"), dgate=ins + ("d_x1", "dx", "dy")).items():
        for n in others:
            m = {k: place[k] for k in ("x1", "y", "gate", "d_x1", "d_z", "dx", "dy", "dgate")} | {out: place[n]}
            assert backward(L, join(), **m) == 1 and b"in the place of another" in L.hwsel_last_error(), (out, n)
    for out in (0x10000, 0x10000 + 4 * 99, 0x10000 - 4 * 99):
        assert L.hwsel_logprob_gradient(0x10000, 100, FAKE, 4, 1.0, None, FAKE, None, 0, None, FAKE, FAKE, out, None) == 1
        assert L.hwsel_last_error() == b"hwsel_logprob_gradient: d_scores overlaps the scores"


def join(**over):
    a = dict(rows=10, cols=64, w_branch=FAKE, w_pre=FAKE, eps=1e-6, stream_scale=1.0, branch_scale=1.0, post_norm=1, gate_sigmoid=0,
             gate_cols=64)
    p, state = over.pop("p", 0.1), over.pop("state", None)
    a.update(over)
    return hwsel.hwsel_join_t(dropout=hwsel.hwsel_dropout_t(1, 2, state, p), **a)


BAD_JOINS = [(dict(rows=0), 1), (dict(cols=0), 1), (dict(rows=1 << 31), 2), (dict(cols=1 << 31), 2), (dict(eps=0.0), 1), (dict(eps=-1.0), 1),
             (dict(eps=math.nan), 1), (dict(eps=math.inf), 1), (dict(stream_scale=math.inf), 1), (dict(branch_scale=math.nan), 1),
             (dict(post_norm=2), 1), (dict(gate_sigmoid=-1), 1), (dict(gate_cols=2), 1), (dict(gate_cols=-1), 1), (dict(p=2.0), 1),
             (dict(state=FAKE + 1), 1), (dict(w_branch=FAKE + 2), 1), (dict(w_pre=FAKE + 1), 1)]
N = 9                                                       # matrices of a gradient call


def forward(L, j, x=mat(), y=mat(), gate=mat(), x1=mat(), z=mat()):
    return L.hwsel_block_join(None if j is None else C.byref(j), *[None if m is None else C.byref(m) for m in (x, y, gate, x1, z)], None)


def backward(L, j, dwb=FAKE, dwp=FAKE, ws=FAKE, nbytes=1 << 40, **over):
    names = ("x1", "y", "gate", "d_x1", "d_z", "dx", "dy", "dgate")
    ms = [over.get(n, mat()) for n in names]
    return L.hwsel_block_join_gradient(None if j is None else C.byref(j), *[None if m is None else C.byref(m) for m in ms], dwb, dwp, ws,
                                       nbytes, None)


@pytest.mark.parametrize("over,status", BAD_JOINS)
def test_joins_reject_their_settings(L, over, status):
    n = C.c_size_t(0)
    assert forward(L, join(**over)) == status
    assert backward(L, join(**over)) == status
    assert L.hwsel_block_join_gradient_workspace_bytes(C.byref(join(**over)), C.byref(n)) == status
    assert L.hwsel_last_error().startswith(b"hwsel_block_join_gradient_workspace_bytes: ")


def test_joins_reject_their_matrices(L):
    assert forward(L, None) == 1 and forward(L, join(), x=None) == 1 and forward(L, join(), x1=None, z=None) == 1
    assert forward(L, join(), y=None) == 1 and forward(L, join(gate_cols=0), y=None, gate=None) == 1     # (a gate, w_branch)
    assert forward(L, join(gate_cols=0)) == 1 and forward(L, join(), gate=None) == 1
    for name in ("x", "y", "gate", "x1", "z"):
        assert forward(L, join(), **{name: mat(ld=63)}) == 1
        assert forward(L, join(), **{name: mat(FAKE + 2)}) == 1
        assert forward(L, join(), **{name: mat(dtype=1)}) == 2
    for name in ("gate", "x1", "z"):
        assert forward(L, join(), **{name: mat(dtype=B)}) == 1
    assert L.hwsel_last_error().startswith(b"hwsel_block_join: z")


def test_join_gradients_reject_their_matrices(L):
    assert backward(L, None) == 1 and backward(L, join(), x1=None) == 1 and backward(L, join(), d_x1=None, d_z=None) == 1
    assert backward(L, join(), None, None, dx=None, dy=None, dgate=None) == 1
    bare = dict(gate_cols=0, w_branch=None)
    assert backward(L, join(**bare), None, y=None, gate=None, dgate=None) == 1              # dy without y
    assert backward(L, join(**bare), y=None, gate=None, dy=None, dgate=None) == 1           # dw_branch without y
    assert backward(L, join(gate_cols=0), gate=None) == 1                                   # dgate without a gate
    assert backward(L, join(), d_z=None) == 1                                               # dw_pre without d_z
    for name in ("x1", "y", "gate", "d_x1", "d_z", "dx", "dy", "dgate"):
        assert backward(L, join(), **{name: mat(ld=63)}) == 1
        assert backward(L, join(), **{name: mat(FAKE + 2)}) == 1
        assert backward(L, join(), **{name: mat(dtype=2)}) == 2
    for name in ("gate", "d_x1", "d_z", "dx", "dy", "dgate"):
        assert backward(L, join(), **{name: mat(dtype=B)}) == 1
    assert backward(L, join(), FAKE + 2) == 1 and backward(L, join(), FAKE, FAKE + 1) == 1
    n = C.c_size_t(0)
    assert L.hwsel_block_join_gradient_workspace_bytes(C.byref(join()), C.byref(n)) == 0 and n.value > 0
    assert L.hwsel_block_join_gradient_workspace_bytes(C.byref(join()), None) == 1
    assert backward(L, join(), ws=None) == 1 and backward(L, join(), ws=FAKE + 16) == 1 and backward(L, join(), nbytes=n.value - 1) == 1
    assert L.hwsel_last_error().startswith(b"hwsel_block_join_gradient: workspace")


def test_binding_rejects_host_tensors():
    s, seg, x = torch.zeros(4), torch.tensor([0, 4]), torch.zeros(4, 8)
    for call in (lambda: hwsel.hwsel_logprob_per_problem(s, seg), lambda: hwsel.hwsel_logprob_gradient(s, seg, torch.zeros(1, 2)),
                 lambda: hwsel.hwsel_dropout(x, 0.5), lambda: hwsel.hwsel_block_join({}, x), lambda: hwsel.hwsel_block_join_gradient({}, x)):
        with pytest.raises(ValueError):
            call()


def test_binding_takes_its_arguments_whole():
    b = hwsel._calls()
    for name, n in (("logprob_per_problem", 12), ("logprob_gradient", 10), ("dropout", 8), ("block_join", 10), ("block_join_gradient", 13)):
        for bad in (0, n - 1, n + 1):
            with pytest.raises(RuntimeError):
                getattr(b, name)(*[None] * bad)
        with pytest.raises((ValueError, TypeError)):
            getattr(b, name)(*[None] * n)
