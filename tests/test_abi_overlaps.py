"""Results of dropout and joins that share a part of another operand's or result's memory: refused on the host, so
these run without a GPU."""
import ctypes as C

import pytest

from paper_2609_35587_amd import hwsel

F, B = 3, 0
ROWS, COLS = 10, 64
SPAN = (9 * COLS + COLS) * 4                                # bytes of a matrix of fp32


@pytest.fixture(scope="module")
def L():
    return hwsel.lib()


def mat(data, ld=COLS, dtype=F):
    return hwsel.hwsel_matrix_t(data, ld, dtype)


def place(i):
    return 0x100000 * (i + 1)


FORWARD = ("x", "y", "gate", "x1", "z")
BACKWARD = ("x1", "y", "gate", "d_x1", "d_z", "dx", "dy", "dgate")


def join(**over):
    a = dict(rows=ROWS, cols=COLS, w_branch=place(20), w_pre=place(21), eps=1e-6, stream_scale=1.0, branch_scale=1.0, post_norm=1,
             gate_sigmoid=0, gate_cols=COLS)
    state = over.pop("state", place(22))
    a.update(over)
    return hwsel.hwsel_join_t(dropout=hwsel.hwsel_dropout_t(1, 2, state, 0.1), **a)


def forward(L, j=None, **over):
    m = {n: mat(place(i)) for i, n in enumerate(FORWARD)} | over
    return L.hwsel_block_join(C.byref(j or join()), *[C.byref(m[n]) for n in FORWARD], None), L.hwsel_last_error()


def backward(L, j=None, dwb=place(23), dwp=place(24), ws=place(25), **over):
    m = {n: mat(place(i)) for i, n in enumerate(BACKWARD)} | over
    st = L.hwsel_block_join_gradient(C.byref(j or join()), *[C.byref(m[n]) for n in BACKWARD], dwb, dwp, ws, 1 << 40, None)
    return st, L.hwsel_last_error()


def dropout(L, x, r, y, rows=ROWS, state=None):
    how = hwsel.hwsel_dropout_t(1, 2, state, 0.5)
    return L.hwsel_dropout(C.byref(how), rows, COLS, C.byref(x), C.byref(r), C.byref(y), None), L.hwsel_last_error()


def refused(answer, name):
    return answer[0] == 1 and (b": %s in the place of another" % name.encode()) in answer[1]


def taken(answer):
    """Past the checks: there is no GPU here to run it, or it is of no concern (the addresses are never used on one)."""
    return b"in the place of another" not in answer[1]


SHIFTS = (SPAN - 4, -(SPAN - 4), 4, -256, 4 * COLS)


@pytest.mark.parametrize("by", SHIFTS)
def test_parts_of_matrices(L, by):
    for out, others in dict(x1=("x", "y", "gate", "z"), z=("x", "y", "gate")).items():
        for n in others:
            assert refused(forward(L, **{out: mat(place(FORWARD.index(n)) + by)}), out), (out, n)
    ins = ("x1", "y", "gate", "d_x1", "d_z")
    for out, others in dict(dx=ins, dy=ins + ("dx",), dgate=ins + ("dx", "dy")).items():
        for n in others:
            assert refused(backward(L, **{out: mat(place(BACKWARD.index(n)) + by)}), out), (out, n)
    far = mat(place(3))
    assert refused(dropout(L, mat(place(0)), far, mat(place(0) + by)), "Y") and refused(dropout(L, far, mat(place(0)), mat(place(0) + by)), "Y")


@pytest.mark.parametrize("by", (0, 4 * COLS - 4, 4 - 4 * COLS))
def test_weights_and_their_gradients(L, by):
    assert refused(forward(L, join(w_branch=place(3) + 256 + by)), "x1") and refused(forward(L, join(w_pre=place(4) + 256 + by)), "z")
    for n in BACKWARD[:5]:
        assert refused(backward(L, dwb=place(BACKWARD.index(n)) + 256 + by), "dw_branch"), n
        assert refused(backward(L, dwp=place(BACKWARD.index(n)) + 256 + by), "dw_pre"), n
    for n in ("dx", "dy", "dgate"):
        assert refused(backward(L, dwp=place(BACKWARD.index(n)) + 256 + by), "dw_pre"), n
    for i in (20, 21):
        assert refused(backward(L, dwb=place(i) + by), "dw_branch") and refused(backward(L, dwp=place(i) + by), "dw_pre")
    assert refused(backward(L, dwp=place(23) + by), "dw_pre")


def test_the_state_and_the_workspace(L):
    assert refused(forward(L, join(state=place(3) + 8)), "x1") and refused(backward(L, join(state=place(6) + 8)), "dy")
    assert refused(dropout(L, mat(place(0)), mat(place(1)), mat(place(2)), state=place(2) + 16), "Y")
    for i in (0, 4, 5, 20, 23):
        assert refused(backward(L, ws=place(i)), "the workspace"), i


if_no_gpu = pytest.mark.skipif(__import__("torch").cuda.is_available(), reason="the addresses are none of a GPU's")


@if_no_gpu
def test_what_lies_apart(L):
    """Neighbours, columns of one buffer, in place: as before."""
    assert taken(forward(L)) and taken(backward(L))
    assert taken(forward(L, x1=mat(place(0)))) and taken(backward(L, dx=mat(place(3))))
    assert taken(forward(L, z=mat(place(0) + SPAN))) and taken(backward(L, dy=mat(place(0) - SPAN)))
    wide = 3 * COLS                                         # x, x1, z side by side
    assert taken(forward(L, x=mat(place(0), wide), x1=mat(place(0) + 4 * COLS, wide), z=mat(place(0) + 8 * COLS, wide),
                         y=mat(place(10)), gate=mat(place(11))))
    assert refused(forward(L, x=mat(place(0), wide), x1=mat(place(0) + 4 * COLS - 4, wide)), "x1")
    # a bf16 matrix beside an fp32 one, rows equally far apart; every second row of a buffer against its other columns
    assert taken(forward(L, x=mat(place(0), wide), y=mat(place(10), COLS, B), gate=mat(place(11), COLS, B), z=mat(place(0) + 4 * COLS, 2 * wide, B)))
    assert taken(dropout(L, mat(place(0), wide), mat(place(9)), mat(place(0) + 4 * COLS, 2 * wide)))
    assert refused(dropout(L, mat(place(0), wide), mat(place(9)), mat(place(0) + 4 * COLS, 2 * wide + 1)), "Y")
    # a row alone is as long as it is, whatever its step
    assert taken(dropout(L, mat(place(0), 1 << 20), mat(place(9)), mat(place(0) + 4 * COLS, 1 << 20), rows=1))
    assert taken(dropout(L, mat(place(0)), mat(0), mat(place(0))))
