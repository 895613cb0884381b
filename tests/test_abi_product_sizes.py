"""Results of a product that a launch cannot cover are refused on the host: a
launch of 2^32 threads or more would wrap without an error."""
import ctypes as C

import pytest

from paper_2609_35587_amd import hwsel

FAKE = 0x1000   # never dereferenced: every call below is rejected


def fp8(rows, cols, block_rows=1):
    width = -(-cols // 128) * 128
    return hwsel.hwsel_fp8_t(rows, cols, FAKE, width, FAKE, -(-width // 512) * 4, 0, block_rows)


# 2^24 tiles of 128 x 128, five to seven blocks of K; fp32 whatever K is
@pytest.mark.parametrize("M,N,K,kind", [(1 << 24, 1 << 14, 640, "codes"), ((1 << 24) - 127, (1 << 14) - 127, 896, "codes"),
                                        (1 << 30, 129, 700, "bf16"), (1 << 24, 1 << 14, 640, "bf16"),
                                        (1 << 24, 1 << 14, 640, "fp32"), (1 << 30, 129, 4096, "fp32"), (1 << 30, 200, 1, "fp32")])
def test_results_past_a_launch(M, N, K, kind):
    L, A, B = hwsel.lib(), fp8(M, K), fp8(N, K, 128)
    if kind == "codes":
        status = L.hwsel_fp8_layer(C.byref(A), C.byref(B), None, 0, C.byref(fp8(M, N)), None, 0, None)
    else:
        status = L.hwsel_fp8_matmul(C.byref(A), C.byref(B), None, 0, FAKE, 3 if kind == "fp32" else 0, N, None, 0, None)
    assert status == 2
    assert b"a result of %d x %d" % (M, N) in L.hwsel_last_error()


@pytest.mark.parametrize("M,N,K,kind", [((1 << 24) - 128, 1 << 14, 640, "codes"), (1 << 24, 1 << 14, 1024, "codes"),
                                        (1 << 24, 1 << 14, 512, "codes"), (1 << 30, 129, 512, "bf16"), (32, 1 << 30, 4096, "bf16"),
                                        (1 << 30, 128, 128, "fp32"), (16, 1 << 30, 128, "fp32")])
def test_results_just_within(M, N, K, kind):
    """They come past this check: what is refused is their misaligned bias, looked at behind it, or result."""
    L, A, B = hwsel.lib(), fp8(M, K), fp8(N, K, 128)
    if kind == "codes":
        status = L.hwsel_fp8_layer(C.byref(A), C.byref(B), FAKE + 2, 0, C.byref(fp8(M, N)), None, 0, None)
    else:
        status = L.hwsel_fp8_matmul(C.byref(A), C.byref(B), FAKE + 2, 0, FAKE, 3 if kind == "fp32" else 0, N, None, 0, None)
    assert status == 1 and b"bias misaligned" in L.hwsel_last_error()
