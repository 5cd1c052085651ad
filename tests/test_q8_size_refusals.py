"""Sizes beyond what the 8-bit calls count in 32 bits are refused by name, before any launch (no GPU needed)."""
import ctypes as C

import pytest

from paper_2411_00853_amd import binding as sv

P = C.c_void_p(4096)      # never dereferenced
SHAPE, MOST, INT = -2, 1 << 30, (1 << 31) - 1


@pytest.fixture(scope="module")
def lib():
    return sv.lib()


def refused(rc, lib, word):
    assert rc == SHAPE and word.encode() in lib.spec_last_error(), (rc, lib.spec_last_error())


@pytest.mark.parametrize("cols", [MOST + 1, INT - 127, INT - 1, INT])
def test_rows(lib, cols):
    refused(lib.spec_q8_quantize(P, 0, cols, 1, cols, P, P, None), lib, str(cols))
    refused(lib.spec_q8_swiglu(P, 1, 1, cols, P, P, None), lib, str(cols))
    refused(lib.spec_q8_add_rmsnorm(P, 0, None, 0, P, 1e-5, 1, cols, None, P, P, None), lib, str(cols))


@pytest.mark.parametrize("n", [MOST + 1, INT - 127, INT - 15, INT])
def test_matrices(lib, n):
    refused(lib.spec_q8_gemm(P, P, P, P, P, 0, 1, n, 128, None), lib, str(n))
    refused(lib.spec_q8_gemm(P, P, P, P, P, 0, 1, 16, n, None), lib, str(n))
    refused(lib.spec_q8_pack_weight(P, P, n, 128, None), lib, str(n))
    refused(lib.spec_q8_pack_weight(P, P, 16, n, None), lib, str(n))
    assert lib.spec_q8_packed_weight_bytes(n, 128) == 0 and lib.spec_q8_packed_weight_bytes(16, n) == 0


def test_the_largest_sizes_are_counted(lib):
    assert lib.spec_q8_packed_weight_bytes(MOST, 128) == MOST * 128
    assert lib.spec_q8_packed_weight_bytes(16, MOST) == 16 * MOST
    refused(lib.spec_q8_gemm(P, P, P, P, P, 0, 1048561, 16, 128, None), lib, "1048560")
