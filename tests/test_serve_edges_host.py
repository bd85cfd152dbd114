"""Host-side checks, without a GPU, of what the operators for sequences of different lengths refuse at their largest sizes, and of
the arithmetic that their kernels share with the host."""
import ctypes

import paper_2401_06104_b200 as tova

SHAPE = -2
A = ctypes.c_void_p(4096)          # never dereferenced: the calls below are refused
NO_SIZE = ctypes.c_size_t(-1).value


def test_paged_bounds_that_row_numbers_do_not_hold_are_refused():
    """A table of 65536 pages of 32768 rows is valid; a bound above 2^30 rows is not (row numbers, and the rows that are looked at
    ahead of them, are 32-bit)."""
    L = tova.lib()
    for dtype in (tova.TOVA_DTYPE_BF16, tova.TOVA_DTYPE_FP32):
        c = tova.tova_paged_config(1, 1, 1, 64, 1, 1 << 15, 1 << 16, dtype, 0.0)
        for n in (2**30 + 1, 2**31 - 130, 2**31 - 64, 2**31 - 1):
            assert L.tova_paged_attention(ctypes.byref(c), A, A, A, A, n, A, 0, A, A, 1 << 40, None) == SHAPE
            assert L.tova_paged_workspace_bytes(ctypes.byref(c), n) == NO_SIZE
