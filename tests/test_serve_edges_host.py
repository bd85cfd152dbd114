"""Host-side checks, without a GPU, of what the operators for sequences of different lengths refuse at their largest sizes, and of
the arithmetic that their kernels share with the host."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2401_06104_b200 as tova
from paper_2401_06104_b200 import build as tbuild

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


@pytest.fixture(scope="module")
def packed_ring(tmp_path_factory):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "packed_ring_host.cu")
    so = str(tmp_path_factory.mktemp("packed_ring") / "packed_ring.so")
    flags = [f for f in tbuild.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
    subprocess.run([tbuild._nvcc(), *flags, "-O1", "-o", so, src], check=True, capture_output=True, text=True)
    f = ctypes.CDLL(so).check_packed_ring
    f.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(ctypes.c_longlong)]
    f.restype = ctypes.c_longlong
    return f


@pytest.mark.parametrize("slots", [5, 8])          # of head_dim 128 and 64
def test_packed_ring_places_hold_beyond_32_bits(packed_ring, slots):
    """A block's copies of K and V may be more than 2^32 in one call: slots, phases and the first turn are those of a count in 64
    bits, whatever the items' numbers of copies (two a column tile, up to those of 2^24 tokens)."""
    rng = random.Random(slots)
    for copies, items in (([2], 1000), ([2, 4, 6], 1000), ([2 * rng.randint(1, 40) for _ in range(97)], 5000),
                          ([2 * rng.randint(1, 2**17 + 2) for _ in range(31)], 2**32 // 2**17 + 5000)):
        total = ctypes.c_longlong(0)
        assert packed_ring(slots, (ctypes.c_int * len(copies))(*copies), len(copies), items, ctypes.byref(total)) == 0, copies
    assert total.value > 2**32
