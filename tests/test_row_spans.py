"""What the norms read beside a row (csrc/residual_norm.cuh, compiled for the host): whole 16-byte pieces, at most 15 bytes on each side, and
nothing outside of the matrix."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2507_19131_b200 import build as mq_build

HERE = os.path.dirname(os.path.abspath(__file__))
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
BASE = 1 << 40


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    if not os.path.exists(NVCC):
        pytest.skip("no nvcc")
    out = str(tmp_path_factory.mktemp("spans") / "libspans.so")
    flags = [f for f in mq_build.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
    subprocess.check_call([NVCC] + flags + ["-o", out, os.path.join(HERE, "host_path", "row_spans.cu")])
    lib = C.CDLL(out)
    lib.row_copy.argtypes = [C.c_long, C.c_long, C.c_long, C.c_int, C.c_int, C.c_int, C.c_long, C.POINTER(C.c_long), C.POINTER(C.c_long)]
    return lib


def span(L, address, stride, rows, dim, size, vec, row):
    lo, hi = C.c_long(), C.c_long()
    L.row_copy(address, stride, rows, dim, size, vec, row, C.byref(lo), C.byref(hi))
    return lo.value, hi.value


@pytest.mark.parametrize("size", [2, 4])
@pytest.mark.parametrize("dim", [1, 2, 3, 7, 8, 9, 31, 257, 1001, 16383])
@pytest.mark.parametrize("pad", [0, 1, 3, 8, 100])
def test_rows_are_copied_inside_the_matrix(L, size, dim, pad):
    stride = dim + pad
    for odd in range(16 // size):
        for rows in (1, 2, 5):
            address = BASE + odd * size
            end = address + ((rows - 1) * stride + dim) * size
            for row in range(rows):
                start = address + row * stride * size
                lo, hi = span(L, address, stride, rows, dim, size, 0, row)
                assert (start + lo) % 16 == 0 and (start + hi) % 16 == 0 and hi >= lo
                if hi > lo:
                    assert start + lo >= address and start + hi <= end
                assert lo > -16 and hi < dim * size + 16
                # a row without neighbours to share a piece with lacks at most its two ends
                assert hi - lo >= dim * size - 30 and (lo <= 15) and (hi >= dim * size - 15 or hi == lo)


@pytest.mark.parametrize("size", [2, 4])
def test_rows_of_whole_vectors_are_copied_as_they_are(L, size):
    for row in range(3):
        assert span(L, BASE, 128, 3, 96, size, 1, row) == (0, 96 * size)
