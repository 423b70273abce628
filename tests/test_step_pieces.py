"""Which bytes the layer norm's gradient copies to shared memory: the kernels' own index arithmetic, compiled for the host.

An asynchronous copy of 16 bytes has to begin on a 16-byte boundary, also where it copies nothing."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2206_01299_b200", "csrc")
PROGRAM = """
#include "aq_stage.h"
extern "C" void piece(int index, int n, int shift, int hidden, int* out) {
  const aq::NormPiece p = aq::norm_piece(index, n, shift, hidden);
  out[0] = p.column; out[1] = p.lo; out[2] = p.hi; out[3] = aq::norm_copy_from(p.column, p.hi, shift);
}
"""


@pytest.fixture(scope="module")
def piece(tmp_path_factory):
    where = tmp_path_factory.mktemp("pieces")
    (where / "piece.cpp").write_text(PROGRAM)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", CSRC, "-I", os.path.join(cuda, "include"), "-o", str(where / "piece.so"),
                           str(where / "piece.cpp")])
    call = ctypes.CDLL(str(where / "piece.so")).piece
    out = (ctypes.c_int * 4)()

    def f(*args):
        call(*args, out)
        return list(out)
    return f


@pytest.mark.parametrize("size", [2, 4])
@pytest.mark.parametrize("hidden", [1, 3, 7, 8, 24, 65, 250, 255, 257, 1021, 1600, 1601, 2045, 4097, 8185])
def test_copies_begin_on_boundaries_and_stay_in_the_row(piece, size, hidden):
    n = 16 // size
    threads = -(-(hidden + n - 1) // (n * 32)) * 32 + 32               # of whole warps, some without elements
    for pad in range(n):
        ld = hidden + pad
        for row in range(n):
            shift = row * (ld % n) % n
            seen = []
            for index in range(threads):
                column, lo, hi, at = piece(index, n, shift, hidden)
                assert (row * ld + at) * size % 16 == 0, (pad, row, index)
                assert at >= -shift and at + hi <= hidden and 0 <= hi <= n
                assert hi == 0 or at == column                         # elements before the row are those of the row before, or of its padding
                seen += range(column + lo, column + hi)
            assert seen == list(range(hidden))                         # every element once
