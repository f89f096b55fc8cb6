"""Which tiles the library's products choose, from its own header compiled for the host: a test that means a tile's kernel asks here
whether its sizes reach it."""
import ctypes
import functools
import os
import subprocess
import tempfile

from paper_2210_07454_amd import build

LARGE, WIDE, MIDDLE, SMALL = range(4)

SOURCE = """
#include "sams_gemm.h"
extern "C" int tile_of(int pairs, int64_t batch, int64_t m, int64_t n, int triangular, int64_t k)
{
    return sams::gemm::choose_tiles(pairs, batch, m, n, triangular, k, 1, 0.0).shape;
}
"""


@functools.lru_cache(None)
def _library():
    with tempfile.TemporaryDirectory() as at:
        source, so = os.path.join(at, "tiles.hip"), os.path.join(at, "tiles.so")
        with open(source, "w") as f:
            f.write(SOURCE)
        subprocess.run([build.HIPCC, "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-shared", "-I" + build.CSRC, source, "-o", so], check=True, capture_output=True)
        lib = ctypes.CDLL(so)
    lib.tile_of.argtypes = [ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_int64]
    return lib


def tile_of(pairs, batch, m, n, k, triangular=False):
    return _library().tile_of(pairs, batch, m, n, triangular, k)


def of_ortho(pairs, batch, rows, cols):
    """The tiles of an orthogonalisation's Gram matrix, its square and the product with X."""
    small, large = min(rows, cols), max(rows, cols)
    return (tile_of(pairs, batch, small, small, large, True), tile_of(pairs, batch, small, small, small, True), tile_of(pairs, batch, cols, rows, small))
