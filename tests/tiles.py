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
extern "C" int tile_of(int pairs, int64_t batch, int64_t m, int64_t n, int triangular, int64_t k, int most_parts, double part_ns)
{
    return sams::gemm::choose_tiles(pairs, batch, m, n, triangular, k, most_parts, part_ns).shape;
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
    lib.tile_of.argtypes = [ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_double]
    return lib


def tile_of(pairs, batch, m, n, k, triangular=False, most_parts=1, part_ns=0.0):
    return _library().tile_of(pairs, batch, m, n, triangular, k, most_parts, part_ns)


def of_ortho(pairs, batch, rows, cols):
    """The tiles of an orthogonalisation's Gram matrix, its square and the product with X."""
    small, large = min(rows, cols), max(rows, cols)
    return (tile_of(pairs, batch, small, small, large, True), tile_of(pairs, batch, small, small, small, True), tile_of(pairs, batch, cols, rows, small))


def of_xent(pairs, n, t, dim, vocab):
    """The tiles of a cross entropy's logits, of dW and of dh (cut along the vocabulary into parts, of 256 MiB and 64 at most)."""
    rows = n * t
    part = rows * ((dim + 3) // 4 * 4) * 4
    most = max(1, min((256 << 20) // part, 64, (vocab + 255) // 256))
    return tile_of(pairs, 1, vocab, rows, dim), tile_of(pairs, n, dim, vocab, t), tile_of(pairs, 1, dim, rows, vocab, most_parts=most, part_ns=part * 2 / 4000.0)
