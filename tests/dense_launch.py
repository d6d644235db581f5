"""The tile that a product takes: the library's own rule (dense_launch.h), compiled for the host."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2010_11305_amd", "csrc")
SOURCE = """
#include "dense_launch.h"
extern "C" int side(int64_t a, int64_t b) { return embd::product_side(a, b); }
"""


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "side.cpp"), os.path.join(d, "side.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", so], check=True)
        lib = ctypes.CDLL(so)
        lib.side.argtypes = [ctypes.c_int64, ctypes.c_int64]
        return lib


def tile_rows(m, n):
    """256, 128 or 64 rows and columns of a workgroup's tile, where the product does not go by few rows."""
    return 32 * _lib().side(-(-m // 16), -(-n // 16))
