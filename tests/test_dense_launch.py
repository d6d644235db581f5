"""Launch sizes of the dense operators (dense_launch.h), compiled for the host: HIP takes fewer than 2^32 threads a
launch, and sizes that a device holds pass that."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2010_11305_amd", "csrc")

SOURCE = """
#include "dense_launch.h"
using namespace embd;
extern "C" int64_t workgroups(int64_t rows, int64_t cols, int by_columns) { return quantize_workgroups(rows, cols, by_columns); }
extern "C" int parts(int64_t n, int threads, int64_t* out, int most, int fail_at) {
  int k = 0;
  const int e = in_launches(n, threads, [&](int64_t first, unsigned some) {
    if (k == fail_at) return 7;
    if (k < most) out[2 * k] = first, out[2 * k + 1] = some;
    ++k;
    return 0;
  });
  return e ? -e : k;
}
extern "C" int side(int64_t a, int64_t b) { return product_side(a, b); }
extern "C" int64_t tiles(int64_t a, int64_t b, int f) { return product_tiles(a, b, f); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("launch")
    src, so = d / "launch.cpp", d / "launch.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", str(src), "-o", str(so)],
                   check=True)
    L = ctypes.CDLL(str(so))
    i64 = ctypes.c_int64
    L.workgroups.restype, L.workgroups.argtypes = i64, [i64, i64, ctypes.c_int]
    L.parts.argtypes = [i64, ctypes.c_int, ctypes.POINTER(i64), ctypes.c_int, ctypes.c_int]
    L.side.argtypes = [i64, i64]
    L.tiles.restype, L.tiles.argtypes = i64, [i64, i64, ctypes.c_int]
    return L


def parts(lib, n, threads):
    out = (ctypes.c_int64 * 2000)()
    k = lib.parts(n, threads, out, 1000, -1)
    assert 0 < k <= 1000
    return [(out[2 * i], out[2 * i + 1]) for i in range(k)]


@pytest.mark.parametrize("threads", [64, 256, 832, 1024])
@pytest.mark.parametrize("n", [1, 255, 2**20, 2**21, 2**21 + 1, 2**23, 2**24, 2**27 + 3, 2**30 + 1])
def test_parts_cover_the_workgroups_and_fit_a_launch(lib, n, threads):
    at = 0
    for first, some in parts(lib, n, threads):
        assert first == at and some >= 1 and some * threads < 2**32
        at += some
    assert at == n
    assert len(parts(lib, n, threads)) == 1 or n * threads > 2**31


def test_a_failure_ends_the_parts(lib):
    out = (ctypes.c_int64 * 20)()
    assert lib.parts(2**24, 256, out, 10, 1) == -7 and lib.parts(2**24, 256, out, 10, 0) == -7


@pytest.mark.parametrize("rows,cols", [(1, 1), (256, 416), (16384, 12800), (2**27, 1), (2**27, 128), (1, 2**27), (2**28, 1),
                                       (2**31 - 1, 1), (1, 2**31 - 1), (2**20, 2**19)])
def test_quantisation_reaches_every_tile(lib, rows, cols):
    """At least a workgroup for each 32 x 128 values (the rows, by columns, to the end of their tile of 128), with numbers that
    the kernel keeps in 32 bits; below 2^32 threads a launch."""
    for by_columns in (0, 1):
        n = lib.workgroups(rows, cols, by_columns)
        rows_to = -(-rows // 128) * 128 if by_columns else rows
        assert -(-rows_to // 32) * -(-cols // 128) <= n < 2**32
        assert all(some * 256 < 2**32 for _, some in parts(lib, n, 256))


def test_product_launches_fit(lib):
    """Tiles of 256 stay at 256 workgroups; the others are chosen only where a launch holds them all."""
    seen = set()
    for a in (1, 2, 3, 5, 16, 63, 1024, 2**14, 2**20, 2**26, 2**27):
        for b in (1, 3, 9, 100, 2**13, 2**21, 2**26, 2**27):
            f = lib.side(a, b)
            seen.add(f)
            assert f == 8 or lib.tiles(a, b, f) * 256 < 2**32
    assert seen == {2, 4, 8}
    assert lib.side(63, 65) == 2 and lib.side(3, 2**27) == 8 and lib.side(1024, 512) == 8
