"""The host side of the operators between a tower's products (csrc/tower.cpp) with stand-ins for its launches and for HIP's copies,
so that its checks and the launches it chooses can be tested where there is no GPU.  A launch leaves its name in a log."""
import ctypes
import functools
import os
import subprocess
import tempfile

from paper_2010_11305_amd import dense_lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2010_11305_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
STANDINS = """
#include <string.h>
#include <string>
#include "dense_internal.h"
static std::string seen;
static hipError_t note(const char* name) { seen += name; seen += ' '; return hipSuccess; }
extern "C" const char* launches() { return seen.c_str(); }
extern "C" void forget() { seen.clear(); }
extern "C" hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t) { memcpy(to, from, n); return hipSuccess; }
extern "C" hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
namespace embd {
hipError_t launch_norm(const NormForward&, int, bool, hipStream_t) { return note("norm"); }
int64_t norm_slabs(int64_t, int64_t, int) { return 1; }
bool norm_in_registers(int64_t, int) { return true; }
hipError_t launch_norm_backward(const NormBackward&, int, bool, hipStream_t) { return note("norm_backward"); }
hipError_t launch_rows8_dequantize(const int8_t*, int64_t, int64_t, int64_t, const float*, void*, int, int64_t, hipStream_t) { return note("rows8"); }
hipError_t launch_w4_quantize(const void*, int, int64_t, const W4&, hipStream_t) { return note("quantize"); }
hipError_t launch_w4_dequantize(const W4&, void*, int, int64_t, hipStream_t) { return note("dequantize"); }
hipError_t launch_w4_pack(const uint8_t*, const uint16_t*, const uint16_t*, const W4&, hipStream_t) { return note("pack"); }
hipError_t launch_w4_unpack(const W4&, uint8_t*, uint16_t*, uint16_t*, hipStream_t) { return note("unpack"); }
size_t w4_linear_workspace(int, int64_t, int64_t, int64_t, int) { return 0; }
hipError_t launch_w4_linear(const W4Linear&, int, const W4&, void*, hipStream_t) { return note("linear"); }
hipError_t launch_clip_squares(const ClipDev&, const ClipPointers&, uint32_t, int64_t, unsigned, double*, hipStream_t) { return note("squares"); }
hipError_t launch_clip_join(const double*, int64_t, double, float*, hipStream_t) { return note("join"); }
hipError_t launch_clip_join_scale(const ClipDev&, const ClipPointers&, uint32_t, int64_t, unsigned, const double*, int64_t, double, float*, hipStream_t) {
  return note("join_scale");
}
hipError_t launch_clip_scale(const ClipDev&, const ClipPointers&, uint32_t, int64_t, unsigned, const float*, hipStream_t) { return note("scale"); }
}  // namespace embd
"""


@functools.lru_cache(maxsize=None)
def load():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "standins.cpp"), os.path.join(d, "tower.so")
        with open(src, "w") as f:
            f.write(STANDINS)
        subprocess.run(["g++", "-std=c++20", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", f"-I{CSRC}", f"-I{os.path.join(ROOT, 'include')}",
                        f"-I{ROCM}/include", "-Wl,-Bsymbolic", os.path.join(CSRC, "tower.cpp"), src, "-o", so], check=True)
        L = ctypes.CDLL(so)
    P, i32, i64, f64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
    for name, args in {
        "emb_clip_query_sizes": [ctypes.POINTER(dense_lib.ClipConfig), ctypes.POINTER(dense_lib.ClipSizes)],
        "emb_clip_create": [ctypes.POINTER(dense_lib.ClipConfig), P, size, P, ctypes.POINTER(P)],
        "emb_clip_destroy": [P],
        "emb_clip_norm": [P, P, f64, P, P, size, P],
        "emb_clip_scale": [P, P, P, P],
        "emb_clip_apply": [P, P, f64, P, P, size, P],
        "emb_w4_pack": [P, P, P, i64, i64, i32, P, P],
        "emb_w4_unpack": [P, i64, i64, i32, P, P, P, P],
    }.items():
        getattr(L, name).argtypes = args
    L.launches.restype = ctypes.c_char_p
    return L


def launches(L):
    """The launches since the last time."""
    names = L.launches().decode().split()
    L.forget()
    return names


class Clip:
    """A handle whose state is host memory; other buffers may be at any address."""

    def __init__(self, sizes, types=None):
        self.L, n = load(), len(sizes)
        self.keep = ((ctypes.c_int64 * n)(*sizes), (ctypes.c_int32 * n)(*types) if types else None)
        c = dense_lib.ClipConfig(n, 0, self.keep[0], self.keep[1])
        self.sizes = dense_lib.ClipSizes()
        assert self.L.emb_clip_query_sizes(ctypes.byref(c), ctypes.byref(self.sizes)) == 0
        self.buffer = ctypes.create_string_buffer(self.sizes.state_bytes + 256)
        self.state = -(-ctypes.addressof(self.buffer) // 256) * 256
        self.h = ctypes.c_void_p()
        assert self.L.emb_clip_create(ctypes.byref(c), self.state, self.sizes.state_bytes, None, ctypes.byref(self.h)) == 0

    def _call(self, f, grads, *args):
        p = (ctypes.c_uint64 * len(grads))(*[g or 0 for g in grads])
        return f(self.h, ctypes.addressof(p), *args, None), launches(self.L)

    def norm(self, grads, result, workspace, nbytes=None):
        return self._call(self.L.emb_clip_norm, grads, 1.0, result, workspace, self.sizes.workspace_bytes if nbytes is None else nbytes)

    def apply(self, grads, result, workspace, nbytes=None):
        return self._call(self.L.emb_clip_apply, grads, 1.0, result, workspace, self.sizes.workspace_bytes if nbytes is None else nbytes)

    def scale(self, grads, factor):
        return self._call(self.L.emb_clip_scale, grads, factor)

    def __del__(self):
        if self.h:
            self.L.emb_clip_destroy(self.h)
