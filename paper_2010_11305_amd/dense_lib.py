"""What the bindings of the dense operators (include/emb_dense.h) share: the signatures of the
library's functions, element types, streams and checks of tensors."""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.graph import increment_version

from . import emb_cache

ROUNDING = {"nearest": 0, "stochastic": 1}
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_lib = None


class AdamwConfig(ctypes.Structure):
    _fields_ = [
        ("num_tensors", ctypes.c_int32),
        ("param_type", ctypes.c_int32),
        ("sizes", ctypes.POINTER(ctypes.c_int64)),
        ("weight_decays", ctypes.POINTER(ctypes.c_double)),
        ("grad_type", ctypes.c_int32),
        ("state_bits", ctypes.c_int32),
        ("rounding", ctypes.c_int32),
        ("pad", ctypes.c_int32),
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("weight_decay", ctypes.c_double),
        ("seed", ctypes.c_uint64),
    ]


class AdamwSizes(ctypes.Structure):
    _fields_ = [
        ("state_bytes", ctypes.c_size_t),
        ("elements", ctypes.c_int64),
        ("first_offset", ctypes.c_size_t),
        ("second_offset", ctypes.c_size_t),
        ("first_scale_offset", ctypes.c_size_t),
        ("second_scale_offset", ctypes.c_size_t),
    ]


def load():
    """libembcache with the signatures of the dense operators (raises if it is not built)."""
    global _lib
    if _lib is not None:
        return _lib
    L = emb_cache.load()
    c, P = ctypes, ctypes.c_void_p
    i32, i64, u32, u64, f64, size = c.c_int32, c.c_int64, c.c_uint32, c.c_uint64, c.c_double, c.c_size_t
    sig = {
        "emb_mx4_query_bytes": [i64, i64, c.POINTER(size)],
        "emb_mx4_quantize": [P, i32, i64, i64, i64, P, P, i32, u64, u32, P],
        "emb_mx4_dequantize": [P, i64, i64, P, i32, i64, P],
        "emb_mx4_pack": [P, P, i64, i64, P, P],
        "emb_mx4_unpack": [P, i64, i64, P, P, P],
        "emb_mx4_matmul": [P, P, i64, i64, i64, P, i32, i64, P],
        "emb_mx4_linear_workspace": [i64, i64, i64, c.POINTER(size)],
        "emb_mx4_linear": [P, i32, i64, i64, i64, P, i64, P, i64, P, size, P],
        "emb_mx4_linear_train_workspace": [i64, i64, i64, c.POINTER(size)],
        "emb_mx4_linear_train": [P, i32, i64, i64, i64, P, i64, P, i64, P, i32, u64, u32, P, size, P],
        "emb_mx4_linear_grad_workspace": [i64, i64, i64, c.POINTER(size)],
        "emb_mx4_linear_grad": [P, i32, i64, i64, i64, P, i64, P, P, i64, P, i32, i64, i32, u64, u32, P, size, P],
        "emb_adamw_query_sizes": [c.POINTER(AdamwConfig), c.POINTER(AdamwSizes)],
        "emb_adamw_create": [c.POINTER(AdamwConfig), P, size, P, c.POINTER(P)],
        "emb_adamw_destroy": [P],
        "emb_adamw_step": [P, P, P, f64, P, P],
        "emb_adamw_get_step": [P, c.POINTER(u64)],
        "emb_adamw_set_step": [P, u64],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = c.c_int
    _lib = L
    return L


def check(status: int, what: str):
    if status != emb_cache.EMB_OK:
        raise emb_cache.EmbCacheError(status, what)


def call(name: str, device, *args):
    """One enqueue-only function of the library on the current stream of `device`, which is made current where it
    is not.  Small operators last a few microseconds, as long as this does: hence torch's raw
    accessors, and no context manager on the usual way."""
    f = getattr(_lib or load(), name)
    index = device.index
    if torch._C._cuda_getDevice() == index:
        status = f(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if status:
        raise emb_cache.EmbCacheError(status, name)


def written(tensors):
    """Count tensors that a kernel wrote in place as changed: a backward pass that had kept one raises then, as it
    does for torch's own operations in place."""
    try:
        increment_version(tensors)
    except RuntimeError:    # some are of inference mode and have no such count
        increment_version([t for t in tensors if not t.is_inference()])


def rounding_of(name: str) -> int:
    if name not in ROUNDING:
        raise ValueError(f"rounding must be 'nearest' or 'stochastic', not {name!r}")
    return ROUNDING[name]


def type_of(dtype) -> int:
    t = TYPES.get(dtype)
    if t is None:
        raise ValueError(f"element type must be float32, bfloat16 or float16, not {dtype}")
    return t


def matrix(x, what: str):
    """(pointer, type, rows, cols, row stride) of a matrix on the GPU whose rows are contiguous."""
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError(f"{what} must be a matrix on the GPU")
    t = type_of(x.dtype)
    rows, cols = x.shape
    if cols > 1 and x.stride(1) != 1:
        raise ValueError(f"{what} must have contiguous rows (stride 1 along them)")
    return x.data_ptr(), t, rows, cols, x.stride(0) if rows > 1 else max(cols, 1)
