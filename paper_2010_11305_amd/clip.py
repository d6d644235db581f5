"""The norm of all gradients of a model together, and clipping by it (include/emb_dense.h).

    clip = GradClip(params, max_norm=1.0)
    norm, factor = clip.norm(grads)
    opt.step(grads, grad_scale=factor)         # AdamW multiplies by it on the way
    norm, factor = clip.clip_(grads)           # or: the gradients themselves are scaled down

norm and factor stay on the GPU.
"""
from __future__ import annotations

import ctypes
from array import array
from operator import attrgetter

import torch
from torch import Tensor

from . import dense_lib as lib

dtype_of = attrgetter("dtype")


class GradClip:
    """params: tensors on one GPU whose gradients have their sizes and types (or all the type grad_dtype); any mixture of
    float32, bfloat16 and float16.  max_norm: the largest norm, above 0 (infinity for none).  Graphs that captured its calls
    need it as long as they are replayed."""

    def __init__(self, params, max_norm: float = 1.0, grad_dtype=None):
        params = list(params)
        if not params or not all(p.is_cuda and p.device == params[0].device for p in params):
            raise ValueError("params must hold at least one tensor, all on one GPU")
        if not float(max_norm) > 0.0:
            raise ValueError(f"max_norm must be above 0, not {max_norm}")
        self.device, self.max_norm = params[0].device, float(max_norm)
        n = len(params)
        self.sizes = [p.numel() for p in params]
        self.dtypes = [grad_dtype or p.dtype for p in params]
        sizes, types = (ctypes.c_int64 * n)(*self.sizes), (ctypes.c_int32 * n)(*map(lib.type_of, self.dtypes))
        c, s = lib.ClipConfig(n, 0, sizes, types), lib.ClipSizes()
        L = lib.load()
        lib.check(L.emb_clip_query_sizes(ctypes.byref(c), ctypes.byref(s)), "emb_clip_query_sizes")
        self._workspace_bytes = s.workspace_bytes
        self._state = torch.empty(max(s.state_bytes, 256), dtype=torch.uint8, device=self.device)
        self._h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            self._stream = torch.cuda.current_stream().cuda_stream
            lib.check(L.emb_clip_create(ctypes.byref(c), self._state.data_ptr(), s.state_bytes, self._stream, ctypes.byref(self._h)),
                      "emb_clip_create")

    def close(self):
        if getattr(self, "_h", None):
            lib.load().emb_clip_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _pointers(self, grads):
        """(the gradients that are there, an array of all addresses)"""
        if len(grads) != len(self.sizes):
            raise ValueError(f"{len(grads)} gradients for {len(self.sizes)} tensors")
        given, sizes, dtypes = grads, self.sizes, self.dtypes
        if type(None) in set(map(type, grads)):
            kept = [k for k, g in enumerate(grads) if g is not None]
            given, sizes, dtypes = ([of[k] for k in kept] for of in (grads, sizes, dtypes))
        if (list(map(Tensor.numel, given)) != sizes or not all(map(Tensor.is_contiguous, given))
                or list(map(dtype_of, given)) != dtypes or not set(map(Tensor.get_device, given)) <= {self.device.index}):
            raise ValueError(f"gradients must be contiguous, on {self.device}, and each of the size and type of its parameter")
        if torch._C._cuda_getCurrentRawStream(self.device.index) != self._stream:
            self._state.record_stream(torch.cuda.current_stream(self.device))   # else the tables were anyone's once self is dropped
        return given, array("Q", map(Tensor.data_ptr, grads) if given is grads else [0 if g is None else g.data_ptr() for g in grads])

    def norm(self, grads):
        """(norm, factor) as float32 scalars on the GPU: factor = min(1, max_norm / norm).  A gradient that is None counts as
        zeros."""
        result = torch.empty(2, dtype=torch.float32, device=self.device)
        pointers = self._pointers(list(grads))[1]
        lib.call_in("emb_clip_norm", self.device, self._workspace_bytes, self._h, pointers.buffer_info()[0], self.max_norm,
                    result.data_ptr())
        return result.unbind()

    def clip_(self, grads):
        """norm(grads), and the gradients multiplied by the factor in place.  No two of them may share memory."""
        result = torch.empty(2, dtype=torch.float32, device=self.device)
        given, pointers = self._pointers(list(grads))
        lib.call_in("emb_clip_apply", self.device, self._workspace_bytes, self._h, pointers.buffer_info()[0], self.max_norm,
                    result.data_ptr())
        lib.written(given)
        return result.unbind()

    def scale_(self, grads, factor):
        """The gradients multiplied in place by a float32 scalar on the GPU (a factor that several processes agreed on, say)."""
        if factor.dtype != torch.float32 or factor.numel() != 1 or factor.device != self.device:
            raise ValueError(f"factor must be one float32 value on {self.device}")
        given, pointers = self._pointers(list(grads))
        lib.call("emb_clip_scale", self.device, self._h, pointers.buffer_info()[0], factor.data_ptr())
        lib.written(given)
