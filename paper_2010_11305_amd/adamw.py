"""AdamW over many tensors in one step, with moments in FP32 or in 8 bits (include/emb_dense.h).

    opt = adamw.AdamW(params, lr=1e-3, state_bits=8, rounding="stochastic")
    opt.step(grads)            # or opt.step(grads, lr=..., grad_scale=clip_factor)

Parameters are updated in place.  The update runs in one HIP kernel per 240 tensors.
"""
from __future__ import annotations

import ctypes
from array import array
from operator import attrgetter

import torch
from torch import Tensor

from . import dense_lib as lib

dtype_of = attrgetter("dtype")
NOWHERE = 2**64 - 1    # the address of no tensor


class AdamW:
    """params: float32 or bfloat16 tensors on one GPU, all of one type, contiguous, none sharing memory with
    another.  A parameter may be given other memory later (through `data`), of the same type, device and size.
    seed: of stochastic rounding, another one than those of the model's 4-bit layers.
    weight_decay: one number, or one per tensor.  grad_dtype: the type of the gradients (default:
    that of the parameters)."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_dtype=None,
                 state_bits=32, rounding="nearest", seed=0):
        self.params = list(params)
        if not self.params:
            raise ValueError("params must hold at least one tensor")
        p0 = self.params[0]
        self.dtype, self.device = p0.dtype, p0.device
        self.grad_dtype = grad_dtype or self.dtype
        n = len(self.params)
        self.sizes = [p.numel() for p in self.params]
        self._hold()
        self.lr, self.state_bits, self.seed = float(lr), state_bits, int(seed)
        c = lib.AdamwConfig()
        self._sizes = (ctypes.c_int64 * n)(*self.sizes)
        c.num_tensors, c.param_type, c.sizes = n, lib.type_of(self.dtype), self._sizes
        if isinstance(weight_decay, (int, float)):
            c.weight_decay = float(weight_decay)
        else:
            weight_decay = [float(w) for w in weight_decay]
            if len(weight_decay) != n:
                raise ValueError("weight_decay must be a number, or one for each tensor")
            self._decays = (ctypes.c_double * n)(*weight_decay)
            c.weight_decays = self._decays
        c.grad_type, c.state_bits, c.rounding = lib.type_of(self.grad_dtype), int(state_bits), lib.rounding_of(rounding)
        c.beta1, c.beta2, c.eps, c.seed = float(betas[0]), float(betas[1]), float(eps), self.seed
        L = lib.load()
        self._layout = lib.AdamwSizes()
        lib.check(L.emb_adamw_query_sizes(ctypes.byref(c), ctypes.byref(self._layout)), "emb_adamw_query_sizes")
        self.state_buffer = torch.empty(max(self._layout.state_bytes, 256), dtype=torch.uint8, device=self.device)
        self._h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            lib.check(L.emb_adamw_create(ctypes.byref(c), self.state_buffer.data_ptr(), self._layout.state_bytes,
                                         torch.cuda.current_stream().cuda_stream, ctypes.byref(self._h)),
                      "emb_adamw_create")

    def _hold(self, which=None):
        """Check the parameters (those of `which` alone: a step writes no other) and keep their memory by views of it: as
        long as a parameter's address is that of its view, nothing else can have come to lie there, and step() need not
        look at type, device and size again."""
        which = range(len(self.params)) if which is None else which
        places = []
        for p, size in ((self.params[k], self.sizes[k]) for k in which):
            if (p.dtype != self.dtype or p.device != self.device or not p.is_cuda or not p.is_contiguous()
                    or p.numel() != size):
                raise ValueError("params must be contiguous tensors of one type on one GPU, and keep type, device and size")
            if size:
                places.append((p.data_ptr(), size * p.element_size()))
        end = 0
        for start, size in sorted(places):
            if start < end:
                raise ValueError("params must not share memory (a tied parameter is given once)")
            end = start + size
        self._held = {k: self.params[k].detach() for k in which}
        self._pointers = array("Q", [self._held[k].data_ptr() if k in self._held else NOWHERE for k in range(len(self.params))])
        # a tensor of one dimension and the same elements cannot lie otherwise
        self._wide = [p for p in self.params if p.dim() > 1]

    def close(self):
        if getattr(self, "_h", None):
            lib.load().emb_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, grads, lr=None, grad_scale=None):
        """One step.  grads: one tensor per parameter, contiguous, of grad_dtype; None leaves the parameter and
        its moments as they are.  grad_scale: a float32 scalar tensor on the GPU that multiplies them."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} tensors")
        # a model has hundreds of tensors and a step lasts some hundred microseconds: C-level maps, one a property
        given, sizes, changed, kept = grads, self.sizes, self.params, None
        if type(None) in set(map(type, grads)):
            kept = [k for k, g in enumerate(grads) if g is not None]
            given, sizes, changed = ([of[k] for k in kept] for of in (grads, sizes, changed))
        index = self.device.index
        if (list(map(Tensor.numel, given)) != sizes or not all(map(Tensor.is_contiguous, given))
                or not set(map(dtype_of, given)) <= {self.grad_dtype} or not set(map(Tensor.get_device, given)) <= {index}):
            raise ValueError(f"gradients must be contiguous, {self.grad_dtype}, on {self.device}, and each as large as its parameter")
        scale = None
        if grad_scale is not None:
            if grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or grad_scale.get_device() != index:
                raise ValueError(f"grad_scale must be one float32 value on {self.device}")
            scale = grad_scale.data_ptr()
        pp = array("Q", map(Tensor.data_ptr, self.params))
        if pp != self._pointers or not all(map(Tensor.is_contiguous, self._wide)):
            self._hold(kept)   # another storage, as a parameter's `data` may be given
        gp = array("Q", map(Tensor.data_ptr, grads) if given is grads else [0 if g is None else g.data_ptr() for g in grads])
        lib.call("emb_adamw_step", self.device, self._h, pp.buffer_info()[0], gp.buffer_info()[0],
                 self.lr if lr is None else float(lr), scale)
        lib.written(changed)

    def state(self) -> dict:
        """The moments, as views of the state buffer over all tensors, each tensor's part padded to a multiple of 32
        elements: exp_avg and exp_avg_sq (32 bits), or exp_avg and exp_avg_root (E4M3 elements) with the scale
        byte of each 32 in exp_avg_scale and exp_avg_root_scale."""
        s, n = self._layout, self._layout.elements

        def view(offset, count, dtype):
            size = torch.empty((), dtype=dtype).element_size()
            return self.state_buffer[offset:offset + count * size].view(dtype)

        if self.state_bits == 32:
            return {"exp_avg": view(s.first_offset, n, torch.float32),
                    "exp_avg_sq": view(s.second_offset, n, torch.float32)}
        return {"exp_avg": view(s.first_offset, n, torch.float8_e4m3fn),
                "exp_avg_root": view(s.second_offset, n, torch.float8_e4m3fn),
                "exp_avg_scale": view(s.first_scale_offset, n // 32, torch.uint8),
                "exp_avg_root_scale": view(s.second_scale_offset, n // 32, torch.uint8)}

    @property
    def step_count(self) -> int:
        """Steps done."""
        v = ctypes.c_uint64()
        lib.check(lib.load().emb_adamw_get_step(self._h, ctypes.byref(v)), "emb_adamw_get_step")
        return int(v.value)

    @step_count.setter
    def step_count(self, steps: int):
        lib.check(lib.load().emb_adamw_set_step(self._h, int(steps)), "emb_adamw_set_step")
