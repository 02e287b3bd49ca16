"""The training operators of include/dmx.h for torch callers: AdamW over many tensors, group norm with an
activation on channels-last data, and the matrix product with bias, activation and residual in its epilogue.

Tensors in, raw pointers through the C ABI; every call runs on the current stream of its tensors' device, takes its
workspace from torch's allocator there, and raises DmxError with the library's code for arguments it refuses.
Nothing synchronises. The functional operators go through a compiled module (csrc/dmx_torch.cpp), which checks their
arguments, and so do AdamW's norm and step; the rest of AdamW goes through ctypes.
"""
from __future__ import annotations

import ctypes
import os

from . import binding as B
from . import build as _build

ACT = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = range(4)
ADAMW_BLOCK = 256

_torch = None
_dtypes = None


def _t():
    global _torch, _dtypes
    if _torch is None:
        import torch
        _torch, _dtypes = torch, {torch.float32: B.F32, torch.bfloat16: B.BF16}
    return _torch


def _stream(x):
    return _torch._C._cuda_getCurrentRawStream(x.device.index)


def _refuse(where, code=B.ERR_ARG):
    raise B.DmxError(code, where)


class _Nothing:
    def __enter__(self):
        pass

    def __exit__(self, *a):
        pass


_nothing = _Nothing()


def _on(x):
    """A context in which x's device is current (launches go to the current device)."""
    return _nothing if x.device.index == _torch._C._cuda_getDevice() else _torch.cuda.device(x.device)


def _ptr(x):
    return None if x is None else x.data_ptr()


def _order(x):
    """x's (extent, stride) pairs where extents are above one; None unless its elements fill one range, each in a place of its own."""
    dims = [(n, s) for n, s in zip(x.shape, x.stride()) if n != 1]
    at = 1
    for n, s in sorted(dims, key=lambda d: d[1]):
        if s != at:
            return None
        at *= n
    return dims


def _lies_like(x, p):
    """x has p's elements in p's order in memory (contiguous tensors of any shapes lie alike)."""
    if x.is_contiguous() and p.is_contiguous():
        return True
    order = _order(x)
    return order is not None and order == _order(p)


class AdamW:
    """AdamW over a list of tensors (dmx_adamw_*). The tensors stay the caller's and are updated in place.

    params, grads: lists of CUDA tensors, any shapes, dense in any order of dimensions (channels last, transposed), a gradient
    in its parameter's; one dtype (fp32 or bf16) for all of each list, that of gradients set by the first one bound. A None
    gradient leaves its tensor alone. copies: bf16 tensors that receive the updated parameters (entries may be None).
    decay: one truth value per tensor (default: all). state_bits: 32 or 8.
    The moments are the caller's too: `new_state()` makes zeroed ones, `state_view(x, i)` is tensor i's part.
    """

    def __init__(self, params, grads, state_bits=32, copies=None, decay=None):
        torch = _t()
        self._h, self._fast = None, _module()
        params, n = list(params), len(params)
        if not all(isinstance(p, torch.Tensor) for p in params) or not all(g is None or isinstance(g, torch.Tensor) for g in grads):
            _refuse("AdamW (what is no tensor)")
        if n == 0 or (decay is not None and len(decay) != n) or params[0].dtype not in _dtypes or not params[0].is_cuda:
            _refuse("AdamW (params)")
        self.device, self.bits, self._params, self._dtype = params[0].device, int(state_bits), params, params[0].dtype
        self._sizes = [p.numel() for p in params]
        self._decay = None if decay is None else [1 if d else 0 for d in decay]
        self._grad_dtype, self._settled, self._set_aside = None, False, []     # settled: a gradient has shown the type
        self._create(next((g.dtype for g in grads if g is not None), torch.float32))
        self.blocks = B.lib().dmx_adamw_blocks(self._h)
        self.bind(grads, copies)

    def _create(self, grad_dtype):
        if grad_dtype not in _dtypes:
            _refuse("AdamW (gradient dtype)")
        n = len(self._sizes)
        sizes = (ctypes.c_int64 * n)(*self._sizes)
        dec = None if self._decay is None else (ctypes.c_uint8 * n)(*self._decay)
        h = ctypes.c_void_p()
        with _torch.cuda.device(self.device):
            rc = B.lib().dmx_adamw_create(n, sizes, dec, _dtypes[self._dtype], _dtypes[grad_dtype], self.bits, ctypes.byref(h))
        if rc != B.OK:
            _refuse("dmx_adamw_create", rc)
        if self._h:
            self._set_aside.append(self._h)      # a captured step may still read its tables
        self._grad_dtype, self._at = grad_dtype, h.value
        self._h, self._destroy = h, B.lib().dmx_adamw_destroy     # (module globals may be gone when __del__ runs)

    def bind(self, grads, copies=None):
        """Take these gradient (and copy) tensors from now on; needed when their memory moves."""
        n = len(self._params)
        if len(grads) != n or (copies is not None and len(copies) != n):
            _refuse("AdamW.bind")
        if not all(x is None or isinstance(x, _torch.Tensor) for x in (*grads, *(copies or []))):
            _refuse("AdamW.bind (what is no tensor)")
        given = next((g.dtype for g in grads if g is not None), self._grad_dtype)
        if given != self._grad_dtype and self._settled:
            _refuse("AdamW.bind (gradient dtype)")
        for xs, dtype in ((self._params, self._dtype), (grads, given), (copies or [], _torch.bfloat16)):
            for x, p, size in zip(xs, self._params, self._sizes):
                if x is not None and (x.dtype != dtype or x.numel() != size or x.device != self.device or not _lies_like(x, p)):
                    _refuse("AdamW.bind (tensor)")
        if given != self._grad_dtype:            # the first gradients there are
            self._create(given)
        arr = lambda xs: (ctypes.c_void_p * n)(*[None if x is None else x.data_ptr() for x in xs])  # noqa: E731
        with _on(self._params[0]):
            rc = B.lib().dmx_adamw_bind(self._h, arr(self._params), arr(grads), arr(copies) if copies is not None else None, _stream(self._params[0]))
        if rc != B.OK:
            _refuse("dmx_adamw_bind", rc)
        self._settled = self._settled or any(g is not None for g in grads)
        self._written = [x for xs in (self._params, copies or []) for x, g in zip(xs, grads) if x is not None and g is not None]
        self._grads, self._copies = list(grads), None if copies is None else list(copies)      # kept alive: the handle holds their addresses

    def new_state(self):
        """(m, v, m_scale, v_scale), zeroed; the scales are None for 32-bit moments."""
        torch, n = _torch, self.blocks * ADAMW_BLOCK
        if self.bits == 32:
            return torch.zeros(n, device=self.device), torch.zeros(n, device=self.device), None, None
        return (torch.zeros(n, dtype=torch.int8, device=self.device), torch.zeros(n, dtype=torch.uint8, device=self.device),
                torch.zeros(self.blocks, device=self.device), torch.zeros(self.blocks, device=self.device))

    def state_view(self, x, i):
        """Tensor i's entries of a state array with one entry per element."""
        first = B.lib().dmx_adamw_first_block(self._h, i)
        if first < 0:
            _refuse("dmx_adamw_first_block", int(first))
        p, x = self._params[i], x[first * ADAMW_BLOCK: first * ADAMW_BLOCK + self._sizes[i]]
        return x.view(p.shape) if p.is_contiguous() else x.as_strided(p.shape, p.stride())

    def _check(self, where, m, v, m_scale, v_scale):
        t, n = _torch, self.blocks * ADAMW_BLOCK
        kinds = ((m, t.float32, n), (v, t.float32, n)) if self.bits == 32 else (
            (m, t.int8, n), (v, t.uint8, n), (m_scale, t.float32, self.blocks), (v_scale, t.float32, self.blocks))
        for x, dtype, size in kinds:
            if x is None or x.dtype != dtype or x.numel() != size or x.device != self.device or not x.is_contiguous():
                _refuse(where)

    def grad_norm(self, max_norm, out=None):
        """out[0] = the gradients' global norm, out[1] = min(1, max_norm / (norm + 1e-6)) (NaN: not finite)."""
        if out is None:
            out = _torch.empty(2, device=self.device)
        r = self._fast.adamw_grad_norm(self._at, self.device.index, max_norm, out)
        return _refuse("AdamW.grad_norm", r) if r.__class__ is int else r

    def step(self, m, v, m_scale=None, v_scale=None, *, lr, t, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=None, seed=None):
        """One update. t: this step's number, from 1. seed: dither 8-bit codes with it (None: to nearest)."""
        r = self._fast.adamw_step(self._at, self.device.index, self.bits, self.blocks, m, v, m_scale, v_scale, grad_scale, lr, beta1, beta2, eps,
                                  weight_decay, t, seed, self._written)
        if r is not None:
            _refuse("AdamW.step", r)

    def moments(self, m, v, m_scale, v_scale, out_m=None, out_v=None):
        """The values of 8-bit moments (fp32 unless outputs are given)."""
        self._check("AdamW.moments (state)", m, v, m_scale, v_scale)
        out_m = _torch.empty(m.numel(), device=self.device) if out_m is None else out_m
        out_v = _torch.empty(m.numel(), dtype=out_m.dtype, device=self.device) if out_v is None else out_v
        for o in (out_m, out_v):
            if o.dtype not in _dtypes or o.dtype != out_m.dtype or o.numel() != m.numel() or o.device != self.device or not o.is_contiguous():
                _refuse("AdamW.moments (outputs)")
        with _on(m):
            rc = B.lib().dmx_adamw_moments(self._h, m.data_ptr(), v.data_ptr(), _ptr(m_scale), _ptr(v_scale), _dtypes[out_m.dtype],
                                           out_m.data_ptr(), out_v.data_ptr(), _stream(m))
        if rc != B.OK:
            _refuse("dmx_adamw_moments", rc)
        _torch.autograd.graph.increment_version([o for o in (out_m, out_v) if not o.is_inference()])
        return out_m, out_v

    def close(self):
        if getattr(self, "_h", None):
            for h in self._set_aside + [self._h]:
                self._destroy(h)
            self._h, self._at, self._set_aside = None, None, []

    __del__ = close


_fast = None
_RECORD = 1          # the compiled module's answer where torch has to record the call


def _module():
    """The compiled module (lib/_dmx_torch.so), connected to the library that the binding loads."""
    global _fast
    if _fast is None:
        import importlib.machinery
        import importlib.util
        _t()
        L, path = B.lib(), _build.lib_path(_build.TORCH_MODULE)
        if not os.path.exists(path):
            raise RuntimeError("%s is not built; run `python -m paper_2510_08522_b200.build`" % path)
        loader = importlib.machinery.ExtensionFileLoader("_dmx_torch", path)
        m = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_dmx_torch", path, loader=loader))
        loader.exec_module(m)
        m.connect(*[ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.dmx_group_norm_workspace, L.dmx_group_norm_forward, L.dmx_group_norm_backward, L.dmx_linear_workspace, L.dmx_linear_forward,
            L.dmx_linear_backward_workspace, L.dmx_linear_backward, L.dmx_adamw_grad_norm, L.dmx_adamw_step)])
        _fast = m
    return _fast


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, act="none", out=None):
    """act(group_norm(x)) of a channels-last tensor (N, ..., C), fp32 or bf16 -> (y, mean, rstd), the statistics
    fp32 (N, groups). weight, bias: fp32 (C,). x may be a channel slice of a wider tensor; out may be x. Where an input
    requires a gradient torch records the call (y's gradient; the statistics carry none), unless `out` is given."""
    r = (_fast or _module()).group_norm(x, groups, weight, bias, eps, ACT.get(act, -1), out)
    if r.__class__ is tuple:
        return r
    if r != _RECORD:
        _refuse("group_norm", r)
    from .train_grad import GroupNorm
    return GroupNorm.apply(x, groups, weight, bias, eps, act)


def group_norm_backward(dy, x, mean, rstd, groups, weight=None, bias=None, act="none", out=None):
    """Gradient of group_norm from its saved statistics -> (dx, dweight, dbias). out may be dy or x."""
    r = (_fast or _module()).group_norm_backward(dy, x, mean, rstd, groups, weight, bias, ACT.get(act, -1), out)
    return r if r.__class__ is tuple else _refuse("group_norm_backward", r)


def linear(x, weight, bias=None, act="none", residual=None, save=False, out=None):
    """act(x @ weight.T + bias) + residual, bf16 matrices -> (y, z). z is the value before the activation, kept for
    linear_backward when `save` is set and there is an activation, else None. out may be the residual. Where an input
    requires a gradient torch records the call (y's gradient; z carries none), unless `out` is given."""
    r = (_fast or _module()).linear(x, weight, bias, ACT.get(act, -1), residual, save, out)
    if r.__class__ is tuple:
        return r
    if r != _RECORD:
        _refuse("linear", r)
    from .train_grad import Linear
    r = Linear.apply(x, weight, bias, act, residual, save)
    return r if r.__class__ is tuple else (r, None)


def linear_backward(dy, x, weight, z=None, act="none", need=(True, True, True), out=(None, None, None)):
    """Gradient of linear -> (dx, dweight, dbias), those not in `need` None. `out`: tensors to write them to, e.g.
    views of a flat gradient vector."""
    r = (_fast or _module()).linear_backward(dy, x, weight, z, ACT.get(act, -1), (1 if need[0] else 0) + (2 if need[1] else 0) + (4 if need[2] else 0), *out)
    return r if r.__class__ is tuple else _refuse("linear_backward", r)


def linear_status():
    """How many warps of the linear kernels gave up a wait on the current device since the last call. Waits for the
    device's work on all streams."""
    n = ctypes.c_int()
    rc = B.lib().dmx_linear_status(ctypes.byref(n))
    if rc != B.OK:
        _refuse("dmx_linear_status", rc)
    return n.value
