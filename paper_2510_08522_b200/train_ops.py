"""The training operators of include/dmx.h for torch callers: AdamW over many tensors, group norm with an
activation on channels-last data, and the matrix product with bias, activation and residual in its epilogue.

Tensors in, raw pointers through the C ABI; every call runs on the current stream of its tensors' device, takes its
workspace from torch's allocator there, and raises DmxError with the library's code for arguments it refuses.
Nothing synchronises.
"""
from __future__ import annotations

import ctypes
import functools

from . import binding as B

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


def _workspace(nbytes, like, where):
    if nbytes < 0:
        _refuse(where, int(nbytes))
    # (bf16 and fp32 callers alike: of the caller's type, which is the cheapest to ask torch for)
    return like.new_empty((nbytes + 1) // 2) if nbytes else None


class AdamW:
    """AdamW over a list of tensors (dmx_adamw_*). The tensors stay the caller's and are updated in place.

    params, grads: lists of CUDA tensors, any shapes, dense; one dtype (fp32 or bf16) for all of each list. A None
    gradient leaves its tensor alone. copies: bf16 tensors that receive the updated parameters (entries may be None).
    decay: one truth value per tensor (default: all). state_bits: 32 or 8.
    The moments are the caller's too: `new_state()` makes zeroed ones, `state_view(x, i)` is tensor i's part.
    """

    def __init__(self, params, grads, state_bits=32, copies=None, decay=None):
        torch = _t()
        self._h = None
        params, n = list(params), len(params)
        if n == 0 or (decay is not None and len(decay) != n) or params[0].dtype not in _dtypes or not params[0].is_cuda:
            _refuse("AdamW (params)")
        self.device, self.bits, self._params, self._dtype = params[0].device, int(state_bits), params, params[0].dtype
        self._grad_dtype = next((g.dtype for g in grads if g is not None), torch.float32)
        if self._grad_dtype not in _dtypes:
            _refuse("AdamW (gradient dtype)")
        self._sizes = [p.numel() for p in params]
        sizes = (ctypes.c_int64 * n)(*self._sizes)
        dec = None if decay is None else (ctypes.c_uint8 * n)(*[1 if d else 0 for d in decay])
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            rc = B.lib().dmx_adamw_create(n, sizes, dec, _dtypes[self._dtype], _dtypes[self._grad_dtype], self.bits, ctypes.byref(h))
        if rc != B.OK:
            _refuse("dmx_adamw_create", rc)
        self._h, self._destroy = h, B.lib().dmx_adamw_destroy     # (module globals may be gone when __del__ runs)
        self.blocks = B.lib().dmx_adamw_blocks(h)
        self.bind(grads, copies)

    def bind(self, grads, copies=None):
        """Take these gradient (and copy) tensors from now on; needed when their memory moves."""
        n = len(self._params)
        if len(grads) != n or (copies is not None and len(copies) != n):
            _refuse("AdamW.bind")
        for xs, dtype in ((self._params, self._dtype), (grads, self._grad_dtype), (copies or [], _torch.bfloat16)):
            for x, size in zip(xs, self._sizes):
                if x is not None and (x.dtype != dtype or x.numel() != size or x.device != self.device or not x.is_contiguous()):
                    _refuse("AdamW.bind (tensor)")
        arr = lambda xs: (ctypes.c_void_p * n)(*[None if x is None else x.data_ptr() for x in xs])  # noqa: E731
        with _on(self._params[0]):
            rc = B.lib().dmx_adamw_bind(self._h, arr(self._params), arr(grads), arr(copies) if copies is not None else None, _stream(self._params[0]))
        if rc != B.OK:
            _refuse("dmx_adamw_bind", rc)
        self._grads, self._copies = list(grads), copies      # kept alive: the handle holds their addresses

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
        return x[first * ADAMW_BLOCK: first * ADAMW_BLOCK + self._sizes[i]].view(self._params[i].shape)

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
        elif out.dtype != _torch.float32 or out.numel() != 2 or out.device != self.device or not out.is_contiguous():
            _refuse("AdamW.grad_norm (out)")
        with _on(out):
            rc = B.lib().dmx_adamw_grad_norm(self._h, max_norm, out.data_ptr(), _stream(out))
        if rc != B.OK:
            _refuse("dmx_adamw_grad_norm", rc)
        return out

    def step(self, m, v, m_scale=None, v_scale=None, *, lr, t, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=None, seed=None):
        """One update. t: this step's number, from 1. seed: dither 8-bit codes with it (None: to nearest)."""
        self._check("AdamW.step (state)", m, v, m_scale, v_scale)
        if grad_scale is not None and (grad_scale.dtype != _torch.float32 or grad_scale.numel() != 1 or grad_scale.device != self.device):
            _refuse("AdamW.step (grad_scale)")
        with _on(m):
            rc = B.lib().dmx_adamw_step(self._h, m.data_ptr(), v.data_ptr(), _ptr(m_scale), _ptr(v_scale), _ptr(grad_scale), lr, beta1, beta2, eps,
                                        weight_decay, t, 0 if seed is None else 1, 0 if seed is None else seed & 0xFFFFFFFF, _stream(m))
        if rc != B.OK:
            _refuse("dmx_adamw_step", rc)

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
        return out_m, out_v

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    __del__ = close


def _image(x, shape, dtype, like, where):
    """Strides (image, row) of an (N, ..., C) tensor whose positions lie at one stride and whose channels are dense."""
    if x is not like and (x.dtype != dtype or x.device != like.device or x.shape != shape):
        _refuse(where)
    st = x.stride()
    if x.dim() == 3:
        if shape[2] > 1 and st[2] != 1:
            _refuse(where)
        return st[0], st[1]
    if shape[-1] > 1 and st[-1] != 1:
        _refuse(where)
    row = st[-2]
    for i in range(x.dim() - 3, 0, -1):                  # (N, H, W, C): rows of the image must follow on
        if shape[i] > 1 and st[i] != row * _prod(shape[i + 1:-1]):
            _refuse(where)
    return st[0], row


def _prod(v):
    n = 1
    for x in v:
        n *= x
    return n


def _norm_args(x, groups, weight, bias, act, where):
    _t()
    if x.dim() < 3 or x.dtype not in _dtypes or not x.is_cuda or act not in ACT:
        _refuse(where)
    shape = x.shape
    C = shape[-1]
    for p in (weight, bias):
        if p is not None and (p.dtype != _torch.float32 or p.numel() != C or p.device != x.device or not p.is_contiguous()):
            _refuse(where + " (weight, bias)")
    return shape[0], shape[1] if len(shape) == 3 else _prod(shape[1:-1]), C, _dtypes[x.dtype]


def _fp32(shape, x, weight):
    return x.new_empty(shape) if x.dtype == _torch.float32 else weight.new_empty(shape) if weight is not None else _torch.empty(shape, dtype=_torch.float32, device=x.device)


@functools.lru_cache(maxsize=256)
def _norm_workspace(*shape):
    return B.lib().dmx_group_norm_workspace(*shape)


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, act="none", out=None):
    """act(group_norm(x)) of a channels-last tensor (N, ..., C), fp32 or bf16 -> (y, mean, rstd), the statistics
    fp32 (N, groups). weight, bias: fp32 (C,). x may be a channel slice of a wider tensor; out may be x."""
    N, L, C, dt = _norm_args(x, groups, weight, bias, act, "group_norm")
    xs = _image(x, x.shape, x.dtype, x, "group_norm (x)")
    if out is None:
        y = _torch.empty_like(x, memory_format=_torch.contiguous_format)
        ys = (L * C, C)
    else:
        y = out
        ys = _image(y, x.shape, x.dtype, x, "group_norm (out)")
    if groups < 1:
        _refuse("group_norm (groups)")
    mean, rstd = _fp32((2, N, groups), x, weight).unbind()
    need = _norm_workspace(N, L, C, groups, dt, 0)
    ws = _workspace(need, x, "group_norm") if need else None
    with _on(x):
        rc = B.lib().dmx_group_norm_forward(N, L, C, groups, dt, x.data_ptr(), xs[0], xs[1], _ptr(weight), _ptr(bias), eps, ACT[act], y.data_ptr(), ys[0], ys[1],
                                            mean.data_ptr(), rstd.data_ptr(), _ptr(ws), need, _stream(x))
    if rc != B.OK:
        _refuse("dmx_group_norm_forward", rc)
    return y, mean, rstd


def group_norm_backward(dy, x, mean, rstd, groups, weight=None, bias=None, act="none", out=None):
    """Gradient of group_norm from its saved statistics -> (dx, dweight, dbias)."""
    N, L, C, dt = _norm_args(x, groups, weight, bias, act, "group_norm_backward")
    xs = _image(x, x.shape, x.dtype, x, "group_norm_backward (x)")
    gs = _image(dy, x.shape, x.dtype, x, "group_norm_backward (dy)")
    if out is None:
        dx = _torch.empty_like(x, memory_format=_torch.contiguous_format)
        ds = (L * C, C)
    else:
        dx = out
        ds = _image(dx, x.shape, x.dtype, x, "group_norm_backward (out)")
    for s in (mean, rstd):
        if s.dtype != _torch.float32 or s.numel() != N * groups or s.device != x.device or not s.is_contiguous():
            _refuse("group_norm_backward (statistics)")
    dweight, dbias = _fp32((2, C), x, weight).unbind()
    need = _norm_workspace(N, L, C, groups, dt, 1)
    ws = _workspace(need, x, "group_norm_backward") if need else None
    with _on(x):
        rc = B.lib().dmx_group_norm_backward(N, L, C, groups, dt, dy.data_ptr(), gs[0], gs[1], x.data_ptr(), xs[0], xs[1], mean.data_ptr(), rstd.data_ptr(),
                                        _ptr(weight), _ptr(bias), ACT[act], dx.data_ptr(), ds[0], ds[1], dweight.data_ptr(),
                                             dbias.data_ptr(), _ptr(ws), need, _stream(x))
    if rc != B.OK:
        _refuse("dmx_group_norm_backward", rc)
    return dx, dweight, dbias


def _rows(x, shape, like, where):
    """Leading dimension of a bf16 matrix with dense rows."""
    if x.dtype != _torch.bfloat16 or x.device != like.device or tuple(x.shape) != shape or (shape[1] > 1 and x.stride(1) != 1):
        _refuse(where)
    return x.stride(0) if shape[0] > 1 else shape[1]


def _matrix(x, like, where):
    if x is None or x.dim() != 2 or not x.is_cuda:
        _refuse(where)
    return _rows(x, tuple(x.shape), like, where)


def linear(x, weight, bias=None, act="none", residual=None, save=False, out=None):
    """act(x @ weight.T + bias) + residual, bf16 matrices -> (y, z). z is the value before the activation, kept for
    linear_backward when `save` is set and there is an activation, else None. out may be the residual."""
    _t()
    if act not in ACT:
        _refuse("linear (act)")
    ldx, ldw = _matrix(x, x, "linear (x)"), _matrix(weight, x, "linear (weight)")
    (M, K), N = x.shape, weight.shape[0]
    if weight.shape[1] != K:
        _refuse("linear (weight)")
    if bias is not None and (bias.dtype != _torch.bfloat16 or bias.numel() != N or bias.device != x.device or not bias.is_contiguous()):
        _refuse("linear (bias)")
    ldr = 0 if residual is None else _rows(residual, (M, N), x, "linear (residual)")
    y = x.new_empty((M, N)) if out is None else out
    ldy = N if out is None else _rows(y, (M, N), x, "linear (out)")
    z = x.new_empty((M, N)) if save and act != "none" else None
    L = B.lib()
    xp, wp = x.data_ptr(), weight.data_ptr()
    with _on(x):
        if (xp | wp | 2 * ldx | 2 * ldw) & 15 or ldx < K or ldw < K:           # an operand has to be laid out (or is one row)
            ws = _workspace(L.dmx_linear_workspace(M, N, K, xp, ldx, wp, ldw), x, "linear")
        else:
            ws = None
        rc = L.dmx_linear_forward(M, N, K, xp, ldx, wp, ldw, _ptr(bias), ACT[act], _ptr(residual), ldr, y.data_ptr(), ldy, _ptr(z), N, _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(), _stream(x))
    if rc != B.OK:
        _refuse("dmx_linear_forward", rc)
    return y, z


def linear_backward(dy, x, weight, z=None, act="none", need=(True, True, True), out=(None, None, None)):
    """Gradient of linear -> (dx, dweight, dbias), those not in `need` None. `out`: tensors to write them to, e.g.
    views of a flat gradient vector."""
    _t()
    if act not in ACT:
        _refuse("linear_backward (act)")
    ldx, ldw = _matrix(x, x, "linear_backward (x)"), _matrix(weight, x, "linear_backward (weight)")
    (M, K), N = x.shape, weight.shape[0]
    if weight.shape[1] != K or (z is None and act != "none"):
        _refuse("linear_backward")
    ldg = _rows(dy, (M, N), x, "linear_backward (dy)")
    ldz = 0 if z is None else _rows(z, (M, N), x, "linear_backward (z)")
    mk = lambda k, shape: None if not need[k] else (x.new_empty(shape) if out[k] is None else out[k])  # noqa: E731
    dx, dw, db = mk(0, (M, K)), mk(1, (N, K)), mk(2, (N,))
    lddx = 0 if dx is None else _rows(dx, (M, K), x, "linear_backward (dx)")
    lddw = 0 if dw is None else _rows(dw, (N, K), x, "linear_backward (dweight)")
    if db is not None and (db.dtype != _torch.bfloat16 or db.numel() != N or db.device != x.device or not db.is_contiguous()):
        _refuse("linear_backward (dbias)")
    L = B.lib()
    gp, xp, wp = dy.data_ptr(), x.data_ptr(), weight.data_ptr()
    with _on(x):
        ws = _workspace(L.dmx_linear_backward_workspace(M, N, K, gp, ldg, xp, ldx, wp, ldw, ACT[act]), x, "linear_backward")
        rc = L.dmx_linear_backward(M, N, K, gp, ldg, xp, ldx, wp, ldw, _ptr(z), ldz, ACT[act], _ptr(dx), lddx, _ptr(dw), lddw, _ptr(db), _ptr(ws),
                                   0 if ws is None else ws.numel() * ws.element_size(), _stream(x))
    if rc != B.OK:
        _refuse("dmx_linear_backward", rc)
    return dx, dw, db


def linear_status():
    """How many warps of the linear kernels gave up a wait on the current device since the last call (synchronous)."""
    n = ctypes.c_int()
    rc = B.lib().dmx_linear_status(ctypes.byref(n))
    if rc != B.OK:
        _refuse("dmx_linear_status", rc)
    return n.value
