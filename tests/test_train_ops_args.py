"""Argument checks of the training operators that need no GPU: the C entry points refuse what they document
before any device call."""
import ctypes

import pytest

import paper_2510_08522_b200 as D
from paper_2510_08522_b200 import binding as B


def test_adamw_create_refuses_bad_descriptions():
    L = B.lib()
    h = ctypes.c_void_p(1)
    one = (ctypes.c_int64 * 1)(5)
    for n, sizes, pd, gd, bits in ((0, one, 0, 0, 32), (-1, one, 0, 0, 32), (65537, one, 0, 0, 32), (1, None, 0, 0, 32), (1, one, 2, 0, 32),
                                   (1, one, 0, -1, 8), (1, one, 0, 0, 16), (1, (ctypes.c_int64 * 1)(-1), 0, 0, 32),
                                   (1, (ctypes.c_int64 * 1)(1 << 40), 0, 0, 32)):
        assert L.dmx_adamw_create(n, sizes, None, pd, gd, bits, ctypes.byref(h)) == B.ERR_ARG
        assert not h.value
    assert L.dmx_adamw_create(1, one, None, 0, 0, 32, None) == B.ERR_ARG


def test_adamw_refuses_what_is_no_handle():
    L = B.lib()
    for h in (None, ctypes.c_void_p(0x10)):
        assert L.dmx_adamw_blocks(h) == B.ERR_HANDLE
        assert L.dmx_adamw_first_block(h, 0) == B.ERR_HANDLE
        assert L.dmx_adamw_bind(h, None, None, None, None) == B.ERR_HANDLE
        assert L.dmx_adamw_grad_norm(h, 1.0, 16, None) == B.ERR_HANDLE
        assert L.dmx_adamw_step(h, 16, 32, None, None, None, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0, None) == B.ERR_HANDLE
        assert L.dmx_adamw_moments(h, 16, 32, 48, 64, 0, 80, 96, None) == B.ERR_HANDLE
    assert L.dmx_adamw_destroy(None) == B.OK
    assert L.dmx_adamw_destroy(ctypes.c_void_p(0x10)) == B.ERR_HANDLE


def test_group_norm_refuses_bad_shapes_strides_and_pointers():
    L = B.lib()
    ok = dict(N=2, L=10, C=12, G=3, dt=0)
    for bad in (dict(C=0), dict(G=0), dict(G=5), dict(dt=2), dict(N=-1), dict(L=-1), dict(C=65537, G=65537), dict(C=1025, G=1), dict(L=1 << 31)):
        a = dict(ok, **bad)
        assert L.dmx_group_norm_workspace(a["N"], a["L"], a["C"], a["G"], a["dt"], 0) == B.ERR_ARG
    assert L.dmx_group_norm_workspace(0, 10, 12, 3, 0, 1) == 0
    assert L.dmx_group_norm_workspace(2, 10, 12, 3, 0, 1) >= 2 * 2 * 12 * 4
    assert L.dmx_group_norm_workspace(1, 1 << 20, 64, 8, 1, 0) > 0              # larger than a cluster holds: chunked

    def forward(x=16, xi=120, xr=12, y=1024, yi=120, yr=12, eps=1e-5, act=0, mean=2048, rstd=3072):
        return L.dmx_group_norm_forward(2, 10, 12, 3, 0, x, xi, xr, None, None, eps, act, y, yi, yr, mean, rstd, None, 0, None)
    assert forward(x=None) == B.ERR_ARG and forward(y=None) == B.ERR_ARG and forward(mean=None) == B.ERR_ARG
    assert forward(yr=11) == B.ERR_ARG and forward(xr=-12) == B.ERR_ARG and forward(act=4) == B.ERR_ARG and forward(eps=-1.0) == B.ERR_ARG
    assert forward(eps=float("nan")) == B.ERR_ARG and forward(x=18) == B.ERR_ALIGN and forward(rstd=2050) == B.ERR_ALIGN
    assert L.dmx_group_norm_forward(0, 10, 12, 3, 0, None, 0, 12, None, None, 1e-5, 0, None, 0, 12, None, None, None, 0, None) == B.OK
    assert forward(yi=0) == B.ERR_ARG and forward(yi=119) == B.ERR_ARG and forward(yi=12, yr=23) == B.ERR_ARG and forward(yi=11, yr=24) == B.ERR_ARG   # two elements in one place
    back = lambda ws, n: L.dmx_group_norm_backward(2, 10, 12, 3, 0, 16, 120, 12, 1024, 120, 12, 2048, 3072, None, None, 0, 4096, 120, 12, None, None,  # noqa: E731
                                                   ws, n, None)
    assert back(None, 0) == B.ERR_ARG and back(8192, 64) == B.ERR_ARG and back(8200, 1 << 20) == B.ERR_ALIGN


def test_linear_refuses_bad_extents_strides_and_pointers():
    L = B.lib()
    big = 4194241
    assert L.dmx_linear_workspace(big, 8, 8, 16, 8, 32, 8) == B.ERR_ARG and L.dmx_linear_workspace(-1, 8, 8, 16, 8, 32, 8) == B.ERR_ARG
    assert L.dmx_linear_workspace(4, 8, 16, 16, 16, 32, 16) == 0                  # operands as TMA takes them
    assert L.dmx_linear_workspace(4, 8, 16, 18, 16, 32, 16) == 256                # x starts off 16 bytes: laid out
    assert L.dmx_linear_workspace(4, 8, 16, 16, 17, 32, 0) == 512                 # odd rows, repeated rows
    assert L.dmx_linear_backward_workspace(4, 8, 16, 16, 8, 32, 16, 48, 16, 9) == B.ERR_ARG

    def forward(M=4, N=8, K=16, x=256, ldx=16, w=512, ldw=16, act=0, y=1024, ldy=8, z=None, ldz=0, r=None, ldr=0, bias=None, ws=None, n=0):
        return L.dmx_linear_forward(M, N, K, x, ldx, w, ldw, bias, act, r, ldr, y, ldy, z, ldz, ws, n, None)
    assert forward(M=big) == B.ERR_ARG and forward(act=-1) == B.ERR_ARG and forward(act=4) == B.ERR_ARG
    assert forward(x=None) == B.ERR_ARG and forward(w=None) == B.ERR_ARG and forward(y=None) == B.ERR_ARG
    assert forward(ldy=7) == B.ERR_ARG and forward(ldx=-1) == B.ERR_ARG and forward(z=2048, ldz=7) == B.ERR_ARG
    assert forward(x=257) == B.ERR_ALIGN and forward(bias=3) == B.ERR_ALIGN
    assert forward(x=258) == B.ERR_ARG and forward(x=258, ws=4096, n=128) == B.ERR_ARG and forward(x=258, ws=4100, n=4096) == B.ERR_ALIGN   # no (or too little) workspace
    assert forward(M=0) == B.OK and forward(N=0) == B.OK

    def backward(z=None, act=0, dy=256, x=512, w=1024, dx=2048, dw=4096, lddx=16, ws=8192, n=1 << 20):
        return L.dmx_linear_backward(4, 8, 16, dy, 8, x, 16, w, 16, z, 8, act, dx, lddx, dw, 16, None, ws, n, None)
    assert backward(act=1) == B.ERR_ARG and backward(dy=None) == B.ERR_ARG and backward(w=None) == B.ERR_ARG and backward(x=None) == B.ERR_ARG
    assert backward(lddx=15) == B.ERR_ARG and backward(ws=None) == B.ERR_ARG and backward(n=16) == B.ERR_ARG and backward(dw=4097) == B.ERR_ALIGN
    assert L.dmx_linear_status(None) == B.ERR_ARG


def test_torch_callers_get_errors_for_what_is_no_cuda_tensor():
    torch = pytest.importorskip("torch")
    x, m = torch.zeros(2, 5, 8), torch.zeros(4, 8, dtype=torch.bfloat16)
    for call in (lambda: D.group_norm(x, 2), lambda: D.group_norm(None, 2), lambda: D.group_norm([1.0], 2), lambda: D.group_norm(x, "2"),
                 lambda: D.group_norm(x, 2, eps="small"), lambda: D.group_norm(x.double(), 2), lambda: D.group_norm_backward(x, x, x[0], x[0], 2),
                 lambda: D.linear(m, m), lambda: D.linear(m, None), lambda: D.linear(m.float(), m.float()), lambda: D.linear_backward(m, m, m),
                 lambda: D.linear_backward(m, 1, m)):
        with pytest.raises(D.DmxError):
            call()
