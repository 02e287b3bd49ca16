"""Argument checks of layer norm that need no GPU: the C entry points refuse what they document before any device call."""
import pytest

import paper_2510_08522_b200 as D
from paper_2510_08522_b200 import binding as B


def test_layer_norm_refuses_bad_shapes_strides_and_pointers():
    L = B.lib()
    for M, n, dt in ((-1, 8, 0), (1 << 40, 8, 0), (4, 0, 0), (4, -1, 1), (4, 65537, 1), (4, 8, 2), (4, 8, -1)):
        assert L.dmx_layer_norm_workspace(M, n, dt) == B.ERR_ARG
    assert L.dmx_layer_norm_workspace(0, 8, 0) == 0 and L.dmx_layer_norm_workspace(5, 1024, 1) >= 2 * 1024 * 4

    def forward(M=4, n=8, dt=0, x=64, ldx=8, eps=1e-5, y=1024, ldy=8, mean=2048, rstd=4096, w=None, b=None):
        return L.dmx_layer_norm_forward(M, n, dt, x, ldx, w, b, eps, y, ldy, mean, rstd, None)
    for bad in (dict(M=-1), dict(n=0), dict(n=65537), dict(dt=7), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(ldx=-1), dict(ldy=7), dict(ldy=0), dict(eps=-1e-9),
                dict(eps=float("nan"))):
        assert forward(**bad) == B.ERR_ARG, bad
    for bad in (dict(x=66), dict(y=1026), dict(mean=2049), dict(rstd=4098), dict(w=6), dict(b=2), dict(dt=1, x=65)):
        assert forward(**bad) == B.ERR_ALIGN, bad
    assert forward(M=0, x=None, y=None, mean=None, rstd=None) == B.OK

    def backward(M=4, n=8, dt=0, dy=64, lddy=8, x=512, ldx=8, mean=2048, rstd=4096, w=None, add=None, ldadd=8, dx=1024, lddx=8, dw=8192, db=8256, ws=16384, size=1 << 20):
        return L.dmx_layer_norm_backward(M, n, dt, dy, lddy, x, ldx, mean, rstd, w, add, ldadd, dx, lddx, dw, db, ws, size, None)
    for bad in (dict(M=-1), dict(n=65537), dict(dt=2), dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(lddy=-1), dict(ldx=-8), dict(lddx=7),
                dict(add=128, ldadd=-1), dict(ws=None), dict(size=255)):
        assert backward(**bad) == B.ERR_ARG, bad
    for bad in (dict(dy=65), dict(x=514), dict(add=130), dict(dx=1025), dict(w=7), dict(dw=8193), dict(db=8258), dict(ws=16392)):
        assert backward(**bad) == B.ERR_ALIGN, bad


def test_torch_callers_get_errors_for_what_is_no_cuda_tensor():
    torch = pytest.importorskip("torch")
    x, m = torch.zeros(4, 8), torch.zeros(4)
    for call in (lambda: D.layer_norm(x), lambda: D.layer_norm(None), lambda: D.layer_norm(x, "w"), lambda: D.layer_norm([1.0]),
                 lambda: D.layer_norm_backward(x, x, m, m), lambda: D.layer_norm_backward(x, None, m, m), lambda: D.layer_norm_backward(x, x, m, 3)):
        with pytest.raises(D.DmxError):
            call()
