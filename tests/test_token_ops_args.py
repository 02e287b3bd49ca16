"""Argument checks of layer norm, the embedding lookup and the cross entropy that need no GPU: the C entry points refuse what they document before any device call."""
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


def test_embedding_refuses_bad_sizes_types_strides_and_pointers():
    L = B.lib()
    big = 1 << 31
    for a in ((-1, 4, 8), (4, -1, 8), (4, 4, -1), (big, 4, 8), (4, big, 8), (4, 4, 65537)):
        assert L.dmx_embedding_backward_workspace(*a) == B.ERR_ARG
    assert L.dmx_embedding_backward_workspace(0, 4, 8) == 0 and L.dmx_embedding_backward_workspace(100, 4, 8) >= 4 * 400

    def forward(N=4, V=5, n=8, dt=0, ib=8, ids=64, table=128, ldt=8, scale=1.0, y=1024, ldy=8):
        return L.dmx_embedding_forward(N, V, n, dt, ib, ids, table, ldt, scale, y, ldy, None)
    for bad in (dict(N=-1), dict(N=big), dict(V=big), dict(n=65537), dict(dt=2), dict(ib=2), dict(ids=None), dict(table=None), dict(y=None), dict(ldt=-1), dict(ldy=7)):
        assert forward(**bad) == B.ERR_ARG, bad
    for bad in (dict(ids=68), dict(ids=66, ib=4), dict(table=130), dict(y=1026), dict(dt=1, table=129)):
        assert forward(**bad) == B.ERR_ALIGN, bad
    assert forward(N=0) == B.OK and forward(n=0, ldy=0) == B.OK

    def backward(N=4, V=5, n=8, ib=8, ids=64, dt=0, dy=128, lddy=8, odt=0, out=1024, ldt=8, add=0, ws=4096, size=1 << 20):
        return L.dmx_embedding_backward(N, V, n, ib, ids, dt, dy, lddy, 1.0, odt, out, ldt, add, ws, size, None)
    for bad in (dict(N=big), dict(V=-1), dict(n=65537), dict(ib=1), dict(dt=3), dict(odt=-1), dict(lddy=-1), dict(ldt=7), dict(ids=None), dict(dy=None), dict(out=None), dict(ws=None), dict(size=100)):
        assert backward(**bad) == B.ERR_ARG, bad
    for bad in (dict(ids=60), dict(dy=130), dict(out=1026), dict(ws=4112)):
        assert backward(**bad) == B.ERR_ALIGN, bad
    assert backward(V=0) == B.OK and backward(n=0, ldt=0) == B.OK and backward(N=0, add=1) == B.OK


def test_cross_entropy_refuses_bad_extents_strides_and_pointers():
    L = B.lib()
    big = 4194241
    for f in (L.dmx_cross_entropy_workspace, L.dmx_cross_entropy_backward_workspace):
        for a in ((-1, 8, 8), (big, 8, 8), (4, 0, 8), (4, big, 8), (4, 8, 0), (4, 8, big)):
            assert f(*a, 256, 8, 512, 8) == B.ERR_ARG
        assert f(0, 8, 8, None, 8, 512, 8) == 0 and 0 < f(4, 8, 8, 256, 8, 512, 8) < f(4, 8, 8, 258, 8, 512, 8)

    def forward(N=4, V=8, n=16, x=256, ldx=16, w=512, ldw=16, bias=None, tb=8, t=1024, loss=2048, lse=4096, ws=8192, size=1 << 20):
        return L.dmx_cross_entropy_forward(N, V, n, x, ldx, w, ldw, bias, tb, t, loss, lse, ws, size, None)
    for bad in (dict(N=-1), dict(V=0), dict(n=0), dict(V=big), dict(ldx=-1), dict(ldw=-1), dict(tb=2), dict(x=None), dict(w=None), dict(t=None), dict(loss=None), dict(lse=None), dict(ws=None), dict(size=64)):
        assert forward(**bad) == B.ERR_ARG, bad
    for bad in (dict(x=257), dict(w=513), dict(bias=3), dict(t=1028), dict(loss=2050), dict(lse=4097), dict(ws=8200)):
        assert forward(**bad) == B.ERR_ALIGN, bad
    assert forward(N=0, x=None, t=None) == B.OK

    def backward(N=4, V=8, n=16, g=128, gs=1, x=256, ldx=16, w=512, ldw=16, bias=None, tb=4, t=1024, lse=2048, dx=4096, lddx=16, dw=8192, lddw=16, db=6144, ws=16384, size=1 << 20):
        return L.dmx_cross_entropy_backward(N, V, n, g, gs, x, ldx, w, ldw, bias, tb, t, lse, dx, lddx, dw, lddw, db, ws, size, None)
    for bad in (dict(N=big), dict(V=0), dict(gs=-1), dict(ldx=-1), dict(lddx=15), dict(lddw=0), dict(tb=1), dict(g=None), dict(x=None), dict(w=None), dict(t=None), dict(lse=None), dict(ws=None),
                dict(size=64)):
        assert backward(**bad) == B.ERR_ARG, bad
    for bad in (dict(g=130), dict(x=257), dict(w=513), dict(bias=3), dict(t=1026), dict(lse=2049), dict(dx=4097), dict(dw=8193), dict(db=6145), dict(ws=16388)):
        assert backward(**bad) == B.ERR_ALIGN, bad
    assert backward(dx=None, dw=None, db=None) == B.OK


def test_torch_callers_get_errors_for_what_is_no_cuda_tensor():
    torch = pytest.importorskip("torch")
    x, m = torch.zeros(4, 8), torch.zeros(4)
    h = x.bfloat16()
    for call in (lambda: D.linear_cross_entropy(h, h, m.long()), lambda: D.linear_cross_entropy(h, None, m.long()), lambda: D.linear_cross_entropy(h, h, 3),
                 lambda: D.linear_cross_entropy_backward(m, h, h, m.long(), m), lambda: D.linear_cross_entropy_backward(None, h, h, m.long(), m), lambda: D.layer_norm(x), lambda: D.layer_norm(None), lambda: D.layer_norm(x, "w"), lambda: D.layer_norm([1.0]),
                 lambda: D.embedding(m.long(), x), lambda: D.embedding(3, x), lambda: D.embedding(m.long(), None), lambda: D.embedding_backward(x, m.long(), 5),
                 lambda: D.embedding_backward(x, [1], 5), lambda: D.layer_norm_backward(x, x, m, m), lambda: D.layer_norm_backward(x, None, m, m), lambda: D.layer_norm_backward(x, x, m, 3)):
        with pytest.raises(D.DmxError):
            call()
