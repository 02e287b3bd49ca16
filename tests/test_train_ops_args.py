"""Argument checks of the training operators that need no GPU: the C entry points refuse what they document
before any device call."""
import ctypes

import paper_2510_08522_b200  # noqa: F401
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
