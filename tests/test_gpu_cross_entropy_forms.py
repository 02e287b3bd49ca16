"""Every form in which the cross entropy's products are cut, against the definition in fp64 (checks and tolerances are those of the
tests beside this one). The list of shapes is kept complete by a test that needs no GPU."""
import ctypes

import pytest

from paper_2510_08522_b200 import binding as B

SHAPES = [(1, 1, 1), (1811, 1, 1), (11663, 1, 466), (1, 4882, 1), (3, 15639, 338), (1, 65, 1), (299, 15843, 1), (159, 26978, 1), (11480, 78, 132), (1557, 22002, 1),
          (3377, 7745, 1), (13564, 142, 367), (70000, 5003, 40), (1, 9585, 1), (1, 19676, 1), (9592, 67, 4), (10462, 130, 3), (258, 6372, 469), (12018, 130, 538),
          (2, 11577, 455), (44229, 1, 67), (1001, 1, 4741), (518, 10393, 141), (1, 892, 4966), (35, 736, 5054), (33, 1, 1),
          (37, 635, 1), (1, 663, 1), (732, 1, 1), (9715, 1, 66), (1, 9938, 137), (408, 2501, 988), (9820, 66, 997), (1563, 716, 1162), (11441, 147, 434),
          (9613, 1118, 68), (7314, 37228, 499)]


def forms(N, V, n):
    """{(product, tile width, pairs, one tile across the vocabulary)}, of the gradient's first one: several pieces; of dx, dw: ranges added afterwards"""
    p = (ctypes.c_int64 * 11)()
    assert B.lib().dmx_cross_entropy_plan(N, V, n, p) == B.OK
    out = {("loss", p[0], p[1], p[2] == 1), ("slope", p[5], p[6], p[3] > 1)}
    return out | ({("dx", p[7]), ("dw", p[9])} if p[3] == 1 else set())


def test_the_shapes_reach_every_form():
    every = {("loss", *f) for f in ((64, 0, True), (64, 0, False), (128, 0, True), (128, 0, False), (128, 1, True), (128, 1, False), (256, 0, True), (256, 0, False), (256, 1, True), (256, 1, False))}
    every |= {("slope", *f) for f in ((64, 0, False), (128, 0, False), (128, 1, False), (256, 0, False), (256, 0, True), (256, 1, False), (256, 1, True))}
    every |= {(name, bn) for name in ("dx", "dw") for bn in (0, 64, 128)}
    reached = set().union(*[forms(*s) for s in SHAPES])
    assert every == reached, (every - reached, reached - every)


def test_plan_refuses_bad_extents():
    p = (ctypes.c_int64 * 11)()
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, -1), (4194241, 8, 8)):
        assert B.lib().dmx_cross_entropy_plan(*bad, p) == B.ERR_ARG
    assert B.lib().dmx_cross_entropy_plan(8, 8, 8, None) == B.ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_forms(shape):
    from tests.test_gpu_cross_entropy import _d, compare, problem
    torch, D = _d()
    x, w, t, b = problem(torch, *shape, seed=1)
    compare(torch, D, x, w, t, b)
