"""Every form in which the matrix product is cut (tile width, pairs of CTAs, ranges of k, exchanged operands, one or several tiles per
CTA, for each of y, dx and dw, whose operands lie differently), against the definition in fp64. The list of shapes is kept complete by a
test that needs no GPU. Checks, tolerances and repeats are those of the tests beside this one."""
import ctypes

import pytest

from paper_2510_08522_b200 import binding as B

# M, N, K: odd ones, whose operands are laid out first, and ones that the tensor maps take as they lie
SHAPES = [(1, 1, 1), (776, 1, 1), (1, 19336, 1), (130, 3, 9636), (142, 7860, 131), (3, 904, 5919), (34, 265, 19383), (1492, 387, 1224), (48, 1, 1),
          (33, 19012, 7), (812, 2748, 901), (19712, 8, 328), (541, 7, 19107), (48, 4741, 5456), (7698, 336, 304), (314, 280, 19824), (3587, 1235, 635),
          (14696, 418, 386), (2, 2, 19005), (2602, 884, 1626), (1, 4819, 840), (295, 15960, 4), (1289, 6284, 219),
          (4096, 2048, 1024), (8192, 4096, 1024), (8192, 64, 64), (200, 2544, 2064), (8, 4792, 2240), (40, 4960, 1504)]


def forms(M, N, K):
    """{(product, tile width, pairs, ranges of k, exchanged, several tiles per CTA)}"""
    out, p = set(), (ctypes.c_int64 * 5)()
    for name, rows, cols, k, across in (("y", M, N, K, 0), ("dx", M, K, N, 0), ("dw", N, K, M, 1)):
        assert B.lib().dmx_linear_plan(rows, cols, k, across, p) == B.OK
        out.add((name, p[0], p[1], p[2], p[3], p[4] > 1))
    return out


def test_the_shapes_reach_every_form():
    plain = [(w, pair, 1, 0, many) for w, pair in ((256, 1), (256, 0), (128, 1), (128, 0), (64, 0)) for many in (False, True)]
    plain += [(128, 0, 2, 0, False), (64, 0, 2, 0, False)]
    exchanged = [(w, 0, 1, 1, many) for w in (32, 64) for many in (False, True)] + [(w, 0, split, 1, False) for w in (32, 64) for split in (2, 4)]
    every = {("dw", *f) for f in plain} | {(name, *f) for name in ("y", "dx") for f in plain + exchanged}
    reached = set().union(*[forms(*s) for s in SHAPES])
    assert every <= reached, sorted(every - reached)
    assert reached <= every, sorted(reached - every)


def test_plan_refuses_bad_extents():
    p = (ctypes.c_int64 * 5)()
    for bad in ((0, 8, 8), (8, -1, 8), (8, 8, 0), (4194241, 8, 8)):
        assert B.lib().dmx_linear_plan(*bad, 0, p) == B.ERR_ARG
    assert B.lib().dmx_linear_plan(8, 8, 8, 0, None) == B.ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_forms(shape):
    from tests.test_gpu_linear import run
    run(*shape, act=["gelu", "none", "silu", "relu"][sum(shape) % 4], residual=sum(shape) % 3 == 0)
