"""Group norm where every CTA (or cluster of CTAs) takes three items and more in turn: buffers are turned, slots refilled and
parameters fetched ahead, in each mode (a slab in one CTA, in clusters of two, four and eight, images in chunks), for both types, both
directions and both access widths. Against the definition in fp64, in place, and repeated. Checks and tolerances are those of the tests beside this one."""
import ctypes

import pytest

from paper_2510_08522_b200 import binding as B

# type, backward, wide accesses, CTAs that share a slab (0: chunks), N, L, C, G
CASES = [
    ("float32", 0, 0, 0, 7, 16538, 65, 5), ("float32", 0, 0, 1, 5000, 7, 33, 3), ("float32", 0, 0, 2, 151, 4930, 12, 6), ("float32", 0, 0, 4, 77, 10464, 11, 11),
    ("float32", 0, 0, 8, 38, 23077, 9, 9), ("float32", 0, 1, 0, 4, 29459, 72, 18), ("float32", 0, 1, 1, 2450, 5, 132, 22), ("float32", 0, 1, 2, 151, 4930, 12, 6),
    ("float32", 0, 1, 4, 152, 422, 156, 4), ("float32", 0, 1, 8, 38, 22491, 12, 6),
    ("float32", 1, 0, 0, 3, 19505, 65, 5), ("float32", 1, 0, 1, 5000, 7, 33, 3), ("float32", 1, 0, 2, 154, 2555, 10, 5), ("float32", 1, 0, 4, 79, 5271, 10, 5),
    ("float32", 1, 0, 8, 41, 9521, 11, 11), ("float32", 1, 1, 0, 6, 1625, 440, 8), ("float32", 1, 1, 1, 2450, 5, 132, 22), ("float32", 1, 1, 2, 371, 67, 172, 4),
    ("float32", 1, 1, 4, 88, 290, 132, 4), ("float32", 1, 1, 8, 79, 224, 172, 4),
    ("bfloat16", 0, 0, 0, 5, 23284, 132, 22), ("bfloat16", 0, 0, 1, 5000, 7, 33, 3), ("bfloat16", 0, 0, 2, 229, 3584, 21, 21), ("bfloat16", 0, 0, 4, 113, 6815, 20, 20),
    ("bfloat16", 0, 0, 8, 56, 16581, 18, 6), ("bfloat16", 0, 1, 0, 9, 10206, 168, 24), ("bfloat16", 0, 1, 1, 2388, 5, 320, 10), ("bfloat16", 0, 1, 2, 162, 2812, 40, 20),
    ("bfloat16", 0, 1, 4, 77, 6913, 40, 20), ("bfloat16", 0, 1, 8, 77, 1430, 184, 8),
    ("bfloat16", 1, 0, 0, 8, 7553, 130, 5), ("bfloat16", 1, 0, 1, 5000, 7, 33, 3), ("bfloat16", 1, 0, 2, 149, 2483, 21, 7), ("bfloat16", 1, 0, 4, 77, 5412, 19, 19),
    ("bfloat16", 1, 0, 8, 39, 9958, 20, 4), ("bfloat16", 1, 1, 0, 2, 20160, 152, 19), ("bfloat16", 1, 1, 1, 2388, 5, 280, 14), ("bfloat16", 1, 1, 2, 78, 195, 312, 6),
    ("bfloat16", 1, 1, 4, 77, 171, 408, 8), ("bfloat16", 1, 1, 8, 41, 231, 504, 8), ("bfloat16", 1, 1, 2, 64, 3136, 256, 32), ("bfloat16", 1, 1, 2, 1024, 1024, 64, 16),
]


@pytest.mark.parametrize("case", CASES)
def test_the_cases_take_their_mode_and_several_items(case):
    dtype, backward, wide, parts, N, L, C, G = case
    p = (ctypes.c_int64 * 6)()
    assert B.lib().dmx_group_norm_plan(N, L, C, G, B.F32 if dtype == "float32" else B.BF16, wide, backward, p) == B.OK
    V, resident, shared_by, items, threads, smem = p
    assert (V > 1) == bool(wide) and (shared_by if resident else 0) == parts
    # more CTAs than these cannot run at once: 2048 threads and 228 KB per SM, each CTA's shared memory and 1 KB
    at_once = 148 * min(32, 2048 // threads, 228 * 1024 // (smem + 1024)) // max(1, parts)
    if (N, L, C) not in ((64, 3136, 256), (1024, 1024, 64)):        # (sizes as they are met; registers allow them three and two CTAs per SM)
        assert items > 2 * at_once, (items, at_once)


def test_plan_refuses_bad_shapes():
    p = (ctypes.c_int64 * 6)()
    for bad in ((0, 5, 8, 2), (2, 0, 8, 2), (2, 5, 8, 3), (2, 5, 70000, 70000)):
        assert B.lib().dmx_group_norm_plan(*bad, 0, 1, 0, p) == B.ERR_ARG
    assert B.lib().dmx_group_norm_plan(2, 5, 8, 2, 0, 1, 0, None) == B.ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_items_in_turn(case):
    from tests.test_gpu_group_norm import _d, check_backward, check_forward, make
    torch, D = _d()
    dtype, backward, wide, _, N, L, C, G = case
    act = ["none", "relu", "silu", "gelu"][(N + L + C) % 4]
    x, dy, w, b = make(N, L, C, getattr(torch, dtype), 0 if wide else 1, seed=N)

    def same(t):                               # a copy that lies as t does
        z = torch.empty_strided((N, L, x.stride(1)), (L * x.stride(1), x.stride(1), 1), dtype=x.dtype, device="cuda")[:, :, :C]
        assert z.stride() == t.stride()
        return z.copy_(t)

    got = D.group_norm(x, G, w, b, 1e-5, act)
    if not backward:
        check_forward(x, G, w, b, 1e-5, act, got)
        again = D.group_norm(x, G, w, b, 1e-5, act)
        assert all(torch.equal(p, q) for p, q in zip(got, again))
        z = same(x)
        D.group_norm(z, G, w, b, 1e-5, act, out=z)
        assert torch.equal(z, got[0])
        return
    want = D.group_norm_backward(dy, x, got[1], got[2], G, w, b, act)
    check_backward(dy, x, got[1], got[2], G, w, b, act, want)
    assert all(torch.equal(p, q) for p, q in zip(want, D.group_norm_backward(dy, x, got[1], got[2], G, w, b, act)))
    z = same(dy)
    assert all(torch.equal(p, q) for p, q in zip(want, D.group_norm_backward(z, x, got[1], got[2], G, w, b, act, out=z)))
    z = same(x)
    assert all(torch.equal(p, q) for p, q in zip(want, D.group_norm_backward(dy, z, got[1], got[2], G, w, b, act, out=z)))
