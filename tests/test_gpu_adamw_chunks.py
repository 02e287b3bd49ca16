"""AdamW on models large enough for the long chunks of fp32 moments (32 blocks, 256 blocks per SM and more), with last blocks that are
parts of a block at several places of a chunk. Checks and tolerances are those of the tests beside this one."""
import math

import pytest

pytestmark = pytest.mark.gpu

CHUNK = 32 * 256
SIZES = [3_000_001, 4 * CHUNK, 1 * CHUNK + 17, 2 * CHUNK + 7 * 256 + 255, 8 * 256 + 1, 31 * 256 + 100, 9_345_679, 5, 16 * 256, 24 * 256 + 8]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gd", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [0, 1])
def test_long_chunks(bits, gd, offset):
    import torch
    from tests.test_gpu_adamw import E, Case
    c = Case(SIZES, torch.float32, getattr(torch, gd), bits, offset, copies=True, seed=11)
    assert c.opt.blocks >= 148 * 256
    for t in (1, 2):
        ref = math.sqrt(sum(float((x.double() ** 2).sum()) for x in c.g))
        n = c.opt.grad_norm(0.5)
        assert abs(float(n[0]) - ref) <= 6 * E * ref and torch.equal(n, c.opt.grad_norm(0.5))
        c.check_step(t, scale=float(n[1]) * 1000, seed=t if bits == 8 else None)
        c.new_grads()
