"""Edges of the training operators' domain that a user meets: nothing to sum over, values that overflow or underflow, images cut out
of wider ones, tensors in other dense orders, calls from several threads and streams."""

import pytest

pytestmark = pytest.mark.gpu


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_statistics_of_no_positions_are_nan(dtype):
    # a sum of nothing over nothing: no mean and no deviation. The memory the results come from held other values before.
    torch, D = _d()
    for N, groups in ((3, 2), (1, 1), (70, 8)):
        x = torch.empty(N, 0, 8, dtype=getattr(torch, dtype), device="cuda")
        old = [torch.full((N, groups), 7.0, device="cuda") for _ in range(8)]
        del old
        y, mean, rstd = D.group_norm(x, groups)
        assert y.shape == x.shape and mean.shape == rstd.shape == (N, groups)
        assert torch.isnan(mean).all() and torch.isnan(rstd).all()
