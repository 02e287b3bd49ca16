"""Edges of the training operators' torch bindings that need no GPU."""
import pytest


def test_a_flag_without_a_truth_value_is_refused():
    torch = pytest.importorskip("torch")
    import paper_2510_08522_b200 as D

    class Neither:
        def __bool__(self):
            raise ValueError("neither")

    m = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(D.DmxError):
        D.linear(m, m, save=Neither())


def test_what_is_no_tensor_is_refused_by_the_optimizer():
    torch = pytest.importorskip("torch")
    import paper_2510_08522_b200 as D
    x = torch.zeros(4)
    for params, grads in (([None], [None]), ([1.0], [None]), ([x], [x]), ([x, None], [None, None]), ([], [])):
        with pytest.raises(D.DmxError):
            D.AdamW(params, grads)
