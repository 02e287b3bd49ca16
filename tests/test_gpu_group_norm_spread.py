"""Group norm of data whose spread is far below its mean, in every mode: values that differ only from channel to channel (a broadcast
input), only from position to position, between an image's halves, or everywhere. The statistics have to be as good as for data around zero.

Tolerances, with e = 2^-24 and G = 150 (additions on the way into a sum, as in the tests beside this one): deviations are summed, so the
variance is within (G + 8) e of itself, whatever the mean; the mean is within 2 e of itself plus G e of the deviations that were
summed, at most twice the largest deviation of the group."""
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
GAMMA = 150 * E


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


SHAPES = [(37, 3, 14, 7), (3, 1120, 226, 113), (14, 2527, 18, 9), (2, 729, 90, 15), (1, 3136, 64, 8), (1, 40000, 32, 4), (2, 9001, 33, 3), (4, 100, 200, 5),
          (70, 16, 512, 32), (1, 20, 1023, 1), (300, 200, 24, 3), (2, 20000, 64, 2), (8, 512, 256, 32)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("mean", [0.0, 30.0, -3000.0])
def test_statistics_do_not_depend_on_the_mean(shape, dtype, mean):
    torch, D = _d()
    N, L, C, G = shape
    g = torch.Generator(device="cuda").manual_seed(L)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    # a spread of some 30 units in the mean's last place (bf16: the type's own), and of one where the mean is zero
    sigma = abs(mean) * (2.0 ** -18 if dtype == "float32" else 2.0 ** -4) if mean else 1.0
    half = (torch.arange(L, device="cuda") >= L // 2).float().view(1, L, 1)
    for name, x in (("channels", r(N, 1, C)), ("positions", r(N, L, 1)), ("halves", half + 0.01 * r(N, 1, C)), ("everywhere", r(N, L, C))):
        x = (mean + sigma * x).to(getattr(torch, dtype))
        x = x.expand(N, L, C) if name == "channels" else x.expand(N, L, C).contiguous()
        _, m, rstd = D.group_norm(x, G, eps=0.0)
        X = x.double().reshape(N, L, G, C // G)
        mu = X.mean((1, 3), keepdim=True)
        dev = X - mu
        var = dev.square().mean((1, 3))
        mu, most = mu[:, 0, :, 0], dev.abs().amax((1, 3))
        assert torch.all((m.double() - mu).abs() <= 2 * E * mu.abs() + 2 * GAMMA * most), (name, float(((m.double() - mu).abs() / mu.abs()).max()))
        some = most > 0                                           # (groups of equal values have no deviation)
        off = (rstd.double()[some] * var[some].sqrt() - 1).abs()
        assert some.any() or L == 1 or name == "positions"
        assert not some.any() or float(off.max()) <= (GAMMA + 8 * E) / 2 + 4 * E, (name, float(off.max()))
