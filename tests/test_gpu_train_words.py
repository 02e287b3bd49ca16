"""Embedding, layer norm, matrix product and cross entropy together, as the small network over words uses them: its gradient against
torch's own differentiation of the same network in 64 bits, explicit calls against recorded ones, and runs with the gradient step and AdamW."""
import pytest

pytestmark = pytest.mark.gpu


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08522_b200 import train_small as S
    return torch, S


def sample(torch, S, words, n=24):
    model = S.Words(words=words, seed=3)
    model.view(model.flat, "head.b").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    model.half = model.flat.to(torch.bfloat16)
    ids, target = model.batch(n, torch.Generator(device="cuda").manual_seed(5), "cuda")
    grad = torch.full((model.P,), float("nan"), dtype=torch.bfloat16, device="cuda")
    return model, ids, target, grad


@pytest.mark.parametrize("words", [1000, 77, 5003])
def test_gradient_matches_autograd(words):
    torch, S = _d()
    model, ids, target, grad = sample(torch, S, words)
    loss = model.learn(ids, target, grad)
    par = {n: model.view(model.flat if ".ln." in n or n.startswith("ln.") else model.half, n).double().requires_grad_(True) for n in model.names}

    def norm(x, w, b):
        d = x - x.mean(1, keepdim=True)
        return d * (d.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * w + b
    ok = (ids >= 0).reshape(-1)
    x = par["table"][ids.reshape(-1).clamp_min(0)] * model.scale * ok[:, None]
    for i in range(model.blocks):
        p = "%d." % i
        u = torch.nn.functional.gelu(norm(x, par[p + "ln.w"], par[p + "ln.b"]) @ par[p + "up.w"].t() + par[p + "up.b"])
        x = u @ par[p + "down.w"].t() + par[p + "down.b"] + x
    ref = torch.nn.functional.cross_entropy(norm(x, par["ln.w"], par["ln.b"]) @ par["table"].t() + par["head.b"], target.reshape(-1), ignore_index=-1)
    ref.backward()
    # some twenty values in a row are rounded to bf16 on the way to a gradient and back, each off by 0.17 % in the mean square:
    # under 1 % if they add as independent errors, taken three times
    assert abs(float(loss) - float(ref.detach())) < 0.03 * float(ref.detach())
    for n in model.names:
        g, r = model.view(grad, n).double(), par[n].grad
        assert float((g - r).norm()) <= 0.03 * float(r.norm()), (n, float((g - r).norm() / r.norm()))


def test_explicit_calls_are_the_recorded_ones():
    """The same network written with the recording forms and `backward()`: head and embedding add their shares of the table as torch does."""
    torch, S = _d()
    import paper_2510_08522_b200 as D
    model, ids, target, grad = sample(torch, S, 300)
    loss = model.learn(ids, target, grad)
    par = {n: model.view(model.flat if ".ln." in n or n.startswith("ln.") else model.half, n).clone().requires_grad_(True) for n in model.names}
    x = D.embedding(ids, par["table"], model.scale).view(-1, model.C)
    for i in range(model.blocks):
        p = "%d." % i
        y = D.layer_norm(x, par[p + "ln.w"], par[p + "ln.b"])[0]
        u = D.linear(y, par[p + "up.w"], par[p + "up.b"], act="gelu")[0]
        x = D.linear(u, par[p + "down.w"], par[p + "down.b"], residual=x)[0]
    y = D.layer_norm(x, par["ln.w"], par["ln.b"])[0]
    each = D.linear_cross_entropy(y, par["table"], target.reshape(-1), par["head.b"])[0]
    (each.sum() / (target >= 0).sum()).backward()
    assert abs(float(each.sum() / (target >= 0).sum()) - float(loss)) <= 1e-5 * float(loss)
    for n in model.names:
        g, r = model.view(grad, n).double(), par[n].grad.double()
        # bit for bit but for what is rounded once more there: the residual's sum, the table's two shares (and 1 / count against a division)
        assert float((g - r).norm()) <= 0.02 * float(r.norm()), n


@pytest.mark.parametrize("bits", [32, 8])
def test_runs(bits):
    torch, S = _d()
    import paper_2510_08522_b200 as D
    a = S.run(steps=8, batch_sizes=(8, 24), bits=bits, network=S.Words)
    b = S.run(steps=8, batch_sizes=(8, 24), bits=bits, network=S.Words)
    assert a == b and all(0 < r["norm"] < float("inf") and 0 < r["loss"] < float("inf") for r in a) and D.linear_status() == 0


def test_captured_step_is_replayed():
    torch, S = _d()
    model, ids, target, grad = sample(torch, S, 500)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model.learn(ids, target, grad)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = model.learn(ids, target, grad)
    again, t2 = model.batch(24, torch.Generator(device="cuda").manual_seed(9), "cuda")
    ids.copy_(again)
    target.copy_(t2)
    graph.replay()
    torch.cuda.synchronize()
    got, got_loss = grad.clone(), float(loss)
    want = float(model.learn(ids, target, grad))
    assert got_loss == want and all(torch.equal(model.view(got, n), model.view(grad, n)) for n in model.names)      # (between tensors nothing is written)
