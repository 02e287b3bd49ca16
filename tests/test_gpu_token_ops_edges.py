"""Layer norm, embedding and cross entropy at calls that are allowed and easily forgotten: several streams and host threads at once, inputs of
another device's or stream's making, weights in any place of a flat vector, the version counters of what is written, batches of padding."""
import threading

import pytest

pytestmark = pytest.mark.gpu


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def work(torch, D, seed, sizes):
    """All six calls at several sizes -> their results"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for M, n, V in sizes:
        x = torch.randn(M, n, generator=g, device="cuda").bfloat16()
        w, b = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
        ids = torch.randint(-1, V, (M,), generator=g, device="cuda")
        table = torch.randn(V, n, generator=g, device="cuda").bfloat16()
        e = D.embedding(ids, table, 1.5)
        y, m, r = D.layer_norm(e, w, b)
        loss, lse = D.linear_cross_entropy(y, table, ids)
        dy, dw, _ = D.linear_cross_entropy_backward(torch.ones_like(loss), y, table, ids, lse, need=(True, True, False))
        dx, lw, lb = D.layer_norm_backward(dy, e, m, r, w, add=x)
        D.embedding_backward(dx, ids, V, 1.5, out=dw, accumulate=True)
        out += [e, y, m, r, loss, lse, dy, dw, dx, lw, lb, D.embedding_backward(dx, ids, V)]
    return out


SIZES = [(33, 64, 200), (700, 72, 1000), (260, 1025, 50), (5000, 40, 300), (90, 10000, 20)]


def test_streams_and_host_threads_at_once():
    torch, D = _d()
    want = [work(torch, D, i, SIZES) for i in range(3)]
    torch.cuda.synchronize()
    got, faults = {}, []

    def one(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                got[i] = [work(torch, D, i, SIZES) for _ in range(4)]
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            faults.append(e)
    threads = [threading.Thread(target=one, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults, faults
    for i in range(3):
        for again in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(again, want[i]))
    assert D.linear_status() == 0


def test_two_captured_graphs_that_are_replayed_together():
    torch, D = _d()
    work(torch, D, 0, SIZES)
    graphs, kept = [], []
    for i in range(2):
        # captured calls may allocate, but their inputs are made outside
        g = torch.Generator(device="cuda").manual_seed(i)
        x, table = torch.randn(400, 96, generator=g, device="cuda").bfloat16(), torch.randn(900, 96, generator=g, device="cuda").bfloat16()
        ids, one = torch.randint(0, 900, (400,), generator=g, device="cuda"), torch.ones(400, device="cuda")

        def calls(x=x, table=table, ids=ids, one=one):
            y, m, r = D.layer_norm(x)
            loss, lse = D.linear_cross_entropy(y, table, ids)
            dy, dw, _ = D.linear_cross_entropy_backward(one, y, table, ids, lse, need=(True, True, False))
            dx, _, _ = D.layer_norm_backward(dy, x, m, r)
            return loss, dw, dx, D.embedding_backward(dx, ids, 900)
        want = calls()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            out = calls()
        graphs.append(graph)
        kept.append((out, want, calls))                          # (with the inputs that the graph reads)
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for out, want, _ in kept:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_parameters_anywhere_in_a_flat_vector():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(4)
    for n in (40, 64, 1000, 1024, 4096, 9000):
        x, dy = torch.randn(37, n, generator=g, device="cuda").bfloat16(), torch.randn(37, n, generator=g, device="cuda").bfloat16()
        flat = torch.randn(2 * n + 9, generator=g, device="cuda")
        for start in (0, 1, 2, 3):
            w, b = flat[start:start + n], flat[start + n + 1:start + 2 * n + 1]
            y, m, r = D.layer_norm(x, w, b)
            want = D.layer_norm(x, w.clone(), b.clone())
            assert all(torch.equal(p, q) for p, q in zip((y, m, r), want))
            a, c = D.layer_norm_backward(dy, x, m, r, w), D.layer_norm_backward(dy, x, m, r, w.clone())
            assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_writes_raise_version_counters():
    torch, D = _d()
    x, ids = torch.randn(6, 16, device="cuda").bfloat16(), torch.tensor([0, 3, -1, 2, 3, 9], device="cuda")
    out, grad = torch.empty_like(x), torch.zeros(5, 16, device="cuda", dtype=torch.bfloat16)
    m = D.layer_norm(x)[1:]
    lse = D.linear_cross_entropy(x, grad, ids)[1]
    db = torch.empty(5, device="cuda", dtype=torch.bfloat16)
    for t, call in ((out, lambda: D.layer_norm(x, out=out)), (out, lambda: D.layer_norm_backward(x, x, *m, out=out)), (out, lambda: D.embedding(ids, grad, out=out)),
                    (grad, lambda: D.embedding_backward(x, ids, 5, out=grad)), (grad, lambda: D.embedding_backward(x, ids, 5, out=grad, accumulate=True)),
                    (out, lambda: D.linear_cross_entropy_backward(lse, x, grad, ids, lse, out=(out, None, None))),
                    (db, lambda: D.linear_cross_entropy_backward(lse, x, grad, ids, lse, out=(None, None, db)))):
        before = t._version
        call()
        assert t._version > before


def test_batches_of_padding():
    """Every token padded, every target ignored: zeros everywhere, no NaN on the way to a tied table."""
    torch, D = _d()
    ids = torch.full((3, 50), -1, device="cuda")
    table = torch.randn(77, 48, device="cuda").bfloat16()
    x = D.embedding(ids, table).view(-1, 48)
    y, m, r = D.layer_norm(x)
    loss, lse = D.linear_cross_entropy(y, table, ids.view(-1))
    each = torch.zeros(1, device="cuda").expand(150)
    dy, dw, db = D.linear_cross_entropy_backward(each, y, table, ids.view(-1), lse, torch.zeros(77, device="cuda", dtype=torch.bfloat16))
    dx, _, _ = D.layer_norm_backward(dy, x, m, r)
    D.embedding_backward(dx, ids.view(-1), 77, out=dw, accumulate=True)
    assert not x.any() and not y.any() and not loss.any() and lse.isfinite().all()
    assert not any(t.any() for t in (dy, dw, db, dx))


def test_other_devices_are_refused_or_served():
    torch, D = _d()
    x = torch.randn(4, 16, device="cuda").bfloat16()
    for call in (lambda: D.layer_norm(x, out=x.cpu()), lambda: D.embedding(torch.zeros(2, dtype=torch.int64), x), lambda: D.embedding_backward(x, torch.zeros(4, dtype=torch.int64), 3),
                 lambda: D.linear_cross_entropy(x, x, torch.zeros(4, dtype=torch.int64)), lambda: D.linear_cross_entropy(x, x.cpu(), torch.zeros(4, dtype=torch.int64, device="cuda"))):
        with pytest.raises(D.DmxError):
            call()
    if torch.cuda.device_count() > 1:
        y = x.to("cuda:1")
        assert torch.equal(D.layer_norm(y)[0].cpu(), D.layer_norm(x)[0].cpu())


def test_inference_tensors():
    torch, D = _d()
    with torch.inference_mode():
        x, ids = torch.randn(9, 24, device="cuda").bfloat16(), torch.arange(9, device="cuda")
        y = D.layer_norm(x, out=torch.empty_like(x))[0]
        loss, lse = D.linear_cross_entropy(D.embedding(ids, y), y, ids)
        assert loss.isfinite().all()
