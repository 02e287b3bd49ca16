"""A small training loop with every step of it in the CUDA library: K emulated workers, each with its own batch size,
run a network forward and backward on one GPU; their flat gradients are aggregated with the statistics a batch-size
controller reads; AdamW updates the model.

The network is a channels-last mixer on 32 x 32 images (Section "Workloads and Datasets" trains on CIFAR; the data
here are synthetic, ten classes told apart by a pattern in noise): patches of 4 x 4 become 64 positions of C channels
(`linear`), then blocks of `group_norm` with SiLU, a widening `linear` with GELU and a narrowing `linear` that adds
the block's input as its residual; at the end `group_norm`, the mean over positions and a `linear` classifier.
Group norm, not batch norm: a worker's result must not depend on the batch size it was given.

The second network (`--model words`) is one of the other kind that the gradient step's workloads are sized like, over words instead of
images: `embedding`, blocks of `layer_norm`, a widening `linear` with GELU and a narrowing one with the residual, `layer_norm`, and the
`linear_cross_entropy` of a head that shares the embedding's table. Its data are sequences in which a word mostly decides the next.

    python -m paper_2510_08522_b200.train_small --steps 40 --bits 8 --model words
"""
from __future__ import annotations

import argparse

CLASSES, PATCH, SIDE = 10, 4, 32
POSITIONS, PATCH_CHANNELS = (SIDE // PATCH) ** 2, 3 * PATCH * PATCH


class _Flat:
    """Parameters as views of one flat fp32 vector and of its bf16 copy, each tensor at a multiple of 8 elements."""

    def _lay_out(self, shapes, device):
        import torch
        self.torch, self.names, self.shapes, self.offsets, at = torch, [n for n, _ in shapes], dict(shapes), {}, 0
        for n, s in shapes:
            self.offsets[n] = at
            at += -(-int(torch.Size(s).numel()) // 8) * 8        # 16 bytes of bf16
        self.P = at
        self.flat = torch.zeros(at, device=device)

    def view(self, flat, name):
        shape = self.shapes[name]
        n = int(self.torch.Size(shape).numel())
        return flat[self.offsets[name]: self.offsets[name] + n].view(shape)

    def segments(self):
        """Segment table of the flat vector, one segment per tensor (with its padding)."""
        return [self.offsets[n] for n in self.names] + [self.P]


class Mixer(_Flat):
    """The network on images; forward and backward by the library's
    operators. Weights and biases of `linear` are used in bf16, those of `group_norm` in fp32."""

    def __init__(self, channels=64, hidden=128, blocks=2, groups=8, seed=0, device="cuda"):
        import torch
        self.C, self.H, self.blocks, self.groups = channels, hidden, blocks, groups
        shapes = [("embed.w", (channels, PATCH_CHANNELS)), ("embed.b", (channels,))]
        for i in range(blocks):
            shapes += [("%d.gn.w" % i, (channels,)), ("%d.gn.b" % i, (channels,)), ("%d.up.w" % i, (hidden, channels)), ("%d.up.b" % i, (hidden,)),
                       ("%d.down.w" % i, (channels, hidden)), ("%d.down.b" % i, (channels,))]
        shapes += [("gn.w", (channels,)), ("gn.b", (channels,)), ("head.w", (CLASSES, channels)), ("head.b", (CLASSES,))]
        self._lay_out(shapes, device)
        g = torch.Generator(device=device).manual_seed(seed)
        for n, s in shapes:
            v = self.view(self.flat, n)
            if n.endswith("gn.w"):
                v.fill_(1.0)
            elif n.endswith(".w"):
                v.copy_(torch.randn(s, generator=g, device=device) * s[1] ** -0.5)
        self.half = self.flat.to(torch.bfloat16)

    def batch(self, n, generator, device):
        return batch(n, generator, device)

    def learn(self, images, label, grad):
        """The gradient of one batch to `grad`; -> its loss"""
        logits, saved = self.forward(images)
        loss, slope = loss_and_slope(logits, label)
        self.backward(slope, saved, grad)
        return loss

    def forward(self, images):
        """images: bf16 (n, 64, 48). -> (logits bf16 (n, 10), what backward needs)"""
        from . import train_ops as T
        h = lambda n: self.view(self.half, n)  # noqa: E731
        f = lambda n: self.view(self.flat, n)  # noqa: E731
        n, kept = images.shape[0], []
        x0 = images.reshape(-1, PATCH_CHANNELS)
        x, _ = T.linear(x0, h("embed.w"), h("embed.b"))
        for i in range(self.blocks):
            p = "%d." % i
            y, mean, rstd = T.group_norm(x.view(n, POSITIONS, self.C), self.groups, f(p + "gn.w"), f(p + "gn.b"), act="silu")
            y = y.view(-1, self.C)
            u, z = T.linear(y, h(p + "up.w"), h(p + "up.b"), act="gelu", save=True)
            x_next, _ = T.linear(u, h(p + "down.w"), h(p + "down.b"), residual=x)
            kept.append((x, y, mean, rstd, u, z))
            x = x_next
        y, mean, rstd = T.group_norm(x.view(n, POSITIONS, self.C), self.groups, f("gn.w"), f("gn.b"), act="silu")
        pooled = y.float().mean(1).to(self.torch.bfloat16)
        logits, _ = T.linear(pooled, h("head.w"), h("head.b"))
        return logits, (x0, kept, x, mean, rstd, pooled)

    def backward(self, dlogits, saved, grad):
        """Writes the gradient of every parameter to the flat bf16 vector `grad`."""
        from . import train_ops as T
        torch = self.torch
        h = lambda n: self.view(self.half, n)  # noqa: E731
        f = lambda n: self.view(self.flat, n)  # noqa: E731
        to = lambda n: self.view(grad, n)  # noqa: E731
        x0, kept, x, mean, rstd, pooled = saved
        n = dlogits.shape[0]
        dp, _, _ = T.linear_backward(dlogits, pooled, h("head.w"), out=(None, to("head.w"), to("head.b")))
        dy = (dp.float() / POSITIONS).to(torch.bfloat16)[:, None, :].expand(n, POSITIONS, self.C)
        dx, dw, db = T.group_norm_backward(dy, x.view(n, POSITIONS, self.C), mean, rstd, self.groups, f("gn.w"), f("gn.b"), act="silu")
        to("gn.w").copy_(dw)
        to("gn.b").copy_(db)
        dx = dx.view(-1, self.C)
        for i in reversed(range(self.blocks)):
            p = "%d." % i
            x, y, mean, rstd, u, z = kept[i]
            du, _, _ = T.linear_backward(dx, u, h(p + "down.w"), out=(None, to(p + "down.w"), to(p + "down.b")))
            dy, _, _ = T.linear_backward(du, y, h(p + "up.w"), z, act="gelu", out=(None, to(p + "up.w"), to(p + "up.b")))
            dn, dw, db = T.group_norm_backward(dy.view(n, POSITIONS, self.C), x.view(n, POSITIONS, self.C), mean, rstd, self.groups, f(p + "gn.w"),
                                               f(p + "gn.b"), act="silu")
            to(p + "gn.w").copy_(dw)
            to(p + "gn.b").copy_(db)
            dx = dx + dn.view(-1, self.C)                  # the residual's share
        T.linear_backward(dx, x0, h("embed.w"), need=(False, True, True), out=(None, to("embed.w"), to("embed.b")))


class Words(_Flat):
    """The network over words: the next word from this one, embedding and head by one table. Weights are used in bf16, those of `layer_norm` in
    fp32."""

    def __init__(self, words=1000, length=65, channels=64, hidden=128, blocks=2, seed=0, device="cuda"):
        import torch
        self.V, self.L, self.C, self.H, self.blocks, self.scale = words, length, channels, hidden, blocks, float(channels) ** 0.5
        shapes = [("table", (words, channels)), ("head.b", (words,))]
        for i in range(blocks):
            shapes += [("%d.ln.w" % i, (channels,)), ("%d.ln.b" % i, (channels,)), ("%d.up.w" % i, (hidden, channels)), ("%d.up.b" % i, (hidden,)),
                       ("%d.down.w" % i, (channels, hidden)), ("%d.down.b" % i, (channels,))]
        self._lay_out(shapes + [("ln.w", (channels,)), ("ln.b", (channels,))], device)
        g = torch.Generator(device=device).manual_seed(seed)
        for n in self.names:
            v = self.view(self.flat, n)
            if n.endswith("ln.w"):
                v.fill_(1.0)
            elif not n.endswith(".b"):
                v.copy_(torch.randn(v.shape, generator=g, device=device) * v.shape[1] ** -0.5)
        self.half = self.flat.to(torch.bfloat16)

    def batch(self, n, generator, device):
        """n sequences and, behind each word, the one to come (-1 where a sequence is padded): mostly 7 w + 3, else any word."""
        import torch
        w = torch.randint(0, self.V, (n, self.L), generator=generator, device=device)
        known = torch.rand(n, self.L, generator=generator, device=device) < 0.9
        for i in range(1, self.L):
            w[:, i] = torch.where(known[:, i], (7 * w[:, i - 1] + 3) % self.V, w[:, i])
        length = torch.randint(self.L // 2, self.L, (n, 1), generator=generator, device=device)
        at = torch.arange(self.L - 1, device=device)
        pad = at >= length
        return torch.where(pad, -1, w[:, :-1]), torch.where(pad, -1, w[:, 1:])

    def learn(self, ids, target, grad):
        """The gradient of the mean loss over the words that count to every parameter's place in the flat bf16 vector `grad`; -> the loss"""
        from . import train_ops as T
        torch = self.torch
        h = lambda n: self.view(self.half, n)  # noqa: E731
        f = lambda n: self.view(self.flat, n)  # noqa: E731
        to = lambda n: self.view(grad, n)  # noqa: E731
        x, target, kept = T.embedding(ids, h("table"), self.scale).view(-1, self.C), target.reshape(-1), []
        for i in range(self.blocks):
            p = "%d." % i
            y, mean, rstd = T.layer_norm(x, f(p + "ln.w"), f(p + "ln.b"))
            u, z = T.linear(y, h(p + "up.w"), h(p + "up.b"), act="gelu", save=True)
            x_next, _ = T.linear(u, h(p + "down.w"), h(p + "down.b"), residual=x)
            kept.append((x, y, mean, rstd, u, z))
            x = x_next
        y, mean, rstd = T.layer_norm(x, f("ln.w"), f("ln.b"))
        loss, lse = T.linear_cross_entropy(y, h("table"), target, h("head.b"))
        each = 1.0 / ((target >= 0) & (target < self.V)).sum().clamp_min(1).float()
        dy, _, _ = T.linear_cross_entropy_backward(each.expand(len(target)), y, h("table"), target, lse, h("head.b"), out=(None, to("table"), to("head.b")))
        dx, dw, db = T.layer_norm_backward(dy, x, mean, rstd, f("ln.w"))
        to("ln.w").copy_(dw)
        to("ln.b").copy_(db)
        for i in reversed(range(self.blocks)):
            p = "%d." % i
            x, y, mean, rstd, u, z = kept[i]
            du, _, _ = T.linear_backward(dx, u, h(p + "down.w"), out=(None, to(p + "down.w"), to(p + "down.b")))
            dy, _, _ = T.linear_backward(du, y, h(p + "up.w"), z, act="gelu", out=(None, to(p + "up.w"), to(p + "up.b")))
            dx, dw, db = T.layer_norm_backward(dy, x, mean, rstd, f(p + "ln.w"), add=dx)      # the residual's share is added
            to(p + "ln.w").copy_(dw)
            to(p + "ln.b").copy_(db)
        T.embedding_backward(dx.view(*ids.shape, self.C), ids, self.V, self.scale, out=to("table"), accumulate=True)      # beside the head's
        return loss.sum() * each


def batch(n, generator, device="cuda"):
    """n synthetic images as patches (bf16) and their classes: a class's pattern (by fixed frequencies) in noise."""
    import torch
    label = torch.randint(0, CLASSES, (n,), generator=generator, device=device)
    pos = torch.arange(POSITIONS, device=device, dtype=torch.float32)[None, :, None]
    ch = torch.arange(PATCH_CHANNELS, device=device, dtype=torch.float32)[None, None, :]
    k = (label + 1).float()[:, None, None]
    pattern = torch.cos(0.37 * k * pos / 8 + 0.11 * k * ch)
    noise = torch.randn(n, POSITIONS, PATCH_CHANNELS, generator=generator, device=device)
    return (0.7 * pattern + noise).to(torch.bfloat16), label


def loss_and_slope(logits, label):
    """Mean cross entropy and its gradient in the logits (bf16)."""
    import torch
    p = torch.softmax(logits.float(), 1)
    loss = -torch.log(p.gather(1, label[:, None])).mean()
    p.scatter_add_(1, label[:, None], torch.full((len(label), 1), -1.0, device=p.device))
    return loss, (p / len(label)).to(torch.bfloat16)


def run(steps=40, batch_sizes=(32, 64, 96, 128), bits=32, lr=3e-3, max_norm=1.0, seed=0, device="cuda:0", verbose=False, network=Mixer):
    """Returns one record per step: loss (batch-weighted mean over the workers), gradient noise scale, cosine to the
    previous aggregate, gradient norm."""
    import torch
    from . import binding as B
    from . import train_ops as T
    torch.cuda.set_device(torch.device(device))
    model = network(seed=seed, device=device)
    K, P = len(batch_sizes), model.P
    grads = [torch.zeros(P, dtype=torch.bfloat16, device=device) for _ in range(K)]
    step = B.Dmx(K, P, model.segments(), B.BF16)
    # with lr = 0 and beta = 0 the step aggregates and measures and leaves the parameters to AdamW
    momentum, agg = torch.zeros(P, device=device), torch.zeros(P, device=device)
    state = torch.empty(step.state_len, device=device)
    views = lambda flat: [model.view(flat, n) for n in model.names]  # noqa: E731
    opt = T.AdamW(views(model.flat), views(agg), state_bits=bits, copies=views(model.half), decay=[len(model.shapes[n]) > 1 for n in model.names])
    moments, norm = opt.new_state(), torch.empty(2, device=device)
    gen = torch.Generator(device=device).manual_seed(seed + 1)
    records = []
    for t in range(1, steps + 1):
        losses = []
        for k, b in enumerate(batch_sizes):
            images, label = model.batch(b, gen, device)
            loss = model.learn(images, label, grads[k])
            losses.append(loss * b)
        step.step(grads, batch_sizes, model.flat, momentum, 0.0, 0.0, agg, state)
        opt.grad_norm(max_norm, out=norm)
        opt.step(*moments, lr=lr, t=t, weight_decay=0.01, grad_scale=norm[1:], seed=t if bits == 8 else None)
        st = state.cpu()
        records.append(dict(loss=float(sum(losses)) / sum(batch_sizes), gns=float(st[B.ST_GNS]), cos=float(st[B.ST_COS_PREV]), norm=float(norm[0])))
        if verbose and (t == 1 or t % 10 == 0):
            print("step %3d: loss %.4f  noise scale %.1f  cosine %.3f  |g| %.3f" % (t, records[-1]["loss"], records[-1]["gns"], records[-1]["cos"], records[-1]["norm"]))
    step.close()
    opt.close()
    return records


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--lr", type=float, default=3e-3)
    ap.add_argument("--model", default="mixer", choices=("mixer", "words"))
    a = ap.parse_args()
    run(a.steps, bits=a.bits, lr=a.lr, verbose=True, network=Words if a.model == "words" else Mixer)


if __name__ == "__main__":
    main()
