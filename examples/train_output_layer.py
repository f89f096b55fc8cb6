"""Trains a small language model whose workers' gradients the library makes and applies: python examples/train_output_layer.py

n workers, batched buffers on one GPU, each with its own batch of a synthetic language (a Markov chain).  The model is an embedding E,
one layer, an output layer W:

    h0 = E[token],   y = layer norm(h0),   h = h0 + y P',   loss = cross entropy of h W'

Every step, layer_norm_forward / linear_xent_forward / linear_xent_backward / layer_norm_backward give each worker's gradients of the norm's
weights and of W straight into that worker's row of g [n][d]; the embedding's rows and the layer's own product are plain torch.  Then
the flat vector (E, norm, W) takes one sketched-AMSGrad iteration, and the matrix P the orthogonalised momentum update.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2210_07454_amd import inputs, sams


class Model:
    def __init__(self, vocab, dim, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.dim = vocab, dim
        # the flat vector's parts, each from a multiple of 4 on
        sizes = {"embed": vocab * dim, "weight": dim, "bias": dim, "head": vocab * dim}
        self.at, d = {}, 0
        for name, size in sizes.items():
            self.at[name] = (d, d + size)
            d += (size + 3) // 4 * 4
        self.d = d
        x = torch.zeros(d, device="cuda")
        for name in ("embed", "head"):
            lo, hi = self.at[name]
            x[lo:hi] = 0.5 * torch.randn(hi - lo, generator=gen, device="cuda") / (dim ** 0.5 if name == "head" else 1)
        x[self.at["weight"][0]:self.at["weight"][1]] = 1
        self.x1 = x
        self.p1 = torch.randn((1, dim, dim), generator=gen, device="cuda") / dim ** 0.5

    def part(self, flat, name):
        """A part of x [d], or of every worker's row of g [n][d], as it lies."""
        lo, hi = self.at[name]
        v = flat[..., lo:hi]
        return v.unflatten(-1, (-1, self.dim)) if name in ("embed", "head") else v


class Workers:
    """Makes the n workers' losses and gradients at the parameters x and P."""

    def __init__(self, model, n, t):
        self.model, self.n, self.t = model, n, t
        full, vocab, dim = (n, t, model.dim), model.vocab, model.dim
        self.norm = sams.LayerNorm(n, t, dim)
        self.xent = sams.LinearCrossEntropy(n, t, dim, vocab)
        self.y, self.dh, self.dx = (torch.empty(full, device="cuda") for _ in range(3))
        self.mean, self.rstd, self.lse = torch.empty((3, n, t), device="cuda")
        self.loss = torch.empty((n,), device="cuda")

    def gradients(self, x, p, tokens, labels, g, g_p):
        m = self.model
        h0 = m.part(x, "embed")[tokens]
        weight, bias, head = m.part(x, "weight"), m.part(x, "bias"), m.part(x, "head")
        self.norm.layer_norm_forward(h0, weight, bias, self.y, self.mean, self.rstd)
        h = h0 + self.y @ p[0].t()
        self.xent.linear_xent_forward(h, head, labels, self.loss, self.lse)
        self.xent.linear_xent_backward(h, head, labels, self.lse, None, self.dh, m.part(g, "head"))
        for i in range(self.n):
            torch.mm(self.dh[i].t(), self.y[i], out=g_p[i, 0])
        self.norm.layer_norm_backward(self.dh @ p[0], h0, weight, self.mean, self.rstd, self.dx, m.part(g, "weight"), m.part(g, "bias"))
        into = m.part(g, "embed")
        for i in range(self.n):
            into[i].zero_().index_add_(0, tokens[i], self.dh[i] + self.dx[i])
        return self.loss


class Language:
    """A Markov chain: from every word the next is one of four, with falling odds."""

    def __init__(self, vocab, seed=1):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.next = torch.randint(0, vocab, (vocab, 4), generator=self.gen, device="cuda")
        self.vocab = vocab

    def batch(self, n, t):
        word = torch.randint(0, self.vocab, (n,), generator=self.gen, device="cuda")
        words = [word]
        odds = torch.tensor([0.6, 0.2, 0.1, 0.1], device="cuda")
        for _ in range(t):
            pick = torch.multinomial(odds, n, replacement=True, generator=self.gen)
            words.append(self.next[words[-1], pick])
        words = torch.stack(words, 1)
        labels = words[:, 1:].contiguous()
        labels[:, -1] = -100                                # the last position is only looked at
        return words[:, :-1].contiguous(), labels


def train(steps=60, n=4, t=256, vocab=1000, dim=64, lr=2e-2, lr_matrix=0.02, report=None):
    """Mean loss over the workers at every step."""
    model, language = Model(vocab, dim), Language(vocab)
    workers = Workers(model, n, t)
    d, k, c, r = model.d, model.d // 8, 1 << 15, 5
    ctx = sams.Context(d, n, r, c, k, inputs.hash_params(r, seed=3))
    ortho = sams.Orthogonalizer(1, dim, dim)
    b = sams.Buffers(d, n, r, c, k, 1e-4, model.x1)
    p, momentum = model.p1.clone(), torch.zeros_like(model.p1)
    g, g_p = torch.zeros((n, d), device="cuda"), torch.empty((n, 1, dim, dim), device="cuda")
    losses = []
    for step in range(steps):
        tokens, labels = language.batch(n, t)
        losses.append(workers.gradients(b.x, p, tokens, labels, g, g_p).mean())
        # the head of the iteration takes g, its tail updates x; both before the next gradients
        sams.run_step(ctx, b, 0.9, 0.99, lr, first=True, g_first=g)
        ortho.muon_update(g_p, momentum, p, momentum, p, beta=0.9, lr=lr_matrix)
        if report and step % 10 == 0:
            report(f"step {step:4d}   loss {float(losses[-1]):.4f}")
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 60), ("workers", 4), ("tokens", 256), ("vocab", 1000), ("dim", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    losses = train(a.steps, a.workers, a.tokens, a.vocab, a.dim, report=lambda s: print(s, flush=True))
    print(f"last    loss {losses[-1]:.4f}   (a uniform guess: {torch.tensor(float(a.vocab)).log():.4f})")


if __name__ == "__main__":
    main()
