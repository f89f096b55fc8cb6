"""Trains a small language model with an attention block on the library's operators: python examples/train_attention_block.py

n workers, batched buffers on one GPU.  A word of the synthetic language depends on the one two places before it, so that what mixes tokens has to
find it by relative position.  The model is an embedding E, one block, an output layer W:

    h0 = E[token],   q, k, v = layer norm(h0) A',   a = attention(q, k, v, bias by relative position),   h = h0 + dropout(a B'),   loss = cross entropy of h W'

Every step the operators make each worker's gradients of the norm's weights, of the bias and of W straight into its row of g [n][d]; the embedding's
rows and the products with A and B are plain torch.  Then the flat vector (E, norm, bias, W) takes one sketched-AMSGrad iteration, and the matrices
A and B the orthogonalised momentum update.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2210_07454_amd import inputs, sams

HEADS = 4
BUCKETS = 8


class Model:
    def __init__(self, vocab, dim, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
        self.vocab, self.dim = vocab, dim
        self.shapes = {"embed": (vocab, dim), "weight": (dim,), "shift": (dim,), "bias": (HEADS, BUCKETS), "head": (vocab, dim)}
        # the flat vector's parts, each from a multiple of 4 on
        self.at, d = {}, 0
        for name, shape in self.shapes.items():
            size = torch.Size(shape).numel()
            self.at[name] = (d, d + size)
            d += (size + 3) // 4 * 4
        self.d = d
        x = torch.zeros(d, device="cuda")
        for name in ("embed", "head"):
            self.part(x, name).copy_(0.5 * rand(vocab, dim) / (dim ** 0.5 if name == "head" else 1))
        self.part(x, "weight").fill_(1)
        self.x1, self.a1, self.b1 = x, rand(1, 3 * dim, dim) / dim ** 0.5, rand(1, dim, dim) / dim ** 0.5

    def part(self, flat, name):
        """A part of x [d], or of every worker's row of g [n][d], as it lies."""
        lo, hi = self.at[name]
        return flat[..., lo:hi].unflatten(-1, self.shapes[name]) if len(self.shapes[name]) > 1 else flat[..., lo:hi]


class Workers:
    """Makes the n workers' losses and gradients at the parameters x, A and B; each worker has `seqs` sequences of equal length."""

    def __init__(self, model, n, t, seqs=1, p=0.1, seed=7):
        self.model, self.n, self.t, self.seqs, self.p = model, n, t, seqs, p
        dim = model.dim
        new = lambda *shape: torch.empty(shape, device="cuda")
        self.norm, self.xent, self.drop = sams.LayerNorm(n, t, dim), sams.LinearCrossEntropy(n, t, dim, model.vocab), sams.Dropout(n, t, dim)
        self.attn = sams.Attention(n, t, HEADS, dim // HEADS, starts=sams.relative_buckets(BUCKETS, 32))
        self.y, self.o, self.h, self.dh, self.dc, self.dx = (new(n, t, dim) for _ in range(6))
        self.dqkv = new(n, t, 3 * dim)
        self.mean, self.rstd, self.lse = new(3, n, t)
        self.row_max, self.row_sum = new(2, n, HEADS, t)
        self.loss = new(n)
        # seed and step of the attention's and of the hidden states' dropout
        self.rng = torch.tensor([[seed, 0], [seed + 1, 0]], device="cuda")

    def gradients(self, x, a, b, tokens, labels, g, g_a, g_b):
        m, n, dim = self.model, self.n, self.model.dim
        weight, shift, bias, head = (m.part(x, name) for name in ("weight", "shift", "bias", "head"))
        how = dict(seqs=self.seqs, rng=self.rng[0], p=self.p)
        h0 = m.part(x, "embed")[tokens]
        self.norm.layer_norm_forward(h0, weight, shift, self.y, self.mean, self.rstd)
        q, k, v = (self.y @ a[0].t()).split(dim, dim=2)
        self.attn.attention_forward(q, k, v, bias, self.o, self.row_max, self.row_sum, **how)
        self.drop.dropout_forward(self.o @ b[0].t(), h0, self.rng[1], self.p, self.h)
        self.xent.linear_xent_forward(self.h, head, labels, self.loss, self.lse)

        self.xent.linear_xent_backward(self.h, head, labels, self.lse, None, self.dh, m.part(g, "head"))
        self.drop.dropout_backward(self.dh, self.rng[1], self.p, self.dc)
        dq, dk, dv = self.dqkv.split(dim, dim=2)
        self.attn.attention_backward(self.dc @ b[0], q, k, v, bias, self.o, self.row_max, self.row_sum, dq, dk, dv, m.part(g, "bias"), **how)
        for i in range(n):
            torch.mm(self.dc[i].t(), self.o[i], out=g_b[i, 0])
            torch.mm(self.dqkv[i].t(), self.y[i], out=g_a[i, 0])
        self.norm.layer_norm_backward(self.dqkv @ a[0], h0, weight, self.mean, self.rstd, self.dx, m.part(g, "weight"), m.part(g, "shift"))
        into = m.part(g, "embed")
        for i in range(n):
            into[i].zero_().index_add_(0, tokens[i], self.dh[i] + self.dx[i])
        self.rng[:, 1] += 1
        return self.loss


class Language:
    """From every word the one two places on is one of two, the likelier nine times in ten."""

    def __init__(self, vocab, seed=1):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.next = torch.randint(0, vocab, (vocab, 2), generator=self.gen, device="cuda")
        self.vocab = vocab

    def batch(self, n, t, seqs=1):
        words = [torch.randint(0, self.vocab, (n * seqs,), generator=self.gen, device="cuda") for _ in range(2)]
        for _ in range(t // seqs - 1):
            other = torch.rand((n * seqs,), generator=self.gen, device="cuda") < 0.1
            words.append(self.next[words[-2], other.long()])
        words = torch.stack(words, 1)
        return words[:, :-1].reshape(n, t), words[:, 1:].reshape(n, t).contiguous()


def train(steps=60, n=4, t=256, seqs=2, vocab=200, dim=64, lr=2e-2, lr_matrix=0.02, p=0.1, report=None):
    """Mean loss over the workers at every step."""
    model, language = Model(vocab, dim), Language(vocab)
    workers = Workers(model, n, t, seqs, p)
    d, k, c, r = model.d, model.d // 8, 1 << 13, 5
    ctx = sams.Context(d, n, r, c, k, inputs.hash_params(r, seed=3))
    buffers = sams.Buffers(d, n, r, c, k, 1e-4, model.x1)
    matrices = [(sams.Orthogonalizer(1, *m.shape[1:]), m.clone(), torch.zeros_like(m), torch.empty((n, *m.shape), device="cuda")) for m in (model.a1, model.b1)]
    g = torch.zeros((n, d), device="cuda")
    losses = []
    for step in range(steps):
        tokens, labels = language.batch(n, t, seqs)
        losses.append(workers.gradients(buffers.x, matrices[0][1], matrices[1][1], tokens, labels, g, matrices[0][3], matrices[1][3]).mean())
        # the head of the iteration takes g, its tail updates x; both before the next gradients
        sams.run_step(ctx, buffers, 0.9, 0.99, lr, first=True, g_first=g)
        for ortho, m, momentum, g_m in matrices:
            ortho.muon_update(g_m, momentum, m, momentum, m, beta=0.9, lr=lr_matrix)
        if report and step % 10 == 0:
            report(f"step {step:4d}   loss {float(losses[-1]):.4f}")
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 60), ("workers", 4), ("tokens", 256), ("sequences", 2), ("vocab", 200), ("dim", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    losses = train(a.steps, a.workers, a.tokens, a.sequences, a.vocab, a.dim, report=lambda s: print(s, flush=True))
    print(f"last    loss {losses[-1]:.4f}   (a uniform guess: {torch.tensor(float(a.vocab)).log():.4f})")


if __name__ == "__main__":
    main()
