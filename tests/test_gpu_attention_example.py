"""The attention, the dropout and the other training operators as they are used together: the example's gradients against autograd in 64 bits, with the
places that are dropped from the generator's definition, and that it runs."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from tests import philox
from tests.attention_oracle import bucket_of

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_attention_block", os.path.join(ROOT, "examples", "train_attention_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("p", [0.0, 0.2])
def test_gradients_against_autograd(example, p):
    """Every number within 4e-5 of its own size plus its tensor's rms: some dozens of 32-bit (2^-24) or 22-bit (2^-22) roundings in a row, the attention's
    among them, whose logits are sums of products too."""
    from paper_2210_07454_amd import sams
    n, seqs, t, vocab, dim, heads = 2, 3, 120, 97, 40, example.HEADS
    length, head_dim = t // seqs, dim // heads
    model, language = example.Model(vocab, dim), example.Language(vocab)
    model.part(model.x1, "bias").normal_()
    workers = example.Workers(model, n, t, seqs, p, seed=11)
    workers.rng[:, 1] = 5
    tokens, labels = language.batch(n, t, seqs)
    nan = lambda *shape: torch.full(shape, float("nan"), device="cuda")
    g, g_a, g_b = nan(n, model.d), nan(n, 1, 3 * dim, dim), nan(n, 1, dim, dim)
    loss = workers.gradients(model.x1, model.a1, model.b1, tokens, labels, g, g_a, g_b).clone()
    assert workers.rng[:, 1].tolist() == [6, 6]
    bucket = bucket_of(sams.relative_buckets(example.BUCKETS, 32), length).cuda()
    share = 1 - philox.least(p) / 65536
    hidden = torch.from_numpy(philox.keep_columns((12, 5), n, t, dim, p)).cuda().double() / share
    for i in range(n):
        x = model.x1.double().requires_grad_()
        a, b = model.a1[0].double().requires_grad_(), model.b1[0].double().requires_grad_()
        h0 = model.part(x, "embed")[tokens[i]]
        y = torch.nn.functional.layer_norm(h0, (dim,), model.part(x, "weight"), model.part(x, "shift"), 1e-5)
        q, k, v = (z.reshape(seqs, length, heads, head_dim).transpose(1, 2) for z in (y @ a.t()).split(dim, dim=1))
        logits = q @ k.transpose(2, 3) / head_dim ** 0.5 + model.part(x, "bias")[:, bucket]
        weights = torch.softmax(logits.masked_fill(~torch.ones(length, length, dtype=torch.bool, device="cuda").tril(), -torch.inf), -1)
        rows = (i * seqs + np.arange(seqs))[:, None] * heads + np.arange(heads)
        keep = torch.from_numpy(philox.keep_pairs((11, 5), rows.reshape(-1), length, p)).cuda().reshape(seqs, heads, length, length)
        o = ((weights * keep / share) @ v).transpose(1, 2).reshape(t, dim)
        h = h0 + hidden[i] * (o @ b.t())
        want = torch.nn.functional.cross_entropy(h @ model.part(x, "head").t(), labels[i])
        want.backward()
        assert abs(float(loss[i]) - want.item()) <= 2e-5 * want.item()
        for name, got, ref in [(key, model.part(g[i], key), model.part(x.grad, key)) for key in model.at] + [("a", g_a[i, 0], a.grad), ("b", g_b[i, 0], b.grad)]:
            rms = ref.pow(2).mean().sqrt()
            assert ((got.double() - ref).abs() <= 4e-5 * (ref.abs() + rms)).all(), (name, float(((got.double() - ref).abs() / (ref.abs() + rms)).max()))


def test_the_example_runs(example):
    losses = example.train(steps=6, n=2, t=64, vocab=50, dim=32)
    assert len(losses) == 6 and all(np.isfinite(losses))
