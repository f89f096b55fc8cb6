"""The training operators as they are used together: the example's gradients against autograd in 64 bits, its loss over some steps, and
the operators inside a HIP graph."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_output_layer", os.path.join(ROOT, "examples", "train_output_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients_against_autograd(example):
    """Every number of g within 2e-5 of its own size plus its tensor's rms: some dozens of 32-bit (2^-24) or 22-bit (2^-22) roundings in a row."""
    n, t, vocab, dim = 3, 70, 301, 40
    model, language = example.Model(vocab, dim), example.Language(vocab)
    workers = example.Workers(model, n, t)
    tokens, labels = language.batch(n, t)
    g, g_p = torch.full((n, model.d), float("nan"), device="cuda"), torch.empty((n, 1, dim, dim), device="cuda")
    loss = workers.gradients(model.x1, model.p1, tokens, labels, g, g_p).clone()
    for i in range(n):
        x = model.x1.double().requires_grad_()
        p = model.p1[0].double().requires_grad_()
        h0 = model.part(x, "embed")[tokens[i]]
        y = torch.nn.functional.layer_norm(h0, (dim,), model.part(x, "weight"), model.part(x, "bias"), 1e-5)
        z = (h0 + y @ p.t()) @ model.part(x, "head").t()
        want = torch.nn.functional.cross_entropy(z, labels[i])
        want.backward()
        assert abs(float(loss[i]) - want.item()) <= 1e-5 * want.item()
        for name, got, ref in [(k, model.part(g[i], k), model.part(x.grad, k)) for k in model.at] + [("p", g_p[i, 0], p.grad)]:
            rms = ref.pow(2).mean().sqrt()
            assert ((got.double() - ref).abs() <= 2e-5 * (ref.abs() + rms)).all(), name


def test_the_example_learns(example):
    losses = example.train(steps=60)
    assert losses[0] > 6.5 and losses[-1] < 0.6 * losses[0], losses[::10]


def test_inside_a_graph(example):
    """Captured once, replayed with other inputs in the same tensors, eager work in between; each replay equals the eager calls."""
    from paper_2210_07454_amd import sams
    n, t, dim, vocab = 2, 50, 96, 700
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        norm, xent = sams.LayerNorm(n, t, dim), sams.LinearCrossEntropy(n, t, dim, vocab)
        small, large = sams.Orthogonalizer(1, dim, dim), sams.Orthogonalizer(1, 300, 520, torch.bfloat16)
        x, weight, bias, w = rand(n, t, dim), 1 + 0.1 * rand(dim), 0.1 * rand(dim), 0.2 * rand(vocab, dim)
        labels = torch.randint(0, vocab, (n, t), generator=gen, device="cuda")
        gm, m, p, big = rand(n, 1, dim, dim), rand(1, dim, dim), rand(1, dim, dim), rand(1, 300, 520).bfloat16()
        y, dh, dx = (torch.empty_like(x) for _ in range(3))
        mean, rstd, lse = torch.empty((3, n, t), device="cuda")
        dweight, dbias = torch.empty((2, n, dim), device="cuda")
        loss, dw = torch.empty((n,), device="cuda"), torch.empty((n, vocab, dim), device="cuda")
        m_out, p_out, out = torch.empty_like(m), torch.empty_like(p), torch.empty_like(big)

        def calls():
            norm.layer_norm_forward(x, weight, bias, y, mean, rstd)
            xent.linear_xent_forward(y, w, labels, loss, lse)
            xent.linear_xent_backward(y, w, labels, lse, None, dh, dw)
            norm.layer_norm_backward(dh, x, weight, mean, rstd, dx, dweight, dbias)
            small.muon_update(gm, m, p, m_out, p_out)
            large.orthogonalize(big, out)

        results = (y, loss, lse, dh, dw, dx, dweight, dbias, m_out, p_out, out)
        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls()
        for _ in range(4):
            for v in (x, w, gm, big):
                v.copy_(rand(*v.shape))
            labels.random_(0, vocab, generator=gen)
            graph.replay()
            torch.cuda.synchronize()
            got = [v.clone() for v in results]
            for v in results:
                v.zero_()
            calls()
            torch.cuda.synchronize()
            for a, b in zip(got, results):
                assert torch.equal(a, b)
