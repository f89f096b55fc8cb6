"""Cross entropy of 32-bit tensors so small that every logit is as good as 0: the loss is the vocabulary's logarithm, and the gradients follow
the tensors down.  Bounds as in the tests of ordinary sizes."""
import math

import pytest
import torch

from tests.test_gpu_linear_xent import check, formulas, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


@pytest.mark.parametrize("vocab", [400, 1, 512, 5000])
@pytest.mark.parametrize("a,b", [(1e-30, 1e-30), (2.0 ** -100, 2.0 ** -110), (1e-36, 1e-3), (0.0, 1e-30), (1e-30, 0.0)])
def test_tensors_that_are_both_small(sams, a, b, vocab):
    n, t, dim = 2, 30, 96
    h, w, labels = make(n, t, dim, vocab, torch.float32)
    h, w = h * a, w * b
    want, tol = formulas(h, w, labels)
    loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
    dh, dw = torch.empty_like(h, device="cuda"), torch.empty((n, vocab, dim), device="cuda")
    with sams.LinearCrossEntropy(n, t, dim, vocab) as op:
        op.linear_xent_forward(h.cuda(), w.cuda(), labels.cuda(), loss, lse)
        op.linear_xent_backward(h.cuda(), w.cuda(), labels.cuda(), lse, None, dh, dw)
    assert torch.allclose(loss.cpu(), torch.full((n,), math.log(vocab)), rtol=1e-6, atol=1e-20)
    for name, got in (("lse", lse), ("loss", loss), ("dh", dh), ("dw", dw)):
        # numbers below 2^-126 have no more than 2^-149 to be right to
        check(got, want[name], tol[name] + 2.0 ** -148 + (2.0 ** -70 if name == "lse" else 0), (name, a, b))
