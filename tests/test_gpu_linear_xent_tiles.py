"""Cross entropy and its gradients in every tile that their products have, in the three types, gradients written and added up, against 64 bits
on the GPU.  Bounds as for the smaller ones."""
import pytest
import torch

from tests import tiles
from tests.test_gpu_linear_xent import HALF_ULP, TINY, formulas, make
from tests.tiles import LARGE, MIDDLE, SMALL, WIDE

TYPES = [torch.float32, torch.bfloat16, torch.float16]

# n, t, dim, vocab; the tiles of the logits, dW and dh in pairs of words and in single ones; sizes that end inside a tile, but for the last, whose tensors are multiplied as they lie
SHAPES = [(2, 2500, 771, 3001, (LARGE, SMALL, LARGE), (LARGE, MIDDLE, LARGE)), (8, 700, 129, 4003, (WIDE, SMALL, WIDE), (LARGE, WIDE, WIDE)),
          (1, 1000, 1027, 2203, (MIDDLE, MIDDLE, MIDDLE), (SMALL, SMALL, MIDDLE)), (3, 130, 259, 9001, (SMALL, LARGE, SMALL), (WIDE, LARGE, SMALL)),
          (8, 130, 129, 3001, (MIDDLE, WIDE, SMALL), (MIDDLE, WIDE, SMALL)), (4, 1000, 768, 4096, (LARGE, MIDDLE, MIDDLE), (LARGE, LARGE, WIDE))]


def test_the_sizes_reach_the_tiles_they_mean():
    for n, t, dim, vocab, *want in SHAPES:
        assert [tiles.of_xent(p, n, t, dim, vocab) for p in (True, False)] == want, (n, t, dim, vocab)
    for words in (4, 5):
        for product in range(3):
            assert {s[words][product] for s in SHAPES} == {LARGE, WIDE, MIDDLE, SMALL}


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def compare(what, got, want, tol):
    slack = tol + HALF_ULP[got.dtype] * (want.abs() + tol) + TINY[got.dtype]
    assert torch.isfinite(got.double()).all(), what
    off = (got.double() - want).abs()
    print(*what, "off by %.3g of what is allowed" % float((off / slack.clamp(min=1e-300)).max()))
    assert (off <= slack).all(), what


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape", [s[:4] for s in SHAPES], ids=str)
def test_every_tile_against_64_bits(sams, kind, shape):
    n, t, dim, vocab = shape
    h, w, labels = (v.cuda() for v in make(*shape, kind))
    grad = torch.linspace(0.5, 2.0, n, device="cuda")
    loss, lse, dh = torch.full((n,), float("nan"), device="cuda"), torch.full((n, t), float("nan"), device="cuda"), torch.full_like(h, float("nan"))
    dw = {k: torch.full((n, vocab, dim), float("nan"), device="cuda", dtype=k) for k in {kind, torch.float32}}
    added = {k: torch.full((n, vocab, dim), 0.25, device="cuda", dtype=k) for k in {kind, torch.float32}}
    again = torch.full_like(dw[kind], float("nan"))
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        op.linear_xent_forward(h, w, labels, loss, lse)
        for k in dw:
            op.linear_xent_backward(h, w, labels, lse, grad, dh, added[k], accumulate=True)
            op.linear_xent_backward(h, w, labels, lse, grad, dh, dw[k])
        op.linear_xent_backward(h, w, labels, lse, grad, dh, again)
    assert torch.equal(again, dw[kind])
    for i in range(n):
        want, tol = formulas(h[i:i + 1], w, labels[i:i + 1], grad[i:i + 1])
        for name, got in (("lse", lse), ("loss", loss), ("dh", dh)):
            compare((name, shape, i), got[i:i + 1], want[name], tol[name])
        for k in dw:
            compare(("dw", shape, i, k), dw[k][i:i + 1], want["dw"], tol["dw"])
            compare(("dw added", shape, i, k), added[k][i:i + 1], want["dw"] + 0.25, tol["dw"] + 2.0 ** -24)
