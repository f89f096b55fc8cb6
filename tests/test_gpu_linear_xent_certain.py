"""Cross entropy of tokens whose label is nearly certain: losses of 1e-9 to 1e-2 beside logits of 200 keep their digits.

Tolerance.  All numbers have few bits and their sums less than 24, so that every logit is exact in any type.  What is left of a token's loss
log(1 + R), R = sum over v but the label of exp(z_v - z_label): a difference of D in the exponent (in units of log 2) carries the rounding
of log2 e and that of one fma, 2^-24 D each, and exp2, the sum over the vocabulary (some 40 adds in a row, then a tree) and log1p
at most 2^-18 of their own.  A sum of t losses of one sign adds 2^-20."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def make(n, t, vocab, kind, common, dim=64, seed=0):
    gen = torch.Generator().manual_seed(seed + n + 10 * t + vocab)
    w = torch.randint(-1, 2, (vocab, dim), generator=gen).float()
    labels = torch.randint(0, vocab, (n, t), generator=gen)
    h = w[labels] * torch.tensor([0.25, 0.375, 0.5])[torch.randint(0, 3, (n, t, 1), generator=gen)]
    w[:, 0], h[..., 0] = 4, common / 4                      # every logit the same number larger
    return h.to(kind), w.to(kind), labels


def reference(h, w, labels):
    """Every token's loss and largest difference of logits, without cancellation."""
    z = h.double() @ w.double().t()
    below = z - z.gather(-1, labels[..., None])
    rest = torch.exp(below).scatter(-1, labels[..., None], 0.0).sum(-1)
    return torch.log1p(rest), below.abs().amax(-1) / math.log(2)


@pytest.mark.parametrize("common", [188.0, 0.0, -192.0])
@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("n,t,vocab", [(24, 1, 1000), (5, 70, 777), (2, 300, 5003), (2, 3, 1)])
def test_losses_keep_their_digits(sams, n, t, vocab, kind, common):
    h, w, labels = make(n, t, vocab, kind, common)
    want, most = reference(h, w, labels)
    loss, lse = torch.full((n,), float("nan"), device="cuda"), torch.empty((n, t), device="cuda")
    with sams.LinearCrossEntropy(n, t, 64, vocab, kind, train=False) as op:
        op.linear_xent_forward(h.cuda(), w.cuda(), labels.cuda(), loss, lse)
    slack = (want * (2.0 ** -23 * most + 2.0 ** -18)).mean(1) + 2.0 ** -20 * want.mean(1)
    off = (loss.cpu().double() - want.mean(1)).abs()
    print(n, t, vocab, kind, common, "losses", float(want.min()), float(want.max()), "off by", float((off / slack.clamp(min=1e-300)).max()), "of what is allowed")
    assert (loss >= 0).all()
    assert (off <= slack).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_labels_far_from_the_largest_logit(sams, kind):
    """The other end: labels 100 or more below the largest, infinitely far among them."""
    h = torch.tensor([[[8.0, 1.0, 0.0]]]).expand(4, 1, 3).contiguous()
    w = torch.tensor([[20.0, 0.0, 0.0], [0.0, 1.0, 0.0], [-20.0, 0.0, 0.0], [-3e4, 0.0, 0.0]])
    labels = torch.tensor([[0], [1], [2], [3]])
    loss, lse = torch.empty((4,), device="cuda"), torch.empty((4, 1), device="cuda")
    with sams.LinearCrossEntropy(4, 1, 3, 4, kind, train=False) as op:
        op.linear_xent_forward(h.to(kind).cuda(), w.to(kind).cuda(), labels.cuda(), loss, lse)
    z = h[0, 0].to(kind).double() @ w.to(kind).double().t()
    want = torch.logsumexp(z, 0) - z
    assert ((loss.cpu().double() - want).abs() <= 2.0 ** -22 * want).all(), loss
    assert ((lse.cpu().double() - 160).abs() <= 2.0 ** -22 * 160).all()


WORD = {torch.float32: 2.0 ** -21, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def check_gradients(sams, h, w, labels):
    """Gradients against 64 bits, a worker at a time on the GPU.  A probability's exponent carries the roundings of lse, of its product with
    log2 e, of log2 e itself and of an fma, each 2^-24 of a logit's size: 2^-22 |z| of the probability, and 2^-18 of exp2 and of the sum
    over the vocabulary; dz is that far off in each number, the label's too, rounded to the words it is held in (and 2^-38), and the products
    add 2^-20 of the magnitudes they add up."""
    (n, t, dim), vocab, kind = h.shape, w.shape[0], h.dtype
    h, w, labels = h.cuda(), w.cuda(), labels.cuda()
    loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
    dh, dw = torch.full_like(h, float("nan")), torch.full((n, vocab, dim), float("nan"), device="cuda", dtype=kind)
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        op.linear_xent_forward(h, w, labels, loss, lse)
        op.linear_xent_backward(h, w, labels, lse, None, dh, dw)
    wd = w.double()
    for i in range(n):
        want_dw, tol_dw = torch.zeros((2, vocab, dim), device="cuda", dtype=torch.float64)
        for lo in range(0, t, 1 << 16):
            part = slice(lo, min(t, lo + (1 << 16)))
            hd, at = h[i, part].double(), labels[i, part, None]
            z = hd @ wd.t().contiguous()
            most = float(z.abs().max())
            p = torch.exp(z - z.gather(-1, at)).scatter_(-1, at, 0.0)
            rest = p.sum(-1, keepdim=True)
            p /= 1 + rest
            dz = p.scatter_(-1, at, -rest / (1 + rest)) / t
            edz = dz.abs() * (2.0 ** -22 * most + 2.0 ** -18 + 2.0 ** -20 + WORD[kind]) + 2.0 ** -38 / t
            compare(("dh", i, (n, t, vocab), kind), dh[i, part], dz @ wd, edz @ wd.abs())
            want_dw += dz.t().contiguous() @ hd
            tol_dw += edz.t().contiguous() @ hd.abs()
        compare(("dw", i, (n, t, vocab), kind), dw[i], want_dw, tol_dw)


def compare(what, got, want, tol):
    slack = tol + HALF_ULP[got.dtype] * (want.abs() + tol) + TINY[got.dtype]
    off = (got.double() - want).abs()
    print(*what, "off by %.3g of what is allowed" % float((off / slack.clamp(min=1e-300)).max()))
    assert (off <= slack).all(), what


@pytest.mark.parametrize("common", [188.0, 0.0, -192.0])
@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("n,t,vocab", [(24, 1, 1000), (5, 70, 777), (2, 300, 5003), (2, 3, 1), (1, 1, 257)])
def test_gradients_keep_their_digits(sams, n, t, vocab, kind, common):
    check_gradients(sams, *make(n, t, vocab, kind, common))


@pytest.mark.parametrize("n,t,vocab,kind", [(3, 22000, 9001, torch.bfloat16), (2, 70000, 5003, torch.float32), (1, 530000, 4001, torch.bfloat16), (2, 3, 2100001, torch.float32),
                                            (1, 3, 4300007, torch.float16)], ids=str)
def test_more_than_the_scratch_has_room_for(sams, n, t, vocab, kind):
    """dz of some workers after the others (two of three, one of two), and by pieces of the vocabulary where a worker's has no room or is too wide."""
    check_gradients(sams, *make(n, t, vocab, kind, 24.0, dim=24))
