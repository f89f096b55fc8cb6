"""Cross entropy of an output layer and its gradients against the formulas in 64 bits.

Tolerances.  A logit is a sum of dim products of words that are exact (16-bit tensors) or hold 22 bits (32-bit ones), added in
32 bits: off by at most E_z = 2^-20 sum |h||w|, and as an argument of exp by 2^-21 |z| more.  lse takes that over, and adds a few
roundings.  dz = p - [label] is off by p times twice that, and by the rounding r of the words it is held in; the products of the
gradients add 2^-20 of the magnitudes they add up, and the output's own rounding."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
WORD = {torch.float32: 2.0 ** -21, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def make(n, t, dim, vocab, kind, masked=0.2, seed=0):
    gen = torch.Generator().manual_seed(seed + 77 * n + 5 * t + 3 * dim + vocab)
    w = (torch.randn(vocab, dim, generator=gen) * 0.3).to(kind)
    labels = torch.randint(0, vocab, (n, t), generator=gen)
    h = (torch.randn(n, t, dim, generator=gen) * 0.5 + w.float()[labels] * torch.rand(n, t, 1, generator=gen) * 4).to(kind)
    labels[torch.rand(n, t, generator=gen) < masked] = -100
    return h, w, labels


def formulas(h, w, labels, grad=None):
    kind, (n, t, dim), vocab = h.dtype, h.shape, w.shape[0]
    used = (labels >= 0) & (labels < vocab)
    h, w = torch.where(used[..., None], h.double(), 0.0), w.double()
    count = used.sum(1)
    inv = torch.where(count > 0, (grad.double() if grad is not None else 1.0) / count.clamp(min=1), 0.0)
    z = h @ w.t()
    lse = torch.where(used, torch.logsumexp(z, -1), 0.0)
    safe = torch.where(used, labels, 0)
    at = z.gather(-1, safe[..., None]).squeeze(-1)
    per = torch.where(used, lse - at, 0.0)
    one = torch.zeros_like(z).scatter_(-1, safe[..., None], 1.0)
    p = torch.exp(z - torch.logsumexp(z, -1, keepdim=True)) * used[..., None]
    dz = p - one * used[..., None]
    out = {"lse": lse, "loss": per.sum(1) / count.clamp(min=1), "dh": inv[:, None, None] * (dz @ w), "dw": inv[:, None, None] * (dz.transpose(1, 2) @ h)}
    ez = 2.0 ** -20 * (h.abs() @ w.abs().t()).amax(-1) + 2.0 ** -21 * z.abs().amax(-1)
    tol = {"lse": used * (ez + 2.0 ** -20 * (lse.abs() + 1))}
    tol["loss"] = (tol["lse"] + used * (ez + 2.0 ** -20 * per.abs())).sum(1) / count.clamp(min=1) + 2.0 ** -20 * out["loss"].abs()
    edz = p * (2 * tol["lse"] + 2.0 ** -20)[..., None] + dz.abs() * (WORD[kind] + 2.0 ** -20) + used[..., None] * 2.0 ** -38
    tol["dh"] = inv.abs()[:, None, None] * (edz @ w.abs())
    tol["dw"] = inv.abs()[:, None, None] * (edz.transpose(1, 2) @ h.abs())
    return out, tol


def check(got, want, tol, what):
    got = got.cpu()
    slack = tol + HALF_ULP[got.dtype] * (want.abs() + tol) + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    assert (off <= slack).all(), (what, float((off / slack.clamp(min=1e-300)).max()))


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 2), (2, 3, 7, 5), (1, 64, 64, 128), (3, 17, 40, 129), (2, 65, 33, 300), (4, 5, 256, 4001), (1, 130, 768, 1000), (2, 200, 200, 517),
          (8, 33, 129, 2049), (1, 700, 96, 777), (2, 1, 1030, 260), (1, 2, 64, 20011)]


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_loss_and_gradients(sams, kind, shape):
    n, t, dim, vocab = shape
    h, w, labels = make(*shape, kind)
    grad = torch.linspace(0.5, 2.0, n)
    want, tol = formulas(h, w, labels, grad)
    hd, wd, ld = h.cuda(), w.cuda(), labels.cuda()
    loss, lse = torch.full((n,), float("nan"), device="cuda"), torch.full((n, t), float("nan"), device="cuda")
    dh, dw = torch.full_like(hd, float("nan")), torch.full((n, vocab, dim), float("nan"), device="cuda", dtype=kind)
    with sams.LinearCrossEntropy(n, t + 2, dim, vocab, kind) as op:
        op.linear_xent_forward(hd, wd, ld, loss, lse)
        op.linear_xent_backward(hd, wd, ld, lse, grad.cuda(), dh, dw)
        for name, got in (("lse", lse), ("loss", loss), ("dh", dh), ("dw", dw)):
            check(got, want[name], tol[name], name)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_tensors_as_they_lie(sams, kind):
    """Rows of longer rows at any element, workers' rows apart, gradients added up in rows of a flat 32-bit vector."""
    n, t, dim, vocab = 3, 21, 50, 333
    h, w, labels = make(n, t, dim, vocab, kind)
    want, tol = formulas(h, w, labels)
    hb = torch.full((t, n, dim + 9), float("nan"), device="cuda", dtype=kind)
    hv = hb[:, :, 1:1 + dim].transpose(0, 1)
    hv.copy_(h)
    wb = torch.full((vocab * (dim + 1) + 1,), float("nan"), device="cuda", dtype=kind)
    wv = wb[1:].view(vocab, dim + 1)[:, :dim]
    wv.copy_(w)
    flat = torch.full((n, 5 + vocab * dim + 2), 0.25, device="cuda")
    dw = flat[:, 5:5 + vocab * dim].unflatten(1, (vocab, dim))
    dhb = torch.full((n, t, dim + 4), 9.0, device="cuda", dtype=kind)
    dh = dhb[:, :, 2:2 + dim]
    loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        op.linear_xent_forward(hv, wv, labels.cuda(), loss, lse)
        op.linear_xent_backward(hv, wv, labels.cuda(), lse, None, dh, dw, accumulate=True)
    check(loss, want["loss"], tol["loss"], "loss")
    check(dh, want["dh"], tol["dh"], "dh")
    check(dw, want["dw"] + 0.25, tol["dw"] + 2.0 ** -24, "dw")
    assert (flat[:, :5] == 0.25).all() and (flat[:, -2:] == 0.25).all() and (dhb[:, :, :2] == 9).all() and (dhb[:, :, -2:] == 9).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_tokens_that_take_no_part_change_nothing(sams, kind):
    n, t, dim, vocab = 3, 40, 64, 500
    h, w, labels = make(n, t, dim, vocab, kind, masked=0.4)
    labels[1] = -100                                        # a worker without labels
    labels[0, 0], labels[2, 1] = vocab, -1                  # outside the vocabulary in any way
    want, tol = formulas(h, w, labels)
    hidden = h.clone()
    out = ~((labels >= 0) & (labels < vocab))
    hidden[out] = torch.tensor([float("nan"), float("inf"), -float("inf"), 6e4]).to(kind)[torch.arange(int(out.sum())) % 4][:, None].expand(-1, dim)
    results = []
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        for x in (h, hidden):
            loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
            dh, dw = torch.empty_like(x, device="cuda"), torch.empty((n, vocab, dim), device="cuda", dtype=kind)
            op.linear_xent_forward(x.cuda(), w.cuda(), labels.cuda(), loss, lse)
            op.linear_xent_backward(x.cuda(), w.cuda(), labels.cuda(), lse, None, dh, dw)
            results.append((loss, lse, dh, dw))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    for name, got in zip(("loss", "lse", "dh", "dw"), results[0]):
        check(got, want[name], tol[name], name)
    assert results[0][0][1] == 0 and (results[0][2][1] == 0).all() and (results[0][3][1] == 0).all()
    assert (results[0][1].cpu()[out] == 0).all() and (results[0][2].cpu()[out] == 0).all()


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_large_logits(sams, kind):
    """Logits of several hundred: the largest is taken out before exp."""
    n, t, dim, vocab = 1, 20, 128, 700
    h, w, labels = make(n, t, dim, vocab, kind, masked=0.0)
    h = (h.float() * 30).to(kind)
    want, tol = formulas(h, w, labels)
    loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
    dh, dw = torch.empty_like(h, device="cuda"), torch.empty((n, vocab, dim), device="cuda", dtype=kind)
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        op.linear_xent_forward(h.cuda(), w.cuda(), labels.cuda(), loss, lse)
        op.linear_xent_backward(h.cuda(), w.cuda(), labels.cuda(), lse, None, dh, dw)
    for name, got in (("lse", lse), ("loss", loss), ("dh", dh), ("dw", dw)):
        check(got, want[name], tol[name], name)


def test_scales_of_32_bit_tensors(sams):
    """Tensors far from 1, in either direction, and one outlier: numbers below 2^-17 of the largest lose bits, to 2^-38 of it."""
    n, t, dim, vocab = 2, 30, 96, 400
    h, w, labels = make(n, t, dim, vocab, torch.float32)
    for a, b in ((1e-12, 1e11), (1e20, 1e-20), (2.0 ** -100, 2.0 ** 99)):
        hs, ws = h * a, w * b
        want, tol = formulas(hs, ws, labels)
        loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
        dh, dw = torch.empty_like(hs, device="cuda"), torch.empty((n, vocab, dim), device="cuda")
        with sams.LinearCrossEntropy(n, t, dim, vocab) as op:
            op.linear_xent_forward(hs.cuda(), ws.cuda(), labels.cuda(), loss, lse)
            op.linear_xent_backward(hs.cuda(), ws.cuda(), labels.cuda(), lse, None, dh, dw)
        for name, got in (("lse", lse), ("loss", loss), ("dh", dh), ("dw", dw)):
            check(got, want[name], tol[name], (name, a, b))


def test_several_pieces_of_the_vocabulary(sams):
    """So many tokens that dz is made in pieces: against a plain computation in 64 bits on the GPU, in 32-bit gradients."""
    n, t, dim, vocab, kind = 2, 30000, 32, 5003, torch.bfloat16
    h, w, labels = make(n, t, dim, vocab, kind)
    hd, wd, ld = h.cuda(), w.cuda(), labels.cuda()
    loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
    dh, dw = torch.empty_like(hd), torch.empty((n, vocab, dim), device="cuda")
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        op.linear_xent_forward(hd, wd, ld, loss, lse)
        op.linear_xent_backward(hd, wd, ld, lse, None, dh, dw)
    for i in range(n):
        want, tol = formulas(hd[i:i + 1], wd, ld[i:i + 1])
        for name, got in (("lse", lse), ("loss", loss), ("dh", dh), ("dw", dw)):
            check(got[i:i + 1], want[name].cpu(), tol[name].cpu(), (name, i))


def test_gradients_against_differences(sams):
    """<gradient, direction> against the difference quotient of the losses' sum in 64 bits."""
    n, t, dim, vocab, step = 2, 9, 24, 111, 1e-5
    h, w, labels = make(n, t, dim, vocab, torch.float32, seed=9)
    loss, lse = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
    dh, dw = torch.empty_like(h, device="cuda"), torch.empty((n, vocab, dim), device="cuda")
    with sams.LinearCrossEntropy(n, t, dim, vocab) as op:
        op.linear_xent_forward(h.cuda(), w.cuda(), labels.cuda(), loss, lse)
        op.linear_xent_backward(h.cuda(), w.cuda(), labels.cuda(), lse, None, dh, dw)
    gen = torch.Generator().manual_seed(1)
    vh, vw = torch.randn(n, t, dim, generator=gen).double(), torch.randn(vocab, dim, generator=gen).double()

    def value(s):
        return _loss(h.double() + s * vh, w.double() + s * vw, labels)

    quotient = float((value(step) - value(-step)) / (2 * step))
    parts = (dh.cpu().double() * vh).sum(), (dw.cpu().double().sum(0) * vw).sum()
    assert abs(float(sum(parts)) - quotient) <= 1e-5 * (abs(quotient) + sum(abs(float(p)) for p in parts) + 1)


def _loss(h, w, labels):
    used = labels >= 0
    per = torch.logsumexp(h @ w.t(), -1) - (h * w[labels.clamp(min=0)]).sum(-1)
    return ((per * used).sum(1) / used.sum(1)).sum()


def test_no_tokens(sams):
    e = torch.empty((2, 0, 16), device="cuda")
    w = torch.randn(40, 16, device="cuda")
    labels, lse = torch.empty((2, 0), device="cuda", dtype=torch.int64), torch.empty((2, 0), device="cuda")
    loss, dw = torch.full((2,), 5.0, device="cuda"), torch.full((2, 40, 16), 3.0, device="cuda")
    with sams.LinearCrossEntropy(2, 4, 16, 40) as op:
        op.linear_xent_forward(e, w, labels, loss, lse)
        op.linear_xent_backward(e, w, labels, lse, None, e, dw, accumulate=True)
        assert (loss == 0).all() and (dw == 3).all()
        op.linear_xent_backward(e, w, labels, lse, None, e, dw)
        assert (dw == 0).all()


def test_the_forward_pass_alone(sams):
    h, w, labels = make(1, 10, 24, 90, torch.float16)
    want, tol = formulas(h, w, labels)
    loss, lse = torch.empty((1,), device="cuda"), torch.empty((1, 10), device="cuda")
    with sams.LinearCrossEntropy(1, 10, 24, 90, torch.float16, train=False) as op, sams.LinearCrossEntropy(1, 10, 24, 90, torch.float16) as full:
        assert op.scratch_bytes < full.scratch_bytes
        op.linear_xent_forward(h.cuda(), w.cuda(), labels.cuda(), loss, lse)
        check(loss, want["loss"], tol["loss"], "loss")
        with pytest.raises(sams.SamsError):
            op.linear_xent_backward(h.cuda(), w.cuda(), labels.cuda(), lse, None, h.cuda(), torch.empty((1, 90, 24), device="cuda", dtype=torch.float16))
