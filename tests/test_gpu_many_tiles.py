"""Calls whose tiles or rows would make a grid of 2^32 threads or more, which no launch takes: they go in several, or from row to row."""
import pytest
import torch

from tests.test_gpu_linear_xent import check, formulas

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_log_sums_of_a_million_tokens_by_half_a_million_words(sams):
    """4097 x 2049 tiles of 256 in 32 bits.  Bounds of `formulas`, at the first, the last and some tokens between."""
    t, dim, vocab = 2 ** 20 + 3, 8, 2 ** 19 + 1
    gen = torch.Generator(device="cuda").manual_seed(0)
    h = torch.randn((1, t, dim), generator=gen, device="cuda")
    w = 0.7 * torch.randn((vocab, dim), generator=gen, device="cuda")
    labels = torch.randint(0, vocab, (1, t), generator=gen, device="cuda")
    loss, lse = torch.full((1,), float("nan"), device="cuda"), torch.full((1, t), float("nan"), device="cuda")
    with sams.LinearCrossEntropy(1, t, dim, vocab, train=False) as op:
        op.linear_xent_forward(h, w, labels, loss, lse)
    at = torch.cat([torch.arange(300), torch.arange(t - 300, t), torch.randint(0, t, (1400,))]).cuda()
    hd, wd = h[0, at].double(), w.double()
    z = hd @ wd.t().contiguous()
    want = torch.logsumexp(z, -1)
    slack = 2.0 ** -20 * (hd.abs() @ wd.abs().t().contiguous()).amax(-1) + 2.0 ** -21 * z.abs().amax(-1) + 2.0 ** -20 * (want.abs() + 1)
    assert ((lse[0, at].double() - want).abs() <= slack).all()
    per = lse[0].double() - (h[0].double() * wd[labels[0]]).sum(-1)
    assert abs(float(loss) - float(per.mean())) <= 2.0 ** -20 * float(lse.abs().max())


def test_gradients_of_more_than_2_to_the_26_tokens(sams):
    n, t, dim, vocab, kind = 1, 2 ** 26 + 5, 8, 8, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn((n, t, dim), generator=gen, device="cuda").to(kind)
    w = torch.randn((vocab, dim), generator=gen, device="cuda").to(kind)
    labels = torch.randint(-1, vocab, (n, t), generator=gen, device="cuda")
    loss, lse = torch.empty((n,), device="cuda"), torch.full((n, t), float("nan"), device="cuda")
    dh, dw = torch.full_like(h, float("nan")), torch.empty((n, vocab, dim), device="cuda")
    with sams.LinearCrossEntropy(n, t, dim, vocab, kind) as op:
        op.linear_xent_forward(h, w, labels, loss, lse)
        op.linear_xent_backward(h, w, labels, lse, torch.full((n,), float(t), device="cuda"), dh, dw)
    count = int((labels >= 0).sum())
    for lo in (0, t // 2, t - 4096):                        # each as if these were all tokens, their share of the gradient
        part = slice(lo, lo + 4096)
        own = int((labels[0, part] >= 0).sum())
        want, tol = formulas(h[:, part], w, labels[:, part], torch.full((1,), float(t) * own / count, device="cuda"))
        check(lse[:, part], want["lse"].cpu(), tol["lse"].cpu(), ("lse", lo))
        check(dh[:, part], want["dh"].cpu(), tol["dh"].cpu(), ("dh", lo))
    sums, slack = torch.zeros((2, vocab, dim), device="cuda", dtype=torch.float64)
    for lo in range(0, t, 2 ** 22):
        part = slice(lo, min(t, lo + 2 ** 22))
        own = int((labels[0, part] >= 0).sum())
        want, tol = formulas(h[:, part], w, labels[:, part], torch.full((1,), float(t) * own / count, device="cuda"))
        sums += want["dw"][0]
        slack += tol["dw"][0]
    check(dw, sums[None].cpu(), slack[None].cpu(), "dw")


def test_thousands_of_long_rows_orthogonalised(sams):
    """8200 matrices of one row each: 2048 tiles of 64 a matrix.  A row's only singular value goes through the polynomial by itself; the
    bound is that of larger matrices, 16 u sum_j K_j |X_j|."""
    batch, cols, coef, steps = 8200, 131072, (3.4445, -4.7750, 2.0315), 5
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = torch.randn((batch, 1, cols), generator=gen, device="cuda")
    out = torch.full_like(g, float("nan"))
    with sams.Orthogonalizer(batch, 1, cols) as op:
        op.orthogonalize(g, out)
    a, b, c = coef
    values = [1.0]
    for _ in range(steps):
        s = values[-1]
        values.append(a * s + b * s ** 3 + c * s ** 5)
    bound = 0.0
    for j in range(steps):
        slope = 1.0
        for s in values[j:-1]:
            slope *= abs(a + 3 * b * s ** 2 + 5 * c * s ** 4)
        bound += max(slope, values[-1] / values[j]) * values[j]
    for lo in range(0, batch, 1025):
        part = g[lo:lo + 1025, 0].double()
        want = values[-1] * part / part.norm(dim=1, keepdim=True)
        off = (out[lo:lo + 1025, 0].double() - want).norm(dim=1)
        assert (off <= 16 * 2.0 ** -22 * bound + 2.0 ** -24 * values[-1]).all(), (lo, float(off.max()))
