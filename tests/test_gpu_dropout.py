"""Dropout against its definition: which places are kept, equal bit for bit; what is kept, within its roundings.

Tolerances.  A product with the share's reciprocal (itself rounded) and a sum: three roundings of 2^-24 in 32 bits of the magnitudes that
are added, and the output's own, half a unit of its type: which takes what lies beyond the type's largest number by half a unit or more to
infinity (16-bit floats: from 65520 on, which x * 65536 reaches where next to everything is dropped)."""
import pytest
import torch

from tests import philox

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = list(HALF_ULP)


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def make(n, t, dim, kind, seed=0):
    gen = torch.Generator().manual_seed(seed + 100 * n + 10 * t + dim)
    return (torch.randn(n, t, dim, generator=gen).to(kind) for _ in range(3))


def check(got, want, size, what):
    kind, got = got.dtype, got.cpu().double()
    beyond = want.abs() >= torch.finfo(kind).max * (1 + HALF_ULP[kind] / 2)
    assert torch.equal(got[beyond], want[beyond].sign() * torch.inf), what
    got, want, size = got[~beyond], want[~beyond], size[~beyond]
    off = (got - want).abs()
    assert (off <= 3 * 2.0 ** -24 * size + HALF_ULP[kind] * (want.abs() + 3 * 2.0 ** -24 * size) + TINY[kind]).all(), what


def rows_like(x, layout):
    n, t, dim = x.shape
    if layout == "plain":
        return x.cuda()
    big = torch.full((n, t, dim + 5) if layout == "wide" else (t, n, dim), 9.0, dtype=x.dtype, device="cuda")
    view = big[:, :, 3:3 + dim] if layout == "wide" else big.transpose(0, 1)
    view.copy_(x)
    return view


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape,layout,p", [((1, 1, 1), "plain", 0.5), ((1, 2, 7), "plain", 0.1), ((2, 3, 8), "wide", 0.9), ((3, 5, 9), "swap", 0.3), ((4, 2, 512), "plain", 0.1),
                                            ((2, 700, 17), "wide", 0.25), ((3, 41, 1283), "swap", 0.1), ((1, 3, 8192), "plain", 2 ** -16), ((2, 2, 20001), "plain", 0.5),
                                            ((1024, 3, 8), "plain", 0.1), ((1, 2, 33), "plain", 0.0), ((1, 2, 33), "plain", 2.0 ** -18), ((1, 64, 64), "plain", 65535 / 65536)])
def test_forward_and_backward(sams, kind, shape, layout, p):
    n, t, dim = shape
    x, residual, dy = make(*shape, kind)
    rng = torch.tensor([-(2 ** 62) + 12345, 2 ** 32 + 7])
    keep = torch.from_numpy(philox.keep_columns(rng, n, t, dim, p))
    share = 1 - philox.least(p) / 65536
    factor = keep.double() / share
    xd, rd, dyd = rows_like(x, layout), rows_like(residual, layout), rows_like(dy, layout)
    y, dx = rows_like(torch.full_like(x, float("nan")), layout), rows_like(torch.full_like(x, float("nan")), layout)
    with sams.Dropout(n, t + 2, dim, kind) as op:
        op.dropout_forward(xd, rd, rng.cuda(), p, y)
        check(y, residual.double() + factor * x.double(), residual.double().abs() + factor * x.double().abs(), "y")
        op.dropout_backward(dyd, rng.cuda(), p, dx)
        check(dx, factor * dy.double(), factor * dy.double().abs(), "dx")
        assert (dx.cpu()[~keep] == 0).all()
        op.dropout_forward(xd, None, rng.cuda(), p, y)
        check(y, factor * x.double(), factor * x.double().abs(), "y without residual")
        assert torch.equal(y.cpu() != 0, keep & (x != 0))
        op.dropout_forward(xd, rd, rng.cuda(), p, rd)                       # over the residual
        check(rd, residual.double() + factor * x.double(), residual.double().abs() + factor * x.double().abs(), "y over the residual")
        op.dropout_forward(xd, None, rng.cuda(), p, xd)                     # in place
        assert torch.equal(xd, y)
    if layout == "wide":
        for v in (y, dx):
            whole = v._base
            assert (whole[:, :, :3] == 9).all() and (whole[:, :, 3 + dim:] == 9).all()


def test_what_is_dropped_may_be_anything(sams):
    """NaN and infinities at places that are dropped leave no trace."""
    n, t, dim, p = 2, 9, 100, 0.4
    x, residual, _ = make(n, t, dim, torch.float32)
    rng = torch.tensor([5, 6])
    keep = torch.from_numpy(philox.keep_columns(rng, n, t, dim, p))
    bad = torch.where(keep, x, torch.tensor([float("nan"), float("inf")])[torch.arange(dim) % 2])
    with sams.Dropout(n, t, dim) as op:
        a, b = torch.empty((2, n, t, dim), device="cuda")
        op.dropout_forward(x.cuda(), residual.cuda(), rng.cuda(), p, a)
        op.dropout_forward(bad.cuda(), residual.cuda(), rng.cuda(), p, b)
    assert torch.equal(a, b)


def test_share_that_is_kept(sams):
    """Of 2^24 places a share of 1 - p is kept, within six standard deviations; seeds, steps, workers and rows drop different places."""
    n, t, dim, p = 4, 1024, 4096, 0.1
    x = torch.ones((n, t, dim), device="cuda")
    y = torch.empty_like(x)
    seen = []
    with sams.Dropout(n, t, dim) as op:
        for seed, step in ((1, 0), (2, 0), (1, 1), (1 << 32 | 1, 0)):
            op.dropout_forward(x, None, torch.tensor([seed, step], device="cuda"), p, y)
            keep = y != 0
            count = keep.numel()
            assert abs(float(keep.double().mean()) - (1 - philox.least(p) / 65536)) < 6 * (p * (1 - p) / count) ** 0.5
            seen += [keep[0, 0], keep[1, 0], keep[0, 1]]
    for i in range(len(seen)):
        for j in range(i):
            both = float((seen[i] ^ seen[j]).double().mean())
            assert abs(both - 2 * p * (1 - p)) < 6 * (0.18 * 0.82 / dim) ** 0.5, (i, j)


def test_no_tokens(sams):
    e = torch.empty((3, 0, 50), device="cuda")
    with sams.Dropout(3, 4, 50) as op:
        op.dropout_forward(e, e, None, 0.0, e)
        op.dropout_backward(e, torch.zeros(2, dtype=torch.int64, device="cuda"), 0.5, e)


def test_replays_draw_anew_and_streams_wait(sams):
    n, t, dim, p = 2, 50, 96, 0.2
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        op = sams.Dropout(n, t, dim, torch.bfloat16)
        x = torch.ones((n, t, dim), device="cuda", dtype=torch.bfloat16)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        rng = torch.tensor([99, 0], device="cuda")

        def calls():
            op.dropout_forward(x, None, rng, p, y)
            op.dropout_backward(y, rng, p, dx)
            rng[1:] += 1

        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls()
        for step in range(1, 5):
            assert int(rng[1]) == step
            graph.replay()
            torch.cuda.synchronize()
            keep = torch.from_numpy(philox.keep_columns((99, step), n, t, dim, p))
            assert torch.equal(y.cpu() != 0, keep) and torch.equal(dx.cpu() != 0, keep)
    # on another stream than the context's, which waits for the tensors made there
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        z = (x.float() * 2).bfloat16()
        out = torch.empty_like(z)
        op.dropout_forward(z, None, torch.tensor([7, 1], device="cuda"), p, out)
        got = out.clone()
    torch.cuda.synchronize()
    assert torch.equal(got.cpu() != 0, torch.from_numpy(philox.keep_columns((7, 1), n, t, dim, p)))
