"""Layer norm, forward and backward, against its formulas in 64 bits.

Tolerances.  With e = 2^-23 and everything in 32 bits: a sum of dim numbers made by 64 lanes is off by at most (dim / 64 + 6) e times
the sum of absolute values, and a handful of roundings follow; so every output lies within C e of what the magnitudes that were
added up allow, C = dim / 64 + 16.  Outputs of 16 bits are rounded once more, by half a unit in the last place."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -23
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # of the larger neighbour
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = list(HALF_ULP)
EPS = 1e-5


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def make(n, t, dim, kind, seed=0):
    gen = torch.Generator().manual_seed(seed + 1000 * n + 10 * t + dim)
    x = (torch.randn(n, t, dim, generator=gen) * torch.exp(torch.randn(dim, generator=gen)) + torch.randn(n, t, 1, generator=gen)).to(kind)
    dy = torch.randn(n, t, dim, generator=gen).to(kind)
    w, b = 1 + 0.3 * torch.randn(dim, generator=gen), 0.2 * torch.randn(dim, generator=gen)
    return x, dy, w, b


def formulas(x, dy, w, b, eps=EPS):
    """Outputs in 64 bits, and the magnitudes that 32-bit rounding errors of each are relative to."""
    x, dy, w, b = x.double(), dy.double(), w.double(), b.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    z = (x - mean) * rstd
    a = dy * w
    out = {"y": z * w + b, "dx": rstd * (a - a.mean(-1, keepdim=True) - z * (a * z).mean(-1, keepdim=True)),
           "dw": (dy * z).sum(1), "db": dy.sum(1), "mean": mean.squeeze(-1), "rstd": rstd.squeeze(-1)}
    zm = z.abs() + x.abs().mean(-1, keepdim=True) * rstd + x.abs() * rstd
    size = {"y": zm * w.abs() + b.abs(), "dx": rstd * (a.abs() + a.abs().mean(-1, keepdim=True) + zm * (a.abs() * zm).mean(-1, keepdim=True)),
            "dw": (dy.abs() * zm).sum(1), "db": dy.abs().sum(1), "mean": x.abs().mean(-1), "rstd": rstd.squeeze(-1)}
    return out, size


def check(got, want, size, steps, what):
    got = got.cpu()
    kind = got.dtype
    slack = steps * E * size + HALF_ULP[kind] * (want.abs() + steps * E * size) + TINY[kind]
    off = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    assert (off <= slack).all(), (what, float((off / slack.clamp(min=1e-300)).max()))


def device_rows(t, layout, fill=float("nan")):
    """A copy on the GPU in one of the layouts a caller may have."""
    n, rows, dim = t.shape
    if layout == "plain":
        return t.cuda()
    if layout == "wide":                                    # rows further apart than they are long, and a first element anywhere
        big = torch.full((n, rows, dim + 5), fill, dtype=t.dtype, device="cuda")
        view = big[:, :, 3:3 + dim]
    else:                                                   # tokens before workers
        big = torch.full((rows, n, dim), fill, dtype=t.dtype, device="cuda")
        view = big.transpose(0, 1)
    view.copy_(t)
    return view


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape,layout", [((1, 1, 1), "plain"), ((1, 1, 7), "plain"), ((2, 3, 64), "plain"), ((3, 5, 65), "wide"), ((4, 2, 512), "swap"),
                                          ((2, 130, 768), "plain"), ((8, 33, 769), "plain"), ((1, 300, 1024), "wide"), ((2, 17, 2055), "swap"),
                                          ((1, 9, 5120), "plain"), ((2, 3, 8192), "swap"), ((1, 5, 20001), "plain"), ((1, 2049, 40), "plain")])
def test_forward_and_backward(sams, kind, shape, layout):
    x, dy, w, b = make(*shape, kind)
    want, size = formulas(x, dy, w, b)
    n, t, dim = shape
    steps = dim / 64 + 16
    steps_t = t + 32                                        # what a sum over a worker's rows may be off by
    xd, dyd = device_rows(x, layout), device_rows(dy, layout)
    y, dx = device_rows(torch.zeros_like(x), layout), device_rows(torch.zeros_like(x), layout)
    mean, rstd = torch.full((2, n, t), float("nan"), device="cuda")
    dw, db = torch.full((2, n, dim), float("nan"), device="cuda")
    with sams.LayerNorm(n, t + 3, dim, kind) as op:
        op.layer_norm_forward(xd, w.cuda(), b.cuda(), y, mean, rstd, EPS)
        op.layer_norm_backward(dyd, xd, w.cuda(), mean, rstd, dx, dw, db)
        check(y, want["y"], size["y"], steps, "y")
        check(mean, want["mean"], size["mean"], steps, "mean")
        check(rstd, want["rstd"], size["rstd"] * (1 + (size["mean"] * want["rstd"]) ** 2), 2 * steps, "rstd")
        check(dx, want["dx"], size["dx"], 4 * steps, "dx")
        check(dw, want["dw"], size["dw"], steps + steps_t, "dw")
        check(db, want["db"], size["db"], steps_t, "db")
        # sums that add to what is there, in rows of a longer vector
        flat = torch.full((n, dim + 11), 2.0, device="cuda")
        op.layer_norm_backward(dyd, xd, w.cuda(), mean, rstd, dx, flat[:, 1:1 + dim], None, accumulate=True)
        check(flat[:, 1:1 + dim], want["dw"] + 2, size["dw"] + 2, steps + steps_t + 1, "dw added up")
        assert (flat[:, 0] == 2).all() and (flat[:, 1 + dim:] == 2).all()
        # no bias; in place
        op.layer_norm_forward(xd, w.cuda(), None, y, mean, rstd, EPS)
        check(y, want["y"] - b.double(), size["y"], steps, "y without bias")
        op.layer_norm_forward(xd, w.cuda(), b.cuda(), xd, mean, rstd, EPS)
        check(xd, want["y"], size["y"], steps, "y in place")


def test_the_backward_pass_may_overwrite_its_inputs(sams):
    n, t, dim = 2, 37, 777
    x, dy, w, b = make(n, t, dim, torch.float32)
    want, size = formulas(x, dy, w, b)
    with sams.LayerNorm(n, t, dim) as op:
        for over in ("x", "dy"):
            xd, dyd = x.cuda(), dy.cuda()
            mean, rstd = torch.empty((2, n, t), device="cuda")
            dw, db = torch.empty((2, n, dim), device="cuda")
            op.layer_norm_forward(xd, w.cuda(), b.cuda(), torch.empty_like(xd), mean, rstd, EPS)
            dx = xd if over == "x" else dyd
            op.layer_norm_backward(dyd, xd, w.cuda(), mean, rstd, dx, dw, db)
            check(dx, want["dx"], size["dx"], 4 * (dim / 64 + 16), "dx over " + over)
            check(dw, want["dw"], size["dw"], dim / 64 + 48 + t, "dw")
            check(db, want["db"], size["db"], 32 + t, "db")


def test_no_tokens(sams):
    dw, db = torch.full((2, 3, 50), 7.0, device="cuda")
    e = torch.empty((3, 0, 50), device="cuda")
    s = torch.empty((3, 0), device="cuda")
    w = torch.ones(50, device="cuda")
    with sams.LayerNorm(3, 4, 50) as op:
        op.layer_norm_forward(e, w, w, e, s, s)
        op.layer_norm_backward(e, e, w, s, s, e, dw, None, accumulate=True)
        assert (dw == 7).all()
        op.layer_norm_backward(e, e, w, s, s, e, dw, db)
        assert (dw == 0).all() and (db == 0).all()


def test_rows_of_equal_numbers_and_rows_beside_nan(sams):
    x = torch.randn(1, 6, 100)
    x[0, 1] = 3.25                                          # no variance: y is the bias, and dx is finite
    x[0, 4, 50] = float("nan")                              # spoils its own row only
    dy = torch.randn(1, 6, 100)
    w, b = torch.randn(100), torch.randn(100)
    want, size = formulas(x, dy, w, b)
    xd = x.cuda()
    y, dx = torch.empty_like(xd), torch.empty_like(xd)
    mean, rstd = torch.empty((2, 1, 6), device="cuda")
    with sams.LayerNorm(1, 6, 100) as op:
        op.layer_norm_forward(xd, w.cuda(), b.cuda(), y, mean, rstd, EPS)
        op.layer_norm_backward(dy.cuda(), xd, w.cuda(), mean, rstd, dx, torch.empty((1, 100), device="cuda"))
    keep = [0, 2, 3, 5]
    check(y[:, keep], want["y"][:, keep], size["y"][:, keep], 20, "y")
    check(dx[:, keep], want["dx"][:, keep], size["dx"][:, keep], 80, "dx")
    assert torch.equal(y[0, 1].cpu(), b) and torch.isfinite(dx[0, 1]).all()
    assert torch.isnan(y[0, 4]).all()


def test_gradients_against_differences(sams):
    """<gradient, direction> against the difference quotient of sum(y * r) in 64 bits; its error is O(h^2) and 64-bit rounding / h."""
    n, t, dim, h = 2, 5, 33, 1e-4
    x, r, w, b = make(n, t, dim, torch.float32, seed=3)
    xd = x.cuda()
    mean, rstd = torch.empty((2, n, t), device="cuda")
    dx, (dw, db) = torch.empty_like(xd), torch.empty((2, n, dim), device="cuda")
    with sams.LayerNorm(n, t, dim) as op:
        op.layer_norm_forward(xd, w.cuda(), b.cuda(), torch.empty_like(xd), mean, rstd, EPS)
        op.layer_norm_backward(r.cuda(), xd, w.cuda(), mean, rstd, dx, dw, db)
    gen = torch.Generator().manual_seed(5)
    vx, vw, vb = torch.randn(n, t, dim, generator=gen).double(), torch.randn(dim, generator=gen).double(), torch.randn(dim, generator=gen).double()

    def value(s):
        return (formulas(x.double() + s * vx, r, w.double() + s * vw, b.double() + s * vb)[0]["y"] * r.double()).sum()

    quotient = float((value(h) - value(-h)) / (2 * h))
    dot = float((dx.cpu().double() * vx).sum() + (dw.cpu().double().sum(0) * vw).sum() + (db.cpu().double().sum(0) * vb).sum())
    assert abs(dot - quotient) <= 1e-5 * (abs(quotient) + float((dx.cpu().double() * vx).abs().sum()))


def test_equal_inputs_give_equal_results_on_any_stream(sams):
    x, dy, w, b = make(3, 70, 900, torch.bfloat16)
    x, dy, w, b = x.cuda(), dy.cuda(), w.cuda(), b.cuda()
    results = []
    with sams.LayerNorm(3, 70, 900, torch.bfloat16) as op:
        for stream in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.current_stream()):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                x2 = x.clone()                              # made on this stream, just before
                y, dx = torch.empty_like(x), torch.empty_like(x)
                mean, rstd = torch.empty((2, 3, 70), device="cuda")
                dw, db = torch.empty((2, 3, 900), device="cuda")
                op.layer_norm_forward(x2, w, b, y, mean, rstd)
                op.layer_norm_backward(dy, x2, w, mean, rstd, dx, dw, db)
                results.append([v.clone() for v in (y, dx, dw, db)])
            torch.cuda.synchronize()
    for other in results[1:]:
        for p, q in zip(results[0], other):
            assert torch.equal(p, q)
