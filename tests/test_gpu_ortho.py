"""Orthogonalised updates against Newton-Schulz steps in 64 bits.

Tolerance.  Matrices are held to u = 2^-22 (32-bit tensors) or 2^-12 (16-bit ones) of each number between the products.  A relative
error of X_j grows by the steps that follow: along singular directions i, k by a divided difference of f = p o ... o p, at most
K_j = max(|f'|, (f(s_i) + f(s_k)) / (s_i + s_k)) over the matrix's singular values.  So with X_j from the 64-bit iteration
    |error|_F <= 16 u sum_j K_j |X_j|_F
(a result of 16-bit floats is off by half of its smallest number, 2^-25, besides) where 16 stands for the roundings of A, P and X of a step, each times a coefficient of up to 4.8.  The inputs have singular values
between 0.3 and 1 (before the norm is divided out), so that K_j stays small and the bound means something."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
CUBIC = (1.5, -0.5, 0.0)
TYPES = [torch.float32, torch.bfloat16, torch.float16]
UNIT = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -12, torch.float16: 2.0 ** -12}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}

TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def matrices(batch, rows, cols, kind, scale=1.0, seed=0):
    gen = torch.Generator().manual_seed(seed + 31 * rows + cols + 7 * batch)
    small = min(rows, cols)
    u = torch.linalg.qr(torch.randn(batch, rows, small, generator=gen).double())[0]
    v = torch.linalg.qr(torch.randn(batch, cols, small, generator=gen).double())[0]
    s = torch.linspace(0.3, 1.0, small).double()
    return ((u * s) @ v.transpose(1, 2) * scale).to(kind)


def reference(g, steps=5, coef=COEF, eps=1e-7):
    """The result and the right side of the bound above, without 16 u."""
    a, b, c = coef
    outs, bounds = [], []
    for m in g.double():
        x = m / (torch.linalg.matrix_norm(m) + eps)
        norms, s0 = [], torch.linalg.svdvals(x)
        for _ in range(steps):
            norms.append(float(torch.linalg.matrix_norm(x)))
            q = x @ x.t() if x.shape[0] <= x.shape[1] else x.t() @ x
            p = a * torch.eye(q.shape[0]) + b * q + c * (q @ q)
            x = p @ x if x.shape[0] <= x.shape[1] else x @ p
        outs.append(x)
        bound, s = 0.0, s0
        for j in range(steps):
            lo, hi = float(s.min()), float(s.max())
            grid = torch.linspace(lo, hi, 2001).double()
            f, slope = grid, torch.ones_like(grid)
            for _ in range(steps - j):
                slope = slope * (a + 3 * b * f ** 2 + 5 * c * f ** 4)
                f = a * f + b * f ** 3 + c * f ** 5
            bound += norms[j] * max(float(slope.abs().max()), float((f.abs() / grid.clamp(min=1e-300)).max()))
            s = (a * s + b * s ** 3 + c * s ** 5).abs()
        bounds.append(bound)
    return torch.stack(outs), bounds


def check(got, want, bounds, kind, what):
    got = got.cpu().double()
    assert torch.isfinite(got).all(), what
    for i in range(got.shape[0]):
        norm = float(torch.linalg.matrix_norm(want[i]))
        off = float(torch.linalg.matrix_norm(got[i] - want[i]))
        assert off <= 16 * UNIT[kind] * bounds[i] + HALF_ULP[kind] * norm + TINY[kind] * math.sqrt(want[i].numel()), (what, off, 16 * UNIT[kind] * bounds[i], norm)


SHAPES = [(1, 1, 1), (2, 1, 9), (2, 9, 1), (1, 5, 3), (3, 16, 16), (2, 63, 65), (50, 20, 12), (1, 84, 120), (2, 128, 128), (1, 129, 257), (2, 300, 120), (1, 33, 700),
          (1, 700, 33), (1, 260, 260), (1, 511, 513), (1, 2000, 70), (1, 70, 2000)]


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_64_bits(sams, kind, shape):
    g = matrices(*shape, kind)
    want, bounds = reference(g)
    out = torch.full_like(g, float("nan"), device="cuda")
    with sams.Orthogonalizer(*shape, kind) as op:
        op.orthogonalize(g.cuda(), out)
    check(out, want, bounds, kind, shape)


@pytest.mark.parametrize("shape", [(4, 96, 128), (4, 120, 84), (2, 300, 400), (2, 400, 130)], ids=str)
def test_no_number_stands_out(sams, shape):
    """The bound above is on the whole matrix, where one number that lost its second part (an error of 2^-12 of it) would hide.  Roundings
    spread over a matrix: no number is off by more than eight times what the bound leaves each on the average."""
    for seed in range(6):
        g = matrices(*shape, torch.float32, seed=100 * seed)
        want, bounds = reference(g, steps=2)
        out = torch.empty_like(g, device="cuda")
        with sams.Orthogonalizer(*shape) as op:
            op.orthogonalize(g.cuda(), out, steps=2)
        for i in range(shape[0]):
            each = 16 * UNIT[torch.float32] * bounds[i] / math.sqrt(want[i].numel())
            assert float((out[i].cpu().double() - want[i]).abs().max()) <= 8 * each, (seed, i)


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("steps,coef", [(1, COEF), (2, CUBIC), (10, CUBIC), (3, (2.0, -1.5, 0.5)), (7, COEF), (2, (0.0, 1.0, 0.0)), (2, (1.0, 0.0, 0.0))], ids=str)
def test_steps_and_coefficients(sams, kind, steps, coef):
    for shape in ((2, 40, 90), (2, 90, 40)):
        g = matrices(*shape, kind)
        want, bounds = reference(g, steps, coef)
        out = torch.empty_like(g, device="cuda")
        with sams.Orthogonalizer(*shape, kind) as op:
            op.orthogonalize(g.cuda(), out, steps=steps, coef=coef)
        check(out, want, bounds, kind, (shape, steps, coef))


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 3e4, 1e25])
def test_any_scale(sams, scale):
    shape = (2, 50, 60)
    kind = torch.float32
    g = matrices(*shape, kind, scale=scale)
    want, bounds = reference(g, eps=0.0)
    out = torch.empty_like(g, device="cuda")
    with sams.Orthogonalizer(*shape, kind) as op:
        op.orthogonalize(g.cuda(), out, eps=0.0)
    check(out, want, bounds, kind, scale)


def test_eps_zeros_and_nan(sams):
    """A matrix of zeros stays zero, eps damps a tiny one, and NaN in one matrix leaves the others alone."""
    g = matrices(4, 30, 40, torch.float32)
    g[1] = 0
    g[2] *= 1e-8
    g[3, 5, 6] = float("nan")
    want, bounds = reference(g[:3])
    out = torch.empty_like(g, device="cuda")
    with sams.Orthogonalizer(4, 30, 40) as op:
        op.orthogonalize(g.cuda(), out)
    check(out[:1], want[:1], bounds[:1], torch.float32, "beside NaN")
    check(out[2:3], want[2:3], bounds[2:3], torch.float32, "tiny")
    assert (out[1] == 0).all() and torch.isnan(out[3]).all()


def test_tensors_as_they_lie(sams):
    for kind in TYPES:
        for rows, cols in ((37, 130), (130, 37)):
            g = matrices(3, rows, cols, kind)
            want, bounds = reference(g)
            big = torch.full((rows, 3, cols + 7), float("nan"), device="cuda", dtype=kind)
            view = big[:, :, 3:3 + cols].transpose(0, 1)
            view.copy_(g)
            with sams.Orthogonalizer(5, rows, cols, kind) as op:
                op.orthogonalize(view, view)                # in place, fewer matrices than the context is for
                check(view, want, bounds, kind, (kind, rows))
                op.orthogonalize(view[:0], view[:0])
            assert torch.isnan(big[:, :, :3]).all() and torch.isnan(big[:, :, 3 + cols:]).all()


@pytest.mark.parametrize("n,shape,nesterov", [(1, (1, 7, 5), True), (50, (1, 84, 120), True), (8, (3, 64, 64), False), (3, (2, 40, 301), True), (4, (2, 301, 40), False)])
def test_momentum_update(sams, n, shape, nesterov):
    batch, rows, cols = shape
    elems = rows * cols
    gen = torch.Generator().manual_seed(n)
    base = matrices(*shape, torch.float32)
    g = base + 0.01 * torch.randn(n, *shape, generator=gen) * base.std()
    m, x = base * 0.7, 0.02 * torch.randn(*shape, generator=gen)
    beta, lr, scale, decay = 0.9, 0.05, 1.3, 0.1
    mean = g.double().mean(0)
    m_want = beta * m.double() + (1 - beta) * mean
    want, bounds = reference(beta * m_want + (1 - beta) * mean if nesterov else m_want)
    x_want = (1 - lr * decay) * x.double() - lr * scale * want
    # gradients in the rows of flat vectors, as the sketched step has them; momentum and parameters too, updated in place
    flat = torch.full((n, 3 + batch * elems), float("nan"), device="cuda")
    gd = flat[:, 3:].unflatten(1, shape)
    gd.copy_(g)
    state = torch.zeros((2, 1 + batch * elems), device="cuda")
    md, xd = state[0, 1:].view(shape), state[1, 1:].view(shape)
    md.copy_(m)
    xd.copy_(x)
    m_out, x_out = torch.empty_like(md), torch.empty_like(xd)
    args = dict(beta=beta, nesterov=nesterov, lr=lr, scale=scale, weight_decay=decay)
    with sams.Orthogonalizer(*shape) as op:
        op.muon_update(gd, md, xd, m_out, x_out, **args)
        assert torch.equal(md.cpu(), m) and torch.equal(xd.cpu(), x)
        op.muon_update(gd, md, xd, md, xd, **args)
    assert torch.equal(md, m_out) and torch.equal(xd, x_out)
    e = 2.0 ** -23
    assert ((m_out.cpu().double() - m_want).abs() <= (n + 4) * e * (m.abs() + g.abs().mean(0))).all()
    for i in range(batch):
        # the rounding of the update's input, up to (n + 8) e of its norm, goes the way of the first step's
        slack = lr * scale * (16 * UNIT[torch.float32] + (n + 8) * e) * bounds[i] + 4 * e * float(torch.linalg.matrix_norm(x_want[i]))
        assert float(torch.linalg.matrix_norm(x_out[i].cpu().double() - x_want[i])) <= slack


def test_singular_values_come_close_to_one(sams):
    """What the operator is for: of a matrix with a spectrum that spans 300 : 1, all singular values end between 0.6 and 1.3."""
    gen = torch.Generator().manual_seed(4)
    u = torch.linalg.qr(torch.randn(200, 100, generator=gen))[0]
    v = torch.linalg.qr(torch.randn(100, 100, generator=gen))[0]
    g = ((u * torch.logspace(0, -2.5, 100)) @ v.t())[None].contiguous()
    for kind in TYPES:
        out = torch.empty_like(g, device="cuda", dtype=kind)
        with sams.Orthogonalizer(1, 200, 100, kind) as op:
            op.orthogonalize(g.cuda().to(kind), out, steps=8)
        s = torch.linalg.svdvals(out[0].float().cpu())
        assert 0.6 < float(s.min()) and float(s.max()) < 1.3, kind


def test_equal_inputs_give_equal_results(sams):
    g = matrices(2, 200, 333, torch.float32).cuda()
    outs = [torch.empty_like(g) for _ in range(3)]
    with sams.Orthogonalizer(2, 200, 333) as op:
        for o in outs:
            op.orthogonalize(g, o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(1, 1, 6000), (2, 19, 3617), (3, 1801, 33), (1, 130, 2500), (1, 2311, 200)], ids=str)
def test_long_thin_matrices(sams, kind, shape):
    """A short side beside a long one, whose products are cut along it."""
    g = matrices(*shape, kind)
    want, bounds = reference(g)
    out = torch.full_like(g, float("nan"), device="cuda")
    with sams.Orthogonalizer(*shape, kind) as op:
        op.orthogonalize(g.cuda(), out)
    check(out, want, bounds, kind, shape)
