"""Orthogonalised updates in every tile that their products have, against the same steps in 64 bits.

Tolerance.  As for the smaller matrices: a relative error u of the numbers between the products (2^-22, and 2^-12 for bfloat16 with both
sides from 1024 on) grows by the steps that follow, along two singular directions by a divided difference of f = p o ... o p, at most
K_j = max(|f'|, |f(s) / s|) over the range of the singular values:
    |error|_F <= 16 u sum_j K_j |X_j|_F
and 16-bit results are rounded besides.  Of thousands of numbers that rounding has the norm that the 64-bit result's own has, to a
tenth.  Roundings spread over a matrix: no row is off by more than eight times what the two leave each on the average."""
import math

import pytest
import torch

from tests import tiles
from tests.tiles import LARGE, MIDDLE, SMALL, WIDE

COEF = (3.4445, -4.7750, 2.0315)
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# batch, rows, cols, the tiles of gram, square and apply; sizes that end inside a tile, but for the first
PAIRS = [(24, 1024, 1024, LARGE, LARGE, MIDDLE), (22, 1001, 1025, LARGE, LARGE, LARGE), (22, 1025, 1001, LARGE, LARGE, LARGE), (12, 1025, 1275, WIDE, WIDE, WIDE),
         (12, 1275, 1025, WIDE, WIDE, WIDE), (13, 513, 1275, MIDDLE, MIDDLE, MIDDLE), (13, 1275, 513, MIDDLE, MIDDLE, MIDDLE), (9, 261, 3001, SMALL, SMALL, LARGE),
         (11, 1531, 261, SMALL, SMALL, WIDE), (19, 387, 387, MIDDLE, MIDDLE, SMALL), (19, 513, 387, MIDDLE, MIDDLE, SMALL)]
SINGLE = [(14, 1275, 1531, LARGE, LARGE, LARGE), (14, 1531, 1275, LARGE, LARGE, LARGE), (7, 1025, 1025, WIDE, WIDE, WIDE), (7, 1027, 1025, WIDE, WIDE, WIDE),
          (4, 1275, 1275, MIDDLE, MIDDLE, MIDDLE), (4, 1279, 1275, MIDDLE, MIDDLE, MIDDLE), (1, 1025, 1111, SMALL, SMALL, SMALL), (1, 1111, 1025, SMALL, SMALL, SMALL),
          (13, 1025, 1790, MIDDLE, LARGE, LARGE)]


def test_the_sizes_reach_the_tiles_they_mean():
    for pairs, shapes in ((True, PAIRS), (False, SINGLE)):
        for batch, rows, cols, *want in shapes:
            assert tiles.of_ortho(pairs, batch, rows, cols) == tuple(want), (pairs, batch, rows, cols)
    for product in range(3):
        assert {s[3 + product] for s in PAIRS} == {s[3 + product] for s in SINGLE} == {LARGE, WIDE, MIDDLE, SMALL}


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def basis(size, count):
    """Columns of an orthogonal matrix: cosines of all frequencies."""
    at, frequency = torch.arange(size, device="cuda").double()[:, None] + 0.5, torch.arange(count, device="cuda").double()
    q = torch.cos(math.pi / size * at * frequency) * math.sqrt(2.0 / size)
    q[:, 0] /= math.sqrt(2.0)
    return q


def matrices(batch, rows, cols, kind, seed=0):
    """Singular values between 0.3 and 1, directions that random signs make each matrix's own."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 31 * rows + cols + 7 * batch)
    small = min(rows, cols)
    u, v, s = basis(rows, small), basis(cols, small).t().contiguous(), torch.linspace(0.3, 1.0, small, device="cuda").double()
    sign = lambda size: torch.randint(0, 2, (batch, size), generator=gen, device="cuda").double() * 2 - 1
    left, middle, right = sign(rows), sign(small) * s, sign(cols)
    return torch.stack([(left[i][:, None] * u * middle[i]) @ (v * right[i]) for i in range(batch)]).to(kind)


def reference(g, steps=5, coef=COEF, eps=1e-7):
    """The result, and sum_j K_j |X_j|_F."""
    a, b, c = coef
    outs, bounds = [], []
    for m in g.double():
        x = m / (torch.linalg.matrix_norm(m) + eps)
        root, norms = float(torch.linalg.matrix_norm(m)), []
        one = torch.eye(min(x.shape), device=x.device, dtype=x.dtype)
        for _ in range(steps):
            norms.append(float(torch.linalg.matrix_norm(x)))
            t = x.t().contiguous()
            q = x @ t if x.shape[0] <= x.shape[1] else t @ x
            p = a * one + b * q + c * (q @ q)
            x = p @ x if x.shape[0] <= x.shape[1] else x @ p
        outs.append(x)
        s, bound = torch.linspace(0.29 / root, 1.01 / root, 2001).double(), 0.0           # the input's rounding moves them by less
        for j in range(steps):
            f, slope = s, torch.ones_like(s)
            for _ in range(steps - j):
                slope = slope * (a + 3 * b * f ** 2 + 5 * c * f ** 4)
                f = a * f + b * f ** 3 + c * f ** 5
            bound += norms[j] * max(float(slope.abs().max()), float((f.abs() / s).max()))
            s = (a * s + b * s ** 3 + c * s ** 5).abs()
            s = torch.linspace(float(s.min()), float(s.max()), 2001).double()
        bounds.append(bound)
    return torch.stack(outs), bounds


def check(got, want, bounds, unit, what, scale=1.0, extra=0.0):
    assert torch.isfinite(got.double()).all(), what
    for i in range(len(want)):
        rounding = 1.1 * float(torch.linalg.matrix_norm(want[i].to(got.dtype).double() - want[i]))
        off, slack = got[i].double() - want[i], 16 * unit * bounds[i] * scale + rounding + extra
        print(what, i, "off by %.3g of what is allowed, a row by %.3g" % (float(off.norm()) / slack, float(off.norm(dim=1).max()) * math.sqrt(off.shape[0]) / (8 * slack)))
        assert float(off.norm()) <= slack, (what, i)
        assert float(off.norm(dim=1).max()) <= 8 * slack / math.sqrt(off.shape[0]), (what, i)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,shape", [(k, s[:3]) for k in (F32, F16) for s in PAIRS] + [(BF16, s[:3]) for s in PAIRS if min(s[1:3]) < 1024] + [(BF16, s[:3]) for s in SINGLE], ids=str)
def test_every_tile_against_64_bits(sams, kind, shape):
    g = matrices(*shape, kind)
    want, bounds = reference(g)
    outs = [torch.full_like(g, float("nan")) for _ in range(3)]
    with sams.Orthogonalizer(*shape, kind) as op:
        for out in outs:
            op.orthogonalize(g, out)
    single = kind is BF16 and min(shape[1:]) >= 1024
    check(outs[0], want, bounds, 2.0 ** -12 if single else 2.0 ** -22, (kind, shape))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(24, 1024, 1024), (22, 1025, 1001)], ids=str)
def test_momentum_update_of_many_layers(sams, shape):
    n, beta, lr, scale, decay = 3, 0.9, 0.05, 1.3, 0.1
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *size: torch.randn(size, generator=gen, device="cuda")
    base = matrices(*shape, F32)
    g = base + 0.01 * base.std() * rand(n, *shape)
    m, x = base * 0.7, 0.02 * rand(*shape)
    mean = g.double().mean(0)
    m_want = beta * m.double() + (1 - beta) * mean
    want, bounds = reference(beta * m_want + (1 - beta) * mean)
    x_want = (1 - lr * decay) * x.double() - lr * scale * want
    outs = [(torch.empty_like(m), torch.empty_like(x)) for _ in range(2)]
    with sams.Orthogonalizer(*shape) as op:
        for m_out, x_out in outs:
            op.muon_update(g, m, x, m_out, x_out, beta=beta, lr=lr, scale=scale, weight_decay=decay)
    e = 2.0 ** -23
    assert ((outs[0][0].double() - m_want).abs() <= (n + 4) * e * (m.abs() + g.abs().mean(0))).all()
    # the rounding of the update's input, up to (n + 8) e of its norm, goes the way of the first step's
    check(outs[0][1], x_want, bounds, 2.0 ** -22 + (n + 8) * e / 16, shape, lr * scale, 4 * e * float(x_want.norm(dim=(1, 2)).max()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
