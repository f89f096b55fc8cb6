"""Orthogonalised updates of 16-bit tensors between whose products the numbers have 22 bits (pairs of words), as every 16-bit float's and
bfloat16's with a side below 1024: off by what 2^-22 between the products allows and by the result's own rounding, which of a thousand
numbers or more has the norm that the 64-bit result's rounding has, to a tenth."""
import pytest
import torch

from tests.test_gpu_ortho import COEF, CUBIC, matrices, reference

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


@pytest.mark.parametrize("kind", list(HALF_ULP), ids=str)
@pytest.mark.parametrize("steps,coef", [(5, COEF), (1, COEF), (10, CUBIC)], ids=str)
@pytest.mark.parametrize("shape", [(3, 16, 16), (2, 63, 65), (1, 84, 120), (2, 128, 128), (1, 129, 257), (2, 300, 120), (1, 33, 700), (1, 700, 33), (1, 260, 260), (1, 511, 513),
                                   (1, 1, 6000), (2, 19, 3617), (1, 2311, 200)], ids=str)
def test_pairs_of_words(sams, kind, shape, steps, coef):
    g = matrices(*shape, kind)
    want, bounds = reference(g, steps, coef)
    out = torch.full_like(g, float("nan"), device="cuda")
    with sams.Orthogonalizer(*shape, kind) as op:
        op.orthogonalize(g.cuda(), out, steps=steps, coef=coef)
    got = out.cpu().double()
    for i in range(shape[0]):
        rounding = float(torch.linalg.matrix_norm(want[i].to(kind).double() - want[i]))
        rounding = 1.1 * rounding if want[i].numel() >= 1000 else HALF_ULP[kind] * float(torch.linalg.matrix_norm(want[i]))
        off = float(torch.linalg.matrix_norm(got[i] - want[i]))
        assert off <= 16 * 2.0 ** -22 * bounds[i] + rounding, (i, off, rounding, bounds[i])


@pytest.mark.parametrize("kind", [torch.float32, *HALF_ULP], ids=str)
@pytest.mark.parametrize("rows,cols", [(30, 40), (300, 200), (1024, 1030)])
def test_zeros_stay_zero_whatever_eps(sams, kind, rows, cols):
    g = torch.zeros((2, rows, cols), device="cuda", dtype=kind)
    g[1] = torch.randn((rows, cols), device="cuda").to(kind)
    out = torch.full_like(g, float("nan"))
    with sams.Orthogonalizer(2, rows, cols, kind) as op:
        op.orthogonalize(g, out, eps=0.0)
    assert (out[0] == 0).all() and torch.isfinite(out[1]).all() and (out[1] != 0).any()
