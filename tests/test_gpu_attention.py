"""Attention with a bias by relative position and dropout, forward and backward, against its formulas in 64 bits (tests/attention_oracle.py has
them, and what each number may be off by)."""
import pytest
import torch

from tests.attention_oracle import check, formulas

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAN = float("nan")


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def make(n, t, heads, kv_heads, dim, buckets, kind, seed=0):
    gen = torch.Generator().manual_seed(seed + 1000 * n + 10 * t + heads + dim)
    rand = lambda *shape: torch.randn(shape, generator=gen)
    x = {"q": rand(n, t, heads * dim).to(kind), "k": rand(n, t, kv_heads * dim).to(kind), "v": rand(n, t, kv_heads * dim).to(kind),
         "do": (rand(n, t, heads * dim) / t).to(kind), "bias": 0.7 * rand(heads, buckets) if buckets else None}
    return x


class Run:
    """One forward and one backward pass on the GPU, outputs full of NaN before."""

    def __init__(self, sams, x, starts, heads, kv_heads, train=True, op=None, accumulate=False, into=None, **how):
        cuda = {name: None if v is None else v.cuda() for name, v in x.items()}
        n, t, wide = cuda["q"].shape
        kind, dim = cuda["q"].dtype, wide // heads
        how = {name: v.cuda() if isinstance(v, torch.Tensor) else v for name, v in how.items()}
        mine = op or sams.Attention(n, t + 3, heads, dim, kv_heads, starts=starts or None, dtype=kind, train=train)
        self.o = torch.full_like(cuda["q"], NAN)
        self.row_max, self.row_sum = torch.full((2, n, heads, t), NAN, device="cuda")
        mine.attention_forward(cuda["q"], cuda["k"], cuda["v"], cuda["bias"], self.o, self.row_max, self.row_sum, **how)
        if train:
            self.dq, self.dk, self.dv = (torch.full_like(cuda[name], NAN) for name in ("q", "k", "v"))
            self.dbias = into if into is not None else torch.full((n, heads, len(starts)), NAN, device="cuda") if starts else None
            mine.attention_backward(cuda["do"], cuda["q"], cuda["k"], cuda["v"], cuda["bias"], self.o, self.row_max, self.row_sum, self.dq, self.dk, self.dv,
                                    self.dbias, accumulate=accumulate, **how)
        if op is None:
            mine.close()

    def outputs(self):
        return {name: v for name, v in (("o", self.o), ("dq", self.dq), ("dk", self.dk), ("dv", self.dv), ("dbias", self.dbias)) if v is not None}


def compare(run, x, starts, heads, kv_heads, **how):
    want, tol = formulas(x["q"], x["k"], x["v"], x["bias"], starts, x["do"], heads=heads, kv_heads=kv_heads, **how)
    for name, got in run.outputs().items():
        check(got, want[name], tol[name], name)


# n, seqs, len, heads, kv_heads, dim, buckets, causal, p
SHAPES = [(1, 1, 1, 1, 1, 8, 1, True, 0.0), (1, 1, 1, 2, 1, 64, 32, True, 0.5), (2, 1, 5, 4, 4, 64, 32, True, 0.1), (1, 3, 31, 2, 2, 32, 8, False, 0.0),
          (2, 2, 33, 2, 1, 40, 9, True, 0.3), (1, 1, 64, 1, 1, 64, 0, False, 0.0), (1, 1, 65, 3, 3, 16, 5, False, 0.1), (1, 2, 127, 2, 2, 72, 32, True, 0.0),
          (1, 1, 128, 2, 1, 96, 17, False, 0.2), (1, 1, 129, 4, 2, 128, 32, True, 0.1), (3, 1, 200, 1, 1, 17, 64, False, 0.0), (1, 1, 333, 6, 2, 80, 33, True, 0.2),
          (1, 1, 515, 2, 2, 64, 32, True, 0.0), (1, 1, 700, 1, 1, 128, 12, False, 0.05), (1, 1, 260, 2, 2, 33, 300, False, 0.0)]


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_output_and_gradients(sams, kind, shape):
    n, seqs, length, heads, kv_heads, dim, buckets, causal, p = shape
    x = make(n, seqs * length, heads, kv_heads, dim, buckets, kind)
    starts = sams.relative_buckets(buckets, 100, causal) if buckets else []
    how = dict(seqs=seqs, causal=causal, p=p, rng=torch.tensor([12345678901234567, 3]) if p else None)
    compare(Run(sams, x, starts, heads, kv_heads, **how), x, starts, heads, kv_heads, **how)
