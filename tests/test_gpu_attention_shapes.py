"""Attention at shapes drawn anew: types, lengths, heads that share keys, widths of 8 to 128 columns, buckets near and far apart, padding, both passes, against
the formulas in 64 bits (tests/attention_oracle.py)."""
import random

import pytest
import torch

from tests.test_gpu_attention import TYPES, Run, compare, make, sams  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(36))
def test_drawn_shape(sams, seed):
    rng = random.Random(seed)
    kind = TYPES[seed % 3]
    n, seqs = rng.randint(1, 3), rng.randint(1, 4)
    length = rng.choice((rng.randint(1, 40), rng.randint(41, 140), rng.randint(141, 420)))
    kv_heads = rng.randint(1, 3)
    heads = kv_heads * rng.choice((1, 1, 2, 3, 5))
    dim = rng.choice((rng.randint(8, 128), 32, 64, 96, 128))
    causal, p = rng.random() < 0.5, rng.choice((0.0, rng.uniform(0.01, 0.6)))
    buckets = rng.choice((0, rng.randint(1, 40), rng.randint(41, 200)))
    if rng.random() < 0.3 and buckets:
        starts = sorted(rng.sample(range(-6000, 6000), buckets))             # most of them beyond any distance, the others anywhere
    else:
        starts = sams.relative_buckets(buckets, rng.choice((5, 64, 300)), causal) if buckets else []
    lengths = None
    if rng.random() < 0.5:
        lengths = torch.tensor([[rng.randint(0, length) for _ in range(seqs)] for _ in range(n)], dtype=torch.int32)
    print((n, seqs, length, heads, kv_heads, dim, buckets, causal, p, str(kind)), flush=True)
    x = make(n, seqs * length, heads, kv_heads, dim, buckets, kind, seed=seed)
    how = dict(seqs=seqs, causal=causal, p=p, lengths=lengths, rng=torch.tensor([seed * 0x9E3779B97F4A7C15 % 2 ** 63, seed]) if p else None)
    compare(Run(sams, x, starts, heads, kv_heads, **how), x, starts, heads, kv_heads, **how)


@pytest.mark.parametrize("length", [74, 420])
@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_no_bias(sams, kind, dim, p, length):
    # nothing is summed up for a bias between the blocks of queries: every column of dk and dv is still whole
    x = make(1, length, 2, 1, dim, 0, kind, seed=3)
    how = dict(seqs=1, causal=False, p=p, lengths=None, rng=torch.tensor([91, 4]) if p else None)
    compare(Run(sams, x, [], 2, 1, **how), x, [], 2, 1, **how)
