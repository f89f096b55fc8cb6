"""Attention where logits are so large that 32 bits of one have no place left for the products beside a bias, or a mask's lowest value is all that a
row has: the output, the row statistics and the gradients of every type.

A bias of 1e7 or more takes the rest of its logit in (products here are below 1.3, less than half of what a logit of 3e7 moves by), so that a row's weights go
by its largest bias: equal ones for the keys that have it where it is that large, the softmax of the others' logits where it is a usual
number.  Tolerances are those of tests/attention_oracle.py with an error of logits, es, only for keys that have a weight: 0 where it is a row's largest
bias alone, which all its keys have in the same 32 bits."""
import pytest
import torch

from tests import philox
from tests.attention_oracle import HALF_ULP, U, bucket_of, check, rounded
from tests.test_gpu_attention import TYPES, Run, make, sams  # noqa: F401

pytestmark = pytest.mark.gpu

LARGE = 1e7
LOWEST = torch.finfo(torch.float32).min


def expected(x, starts, heads, kv_heads, causal=True, lengths=None, p=0.0, rng=None, scale=None):
    """Outputs, gradients and sums of exponentials of one sequence a worker, what each may be off by, and the magnitudes that it is summed up from."""
    kind, (n, t, wide) = x["q"].dtype, x["q"].shape
    dim, group = wide // heads, heads // kv_heads
    scale = dim ** -0.5 if scale is None else scale
    word, tiny = (0.0 if kind == torch.float32 else HALF_ULP[kind]), 2.0 ** -38 if kind == torch.float16 else 0.0
    split = lambda v, h: v.double().unflatten(2, (h, dim)).transpose(1, 2)                  # [n][heads][t][dim]
    q, do = split(x["q"], heads), split(x["do"], heads)
    k, v = (split(x[name], kv_heads).repeat_interleave(group, 1).contiguous() for name in ("k", "v"))
    across = lambda m: m.transpose(-1, -2).contiguous()
    length = torch.full((n,), t) if lengths is None else lengths[:, 0].long().clamp(0, t)
    inside = torch.arange(t)[None, :] < length[:, None]
    allowed = inside[:, None, :, None] & inside[:, None, None, :]
    if causal:
        allowed = allowed & torch.ones(t, t, dtype=torch.bool).tril()
    products = scale * (q @ across(k))
    b = x["bias"].double()[:, bucket_of(starts, t)][None] if starts else torch.zeros(1, heads, t, t, dtype=torch.float64)
    most = torch.where(allowed, b, -torch.inf).amax(3, keepdim=True)
    ruled = most.abs() >= LARGE                                                             # rows that one bias rules
    near = b.abs() < LARGE
    assert not starts or float(products.abs().max()) < 1.3
    live = allowed & torch.where(ruled, b == most, near)
    logits = torch.where(live, torch.where(ruled, 0.0, products + b), -torch.inf)
    top = logits.amax(3, keepdim=True)
    E = torch.where(live, torch.exp(logits - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
    sums = E.sum(3, keepdim=True)
    P = E / sums.clamp(min=1e-300)
    usual = live & ~ruled
    es = torch.where(usual, (dim + 4) * U * abs(scale) * (q.abs() @ across(k.abs())) + 4 * U * (torch.where(usual, logits.abs() + b.abs(), 0.0) + torch.where(usual, top.abs(), 0.0)), 0.0)
    ep = es + es.amax(3, keepdim=True) + (t + 24) * U
    more = word + (t + 24) * U
    m = torch.ones(n, heads, t, t, dtype=torch.float64)
    if p:
        m = torch.from_numpy(philox.keep_pairs(rng, torch.arange(n * heads).numpy(), t, p)).double().reshape(n, heads, t, t) / (1 - philox.least(p) / 65536)
    share = 1 - philox.least(p) / 65536
    PD = P * m
    o = PD @ v
    some = live.any(3, keepdim=True)
    eo = (PD * (ep + more)) @ v.abs() + torch.where(some, tiny * v.abs().sum(2, keepdim=True) / share, 0.0)
    ro = rounded(o, eo, kind)
    dP = (do @ across(v)) * m
    delta = (P * dP).sum(3, keepdim=True)
    dS = P * (dP - delta)
    edp = (dim + 4) * U * m * (do.abs() @ across(v.abs()))
    ed = (P * (edp + dP.abs() * (ep + (t + 4) * U))).sum(3, keepdim=True)
    eds = P * (edp + ed) + dS.abs() * (ep + 4 * U)
    ew = eds + dS.abs() * more
    # the rounding of do . o is taken back at the end by sum P k, whose P's are words
    back = more * (do.abs() * ro).sum(3, keepdim=True)
    joined = lambda w: w.unflatten(1, (kv_heads, group)).sum(2)
    rows = lambda w: w.transpose(1, 2).reshape(n, t, -1)
    want, tol = {"o": rows(o), "dq": rows(scale * (dS @ k)), "dk": rows(joined(scale * (across(dS) @ q))), "dv": rows(joined(across(PD) @ do))}, {"o": rows(ro)}
    tol["dq"] = rows(abs(scale) * (back * (P @ k.abs()) + (ew + back * P + tiny * dS.abs().amax(3, keepdim=True)) @ k.abs()))
    tol["dk"] = rows(joined(abs(scale) * (across(ew + tiny * dS.abs().amax(2, keepdim=True)) @ q.abs()))) * (1 + group * U)
    tol["dv"] = rows(joined(across(PD * (ep + more)) @ do.abs() + tiny * do.abs().sum(2, keepdim=True) / share)) * (1 + group * U)
    for name in ("dq", "dk", "dv"):
        tol[name] = rounded(want[name], tol[name], kind)
    if starts:
        which = torch.nn.functional.one_hot(bucket_of(starts, t), len(starts)).double()
        want["dbias"] = torch.tensordot(dS, which, 2)
        count = which.sum((0, 1))
        tol["dbias"] = rounded(want["dbias"], torch.tensordot(eds, which, 2) + torch.tensordot(dS.abs(), which, 2) * (count + 72) * U, torch.float32)
    want["row_sum"], tol["row_sum"] = sums[..., 0], sums[..., 0] * (ep.amax(3) + (t + 24) * U)
    sd = P * (dP.abs() + delta.abs())
    size = {"o": rows(PD @ v.abs()), "dq": rows(abs(scale) * (sd @ k.abs())), "dk": rows(joined(abs(scale) * (across(sd) @ q.abs()))), "dv": rows(joined(across(PD) @ do.abs())),
            "row_sum": want["row_sum"]}
    if starts:
        size["dbias"] = torch.tensordot(sd, which, 2)
    return want, tol, size


def compare(got, want, tol, size, name):
    """The tolerance is one that only right numbers keep to: 1 % of the magnitudes that a number is summed up from at most."""
    assert float(tol[name].max()) <= 0.01 * float(size[name].max()), name
    check(got, want[name], tol[name], name)


# n, t, heads, kv_heads, dim: two wavefronts for 32 rows, and one (enough workgroups for that)
SIZES = [(1, 130, 2, 1, 64), (1, 50, 2, 2, 40), (2, 130, 104, 52, 16)]
# The bias's large buckets, of distances up to -9, from -8 on to -1, 0 and above: a first row, or the first rows, without another key, tiles of mixed buckets
# and of one, every row
WHERE = {"own": [2], "near": [1, 2], "far": [0], "all": [0, 1, 2, 3]}


def inputs(kind, size, buckets, low):
    n, t, heads, kv_heads, dim = size
    x = make(n, t, heads, kv_heads, dim, 4, kind, seed=5)
    x["q"] = (x["q"].clamp(-3, 3) * 0.125).to(kind)
    x["k"] = x["k"].clamp(-2, 2)
    x["bias"][:, buckets] = low
    return x, [-(2 ** 31), -8, 0, 1]


@pytest.mark.parametrize("low", [-3e7, -5e7, -1e8, -1e9, LOWEST, 3e7, 1e9], ids=str)
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_output_beside_large_biases(sams, kind, size, where, low):
    x, starts = inputs(kind, size, WHERE[where], low)
    n, t, heads, kv_heads, dim = size
    for causal in (True, False):
        run = Run(sams, x, starts, heads, kv_heads, train=False, causal=causal)
        right = expected(x, starts, heads, kv_heads, causal)
        for name, got in (("row_sum", run.row_sum), ("o", run.o)):
            compare(got, *right, name)


@pytest.mark.parametrize("low", [-3e7, -1e8, -1e9, LOWEST, 3e7], ids=str)
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_gradients_beside_large_biases(sams, kind, size, where, low):
    x, starts = inputs(kind, size, WHERE[where], low)
    n, t, heads, kv_heads, dim = size
    lengths = torch.full((n, 1), t - 3, dtype=torch.int32)
    for how in (dict(causal=True), dict(causal=False, p=0.2, rng=torch.tensor([11, 12]), lengths=lengths)):
        run = Run(sams, x, starts, heads, kv_heads, **how)
        right = expected(x, starts, heads, kv_heads, **how)
        for name, got in run.outputs().items():
            compare(got, *right, name)


def signs(size, kind, by):
    """Queries and keys of plus or minus `by`, a row's query like its key, no two rows of a head alike."""
    n, t, heads, dim = size
    gen = torch.Generator().manual_seed(t + dim)
    rows = torch.randint(0, 2, (n, t, heads, dim), generator=gen) * 2 - 1
    if dim < 64:                                                    # by the bits of the row's number
        bits = torch.arange(t)[:, None] >> torch.arange(8)[None, :] & 1
        rows[..., :8] = (bits * 2 - 1)[None, :, None, :]
    x = make(n, t, heads, heads, dim, 0, kind, seed=2)
    x["q"] = (rows * by).reshape(n, t, heads * dim).to(kind)
    x["k"] = x["q"].clone()
    return x


# n, t, heads, dim: tiles of 32 or 64 keys inside the sequence, and such as reach past its end
@pytest.mark.parametrize("size", [(1, 192, 2, 64), (1, 100, 1, 128), (1, 128, 3, 16), (2, 128, 200, 8)], ids=str)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_large_products(sams, kind, causal, size):
    """Rows whose own key's logit is 2^28 (16-bit floats) or 2^38, and the other keys' are 2^25 or 2^35 lower at least: all weight on the own key, whatever
    32 bits make of such a logit.  Products are whole multiples of a power of two that 32 bits hold."""
    n, t, heads, dim = size
    size_of = 2.0 ** 11 if kind == torch.float16 else 2.0 ** 16
    x = signs(size, kind, size_of)
    how = dict(causal=causal, scale=64.0 / dim)
    run = Run(sams, x, [], heads, heads, **how)
    assert torch.equal(run.row_sum, torch.ones_like(run.row_sum))
    assert torch.equal(run.o.cpu(), x["v"])
    assert torch.equal(run.dv.cpu(), x["do"])
    # dS is 0 in 64 bits; in 32, what the sums do . v, made twice, are off by from one another, times the row's own key
    slack = (dim + 4) * U * (x["do"].double() * x["v"].double()).abs().reshape(n, t, heads, dim).sum(-1, keepdim=True)
    slack = (2 * how["scale"] * size_of * slack).expand(-1, -1, -1, dim).reshape(n, t, -1)
    word = 0.0 if kind == torch.float32 else HALF_ULP[kind]
    for got in (run.dq, run.dk):
        check(got, torch.zeros_like(slack), slack * (1 + 2 * word) + 2.0 ** -25, "a row's own key")


@pytest.mark.parametrize("power", [2, 3, 4, 6, 8])
@pytest.mark.parametrize("size", [(1, 192, 2, 64), (1, 100, 1, 128), (2, 128, 200, 8)], ids=str)
@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_products_that_leave_few_bits(sams, kind, size, power):
    """Logits from 2^10 to 2^22, the other keys' an eighth lower at least: the forward pass and the backward one agree on the weight, whatever
    of the largest logit is rounded away.  A word's rounding of P and an output's, and sixteen of 32 bits."""
    n, t, heads, dim = size
    x = signs(size, kind, 2.0 ** power)
    for causal in (True, False):
        run = Run(sams, x, [], heads, heads, causal=causal, scale=64.0 / dim)
        for got, name in ((run.o, "v"), (run.dv, "do")):
            want = x[name].double()
            check(got, want, want.abs() * (2 * HALF_ULP[kind] + 16 * U) + 2.0 ** -25, (name, causal))


# n, t, heads, dim
@pytest.mark.parametrize("size", [(1, 137, 3, 64), (1, 300, 2, 96), (1, 70, 4, 113), (2, 130, 104, 16)], ids=str)
@pytest.mark.parametrize("scale", [1.0, 0.3, -0.5, -1.0])
@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_large_products_of_any_number(sams, kind, scale, size):
    """Logits of 1e7 and more that 32 bits hold to whole numbers or hundreds: which of two near ones is larger is left to rounding, but every kernel has to see it alike.
    A weight is at most 1 and a row's sum to 1, so that o is at most the largest v, a key's dv the sum of all rows' do, dS of a row P (|dP| + |delta|) with P summing to 1; and
    where one logit is above all others by more than its roundings, o is that key's v."""
    n, t, heads, dim = size
    x = make(n, t, heads, heads, dim, 0, kind, seed=8)
    for name in ("q", "k"):
        x[name] = (x[name].clamp(-4, 4) * (4000 if kind == torch.float16 else 1e6)).to(kind)
    run = Run(sams, x, [], heads, heads, scale=scale, causal=False)
    q, k, v, do = (x[name].double().unflatten(2, (heads, dim)).transpose(1, 2) for name in ("q", "k", "v", "do"))
    across = lambda m: m.transpose(-1, -2).contiguous()
    o, dq, dk, dv = (got.cpu().double().unflatten(2, (heads, dim)).transpose(1, 2) for got in (run.o, run.dq, run.dk, run.dv))
    assert all(bool(torch.isfinite(got).all()) for got in (o, dq, dk, dv))
    sums = run.row_sum.cpu()
    assert (sums >= 1).all() and (sums <= t).all()
    # a word's rounding of P and of dS each, an output's, and a rounding of 32 bits for each number of a sum
    word = HALF_ULP[kind] if kind != torch.float32 else U
    more = 1 + 4 * word + 4 * (t + dim) * U
    assert (o.abs() <= v.abs().amax(2, keepdim=True) * more).all()
    assert (dv.abs() <= do.abs().sum(2, keepdim=True) * more).all()
    most = (do.abs() @ across(v.abs())).amax(3)                                             # of |dP| and |delta| in a row
    assert (dq.abs() <= abs(scale) * 2 * most[..., None] * k.abs().amax(2, keepdim=True) * more).all()
    assert (dk.abs() <= abs(scale) * (2 * most[..., None] * q.abs()).sum(2, keepdim=True) * more).all()
    logits = scale * (q @ across(k))
    top, which = logits.max(3)
    below = logits.scatter(3, which[..., None], -torch.inf).amax(3)
    off = 2 * abs(scale) * ((dim + 8) * U * (q.abs() @ across(k.abs()))).amax(3)             # (dim + 4) roundings of a product and four of the logit, two logits
    sure = top - below > off + 120                                                          # e^-120 is no number beside 1, in any type
    assert float(sure.double().mean()) > 0.9
    assert torch.equal(o[sure], v.gather(2, which[..., None].expand(-1, -1, -1, dim))[sure])
