"""Attention and dropout with more workgroups than one launch takes (2^23): they go in several, and every one finds its rows."""
import pytest
import torch

from tests import philox
from tests.attention_oracle import check, formulas
from tests.test_gpu_attention import NAN, sams  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("buckets", [0, 3])
def test_attention_of_short_sequences_with_a_thousand_heads(sams, buckets):
    """8,201 sequences of two tokens, 1024 heads: the same 59 sequences over and over (139 times), so that all of them have the small call's bits; that one
    against the formulas, some heads of it."""
    heads, dim, few, times, length = 1024, 8, 59, 139, 2
    gen = torch.Generator().manual_seed(0)
    rand = lambda: torch.randn((1, few * length, heads * dim), generator=gen)
    x = {name: rand() for name in ("q", "k", "v", "do")}
    bias = 0.7 * torch.randn((heads, buckets), generator=gen) if buckets else None
    starts = [-1, 0, 1][:buckets]
    cuda = {name: v.cuda() for name, v in x.items()}

    def passes(repeats):
        y = {name: v.repeat(1, repeats, 1) for name, v in cuda.items()}
        t = few * length * repeats
        o, dq, dk, dv = (torch.full_like(y["q"], NAN) for _ in range(4))
        row_max, row_sum = torch.full((2, 1, heads, t), NAN, device="cuda")
        dbias = torch.full((1, heads, buckets), NAN, device="cuda") if buckets else None
        b = bias.cuda() if buckets else None
        how = dict(seqs=few * repeats, causal=False)
        with sams.Attention(1, t, heads, dim, starts=starts or None) as op:
            op.attention_forward(y["q"], y["k"], y["v"], b, o, row_max, row_sum, **how)
            op.attention_backward(y["do"], y["q"], y["k"], y["v"], b, o, row_max, row_sum, dq, dk, dv, dbias, **how)
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}, dbias

    assert few * times * heads > 2 ** 23
    small, small_bias = passes(1)
    large, large_bias = passes(times)
    for name, got in large.items():
        assert torch.equal(got.unflatten(1, (times, -1)), small[name][:, None].expand(-1, times, -1, -1)), name
    for h in (0, 1, 511, 1023):
        one = slice(h * dim, (h + 1) * dim)
        y = {name: v[..., one] for name, v in x.items()}
        want, tol = formulas(y["q"], y["k"], y["v"], bias[h:h + 1] if buckets else None, starts, y["do"], seqs=few, causal=False)
        for name, got in small.items():
            check(got[..., one], want[name], tol[name], (name, h))
        if buckets:
            check(small_bias[:, h:h + 1], want["dbias"], tol["dbias"], ("dbias", h))
            # the same terms 139 times: what each sum may be off by, and a rounding of the magnitudes' sum for every term that is added
            split = {name: v[0].double().unflatten(0, (few, length)) for name, v in y.items()}
            across = lambda m: m.transpose(1, 2).contiguous()
            places = torch.tensor([[1, 2], [0, 1]])
            P = torch.softmax(dim ** -0.5 * (split["q"] @ across(split["k"])) + bias[h].double()[places], 2)
            dP = split["do"] @ across(split["v"])
            dS = (P * (dP - (P * dP).sum(2, keepdim=True))).abs().sum(0)
            size = torch.stack([dS[places == b].sum() for b in range(3)])
            check(large_bias[:, h:h + 1], times * want["dbias"], times * (tol["dbias"] + 2.0 ** -24 * (2 * few * times + 72) * size), ("dbias of all", h))


def test_dropout_of_2_to_the_28_rows(sams):
    """2^31 pieces of 8 columns are 2^23 workgroups; these are a quarter more."""
    t, dim, p, kind = 2 ** 28, 73, 0.3, torch.bfloat16
    row = torch.arange(1, dim + 1, device="cuda").to(kind)
    x = row.expand(1, t, dim)                                       # one row for all
    y = torch.full((1, t, dim), NAN, dtype=kind, device="cuda")
    rng = torch.tensor([21, 22])
    with sams.Dropout(1, t, dim, kind) as op:
        op.dropout_forward(x, None, rng.cuda(), p, y)
    share = 1 - philox.least(p) / 65536
    kept = row.double() / share
    near = kept * (2.0 ** -8 + 2.0 ** -22)                          # rounded to 8 bits; its reciprocal and the product to 32 before
    for first in (0, 2 ** 27 - 9, 2 ** 31 // 10 - 1000, t - 2000):
        part = y[0, first:first + 2000]
        keep = torch.from_numpy(philox.numbers(21, 22, torch.arange((dim + 7) // 8).numpy(), torch.arange(first, first + 2000)[:, None].numpy(), 0)).reshape(2000, -1)[:, :dim]
        keep = (keep >= philox.least(p)).cuda()
        assert torch.equal(part != 0, keep), first
        assert ((part.double() - kept).abs() <= near)[keep].all(), first
    for first in range(0, t, 2 ** 25):
        count = (y[0, first:first + 2 ** 25] != 0).sum(0).double()
        assert ((count / 2 ** 25 - share).abs() < 7 * (share * (1 - share) / 2 ** 25) ** 0.5).all(), first
