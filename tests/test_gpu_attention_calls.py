"""Calls of the attention that its documentation allows: padded and empty sequences, buckets of all kinds, masks that leave nothing, tensors as they
lie, other streams, graphs, many sequences, and gradients against differences.  Tolerances: tests/attention_oracle.py."""
import pytest
import torch

from tests.attention_oracle import check, formulas
from tests.test_gpu_attention import NAN, TYPES, Run, compare, make, sams  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_padding_changes_nothing_and_gets_nothing(sams, kind, causal):
    n, seqs, length, heads, kv_heads, dim = 2, 4, 150, 4, 2, 48
    x = make(n, seqs * length, heads, kv_heads, dim, 9, kind)
    starts = sams.relative_buckets(9, 40, causal)
    given = torch.tensor([[150, 0, 1, 77], [64, 149, -5, 1000]], dtype=torch.int32)             # what lies outside 0 .. 150 is taken to the nearer end
    real = given.clamp(0, length)
    how = dict(seqs=seqs, causal=causal, p=0.2, rng=torch.tensor([3, 4]))
    runs = []
    for fill in (0.0, NAN, float("inf")):
        y = dict(x)
        pad = (torch.arange(length)[None, None, :] >= real[:, :, None]).reshape(n, seqs * length)
        for name in ("q", "k", "v", "do"):
            y[name] = torch.where(pad[..., None], torch.tensor(fill, dtype=kind), x[name])
        runs.append(Run(sams, y, starts, heads, kv_heads, lengths=given, **how))
        for name in ("o", "dq", "dk", "dv"):
            assert (runs[-1].outputs()[name][pad.cuda()] == 0).all(), name
    compare(runs[0], x, starts, heads, kv_heads, lengths=real, **how)
    for other in runs[1:]:
        for name, got in other.outputs().items():
            assert torch.equal(got, runs[0].outputs()[name]), name


@pytest.mark.parametrize("starts", [[0], [-7], [-5, 0], [-100000, -90000, -3, 0, 2, 90000], [-60000, -50, -49, 0, 70000], list(range(-200, 312)), [5, 6, 7], [-(2 ** 31), 2 ** 31 - 1],
                                    [-(2 ** 31), -(2 ** 31) + 1, 0]], ids=lambda v: f"{len(v)} from {v[0]}")
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16], ids=str)
def test_buckets(sams, kind, starts):
    """One bucket, buckets that no pair reaches, distances by table and (far apart) by search, as many buckets as there may be."""
    for causal in (True, False):
        x = make(1, 230, 2, 2, 32, len(starts), kind)
        compare(Run(sams, x, starts, 2, 2, causal=causal), x, starts, 2, 2, causal=causal)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_banned_distances(sams, kind):
    """A bias of minus infinity: keys without weight, rows without keys (0, with gradients 0), and tiles that nothing is read for."""
    length, heads = 300, 2
    starts = [-(2 ** 31), -39, 0, 1]                       # far back, the 39 before, the query itself, behind it
    x = make(1, length, heads, heads, 64, 4, kind)
    x["bias"][:, 0] = -torch.inf
    x["bias"][0, 3] = -torch.inf
    x["bias"][1, 2] = -torch.inf
    for causal in (True, False):
        compare(Run(sams, x, starts, heads, heads, causal=causal), x, starts, heads, heads, causal=causal)
    x["bias"][1, 1:] = -torch.inf                           # nothing left for the second head
    for causal in (True, False):
        run = Run(sams, x, starts, heads, heads, causal=causal)
        compare(run, x, starts, heads, heads, causal=causal)
        for v in (run.o, run.dq, run.dk, run.dv):
            assert (v.unflatten(2, (heads, 64))[:, :, 1] == 0).all()
        assert (run.dbias[:, 1] == 0).all()


@pytest.mark.parametrize("low", [-1e9, torch.finfo(torch.float32).min])
def test_large_negative_biases(sams, low):
    """As masks have them: no weight beside other keys.  Where a row has nothing else and the type's lowest value swallows the products, all its keys
    weigh the same, in the gradients too."""
    starts = [-(2 ** 31), -9, 1]
    x = make(1, 200, 1, 1, 32, 3, torch.float32)
    x["bias"][:, 0] = low
    compare(Run(sams, x, starts, 1, 1, causal=True), x, starts, 1, 1, causal=True)
    if low < -1e30:
        x["bias"][:] = low
        run = Run(sams, x, starts, 1, 1, causal=True)
        v = x["v"][0].double()
        mean = v.cumsum(0) / torch.arange(1, 201)[:, None]
        check(run.o[0], mean, 2.0 ** -15 * v.abs().amax().expand_as(mean), "mean")     # 200 weights of 2^-24's and 230 roundings of a sum
        P = torch.ones(200, 200).tril().double() / torch.arange(1, 201)[:, None]
        want = P.t() @ x["do"][0].double()
        check(run.dv[0], want, 2.0 ** -15 * (P.t() @ x["do"][0].double().abs()), "dv")


@pytest.mark.parametrize("kind", TYPES, ids=str)
@pytest.mark.parametrize("scale", [0.0, -0.7, 3.0])
def test_scales(sams, kind, scale):
    x = make(2, 100, 2, 1, 24, 5, kind)
    starts = sams.relative_buckets(5, 30)
    compare(Run(sams, x, starts, 2, 1, scale=scale), x, starts, 2, 1, scale=scale)


def test_sharp_rows(sams):
    """Rows whose weight lies on one key: dq and dk, differences of nearly equal numbers, keep to what their words' rounding gives."""
    for kind in TYPES:
        x = make(1, 190, 2, 2, 64, 4, kind)
        x["q"] = (x["q"].float() * 6).to(kind)
        starts = sams.relative_buckets(4, 20)
        compare(Run(sams, x, starts, 2, 2), x, starts, 2, 2)


def test_small_gradients_of_16_bit_floats(sams):
    """Gradients far below 2^-14 keep their digits between the products, and only the outputs' own smallest numbers limit them."""
    x = make(1, 300, 2, 1, 64, 8, torch.float16)
    x["do"] = (x["do"].float() * 2.0 ** -9).half()
    x["v"] = (x["v"].float() * 64).half()
    starts = sams.relative_buckets(8, 100)
    compare(Run(sams, x, starts, 2, 1), x, starts, 2, 1)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_tensors_as_they_lie(sams, kind):
    """Parts of one projection's rows at any element, tokens before workers, the bias's gradient added up in rows of a flat vector; nothing beside them is written."""
    n, t, heads, kv_heads, dim = 3, 90, 4, 2, 44
    x = make(n, t, heads, kv_heads, dim, 6, kind)
    starts = sams.relative_buckets(6, 30)
    wide, narrow = heads * dim, kv_heads * dim
    full = wide + 2 * narrow + 7
    packed = torch.full((t, n, full), NAN, dtype=kind, device="cuda").transpose(0, 1)
    grads = torch.full((n, t, full), 9.0, dtype=kind, device="cuda")
    cut = lambda v: (v[..., 1:1 + wide], v[..., 1 + wide:1 + wide + narrow], v[..., 1 + wide + narrow:1 + wide + 2 * narrow])
    q, k, v = cut(packed)
    for to, name in ((q, "q"), (k, "k"), (v, "v")):
        to.copy_(x[name])
    o = torch.full((n, t, wide + 3), 9.0, dtype=kind, device="cuda")
    do = torch.full((n, t, wide + 1), NAN, dtype=kind, device="cuda")
    do[..., 1:].copy_(x["do"])
    flat = torch.full((n, 5 + heads * 6 + 2), 0.25, device="cuda")
    dbias = flat[:, 5:5 + heads * 6].unflatten(1, (heads, 6))
    row_max, row_sum = torch.empty((2, n, heads, t), device="cuda")
    bias = x["bias"].cuda()
    with sams.Attention(n, t, heads, dim, kv_heads, starts=starts, dtype=kind) as op:
        op.attention_forward(q, k, v, bias, o[..., 2:2 + wide], row_max, row_sum)
        op.attention_backward(do[..., 1:], q, k, v, bias, o[..., 2:2 + wide], row_max, row_sum, *cut(grads), dbias, accumulate=True)
    want, tol = formulas(x["q"], x["k"], x["v"], x["bias"], starts, x["do"], heads=heads, kv_heads=kv_heads)
    check(o[..., 2:2 + wide], want["o"], tol["o"], "o")
    for got, name in zip(cut(grads), ("dq", "dk", "dv")):
        check(got, want[name], tol[name], name)
    check(dbias, want["dbias"] + 0.25, tol["dbias"] + 2.0 ** -24 * (0.25 + want["dbias"].abs()), "dbias")
    assert (flat[:, :5] == 0.25).all() and (flat[:, -2:] == 0.25).all() and (o[..., :2] == 9).all() and (o[..., -1] == 9).all()
    assert (grads[..., 0] == 9).all() and (grads[..., 1 + wide + 2 * narrow:] == 9).all()


def test_inputs_that_overlap_themselves(sams):
    """Keys and values of one worker for all (distance 0)."""
    n, t, heads, dim = 3, 70, 2, 32
    x = make(n, t, heads, heads, dim, 0, torch.float32)
    for name in ("k", "v"):
        x[name] = x[name][:1].expand(n, -1, -1)
    cuda = {name: v.cuda() for name, v in x.items() if v is not None}
    cuda["k"], cuda["v"] = (x[name][:1].cuda().expand(n, -1, -1) for name in ("k", "v"))
    o = torch.empty_like(cuda["q"])
    row_max, row_sum = torch.empty((2, n, heads, t), device="cuda")
    with sams.Attention(n, t, heads, dim) as op:
        op.attention_forward(cuda["q"], cuda["k"], cuda["v"], None, o, row_max, row_sum)
    want, tol = formulas(x["q"], x["k"], x["v"], None, None, heads=heads, kv_heads=heads)
    check(o, want["o"], tol["o"], "o")


def test_many_short_sequences(sams):
    """More sequences than the scratch has room for at a time: the bias's gradient in several launches, added up."""
    n, seqs, length, heads = 2, 400, 3, 2
    x = make(n, seqs * length, heads, 1, 16, 5, torch.float32)
    starts = sams.relative_buckets(5, 4, False)
    for accumulate in (False, True):
        into = torch.full((n, heads, 5), 2.0, device="cuda")
        run = Run(sams, x, starts, heads, 1, seqs=seqs, causal=False, accumulate=accumulate, into=into)
        want, tol = formulas(x["q"], x["k"], x["v"], x["bias"], starts, x["do"], heads=heads, kv_heads=1, seqs=seqs, causal=False)
        if accumulate:
            want["dbias"] = want["dbias"] + 2
            tol["dbias"] = tol["dbias"] + 8 * 2.0 ** -24 * (2 + want["dbias"].abs())
        for name, got in run.outputs().items():
            check(got, want[name], tol[name], name)


@pytest.mark.parametrize("kind", TYPES, ids=str)
def test_pieces_of_the_keys_sums(sams, kind):
    """A group's heads, and a head's queries, shared out to several workgroups; equal results however often it is done."""
    for n, length, heads, kv_heads, dim, causal in ((1, 1100, 6, 1, 64, True), (1, 1400, 1, 1, 64, False), (2, 130, 12, 2, 128, False), (1, 1300, 4, 2, 24, True)):
        x = make(n, length, heads, kv_heads, dim, 7, kind)
        starts = sams.relative_buckets(7, 64, causal)
        with sams.Attention(n, length, heads, dim, kv_heads, starts=starts, dtype=kind) as op:
            first = Run(sams, x, starts, heads, kv_heads, op=op, causal=causal, p=0.1, rng=torch.tensor([1, 2]))
            again = Run(sams, x, starts, heads, kv_heads, op=op, causal=causal, p=0.1, rng=torch.tensor([1, 2]))
        compare(first, x, starts, heads, kv_heads, causal=causal, p=0.1, rng=torch.tensor([1, 2]))
        for name, got in first.outputs().items():
            assert torch.equal(got, again.outputs()[name]), name


def test_gradients_against_differences(sams):
    """<gradient, direction> against the difference quotient of sum(o * r) in 64 bits; its error is O(h^2) and 64-bit rounding / h."""
    n, seqs, length, heads, kv_heads, dim, h = 1, 2, 37, 4, 2, 24, 1e-4
    x = make(n, seqs * length, heads, kv_heads, dim, 6, torch.float32)
    starts = sams.relative_buckets(6, 20)
    how = dict(seqs=seqs, lengths=torch.tensor([[37, 20]], dtype=torch.int32), p=0.25, rng=torch.tensor([8, 9]))
    run = Run(sams, x, starts, heads, kv_heads, **how)
    gen = torch.Generator().manual_seed(1)
    move = {name: torch.randn(x[name].shape, generator=gen).double() for name in ("q", "k", "v", "bias")}

    def value(s):
        y = {name: x[name].double() + s * move[name] for name in move}
        o = formulas64(y["q"], y["k"], y["v"], y["bias"], starts, heads, kv_heads, **how)
        return float((o * x["do"].double()).sum())

    quotient = (value(h) - value(-h)) / (2 * h)
    terms = [(got.cpu().double() * move[name]) for name, got in (("q", run.dq), ("k", run.dk), ("v", run.dv))] + [run.dbias[0].cpu().double() * move["bias"]]
    dot = sum(float(v.sum()) for v in terms)
    assert abs(dot - quotient) <= 1e-5 * sum(float(v.abs().sum()) for v in terms)


def formulas64(q, k, v, bias, starts, heads, kv_heads, seqs, lengths, p, rng):
    """The output alone, of 64-bit inputs (which the formulas take to be of the type whose rounding they count)."""
    return formulas(q, k, v, bias, starts, heads=heads, kv_heads=kv_heads, seqs=seqs, lengths=lengths, p=p, rng=rng, kind=torch.float32)[0]["o"]


def test_no_tokens(sams):
    e, s = torch.empty((3, 0, 32), device="cuda"), torch.empty((3, 2, 0), device="cuda")
    dbias = torch.full((3, 2, 4), 7.0, device="cuda")
    bias = torch.zeros((2, 4), device="cuda")
    with sams.Attention(3, 4, 2, 16, starts=[0, 1, 2, 3]) as op:
        op.attention_forward(e, e, e, bias, e, s, s)
        op.attention_backward(e, e, e, e, bias, e, s, s, e, e, e, dbias, accumulate=True)
        assert (dbias == 7).all()
        op.attention_backward(e, e, e, e, bias, e, s, s, e, e, e, dbias)
        assert (dbias == 0).all()
    with sams.Attention(1, 0, 1, 8) as op:
        e, s = torch.empty((1, 0, 8), device="cuda"), torch.empty((1, 1, 0), device="cuda")
        op.attention_forward(e, e, e, None, e, s, s)


def test_without_the_biases_gradient_or_training(sams):
    x = make(2, 150, 2, 2, 64, 8, torch.bfloat16)
    starts = sams.relative_buckets(8, 30)
    full = Run(sams, x, starts, 2, 2)
    cuda = {name: v.cuda() for name, v in x.items()}
    with sams.Attention(2, 150, 2, 64, starts=starts, dtype=torch.bfloat16) as op:
        dq, dk, dv = (torch.empty_like(cuda[name]) for name in ("q", "k", "v"))
        op.attention_backward(cuda["do"], cuda["q"], cuda["k"], cuda["v"], cuda["bias"], full.o, full.row_max, full.row_sum, dq, dk, dv)
    for a, b in ((dq, full.dq), (dk, full.dk), (dv, full.dv)):
        assert torch.equal(a, b)
    with sams.Attention(2, 150, 2, 64, starts=starts, dtype=torch.bfloat16, train=False) as op:
        o = torch.empty_like(cuda["q"])
        row_max, row_sum = torch.empty((2, 2, 2, 150), device="cuda")
        op.attention_forward(cuda["q"], cuda["k"], cuda["v"], cuda["bias"], o, row_max, row_sum)
        assert torch.equal(o, full.o)
        with pytest.raises(sams.SamsError):
            op.attention_backward(cuda["do"], cuda["q"], cuda["k"], cuda["v"], cuda["bias"], o, row_max, row_sum, dq, dk, dv)


def test_on_any_stream_and_in_graphs(sams):
    """A step with dropout of hidden states, layer norm, attention and its residual, captured twice with contexts of their own and the steps raised
    inside; replays, with eager work between them and both graphs in turn, equal the eager calls of the same step."""
    n, t, heads, dim = 2, 140, 4, 32
    wide = heads * dim
    starts = sams.relative_buckets(8, 60)
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    class Step:
        def __init__(self):
            self.attn, self.norm, self.drop = sams.Attention(n, t, heads, dim, starts=starts), sams.LayerNorm(n, t, wide), sams.Dropout(n, t, wide)
            self.x, self.weight, self.bias, self.do = rand(n, t, wide), 1 + 0.1 * rand(wide), rand(heads, 8), rand(n, t, wide)
            self.rng = torch.tensor([[5, 0], [6, 0]], device="cuda")
            self.y, self.o, self.out, self.d1, self.dq, self.dk, self.dv = (torch.empty_like(self.x) for _ in range(7))
            self.mean, self.rstd = torch.empty((2, n, t), device="cuda")
            self.row_max, self.row_sum = torch.empty((2, n, heads, t), device="cuda")
            self.dbias = torch.empty((n, heads, 8), device="cuda")

        def calls(self):
            self.norm.layer_norm_forward(self.x, self.weight, None, self.y, self.mean, self.rstd)
            how = dict(rng=self.rng[0], p=0.1)
            self.attn.attention_forward(self.y, self.y, self.y, self.bias, self.o, self.row_max, self.row_sum, **how)
            self.drop.dropout_forward(self.o, self.x, self.rng[1], 0.2, self.out)
            self.drop.dropout_backward(self.do, self.rng[1], 0.2, self.d1)
            self.attn.attention_backward(self.d1, self.y, self.y, self.y, self.bias, self.o, self.row_max, self.row_sum, self.dq, self.dk, self.dv, self.dbias, **how)
            self.rng[:, 1] += 1

        def results(self):
            return [v.clone() for v in (self.y, self.o, self.out, self.d1, self.dq, self.dk, self.dv, self.dbias)]

    with torch.cuda.stream(stream):
        steps = [Step(), Step()]
        for s in steps:
            s.calls()
        torch.cuda.synchronize()
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        for s, graph in zip(steps, graphs):
            with torch.cuda.graph(graph, stream=stream):
                s.calls()
        seen = []
        for turn in range(3):
            for s, graph in zip(steps, graphs):
                s.x.copy_(rand(n, t, wide))
                at = s.rng.clone()
                graph.replay()
                torch.cuda.synchronize()
                got = s.results()
                s.rng.copy_(at)
                for v in (s.y, s.o, s.out, s.d1, s.dq, s.dk, s.dv, s.dbias):
                    v.fill_(NAN)
                s.calls()
                torch.cuda.synchronize()
                for a, b in zip(got, s.results()):
                    assert torch.equal(a, b)
                seen.append(got[2])
        # without either graph, from another stream: it waits for what was made there, and what follows there waits for it
        other = torch.cuda.Stream()
        s = steps[0]
        s.rng[:, 1] -= 1
        with torch.cuda.stream(other):
            other.wait_stream(stream)
            s.x.mul_(1.0)
            for v in (s.o, s.dbias):
                v.zero_()
            s.calls()
            after = [v.clone() for v in (s.o, s.dbias)]
        torch.cuda.synchronize()
        assert all(torch.isfinite(v).all() and (v != 0).any() for v in after)


def test_long_offsets(sams):
    """Rows so far apart that offsets pass 2^32 bytes; only the rows themselves are touched."""
    n, t, heads, dim = 1, 70, 1, 64
    row = 2 ** 26
    x = make(n, t, heads, heads, dim, 0, torch.bfloat16)
    room = torch.zeros(((t - 1) * row + 4 * dim,), dtype=torch.bfloat16, device="cuda")
    views = [torch.as_strided(room, (1, t, dim), (t * row, row, 1), i * dim) for i in range(4)]
    for v, name in zip(views, ("q", "k", "v")):
        v.copy_(x[name])
    row_max, row_sum = torch.empty((2, n, heads, t), device="cuda")
    dq, dk = torch.empty((2, n, t, dim), dtype=torch.bfloat16, device="cuda")
    with sams.Attention(n, t, heads, dim, dtype=torch.bfloat16) as op:
        op.attention_forward(*views[:3], None, views[3], row_max, row_sum)
        o = views[3].clone()
        op.attention_backward(x["do"].cuda(), *views[:3], None, o, row_max, row_sum, dq, dk, views[3])
    want, tol = formulas(x["q"], x["k"], x["v"], None, None, x["do"])
    for got, name in ((o, "o"), (dq, "dq"), (dk, "dk"), (views[3], "dv")):
        check(got, want[name], tol[name], name)
