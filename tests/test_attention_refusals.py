"""What dropout and the attention refuse: sizes, types, pointers, distances and devices, without anything enqueued; and the buckets that
``relative_buckets`` makes."""
import ctypes

import pytest
import torch

from tests import philox


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def test_the_generator_of_the_tests_is_the_published_one():
    """Known answers that the generator's authors give: 10 and 7 rounds of zeros, 10 of ones."""
    assert [int(v) for v in philox.words(0, 0, 0, 0, 0, 10)] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert [int(v) for v in philox.words(0, 0, 0, 0, 0)] == [0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48]
    top = 2 ** 32 - 1
    assert [int(v) for v in philox.words(2 ** 64 - 1, top, top, top, top, 10)] == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_sizes_are_checked_before_any_device_call(sams):
    lib, h = sams.load(), ctypes.c_void_p()
    out = ctypes.byref(h)
    starts = (ctypes.c_int32 * 513)(*range(513))
    same = (ctypes.c_int32 * 3)(0, 1, 1)
    bad = [lib.sams_dropout_create(None, 1, 1, 1, 0, None)]
    bad += [lib.sams_dropout_create(out, *args, None) for args in
            ((0, 4, 8, 0), (1025, 4, 8, 0), (1, -1, 8, 0), (2, 2 ** 28, 8, 0), (1, 4, 0, 0), (1, 4, 131073, 0), (1, 4, 8, 3), (1, 4, 8, -1))]
    bad += [lib.sams_attn_create(None, 1, 1, 1, 1, 8, 0, None, 0, 1, None)]
    # n, t_max, heads, kv_heads, dim, buckets, starts, type, train
    good = dict(n=1, t_max=4, heads=4, kv_heads=2, dim=8, buckets=3, starts=starts, type=0)
    for change in (dict(n=0), dict(n=1025), dict(t_max=-1), dict(n=2, t_max=2 ** 28), dict(heads=0), dict(heads=1025, kv_heads=1), dict(kv_heads=0), dict(kv_heads=3), dict(kv_heads=8),
                   dict(dim=7), dict(dim=0), dict(dim=129), dict(buckets=-1), dict(buckets=513), dict(starts=None), dict(starts=same), dict(type=3), dict(type=-1)):
        a = {**good, **change}
        bad.append(lib.sams_attn_create(out, a["n"], a["t_max"], a["heads"], a["kv_heads"], a["dim"], a["buckets"], a["starts"], a["type"], 1, None))
    assert bad == [sams.SAMS_EINVAL] * len(bad) and h.value is None


def test_no_context_is_an_error_and_destroying_none_is_not(sams):
    lib, row = sams.load(), (None, 0, 0)
    assert lib.dropout_forward(None, 1, *row, *row, None, 0.0, *row) == sams.SAMS_EINVAL
    assert lib.dropout_backward(None, 1, *row, None, 0.0, *row) == sams.SAMS_EINVAL
    assert lib.attention_forward(None, 1, 1, None, *row, *row, *row, None, 1.0, 1, None, 0.0, *row, None, None) == sams.SAMS_EINVAL
    assert lib.attention_backward(None, 1, 1, None, *row, *row, *row, *row, None, 1.0, 1, None, 0.0, *row, None, None, *row, *row, *row, None, 0, 0) == sams.SAMS_EINVAL
    for name in ("sams_dropout", "sams_attn"):
        assert getattr(lib, name + "_destroy")(None) == sams.SAMS_OK
        assert getattr(lib, name + "_scratch_bytes")(None) == 0


def test_without_a_gpu_the_classes_raise(sams):
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    for make in (lambda: sams.Dropout(1, 1, 1), lambda: sams.Attention(1, 1, 1, 8)):
        with pytest.raises(RuntimeError):
            make()


@pytest.mark.parametrize("causal", [True, False])
def test_relative_buckets(sams, causal):
    """Ascending; one distance each near the query; on either side the last bucket begins at max_distance or, where there are more buckets than
    distances up to it, as soon as it can; every start is the least that reaches the bucket's share of the way."""
    for buckets in (1, 2, 3, 4, 7, 32, 33, 64, 129):
        for far in (1, 2, 3, 20, 128, 5000):
            starts = sams.relative_buckets(buckets, far, causal)
            assert len(starts) == buckets and all(a < b for a, b in zip(starts, starts[1:]))
            left = buckets - 1 if causal else buckets // 2
            assert starts[left] == 0                                # the query's own bucket
            sides = [[-s for s in starts[left - 1::-1]] if left else [], starts[left + 1:]]     # last distance of each bucket on the left, first on the right
            least = [[1] + [e + 1 for e in sides[0][:-1]] if left else [], sides[1]]
            assert not causal or not sides[1]
            for side in least:
                near = (len(side) + 1) // 2
                assert side[:near] == list(range(1, near + 1))
                for i, d in enumerate(side[near:], 1):
                    rest = len(side) - near
                    reaches = lambda v: v ** rest >= far ** i * max(near, 1) ** (rest - i)
                    assert d == side[near + i - 2] + 1 or (reaches(d) and not reaches(d - 1)), (buckets, far, side)
                    assert reaches(d) or d >= far
    for bad in ((0, 5), (5, 0)):
        with pytest.raises(ValueError):
            sams.relative_buckets(*bad)


def cuda(*shape, dtype=torch.float32):
    return torch.zeros(shape, device="cuda", dtype=dtype)


@pytest.mark.gpu
def test_dropout_refuses(sams):
    with pytest.raises(TypeError):
        sams.Dropout(1, 1, 8, torch.float64)
    x, rng = cuda(2, 3, 8), cuda(2, dtype=torch.int64)
    with sams.Dropout(2, 3, 8) as op:
        ok = lambda **kw: op.dropout_forward(**{**dict(x=x, residual=x, rng=rng, p=0.1, y=cuda(2, 3, 8)), **kw})
        ok()
        ok(rng=None, p=0.0)
        for kw in (dict(x=x.half()), dict(x=None), dict(x=x.cpu()), dict(residual=x.half()), dict(rng=rng.int()), dict(rng=rng.cpu()), dict(y=None)):
            with pytest.raises(TypeError):
                ok(**kw)
        for kw in (dict(x=cuda(2, 3, 9)), dict(x=cuda(8)), dict(x=cuda(1, 3, 8)), dict(residual=cuda(2, 2, 8)), dict(rng=cuda(3, dtype=torch.int64)), dict(y=cuda(2, 3, 7)),
                   dict(x=cuda(2, 8, 3).transpose(1, 2))):
            with pytest.raises(ValueError):
                ok(**kw)
        for kw in (dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(p=1 - 2.0 ** -18), dict(rng=None), dict(y=cuda(1, 1, 8).expand(2, 3, 8)),
                   dict(x=cuda(2, 4, 8), residual=None, y=cuda(2, 4, 8))):
            with pytest.raises(sams.SamsError):
                ok(**kw)
        back = lambda **kw: op.dropout_backward(**{**dict(dy=x, rng=rng, p=0.1, dx=cuda(2, 3, 8)), **kw})
        back()
        with pytest.raises(TypeError):
            back(dy=None)
        with pytest.raises(ValueError):
            back(dx=cuda(2, 3, 9))
        with pytest.raises(sams.SamsError):
            back(p=2.0)
        op._device += 1                                     # a context on another device than the tensors
        for call in (ok, back):
            with pytest.raises(ValueError):
                call()


@pytest.mark.gpu
def test_attention_refuses(sams):
    for kw in (dict(kv_heads=3), dict(dim=4), dict(dim=160), dict(starts=[0, 0]), dict(starts=[1, 0]), dict(starts=range(513))):
        with pytest.raises(sams.SamsError):
            sams.Attention(**{**dict(n=2, t_max=6, heads=4, dim=8), **kw})
    with pytest.raises(ValueError):
        sams.Attention(2, 6, 4, 8, starts=[0, 2 ** 31])
    with pytest.raises(TypeError):
        sams.Attention(2, 6, 4, 8, dtype=torch.float64)
    q, k, stat, bias, rng = cuda(2, 6, 32), cuda(2, 6, 16), cuda(2, 4, 6), cuda(4, 3), cuda(2, dtype=torch.int64)
    lengths = cuda(2, 2, dtype=torch.int32)
    with sams.Attention(2, 6, 4, 8, 2, starts=[-1, 0, 1]) as op, sams.Attention(2, 6, 4, 8, 2) as bare:
        forward = dict(q=q, k=k, v=k, bias=bias, o=cuda(2, 6, 32), row_max=stat, row_sum=cuda(2, 4, 6), seqs=2, lengths=lengths, rng=rng, p=0.1)
        backward = {**forward, **dict(do=q, dq=cuda(2, 6, 32), dk=cuda(2, 6, 16), dv=cuda(2, 6, 16), dbias=cuda(2, 4, 3))}
        for call, good in ((op.attention_forward, forward), (op.attention_backward, backward)):
            ok = lambda **kw: call(**{**good, **kw})
            ok()
            ok(rng=None, p=0.0, lengths=None, seqs=3)
            for kw in (dict(q=q.half()), dict(q=None), dict(k=k.half()), dict(v=k.cpu()), dict(bias=bias.half()), dict(o=None), dict(rng=rng.int()), dict(lengths=lengths.long()),
                       dict(row_max=stat.double())):
                with pytest.raises(TypeError):
                    ok(**kw)
            for kw in (dict(q=cuda(2, 6, 33)), dict(q=cuda(6, 32)), dict(k=q), dict(v=cuda(2, 5, 16)), dict(bias=cuda(4, 4)), dict(o=cuda(2, 6, 16)), dict(row_sum=cuda(2, 6, 4)),
                       dict(lengths=cuda(4, dtype=torch.int32)), dict(lengths=cuda(2, 3, dtype=torch.int32)), dict(rng=cuda(1, dtype=torch.int64)),
                       dict(q=cuda(2, 32, 6).transpose(1, 2))):
                with pytest.raises(ValueError):
                    ok(**kw)
            for kw in (dict(p=1.0), dict(p=-1e-9), dict(rng=None), dict(bias=None), dict(scale=float("inf")), dict(scale=float("nan")), dict(seqs=4, lengths=None), dict(seqs=0, lengths=None),
                       dict(seqs=-1, lengths=None), dict(row_max=None)):
                with pytest.raises(sams.SamsError):
                    ok(**kw)
        for kw in (dict(o=cuda(1, 1, 32).expand(2, 6, 32)),):
            with pytest.raises(sams.SamsError):
                op.attention_forward(**{**forward, **kw})
        for kw in (dict(dq=cuda(1, 1, 32).expand(2, 6, 32)), dict(dk=cuda(1, 1, 16).expand(2, 6, 16)), dict(dv=cuda(2, 1, 16).expand(2, 6, 16)), dict(dbias=cuda(1, 4, 3).expand(2, 4, 3))):
            with pytest.raises(sams.SamsError):
                op.attention_backward(**{**backward, **kw})
        for kw in (dict(dq=None), dict(dk=cuda(2, 6, 16).half()), dict(dbias=cuda(2, 4, 3).half())):
            with pytest.raises(TypeError):
                op.attention_backward(**{**backward, **kw})
        for kw in (dict(dbias=cuda(2, 4, 4)), dict(dbias=cuda(2, 3, 4).transpose(1, 2)), dict(dv=cuda(2, 6, 15))):
            with pytest.raises(ValueError):
                op.attention_backward(**{**backward, **kw})
        with pytest.raises(ValueError):                    # a bias for a context without buckets
            bare.attention_forward(**forward)
        with pytest.raises(sams.SamsError):                # more tokens than the context is for
            op.attention_forward(cuda(2, 8, 32), cuda(2, 8, 16), cuda(2, 8, 16), bias, cuda(2, 8, 32), cuda(2, 4, 8), cuda(2, 4, 8))
        op._device += 1
        for call, good in ((op.attention_forward, forward), (op.attention_backward, backward)):
            with pytest.raises(ValueError):
                call(**good)
