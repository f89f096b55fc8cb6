"""What the training operators refuse: sizes, types, pointers and distances, without anything enqueued."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def sams():
    from paper_2210_07454_amd import sams as mod
    mod.load()
    return mod


def test_sizes_are_checked_before_any_device_call(sams):
    lib, h = sams.load(), ctypes.c_void_p()
    out = ctypes.byref(h)
    bad = [lib.sams_norm_create(None, 1, 1, 1, 0, None)]
    bad += [lib.sams_norm_create(out, *args, None) for args in
            ((0, 4, 8, 0), (1025, 4, 8, 0), (1, -1, 8, 0), (2, 2 ** 28, 8, 0), (1, 4, 0, 0), (1, 4, 131073, 0), (1, 4, 8, 3), (1, 4, 8, -1))]
    bad += [lib.sams_xent_create(out, *args, None) for args in
            ((0, 4, 8, 9, 0, 1), (1, -1, 8, 9, 0, 1), (2, 2 ** 28, 8, 9, 0, 1), (1, 4, 0, 9, 0, 1), (1, 4, 8, 0, 0, 1), (1, 4, 8, 2 ** 24 + 1, 0, 1), (1, 4, 8, 9, 5, 1),
             (1, 2 ** 27, 8, 2 ** 24, 0, 1))]
    bad += [lib.sams_ortho_create(out, *args, None) for args in
            ((0, 4, 8, 0), (65536, 4, 8, 0), (1, 0, 8, 0), (1, 4, 0, 0), (1, 131073, 8, 0), (1, 8, 131073, 0), (1, 4, 8, 7))]
    assert bad == [sams.SAMS_EINVAL] * len(bad) and h.value is None


def test_no_context_is_an_error_and_destroying_none_is_not(sams):
    lib, coef = sams.load(), (ctypes.c_float * 3)(1, 0, 0)
    assert lib.layer_norm_forward(None, 1, None, 0, 0, None, None, 1e-5, None, 0, 0, None, None) == sams.SAMS_EINVAL
    assert lib.layer_norm_backward(None, 1, None, 0, 0, None, 0, 0, None, None, None, None, 0, 0, None, 0, None, 0, 0) == sams.SAMS_EINVAL
    assert lib.linear_xent_forward(None, 1, None, 0, 0, None, 0, None, None, None) == sams.SAMS_EINVAL
    assert lib.linear_xent_backward(None, 1, None, 0, 0, None, 0, None, None, None, None, 0, 0, None, 0, 0, 0, 0) == sams.SAMS_EINVAL
    assert lib.orthogonalize(None, 1, None, 0, 0, 5, coef, 1e-7, None, 0, 0) == sams.SAMS_EINVAL
    assert lib.muon_update(None, 1, 1, None, 0, 0, None, 0, None, 0, None, 0, None, 0, .9, 1, .1, 1., 0., 5, coef, 1e-7) == sams.SAMS_EINVAL
    for name in ("sams_norm", "sams_xent", "sams_ortho"):
        assert getattr(lib, name + "_destroy")(None) == sams.SAMS_OK
        assert getattr(lib, name + "_scratch_bytes")(None) == 0


def test_without_a_gpu_the_classes_raise(sams):
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    for make in (lambda: sams.LayerNorm(1, 1, 1), lambda: sams.LinearCrossEntropy(1, 1, 1, 1), lambda: sams.Orthogonalizer(1, 1, 1)):
        with pytest.raises(RuntimeError):
            make()


def cuda(*shape, dtype=torch.float32):
    return torch.zeros(shape, device="cuda", dtype=dtype)


@pytest.mark.gpu
def test_layer_norm_refuses(sams):
    with pytest.raises(TypeError):
        sams.LayerNorm(1, 1, 8, torch.float64)
    x, w, s = cuda(2, 3, 8), cuda(8), cuda(2, 3)
    with sams.LayerNorm(2, 3, 8) as op:
        ok = lambda **kw: op.layer_norm_forward(**{**dict(x=x, weight=w, bias=w, y=cuda(2, 3, 8), mean=s, rstd=cuda(2, 3)), **kw})
        ok()
        for kw in (dict(x=x.half()), dict(x=x.cpu()), dict(weight=w.bfloat16()), dict(y=None), dict(mean=None)):
            with pytest.raises((TypeError, sams.SamsError)):
                ok(**kw)
        for kw in (dict(x=cuda(2, 3, 9)), dict(x=cuda(1, 3, 8)), dict(weight=cuda(9)), dict(mean=cuda(3, 2)), dict(x=cuda(2, 8, 3).transpose(1, 2)), dict(y=cuda(2, 2, 8))):
            with pytest.raises(ValueError):
                ok(**kw)
        for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(y=cuda(1, 1, 8).expand(2, 3, 8)), dict(weight=None)):
            with pytest.raises(sams.SamsError):
                ok(**kw)
        with pytest.raises(sams.SamsError):                # more tokens than the context is for
            op.layer_norm_forward(cuda(2, 4, 8), w, w, cuda(2, 4, 8), cuda(2, 4), cuda(2, 4))
        with pytest.raises(sams.SamsError):                # workers' sums over each other
            op.layer_norm_backward(x, x, w, s, s, cuda(2, 3, 8), cuda(1, 8).expand(2, 8))


@pytest.mark.gpu
def test_linear_xent_refuses(sams):
    h, w, labels = cuda(2, 3, 8), cuda(20, 8), cuda(2, 3, dtype=torch.int64)
    with sams.LinearCrossEntropy(2, 3, 8, 20) as op:
        ok = lambda **kw: op.linear_xent_forward(**{**dict(h=h, w=w, labels=labels, loss=cuda(2), lse=cuda(2, 3)), **kw})
        ok()
        for kw in (dict(h=h.half()), dict(w=w.half()), dict(labels=labels.int()), dict(labels=labels.cpu()), dict(loss=cuda(2).half())):
            with pytest.raises(TypeError):
                ok(**kw)
        for kw in (dict(h=cuda(2, 3, 9)), dict(w=cuda(21, 8)), dict(w=cuda(8, 20).t()), dict(labels=labels[:1]), dict(loss=cuda(3)), dict(lse=cuda(3, 2))):
            with pytest.raises(ValueError):
                ok(**kw)
        back = lambda **kw: op.linear_xent_backward(**{**dict(h=h, w=w, labels=labels, lse=cuda(2, 3), grad_loss=None, dh=cuda(2, 3, 8), dw=cuda(2, 20, 8)), **kw})
        back()
        for kw in (dict(dw=cuda(2, 20, 8).half()), dict(dh=None)):
            with pytest.raises(TypeError):
                back(**kw)
        for kw in (dict(dw=cuda(2, 20, 9)), dict(grad_loss=cuda(1))):
            with pytest.raises(ValueError):
                back(**kw)
        for kw in (dict(dw=cuda(1, 20, 8).expand(2, 20, 8)), dict(dh=cuda(1, 1, 8).expand(2, 3, 8)), dict(lse=None)):
            with pytest.raises(sams.SamsError):
                back(**kw)


@pytest.mark.gpu
def test_ortho_refuses(sams):
    g = cuda(2, 6, 8)
    with sams.Orthogonalizer(2, 6, 8) as op, sams.Orthogonalizer(2, 6, 8, torch.bfloat16) as half:
        op.orthogonalize(g, cuda(2, 6, 8))
        for kw in (dict(steps=0), dict(steps=101), dict(eps=-1.0), dict(coef=(1.0, float("inf"), 0.0)), dict(out=cuda(1, 1, 8).expand(2, 6, 8)), dict(g=cuda(3, 6, 8), out=cuda(3, 6, 8))):
            with pytest.raises(sams.SamsError):
                op.orthogonalize(**{**dict(g=g, out=cuda(2, 6, 8)), **kw})
        with pytest.raises(TypeError):
            half.orthogonalize(g, cuda(2, 6, 8))
        with pytest.raises(ValueError):
            op.orthogonalize(cuda(2, 8, 6).transpose(1, 2), g)
        gs = cuda(3, 2, 6, 8)
        op.muon_update(gs, g, g, g.clone(), g.clone())
        with pytest.raises(sams.SamsError):                # the momentum update works on 32-bit tensors
            half.muon_update(gs, g, g, g.clone(), g.clone())
        with pytest.raises(ValueError):
            op.muon_update(gs.transpose(2, 3).contiguous().transpose(2, 3), g, g, g.clone(), g.clone())
        with pytest.raises(sams.SamsError):
            op.muon_update(gs, g, g, cuda(1, 6, 8).expand(2, 6, 8), g.clone())
