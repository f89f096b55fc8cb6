"""Thin ctypes binding over the C ABI of ``include/sams.h`` (argument marshalling only).

Every function has the name and argument order of its C entry point and takes torch
CUDA tensors (device memory and streams are all PyTorch is used for).  There is no
fallback: if the HIP library has not been built, or no GPU is present, the calls raise.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsams.so")

SAMS_OK, SAMS_EINVAL, SAMS_ENOMEM, SAMS_EHIP = 0, -1, -2, -3
_ERR = {SAMS_EINVAL: "SAMS_EINVAL (bad argument)", SAMS_ENOMEM: "SAMS_ENOMEM (scratch allocation failed)",
        SAMS_EHIP: "SAMS_EHIP (HIP runtime error)"}

# every symbol include/sams.h declares
EXPORTS = ["sams_create", "sams_destroy", "sams_scratch_bytes", "sams_precondition_device_memory", "sams_last_hip_error", "sams_hash_dump",
           "sams_configure", "sams_sketch_mode", "sams_accumulate_variant", "sams_record_rows", "sams_profile_kernels", "sams_profile_name", "sams_profile_enable", "sams_profile_only", "sams_profile_read",
           "sketch_accumulate", "sketch_reduce", "unsketch_topk", "unsketch_estimates", "gather_topk", "topk_refine",
           "amsgrad_ef_update", "amsgrad_ef_update_pa", "topk_refine_static", "topk_refine_static_max_candidates",
           "sams_norm_create", "sams_norm_destroy", "sams_norm_scratch_bytes", "layer_norm_forward", "layer_norm_backward",
           "sams_xent_create", "sams_xent_destroy", "sams_xent_scratch_bytes", "linear_xent_forward", "linear_xent_backward",
           "sams_ortho_create", "sams_ortho_destroy", "sams_ortho_scratch_bytes", "orthogonalize", "muon_update",
           "sams_dropout_create", "sams_dropout_destroy", "sams_dropout_scratch_bytes", "dropout_forward", "dropout_backward",
           "sams_attn_create", "sams_attn_destroy", "sams_attn_scratch_bytes", "attention_forward", "attention_backward"]

_lib = None
_F32, _I32 = torch.float32, torch.int32


class SamsError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        extra = ""
        if code == SAMS_EHIP and _lib is not None:
            extra = f" hipError={_lib.sams_last_hip_error()}"
        super().__init__(f"{where}: {_ERR.get(code, code)}{extra}")


def load() -> ctypes.CDLL:
    """Load libsams.so (built by ``paper_2210_07454_amd.build``); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2210_07454_amd.build`")
    # torch has already loaded its HIP runtime (soname libamdhip64.so.7); the library binds to that one
    lib = ctypes.CDLL(LIB_PATH, mode=ctypes.RTLD_GLOBAL)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.sams_create.argtypes = [ctypes.POINTER(vp), i64, i32, i32, i64, i64, vp, vp]
    lib.sams_destroy.argtypes = [vp]
    lib.sams_scratch_bytes.argtypes = [vp]
    lib.sams_scratch_bytes.restype = i64
    lib.sams_precondition_device_memory.argtypes = [ctypes.c_double]
    lib.sams_precondition_device_memory.restype = i64
    lib.sams_last_hip_error.argtypes = []
    lib.sams_hash_dump.argtypes = [vp, vp, vp]
    lib.sams_configure.argtypes = [ctypes.c_char_p, ctypes.c_int]
    lib.sams_sketch_mode.argtypes = [vp]
    lib.sams_accumulate_variant.argtypes = [vp]
    lib.sams_record_rows.argtypes = [vp]
    lib.sams_record_rows.restype = i64
    lib.sams_profile_kernels.argtypes = []
    lib.sams_profile_name.argtypes = [ctypes.c_int]
    lib.sams_profile_enable.argtypes = [vp, ctypes.c_int]
    lib.sams_profile_only.argtypes = [vp, ctypes.c_int]
    lib.sams_profile_read.argtypes = [vp, vp, vp]
    lib.sketch_accumulate.argtypes = [vp, vp, vp]
    lib.sketch_reduce.argtypes = [vp, vp, vp]
    lib.unsketch_topk.argtypes = [vp, vp, vp, vp, vp]
    lib.unsketch_estimates.argtypes = [vp, vp, vp, vp]
    lib.gather_topk.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.topk_refine.argtypes = [vp, vp, vp, i64, vp, vp]
    lib.amsgrad_ef_update.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, f32, f32, f32, f32]
    lib.amsgrad_ef_update_pa.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, f32, f32, f32, f32]
    lib.topk_refine_static.argtypes = [vp, vp, i64, i64, vp, vp, vp]
    lib.topk_refine_static_max_candidates.argtypes = []
    lib.topk_refine_static_max_candidates.restype = i64
    lib.sams_norm_create.argtypes = [ctypes.POINTER(vp), i32, i64, i64, i32, vp]
    lib.layer_norm_forward.argtypes = [vp, i64, vp, i64, i64, vp, vp, f32, vp, i64, i64, vp, vp]
    lib.layer_norm_backward.argtypes = [vp, i64, vp, i64, i64, vp, i64, i64, vp, vp, vp, vp, i64, i64, vp, i64, vp, i64, i32]
    lib.sams_xent_create.argtypes = [ctypes.POINTER(vp), i32, i64, i64, i64, i32, i32, vp]
    lib.linear_xent_forward.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, vp, vp]
    lib.linear_xent_backward.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, vp, vp, vp, i64, i64, vp, i64, i64, i32, i32]
    lib.sams_ortho_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, i32, vp]
    lib.orthogonalize.argtypes = [vp, i64, vp, i64, i64, i32, vp, f32, vp, i64, i64]
    lib.muon_update.argtypes = [vp, i32, i64, vp, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, f32, i32, f32, f32, f32, i32, vp, f32]
    f64, row = ctypes.c_double, [vp, i64, i64]
    lib.sams_dropout_create.argtypes = [ctypes.POINTER(vp), i32, i64, i64, i32, vp]
    lib.dropout_forward.argtypes = [vp, i64, *row, *row, vp, f64, *row]
    lib.dropout_backward.argtypes = [vp, i64, *row, vp, f64, *row]
    lib.sams_attn_create.argtypes = [ctypes.POINTER(vp), i32, i64, i32, i32, i32, i32, vp, i32, i32, vp]
    lib.attention_forward.argtypes = [vp, i64, i64, vp, *row, *row, *row, vp, f32, i32, vp, f64, *row, vp, vp]
    lib.attention_backward.argtypes = [vp, i64, i64, vp, *row, *row, *row, *row, vp, f32, i32, vp, f64, *row, vp, vp, *row, *row, *row, vp, i64, i32]
    for name in ("sams_norm", "sams_xent", "sams_ortho", "sams_dropout", "sams_attn"):
        getattr(lib, name + "_destroy").argtypes = getattr(lib, name + "_scratch_bytes").argtypes = [vp]
        getattr(lib, name + "_scratch_bytes").restype = i64
    for name in EXPORTS:
        if name not in ("sams_scratch_bytes", "sams_profile_name", "sams_precondition_device_memory",
                        "topk_refine_static_max_candidates", "sams_record_rows", "sams_norm_scratch_bytes",
                        "sams_xent_scratch_bytes", "sams_ortho_scratch_bytes", "sams_dropout_scratch_bytes", "sams_attn_scratch_bytes"):
            getattr(lib, name).restype = ctypes.c_int
    lib.sams_profile_name.restype = ctypes.c_char_p
    _lib = lib
    return lib


def sams_configure(key: str, value: int):
    _check(load().sams_configure(key.encode(), int(value)), f"sams_configure({key}={value})")


def sams_precondition_device_memory(fraction: float = 0.995) -> int:
    """Allocate-and-free pass over the free memory of the current device (see sams.h); returns the GiB held."""
    if not torch.cuda.is_available():
        raise RuntimeError("paper_2210_07454_amd needs a GPU: no CPU fallback exists")
    got = int(load().sams_precondition_device_memory(float(fraction)))
    if got < 0:
        raise SamsError(got, "sams_precondition_device_memory")
    return got


def _ptr(t, dtype=None, shape=None, name="tensor"):
    """Device address of a tensor after the checks the C side cannot make (every call of a step goes through here for
    each of its tensors, so the good case comes first and costs a few attribute look-ups)."""
    if t is None:
        return None
    try:
        if (t.dtype is dtype or dtype is None) and (shape is None or t.shape == shape) and t.is_cuda and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise TypeError(f"{name}: expected a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")


def _check(code, where):
    if code != SAMS_OK:
        raise SamsError(code, where)


def topk_refine_static(idx_in, delta_in, k_out, idx_out, delta_out, stream=None):
    """Context-free topk_refine on the library's static scratch (allocates nothing); see sams.h."""
    if not torch.cuda.is_available():
        raise RuntimeError("paper_2210_07454_amd needs a GPU: no CPU fallback exists")
    k_in = idx_in.numel()
    st = stream if stream is not None else torch.cuda.current_stream()
    _check(load().topk_refine_static(
        _ptr(idx_in, torch.int32, (k_in,), "idx_in"), _ptr(delta_in, torch.float32, (k_in,), "delta_in"), int(k_in),
        int(k_out), _ptr(idx_out, torch.int32, (k_out,), "idx_out"), _ptr(delta_out, torch.float32, (k_out,), "delta_out"),
        ctypes.c_void_p(st.cuda_stream)), "topk_refine_static")


class Context:
    """Owns one ``sams_ctx``.  Work is enqueued on the torch stream that is current at creation."""

    def __init__(self, d: int, n: int, r: int, c: int, k: int, hash_params, stream=None):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2210_07454_amd needs a GPU: no CPU fallback exists")
        lib = load()
        hp = np.ascontiguousarray(hash_params, dtype=np.uint32)
        if hp.shape != (r, 4):
            raise ValueError(f"hash_params: expected shape ({r}, 4)")
        self.d, self.n, self.r, self.c, self.k = d, n, r, c, k
        self._nd, self._d, self._k, self._nk = (n, d), (d,), (k,), (n, k)      # the shapes the calls check
        self._nrc, self._rc = (n, r, c), (r, c)
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._h = ctypes.c_void_p()
        self._lib = lib
        code = lib.sams_create(ctypes.byref(self._h), d, n, r, c, k, hp.ctypes.data_as(ctypes.c_void_p),
                               ctypes.c_void_p(self.stream.cuda_stream))
        _check(code, "sams_create")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.sams_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    @property
    def scratch_bytes(self) -> int:
        return int(self._lib.sams_scratch_bytes(self._h))

    @property
    def sketch_mode(self) -> int:
        return int(self._lib.sams_sketch_mode(self._h))

    @property
    def accumulate_variant(self) -> int:
        return int(self._lib.sams_accumulate_variant(self._h))

    @property
    def record_rows(self) -> int:
        """Bit mask of the rows whose second pass reads chunk records (see sams.h)."""
        return int(self._lib.sams_record_rows(self._h))

    def sams_profile_enable(self, on: bool):
        _check(self._lib.sams_profile_enable(self._h, 1 if on else 0), "sams_profile_enable")

    def sams_profile_only(self, name=None):
        """Restrict the timing to the kernel called ``name`` (None: every kernel)."""
        nk = self._lib.sams_profile_kernels()
        names = [self._lib.sams_profile_name(q).decode() for q in range(nk)]
        _check(self._lib.sams_profile_only(self._h, -1 if name is None else names.index(name)), "sams_profile_only")

    def sams_profile_read(self):
        """{kernel name: (total milliseconds, launches)} since profiling was enabled."""
        nk = self._lib.sams_profile_kernels()
        ms = (ctypes.c_double * nk)()
        cnt = (ctypes.c_int64 * nk)()
        _check(self._lib.sams_profile_read(self._h, ms, cnt), "sams_profile_read")
        return {self._lib.sams_profile_name(q).decode(): (ms[q], cnt[q]) for q in range(nk) if cnt[q]}

    # ---- entry points, same names and argument order as the C ABI ----
    def sams_hash_dump(self, bucket, sign):
        _check(self._lib.sams_hash_dump(self._h, _ptr(bucket, torch.int32, (self.r, self.d), "bucket"),
                                        _ptr(sign, torch.int8, (self.r, self.d), "sign")), "sams_hash_dump")

    def sketch_accumulate(self, u, S_workers):
        code = self._lib.sketch_accumulate(self._h, _ptr(u, _F32, self._nd, "u"), _ptr(S_workers, _F32, self._nrc, "S_workers"))
        if code:
            _check(code, "sketch_accumulate")

    def sketch_reduce(self, S_workers, S_mean):
        code = self._lib.sketch_reduce(self._h, _ptr(S_workers, _F32, self._nrc, "S_workers"),
                                       _ptr(S_mean, _F32, self._rc, "S_mean"))
        if code:
            _check(code, "sketch_reduce")

    def unsketch_topk(self, S_mean, vhat, idx, est_sel=None):
        code = self._lib.unsketch_topk(self._h, _ptr(S_mean, _F32, self._rc, "S_mean"), _ptr(vhat, _F32, self._d, "vhat"),
                                       _ptr(idx, _I32, self._k, "idx"), _ptr(est_sel, _F32, self._k, "est_sel"))
        if code:
            _check(code, "unsketch_topk")

    def unsketch_estimates(self, S_mean, vhat, est):
        code = self._lib.unsketch_estimates(self._h, _ptr(S_mean, _F32, self._rc, "S_mean"), _ptr(vhat, _F32, self._d, "vhat"),
                                            _ptr(est, _F32, self._d, "est"))
        if code:
            _check(code, "unsketch_estimates")

    def gather_topk(self, u, vhat, idx, U_workers, delta):
        code = self._lib.gather_topk(self._h, _ptr(u, _F32, self._nd, "u"), _ptr(vhat, _F32, self._d, "vhat"),
                                     _ptr(idx, _I32, self._k, "idx"), _ptr(U_workers, _F32, self._nk, "U_workers"),
                                     _ptr(delta, _F32, self._k, "delta"))
        if code:
            _check(code, "gather_topk")

    def topk_refine(self, idx_in, delta_in, k_out, idx_out, delta_out):
        code = self._lib.topk_refine(self._h, _ptr(idx_in, _I32, self._k, "idx_in"), _ptr(delta_in, _F32, self._k, "delta_in"),
                                     int(k_out), _ptr(idx_out, _I32, (k_out,), "idx_out"),
                                     _ptr(delta_out, _F32, (k_out,), "delta_out"))
        if code:
            _check(code, "topk_refine")

    def amsgrad_ef_update(self, g_next, m, e_u, v, vhat, x, idx, delta, k_sel, beta1, beta2, lr, ef_ratio=1.0):
        if k_sel and (idx is None or delta is None or idx.numel() < k_sel or delta.numel() < k_sel):
            raise ValueError("idx/delta shorter than k_sel")
        nd, d = self._nd, self._d
        code = self._lib.amsgrad_ef_update(
            self._h, _ptr(g_next, _F32, nd, "g_next"), _ptr(m, _F32, nd, "m"), _ptr(e_u, _F32, nd, "e_u"),
            _ptr(v, _F32, d, "v"), _ptr(vhat, _F32, d, "vhat"), _ptr(x, _F32, d, "x"), _ptr(idx, _I32, None, "idx"),
            _ptr(delta, _F32, None, "delta"), int(k_sel), beta1, beta2, lr, ef_ratio)
        if code:
            _check(code, "amsgrad_ef_update")

    def amsgrad_ef_update_pa(self, g_next, m, e_u, v_workers, vhat_workers, x, idx, delta, k_sel, beta1, beta2, lr,
                             ef_ratio=1.0):
        if k_sel and (idx is None or delta is None or idx.numel() < k_sel or delta.numel() < k_sel):
            raise ValueError("idx/delta shorter than k_sel")
        nd = self._nd
        code = self._lib.amsgrad_ef_update_pa(
            self._h, _ptr(g_next, _F32, nd, "g_next"), _ptr(m, _F32, nd, "m"), _ptr(e_u, _F32, nd, "e_u"),
            _ptr(v_workers, _F32, nd, "v_workers"), _ptr(vhat_workers, _F32, nd, "vhat_workers"), _ptr(x, _F32, self._d, "x"),
            _ptr(idx, _I32, None, "idx"), _ptr(delta, _F32, None, "delta"), int(k_sel), beta1, beta2, lr, ef_ratio)
        if code:
            _check(code, "amsgrad_ef_update_pa")


class Buffers:
    """Caller-owned device buffers for a run (the library itself allocates none of these)."""

    def __init__(self, d, n, r, c, k, eps, x1, device="cuda"):
        f = dict(device=device, dtype=torch.float32)
        self.m = torch.zeros((n, d), **f)
        self.e_u = torch.zeros((n, d), **f)
        self.v = torch.full((d,), eps, **f)
        self.vhat = torch.full((d,), eps, **f)
        self.x = x1.to(device=device, dtype=torch.float32).clone()
        self.S_workers = torch.empty((n, r, c), **f)
        self.S_mean = torch.empty((r, c), **f)
        self.idx = torch.empty((k,), device=device, dtype=torch.int32)
        self.U_workers = torch.empty((n, k), **f)
        self.delta = torch.empty((k,), **f)


def run_step(ctx: Context, b: Buffers, beta1, beta2, lr, g_next=None, first=False, g_first=None,
             use_vhat=True):
    """The calling sequence of one iteration, in the order sams.h documents.

    ``first``: enqueue the head-only call for ``g_first`` before the five stages.
    After the stages, ``amsgrad_ef_update`` finishes the iteration and, if ``g_next`` is
    given, starts the next one.
    """
    if first:
        ctx.amsgrad_ef_update(g_first, b.m, b.e_u, b.v, b.vhat, b.x, None, None, 0, beta1, beta2, lr)
    vh = b.vhat if use_vhat else None
    ctx.sketch_accumulate(b.e_u, b.S_workers)
    ctx.sketch_reduce(b.S_workers, b.S_mean)
    ctx.unsketch_topk(b.S_mean, vh, b.idx, None)
    ctx.gather_topk(b.e_u, vh, b.idx, b.U_workers, b.delta)
    ctx.amsgrad_ef_update(g_next, b.m, b.e_u, b.v, b.vhat, b.x, b.idx, b.delta, ctx.k, beta1, beta2, lr)


# ---- training operators ----
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}       # SAMS_F32, SAMS_BF16, SAMS_F16


# the handle of the stream that is current on a device, without making a stream object (3 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _strided(t, dtype, shape, inner, name):
    """(address, distances of the leading axes) of a tensor whose last `inner` axes are contiguous."""
    if inner == 1 and isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_cuda:       # the good case first
        strides = t.stride()
        if strides[-1] == 1 or shape[-1] == 1:
            return (t.data_ptr(), *strides[:-1])
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name}: expected a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    strides, want = t.stride(), 1
    for axis in range(len(shape) - 1, len(shape) - 1 - inner, -1):
        if shape[axis] > 1 and strides[axis] != want:
            raise ValueError(f"{name}: the last {inner} axes have to be contiguous")
        want *= shape[axis]
    return (t.data_ptr(), *strides[:len(shape) - inner])


def _leading(t, axes, name):
    """Extents of a tensor that a call goes by, before its shape is compared with them."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a CUDA tensor")
    if t.dim() != axes:
        raise ValueError(f"{name}: expected {axes} axes, got shape {tuple(t.shape)}")
    return t.shape


def _coefficients(coef):
    coef = tuple(coef)
    if len(coef) != 3:
        raise ValueError(f"coef: expected three numbers, got {len(coef)}")
    return (ctypes.c_float * 3)(*coef)


class _TrainContext:
    """Owns one context of a training operator.  Work is enqueued on the stream given, or on the torch stream that is current at
    creation; a call made while another one is current waits for that one's work, and that one waits for the call's."""

    _name = ""

    def __init__(self, dtype, stream, *sizes):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2210_07454_amd needs a GPU: no CPU fallback exists")
        if dtype not in TYPES:
            raise TypeError(f"expected one of {list(TYPES)}, got {dtype}")
        self.dtype = dtype
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._device, self._raw = self.stream.device_index, self.stream.cuda_stream
        self._lib = load()
        self._h = ctypes.c_void_p()
        _check(getattr(self._lib, self._name + "_create")(ctypes.byref(self._h), *sizes, ctypes.c_void_p(self.stream.cuda_stream)),
               self._name + "_create")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            getattr(self._lib, self._name + "_destroy")(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    @property
    def scratch_bytes(self) -> int:
        return int(getattr(self._lib, self._name + "_scratch_bytes")(self._h))

    def _call(self, name, *args):
        if _raw_stream(self._device) == self._raw:
            code = getattr(self._lib, name)(self._h, *args)
        else:
            current = torch.cuda.current_stream(self._device)
            self.stream.wait_stream(current)
            code = getattr(self._lib, name)(self._h, *args)
            current.wait_stream(self.stream)
        if code:
            _check(code, name)


class LayerNorm(_TrainContext):
    """Layer norm of [n][t][dim] tensors, t up to ``t_max``; see sams.h."""

    _name = "sams_norm"

    def __init__(self, n: int, t_max: int, dim: int, dtype=torch.float32, stream=None):
        self.n, self.t_max, self.dim = n, t_max, dim
        super().__init__(dtype, stream, n, t_max, dim, TYPES.get(dtype, -1))

    def layer_norm_forward(self, x, weight, bias, y, mean, rstd, eps=1e-5):
        t = _leading(x, 3, "x")[1]
        full = (self.n, t, self.dim)
        self._call("layer_norm_forward", t, *_strided(x, self.dtype, full, 1, "x"), _ptr(weight, _F32, (self.dim,), "weight"),
                   _ptr(bias, _F32, (self.dim,), "bias"), eps, *_strided(y, self.dtype, full, 1, "y"),
                   _ptr(mean, _F32, full[:2], "mean"), _ptr(rstd, _F32, full[:2], "rstd"))

    def layer_norm_backward(self, dy, x, weight, mean, rstd, dx, dweight, dbias=None, accumulate=False):
        t = _leading(x, 3, "x")[1]
        full, sums = (self.n, t, self.dim), (self.n, self.dim)
        self._call("layer_norm_backward", t, *_strided(dy, self.dtype, full, 1, "dy"), *_strided(x, self.dtype, full, 1, "x"),
                   _ptr(weight, _F32, (self.dim,), "weight"), _ptr(mean, _F32, full[:2], "mean"), _ptr(rstd, _F32, full[:2], "rstd"),
                   *_strided(dx, self.dtype, full, 1, "dx"), *_strided(dweight, _F32, sums, 1, "dweight"),
                   *(_strided(dbias, _F32, sums, 1, "dbias") if dbias is not None else (None, 0)), int(bool(accumulate)))


class LinearCrossEntropy(_TrainContext):
    """Output layer and softmax cross entropy of [n][t][dim] hidden states, t up to ``t_max``; see sams.h."""

    _name = "sams_xent"

    def __init__(self, n: int, t_max: int, dim: int, vocab: int, dtype=torch.float32, train=True, stream=None):
        self.n, self.t_max, self.dim, self.vocab = n, t_max, dim, vocab
        super().__init__(dtype, stream, n, t_max, dim, vocab, TYPES.get(dtype, -1), int(bool(train)))

    def _inputs(self, h, w, labels):
        t = _leading(h, 3, "h")[1]
        return (t, *_strided(h, self.dtype, (self.n, t, self.dim), 1, "h"), *_strided(w, self.dtype, (self.vocab, self.dim), 1, "w"),
                _ptr(labels, torch.int64, (self.n, t), "labels"))

    def linear_xent_forward(self, h, w, labels, loss, lse):
        self._call("linear_xent_forward", *self._inputs(h, w, labels), _ptr(loss, _F32, (self.n,), "loss"),
                   _ptr(lse, _F32, (self.n, h.shape[1]), "lse"))

    def linear_xent_backward(self, h, w, labels, lse, grad_loss, dh, dw, accumulate=False):
        t = _leading(h, 3, "h")[1]
        kind = dw.dtype if isinstance(dw, torch.Tensor) and dw.dtype in (self.dtype, _F32) else self.dtype
        self._call("linear_xent_backward", *self._inputs(h, w, labels), _ptr(lse, _F32, (self.n, t), "lse"),
                   _ptr(grad_loss, _F32, (self.n,), "grad_loss"), *_strided(dh, self.dtype, (self.n, t, self.dim), 1, "dh"),
                   *_strided(dw, kind, (self.n, self.vocab, self.dim), 1, "dw"), TYPES[kind], int(bool(accumulate)))


class Orthogonalizer(_TrainContext):
    """Newton-Schulz orthogonalisation of up to ``batch`` matrices of one shape, and the momentum update built on it; see sams.h."""

    _name = "sams_ortho"

    def __init__(self, batch: int, rows: int, cols: int, dtype=torch.float32, stream=None):
        self.batch, self.rows, self.cols = batch, rows, cols
        super().__init__(dtype, stream, batch, rows, cols, TYPES.get(dtype, -1))

    def orthogonalize(self, g, out, steps=5, coef=(3.4445, -4.7750, 2.0315), eps=1e-7):
        full = (_leading(g, 3, "g")[0], self.rows, self.cols)
        self._call("orthogonalize", full[0], *_strided(g, self.dtype, full, 1, "g"), steps, _coefficients(coef), eps,
                   *_strided(out, self.dtype, full, 1, "out"))

    def muon_update(self, g, m, x, m_out, x_out, beta=0.95, nesterov=True, lr=0.02, scale=1.0, weight_decay=0.0, steps=5,
                    coef=(3.4445, -4.7750, 2.0315), eps=1e-7):
        n, batch = _leading(g, 4, "g")[:2]
        full = (batch, self.rows, self.cols)
        self._call("muon_update", n, batch, *_strided(g, _F32, (n, *full), 2, "g"), *_strided(m, _F32, full, 2, "m"),
                   *_strided(x, _F32, full, 2, "x"), *_strided(m_out, _F32, full, 2, "m_out"), *_strided(x_out, _F32, full, 2, "x_out"),
                   beta, int(bool(nesterov)), lr, scale, weight_decay, steps, _coefficients(coef), eps)


def _on(device, *tensors):
    """Every tensor given lies on the context's device (those that are none, or on the host, are refused by name later)."""
    for t in tensors:
        if t is not None and isinstance(t, torch.Tensor) and t.get_device() not in (device, -1):
            raise ValueError(f"expected tensors on cuda:{device}, got one on {t.device}")


class Dropout(_TrainContext):
    """Dropout of [n][t][dim] tensors, t up to ``t_max``, by a seed and a step that lie on the device; see sams.h."""

    _name = "sams_dropout"

    def __init__(self, n: int, t_max: int, dim: int, dtype=torch.float32, stream=None):
        self.n, self.t_max, self.dim = n, t_max, dim
        super().__init__(dtype, stream, n, t_max, dim, TYPES.get(dtype, -1))

    def dropout_forward(self, x, residual, rng, p, y):
        t = _leading(x, 3, "x")[1]
        _on(self._device, x, residual, rng, y)
        full = (self.n, t, self.dim)
        self._call("dropout_forward", t, *_strided(x, self.dtype, full, 1, "x"),
                   *(_strided(residual, self.dtype, full, 1, "residual") if residual is not None else (None, 0, 0)), _ptr(rng, torch.int64, (2,), "rng"),
                   p, *_strided(y, self.dtype, full, 1, "y"))

    def dropout_backward(self, dy, rng, p, dx):
        t = _leading(dy, 3, "dy")[1]
        _on(self._device, dy, rng, dx)
        full = (self.n, t, self.dim)
        self._call("dropout_backward", t, *_strided(dy, self.dtype, full, 1, "dy"), _ptr(rng, torch.int64, (2,), "rng"), p,
                   *_strided(dx, self.dtype, full, 1, "dx"))


def relative_buckets(buckets: int, max_distance: int, causal: bool = True):
    """First distances (key minus query) of ``buckets`` buckets, for ``Attention``: one by one near the query, then stretches whose lengths grow
    by a constant factor up to ``max_distance``, from which on all distances share a bucket (with more buckets than distances up to it, from where
    the buckets are used up).  causal: keys up to the query; otherwise one bucket for the query itself, and the others shared out to both sides."""
    if buckets < 1 or max_distance < 1:
        raise ValueError("relative_buckets: buckets and max_distance have to be at least 1")

    def reach(count):
        """The least distance to one side of each of `count` buckets, from 1 on: exact up to half of them, then near * (max / near) ** (i / far)."""
        near = (count + 1) // 2
        far, out = count - near, list(range(1, near + 1))
        for i in range(1, far + 1):
            low = out[-1] + 1
            # the least whole number d with d ** far * near ** (i - far) >= max_distance ** i
            d = low
            top = max(low, max_distance)
            while d < top:
                mid = (d + top) // 2
                if mid ** far >= max_distance ** i * max(near, 1) ** (far - i):
                    top = mid
                else:
                    d = mid + 1
            out.append(d)
        return out

    left = buckets - 1 if causal else (buckets - 1 + 1) // 2
    right = buckets - 1 - left
    # a bucket on the left that begins at distance a and ends before b is the distances -(b - 1) .. -a
    least = reach(left)
    ends = [b - 1 for b in least[1:]] + [2 ** 30]
    return [-e for e in reversed(ends[:left])] + [0] + reach(right)


class Attention(_TrainContext):
    """Self-attention of [n][t][heads * dim] queries with a bias by buckets of the relative position, t up to ``t_max``; see sams.h.
    ``starts``: the buckets' first distances (``relative_buckets`` makes some), or None for no bias."""

    _name = "sams_attn"

    def __init__(self, n: int, t_max: int, heads: int, dim: int, kv_heads=None, starts=None, dtype=torch.float32, train=True, stream=None):
        self.n, self.t_max, self.heads, self.dim = n, t_max, heads, dim
        self.kv_heads = heads if kv_heads is None else kv_heads
        starts = () if starts is None else tuple(int(v) for v in starts)
        if any(not -2 ** 31 <= v < 2 ** 31 for v in starts):
            raise ValueError("starts: expected 32-bit numbers")
        self.buckets = len(starts)
        super().__init__(dtype, stream, n, t_max, heads, self.kv_heads, dim, self.buckets, (ctypes.c_int32 * self.buckets)(*starts) if starts else None,
                         TYPES.get(dtype, -1), int(bool(train)))

    def _inputs(self, t, q, k, v):
        narrow = (self.n, t, self.kv_heads * self.dim)
        return (*_strided(q, self.dtype, (self.n, t, self.heads * self.dim), 1, "q"), *_strided(k, self.dtype, narrow, 1, "k"), *_strided(v, self.dtype, narrow, 1, "v"))

    def _how(self, bias, causal, scale, rng, p):
        return (_ptr(bias, _F32, (self.heads, self.buckets), "bias"), self.dim ** -0.5 if scale is None else scale, int(bool(causal)),
                _ptr(rng, torch.int64, (2,), "rng"), p)

    def attention_forward(self, q, k, v, bias, o, row_max, row_sum, seqs=1, lengths=None, causal=True, scale=None, rng=None, p=0.0):
        t = _leading(q, 3, "q")[1]
        _on(self._device, q, k, v, bias, o, row_max, row_sum, lengths, rng)
        stats = (self.n, self.heads, t)
        self._call("attention_forward", t, seqs, _ptr(lengths, _I32, (self.n, seqs), "lengths"), *self._inputs(t, q, k, v),
                   *self._how(bias, causal, scale, rng, p), *_strided(o, self.dtype, (self.n, t, self.heads * self.dim), 1, "o"),
                   _ptr(row_max, _F32, stats, "row_max"), _ptr(row_sum, _F32, stats, "row_sum"))

    def attention_backward(self, do, q, k, v, bias, o, row_max, row_sum, dq, dk, dv, dbias=None, seqs=1, lengths=None, causal=True, scale=None,
                           rng=None, p=0.0, accumulate=False):
        t = _leading(q, 3, "q")[1]
        _on(self._device, do, q, k, v, bias, o, row_max, row_sum, dq, dk, dv, dbias, lengths, rng)
        wide, narrow, stats = (self.n, t, self.heads * self.dim), (self.n, t, self.kv_heads * self.dim), (self.n, self.heads, t)
        into = (None, 0)
        if dbias is not None:
            into = _strided(dbias, _F32, (self.n, self.heads, self.buckets), 2, "dbias")
        self._call("attention_backward", t, seqs, _ptr(lengths, _I32, (self.n, seqs), "lengths"), *_strided(do, self.dtype, wide, 1, "do"),
                   *self._inputs(t, q, k, v), *self._how(bias, causal, scale, rng, p), *_strided(o, self.dtype, wide, 1, "o"),
                   _ptr(row_max, _F32, stats, "row_max"), _ptr(row_sum, _F32, stats, "row_sum"), *_strided(dq, self.dtype, wide, 1, "dq"),
                   *_strided(dk, self.dtype, narrow, 1, "dk"), *_strided(dv, self.dtype, narrow, 1, "dv"), *into, int(bool(accumulate)))
