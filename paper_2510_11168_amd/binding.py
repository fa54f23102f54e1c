"""Thin ctypes binding of libelmo_head.so: argument marshalling only.

Every step of the head's hot path runs in the library's HIP kernels.  PyTorch is used for device
memory and streams and nothing else.  There is no fallback: if the shared library is missing the
import of this module raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from .build import LIB_PATH

ELMO_BF16 = 0
ELMO_FP8_E4M3 = 1
ELMO_FP32 = 2
ELMO_INT8 = 3
ELMO_SR = 1
ELMO_KAHAN = 2
ELMO_VALIDATE = 4


class ElmoError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"elmo_head error {code}: {text}")
        self.code = code


if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
        "(the HIP library is the only implementation, there is no CPU path)")

_lib = C.CDLL(LIB_PATH)


class elmo_head_opts(C.Structure):
    _fields_ = [
        ("flags", C.c_uint32), ("max_B", C.c_int32), ("max_nnz", C.c_int64),
        ("W", C.c_void_p), ("W_bytes", C.c_size_t),
        ("comp", C.c_void_p), ("comp_bytes", C.c_size_t), ("kahan_rows", C.c_int64), ("weight_decay", C.c_float),
        ("dropout_p", C.c_float),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


_lib.elmo_last_error.restype = C.c_char_p
_lib.elmo_last_error.argtypes = []
_lib.elmo_logit_buffer_bytes.restype = C.c_size_t
_lib.elmo_logit_buffer_bytes.argtypes = [C.c_int64, C.c_int64]
_lib.elmo_head_sizes.restype = C.c_int
_lib.elmo_head_sizes.argtypes = [C.c_int64, C.c_int32, C.c_int, C.c_int64, C.c_int32, C.c_int64, C.c_uint32, C.c_int64,
                                 C.POINTER(C.c_size_t), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
_lib.elmo_head_create.restype = C.c_int
_lib.elmo_head_create.argtypes = [C.c_int64, C.c_int32, C.c_int, C.c_int64, C.POINTER(elmo_head_opts),
                                  C.POINTER(C.c_void_p)]
_lib.elmo_head_step.restype = C.c_int
_lib.elmo_head_step.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_float,
                                C.c_uint64, C.c_uint64, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.elmo_quantize_em.restype = C.c_int
_lib.elmo_quantize_em.argtypes = [C.c_void_p, C.c_int64, C.c_int, C.c_int, C.c_int, C.c_uint64, C.c_uint64, C.c_uint64,
                                  C.c_void_p, C.c_void_p]
_lib.elmo_precision_hits.restype = C.c_int
_lib.elmo_precision_hits.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.elmo_head_topk.restype = C.c_int
_lib.elmo_head_topk.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.elmo_topk_static.restype = C.c_int
_lib.elmo_topk_static.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_int, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                  C.c_void_p, C.c_void_p]
_lib.elmo_head_destroy.restype = C.c_int
_lib.elmo_head_destroy.argtypes = [C.c_void_p]
_lib.elmo_head_profile.restype = C.c_int
_lib.elmo_head_profile.argtypes = [C.c_void_p, C.c_int]
_lib.elmo_head_profile_read.restype = C.c_int
_lib.elmo_head_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
_lib.elmo_quantize.restype = C.c_int
_lib.elmo_quantize.argtypes = [C.c_void_p, C.c_int64, C.c_int, C.c_int, C.c_uint64, C.c_uint64, C.c_uint64,
                               C.c_void_p, C.c_void_p]
_lib.elmo_philox4x32_10.restype = None
_lib.elmo_philox4x32_10.argtypes = [C.POINTER(C.c_uint32), C.POINTER(C.c_uint32), C.POINTER(C.c_uint32)]
_lib.elmo_kahan_adamw.restype = C.c_int
_lib.elmo_kahan_adamw.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_float,
                                  C.c_double, C.c_double, C.c_float, C.c_float, C.c_int64, C.c_void_p]
_lib.elmo_dropout_keep16.restype = C.c_uint32
_lib.elmo_dropout_keep16.argtypes = [C.c_uint64, C.c_uint64, C.c_uint64, C.c_uint32]
_I, _L, _F, _P, _Z = C.c_int, C.c_int64, C.c_float, C.c_void_p, C.c_size_t
_lib.elmo_rms_norm.restype = _I
_lib.elmo_rms_norm.argtypes = [_P, _L, _I, _L, _L, _P, _L, _P, _I, _F, _P, _L, _P, _L, _I, _P, _P]
_lib.elmo_rms_norm_backward_bytes.restype = _Z
_lib.elmo_rms_norm_backward_bytes.argtypes = [_L, _L]
_lib.elmo_rms_norm_backward.restype = _I
_lib.elmo_rms_norm_backward.argtypes = [_P, _L, _P, _L, _I, _L, _L, _P, _I, _F, _P, _L, _P, _L, _P, _P, _Z, _P]
_lib.elmo_int8_matmul.restype = _I
_lib.elmo_int8_matmul.argtypes = [_P, _L, _P, _P, _L, _P, _P, _L, _L, _L, _P, _L, _I, _P]
_lib.elmo_int8_matmul_tile.restype = _I
_lib.elmo_int8_matmul_tile.argtypes = [_L, _L, _L]
_lib.elmo_sample_bytes.restype = _Z
_lib.elmo_sample_bytes.argtypes = [_L, _L]
_lib.elmo_sample.restype = _I
_lib.elmo_sample.argtypes = [_P, _L, _I, _L, _L, _P, _P, _P, _P, _P, _P, _P, _P, _Z, _P]
_lib.elmo_distill_bytes.restype = _Z
_lib.elmo_distill_bytes.argtypes = [_L, _L]
_lib.elmo_distill.restype = _I
_lib.elmo_distill.argtypes = [_P, _L, _I, _L, _L, _P, _P, _I, _L, _F, _P, _P, _P, _L, _P, _Z, _P]

EXPORTS = ("elmo_last_error", "elmo_logit_buffer_bytes", "elmo_head_sizes", "elmo_head_create",
           "elmo_head_step", "elmo_head_topk", "elmo_head_destroy", "elmo_quantize", "elmo_philox4x32_10",
           "elmo_head_profile", "elmo_head_profile_read", "elmo_precision_hits", "elmo_quantize_em",
           "elmo_dropout_keep16", "elmo_kahan_adamw", "elmo_topk_static", "elmo_rms_norm",
           "elmo_rms_norm_backward_bytes", "elmo_rms_norm_backward", "elmo_int8_matmul", "elmo_int8_matmul_tile",
           "elmo_sample_bytes", "elmo_sample",
           "elmo_distill_bytes", "elmo_distill")


def _check(rc: int) -> None:
    if rc != 0:
        raise ElmoError(rc, elmo_last_error())


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        if not torch.cuda.is_available():
            return 0          # no device: only argument checks can run, on the null stream
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


# ------------------------------------------------------------------ the C entry points, same names
def elmo_last_error() -> str:
    return _lib.elmo_last_error().decode()


def elmo_logit_buffer_bytes(batch: int, labels: int) -> int:
    return int(_lib.elmo_logit_buffer_bytes(batch, labels))


def elmo_head_sizes(L, d, weight_dtype, chunk, max_B, max_nnz, flags, kahan_rows=0):
    w, c, s = C.c_size_t(), C.c_size_t(), C.c_size_t()
    _check(_lib.elmo_head_sizes(L, d, weight_dtype, chunk, max_B, max_nnz, flags, kahan_rows, C.byref(w), C.byref(c), C.byref(s)))
    return w.value, c.value, s.value


def elmo_head_create(L, d, weight_dtype, chunk, *, flags, max_B, max_nnz, W, comp, workspace, kahan_rows=0,
                     weight_decay=0.0, dropout_p=0.0) -> int:
    """W, comp, workspace: 1-D torch.uint8 device tensors (comp may be None).  Returns the handle."""
    o = elmo_head_opts(flags=flags, max_B=max_B, max_nnz=max_nnz,
                       W=_ptr(W), W_bytes=0 if W is None else W.numel() * W.element_size(),
                       comp=_ptr(comp), comp_bytes=0 if comp is None else comp.numel() * comp.element_size(),
                       kahan_rows=kahan_rows, weight_decay=weight_decay, dropout_p=dropout_p,
                       workspace=_ptr(workspace),
                       workspace_bytes=0 if workspace is None else workspace.numel() * workspace.element_size())
    h = C.c_void_p()
    _check(_lib.elmo_head_create(L, d, weight_dtype, chunk, C.byref(o), C.byref(h)))
    return h.value


def elmo_head_step(h, X, B, indptr, indices, nnz, lr, seed, step, dX_out=None, loss_out=None, stream=None) -> None:
    _check(_lib.elmo_head_step(h, _ptr(X), B, _ptr(indptr), _ptr(indices), nnz, lr, seed, step,
                               _ptr(dX_out), _ptr(loss_out), _stream(stream)))


def elmo_head_topk(h, X, B, k, idx_out=None, score_out=None, stream=None) -> None:
    _check(_lib.elmo_head_topk(h, _ptr(X), B, k, _ptr(idx_out), _ptr(score_out), _stream(stream)))


def elmo_topk_static(W, L, d, weight_dtype, X, B, k, idx_out=None, score_out=None, stream=None) -> None:
    _check(_lib.elmo_topk_static(_ptr(W), L, d, weight_dtype, _ptr(X), B, k, _ptr(idx_out), _ptr(score_out), _stream(stream)))


def elmo_quantize_em(src, n, exp_bits, man_bits, mode, seed, step, first_elem, dst, stream=None) -> None:
    _check(_lib.elmo_quantize_em(_ptr(src), n, exp_bits, man_bits, mode, seed, step, first_elem, _ptr(dst), _stream(stream)))


def elmo_precision_hits(idx, B, k, indptr, indices, hits_out, stream=None) -> None:
    """hits_out: torch.int64 device tensor of k entries; P@j = hits_out[j-1] / (j * B)."""
    _check(_lib.elmo_precision_hits(_ptr(idx), B, k, _ptr(indptr), _ptr(indices), _ptr(hits_out), _stream(stream)))


def elmo_head_destroy(h) -> None:
    _check(_lib.elmo_head_destroy(h))


PROFILE_CLASSES = ("setup", "logits", "dx", "update", "finalize", "topk")


def elmo_head_profile(h, enable: bool) -> None:
    _check(_lib.elmo_head_profile(h, int(enable)))


def elmo_head_profile_read(h):
    """{class: (milliseconds, spans)} accumulated since profiling was enabled / last read."""
    ms = (C.c_double * 6)()
    n = (C.c_int64 * 6)()
    _check(_lib.elmo_head_profile_read(h, ms, n))
    return {name: (ms[i], n[i]) for i, name in enumerate(PROFILE_CLASSES)}


def elmo_quantize(src, n, dtype, mode, seed, step, first_elem, dst, stream=None) -> None:
    _check(_lib.elmo_quantize(_ptr(src), n, dtype, mode, seed, step, first_elem, _ptr(dst), _stream(stream)))


def elmo_kahan_adamw(param, comp, m, v, grad, n, state_dtype, lr, beta1, beta2, eps, weight_decay, t, stream=None) -> None:
    _check(_lib.elmo_kahan_adamw(_ptr(param), _ptr(comp), _ptr(m), _ptr(v), _ptr(grad), n, state_dtype, lr, beta1, beta2, eps,
                                 weight_decay, t, _stream(stream)))


def elmo_dropout_keep16(seed, step, block, threshold) -> int:
    return int(_lib.elmo_dropout_keep16(seed, step, block, threshold))


def elmo_philox4x32_10(ctr, key):
    c = (C.c_uint32 * 4)(*ctr)
    k = (C.c_uint32 * 2)(*key)
    o = (C.c_uint32 * 4)()
    _lib.elmo_philox4x32_10(c, k, o)
    return list(o)


# ------------------------------------------------------------------ the output end of a language model
# These take shapes, strides and types from the tensors and refuse (ElmoError -1 / -2) what does not fit together.  BF16 values are
# torch.bfloat16 or their bit patterns as torch.int16, E4M3 codes torch.float8_e4m3fn or torch.uint8.  The work runs on the tensors' own
# device, on `stream` or that device's current one.  A workspace that is not given is allocated for the call on that stream.
_REAL = {torch.bfloat16: ELMO_BF16, torch.int16: ELMO_BF16, torch.float32: ELMO_FP32}
_ROWS = {**_REAL, torch.float8_e4m3fn: ELMO_FP8_E4M3, torch.uint8: ELMO_FP8_E4M3, torch.int8: ELMO_INT8}
_ONLY_FP32, _ONLY_INT32, _ONLY_INT8 = {torch.float32: ELMO_FP32}, {torch.int32: 0}, {torch.int8: ELMO_INT8}


_SAME = {code: {t: c for t, c in _REAL.items() if c == code} for code in (ELMO_BF16, ELMO_FP32)}     # the types of one code
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # current_stream() without its Python object, a few us less of a small call


def _matrix(name, t, types, rows=None, cols=None):
    """(address, row stride, type code) of a 2-D tensor whose rows are dense; (None, 0, 0) for None."""
    if t is None:
        return None, 0, 0
    code = types.get(t.dtype)
    if code is None:
        raise ElmoError(-2, f"{name}: unsupported dtype {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ElmoError(-1, f"{name}: shape {tuple(shape)}, expected ({'rows' if rows is None else rows}, {'columns' if cols is None else cols})")
    stride, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ElmoError(-1, f"{name}: the elements of a row must lie next to each other (stride {step})")
    return t.data_ptr(), stride, code


def _vector(name, t, types, n):
    """(address, type code) of a dense 1-D tensor of n elements; (None, 0) for None."""
    if t is None:
        return None, 0
    code = types.get(t.dtype)
    if code is None:
        raise ElmoError(-2, f"{name}: unsupported dtype {t.dtype}")
    if t.shape != (n,) or not t.is_contiguous():
        raise ElmoError(-1, f"{name}: shape {tuple(t.shape)} with strides {t.stride()}, expected {n} dense elements")
    return t.data_ptr(), code


def _needed(names, *tensors):
    for t in tensors:
        if t is None:
            raise ElmoError(-1, f"{names}: all of them are needed")


def _call(fn, args, tensors, stream, workspace=None, bytes_needed=None):
    """fn(*args[, workspace, its size], stream) on the device that holds all `tensors`."""
    index = tensors[0].get_device()         # -1: not on a GPU
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ElmoError(-1, f"tensors on {t.device} and {tensors[0].device}")
    if index < 0:
        raise ElmoError(-1, f"the tensors must be on the GPU (got {tensors[0].device})")
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return _call(fn, args, tensors, stream, workspace, bytes_needed)
    if stream is not None:
        if stream.device.index != index:
            raise ElmoError(-1, f"stream of {stream.device}, tensors on {tensors[0].device}")
        handle = stream.cuda_stream
    else:
        handle = _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream
    if bytes_needed is None:
        return _check(fn(*args, handle))
    if workspace is not None:
        if workspace.get_device() != index or not workspace.is_contiguous():
            raise ElmoError(-1, f"workspace: a dense tensor on {tensors[0].device} is needed")
    elif bytes_needed and stream is None:
        workspace = torch.empty(bytes_needed, dtype=torch.uint8, device=tensors[0].device)
    elif bytes_needed:
        with torch.cuda.stream(stream):     # the caching allocator then reuses it in this stream's order
            workspace = torch.empty(bytes_needed, dtype=torch.uint8, device=tensors[0].device)
    return _check(fn(*args, _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), handle))


def elmo_rms_norm(x, y, weight=None, eps=1e-6, *, residual=None, sum_out=None, scale_out=None, stream=None) -> None:
    """y <- weight * h / sqrt(mean(h^2) + eps), h = x + residual; sum_out <- h; 8-bit y (int8, E4M3): scale_out <- the rows' scales."""
    _needed("x, y", x, y)
    xp, xs, dtype = _matrix("x", x, _REAL)
    rows, d = x.shape
    real = _SAME[dtype]
    rp, rs, _ = _matrix("residual", residual, real, rows, d)
    sp, ss, _ = _matrix("sum_out", sum_out, real, rows, d)
    yp, ys, yt = _matrix("y", y, _ROWS, rows, d)
    wp, wt = _vector("weight", weight, _REAL, d)
    cp, _ = _vector("scale_out", scale_out, _ONLY_FP32, rows)
    _call(_lib.elmo_rms_norm, (xp, xs, dtype, rows, d, rp, rs, wp, wt, eps, sp, ss, yp, ys, yt, cp),
          (x, y, weight, residual, sum_out, scale_out), stream)


def elmo_rms_norm_backward_bytes(rows, d) -> int:
    return int(_lib.elmo_rms_norm_backward_bytes(rows, d))


def elmo_rms_norm_backward(dy, h, dh, weight=None, eps=1e-6, *, dsum=None, dweight=None, workspace=None, stream=None) -> None:
    """dh <- gradient of h (plus dsum), dweight <- gradient of the weight."""
    _needed("dy, h, dh", dy, h, dh)
    yp, ys, dtype = _matrix("dy", dy, _REAL)
    rows, d = dy.shape
    real = _SAME[dtype]
    hp, hs, _ = _matrix("h", h, real, rows, d)
    op, os_, _ = _matrix("dh", dh, real, rows, d)
    sp, ss, _ = _matrix("dsum", dsum, real, rows, d)
    wp, wt = _vector("weight", weight, _REAL, d)
    gp, _ = _vector("dweight", dweight, _ONLY_FP32, d)
    _call(_lib.elmo_rms_norm_backward, (yp, ys, hp, hs, dtype, rows, d, wp, wt, eps, sp, ss, op, os_, gp),
          (dy, h, dh, weight, dsum, dweight), stream, workspace, 0 if dweight is None else elmo_rms_norm_backward_bytes(rows, d))


def elmo_int8_matmul(a, a_scale, b, b_scale, out, bias=None, *, stream=None) -> None:
    """out[m, n] <- (sum_k a[m, k] b[n, k]) a_scale[m] b_scale[n] + bias[n]."""
    _needed("a, a_scale, b, b_scale, out", a, a_scale, b, b_scale, out)
    ap, as_, _ = _matrix("a", a, _ONLY_INT8)
    M, K = a.shape
    bp, bs, _ = _matrix("b", b, _ONLY_INT8, None, K)
    N = b.shape[0]
    op, os_, ot = _matrix("out", out, _REAL, M, N)
    pa, _ = _vector("a_scale", a_scale, _ONLY_FP32, M)
    pb, _ = _vector("b_scale", b_scale, _ONLY_FP32, N)
    pc, _ = _vector("bias", bias, _ONLY_FP32, N)
    _call(_lib.elmo_int8_matmul, (ap, as_, pa, bp, bs, pb, pc, M, N, K, op, os_, ot), (a, a_scale, b, b_scale, out, bias), stream)


def elmo_int8_matmul_tile(M, N, K) -> int:
    """How a product of these sizes is worked on: tiles of 64, 128 or 256 outputs each way, 0: the kernel of few tokens that streams the weights."""
    t = int(_lib.elmo_int8_matmul_tile(M, N, K))
    if t < 0:
        _check(t)
    return t


def elmo_sample_bytes(rows, V) -> int:
    return int(_lib.elmo_sample_bytes(rows, V))


def elmo_sample(logits, u, idx_out, *, temperature=None, top_k=None, top_p=None, min_p=None, prob_out=None, workspace=None, stream=None) -> None:
    """idx_out <- one token a row by temperature, top-k, top-p and min-p from the random numbers u; prob_out <- its probability among the kept."""
    _needed("logits, u, idx_out", logits, u, idx_out)
    zp, zs, dtype = _matrix("logits", logits, _REAL)
    rows, V = logits.shape
    up, _ = _vector("u", u, _ONLY_FP32, rows)
    tp, _ = _vector("temperature", temperature, _ONLY_FP32, rows)
    kp, _ = _vector("top_k", top_k, _ONLY_INT32, rows)
    pp, _ = _vector("top_p", top_p, _ONLY_FP32, rows)
    mp, _ = _vector("min_p", min_p, _ONLY_FP32, rows)
    ip, _ = _vector("idx_out", idx_out, _ONLY_INT32, rows)
    qp, _ = _vector("prob_out", prob_out, _ONLY_FP32, rows)
    _call(_lib.elmo_sample, (zp, zs, dtype, rows, V, up, tp, kp, pp, mp, ip, qp), (logits, u, idx_out, temperature, top_k, top_p, min_p, prob_out),
          stream, workspace, elmo_sample_bytes(rows, V) if top_k is None else 0)


def elmo_distill_bytes(rows, V) -> int:
    return int(_lib.elmo_distill_bytes(rows, V))


def elmo_distill(logits, teacher_idx, teacher_logits, loss_out, grad_out=None, *, temperature=1.0, row_weight=None, workspace=None,
                 stream=None) -> None:
    """loss_out <- row_weight T^2 KL(teacher's top tokens || student) for each row, grad_out <- its gradient by the logits."""
    _needed("logits, teacher_idx, teacher_logits, loss_out", logits, teacher_idx, teacher_logits, loss_out)
    zp, zs, dtype = _matrix("logits", logits, _REAL)
    rows, V = logits.shape
    tp, ts, _ = _matrix("teacher_idx", teacher_idx, _ONLY_INT32, rows)
    K = teacher_idx.shape[1]
    lp, ls, lt = _matrix("teacher_logits", teacher_logits, _REAL, rows, K)
    if rows > 1 and (ts != K or ls != K):
        raise ElmoError(-1, "teacher_idx and teacher_logits must be dense")
    gp, gs, _ = _matrix("grad_out", grad_out, _SAME[dtype], rows, V)
    op, _ = _vector("loss_out", loss_out, _ONLY_FP32, rows)
    vp, _ = _vector("row_weight", row_weight, _ONLY_FP32, rows)
    _call(_lib.elmo_distill, (zp, zs, dtype, rows, V, tp, lp, lt, K, temperature, vp, op, gp, gs),
          (logits, teacher_idx, teacher_logits, loss_out, grad_out, row_weight), stream, workspace, elmo_distill_bytes(rows, V))


# ------------------------------------------------------------------ convenience owner of the buffers
class Head:
    """Allocates W / comp / workspace as torch device tensors and keeps the handle alive."""

    def __init__(self, L, d, weight_dtype, chunk, flags, max_B, max_nnz, device="cuda:0", kahan_rows=0, weight_decay=0.0,
                 dropout_p=0.0):
        self.L, self.d, self.fmt, self.chunk, self.flags = L, d, weight_dtype, chunk, flags
        self.max_B, self.max_nnz = max_B, max_nnz
        self.kahan_rows = (kahan_rows or L) if flags & ELMO_KAHAN else 0   # label rows that carry compensation
        wb, cb, sb = elmo_head_sizes(L, d, weight_dtype, chunk, max_B, max_nnz, flags, kahan_rows)
        self.W = torch.zeros(wb, dtype=torch.uint8, device=device)
        self.comp = torch.zeros(cb, dtype=torch.uint8, device=device) if cb else None
        self.workspace = torch.empty(sb, dtype=torch.uint8, device=device)
        self.bytes = (wb, cb, sb)
        self.h = elmo_head_create(L, d, weight_dtype, chunk, flags=flags, max_B=max_B, max_nnz=max_nnz,
                                  W=self.W, comp=self.comp, workspace=self.workspace, kahan_rows=kahan_rows,
                                  weight_decay=weight_decay, dropout_p=dropout_p)

    def weights(self):
        """[L, d] view of the raw weight bits: uint8 codes (E4M3) or int16 patterns (BF16)."""
        if self.fmt == ELMO_FP8_E4M3:
            return self.W.view(self.L, self.d)
        return self.W.view(torch.int16).view(self.L, self.d)

    def compensation(self):
        return None if self.comp is None else self.comp.view(torch.int16).view(self.kahan_rows, self.d)

    def step(self, X, indptr, indices, lr, seed, step, dX_out=None, loss_out=None, stream=None):
        elmo_head_step(self.h, X, X.shape[0], indptr, indices, int(indices.numel()), lr, seed, step,
                       dX_out, loss_out, stream)

    def topk(self, X, k, idx_out, score_out, stream=None):
        elmo_head_topk(self.h, X, X.shape[0], k, idx_out, score_out, stream)

    def close(self):
        if self.h is not None:
            elmo_head_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
