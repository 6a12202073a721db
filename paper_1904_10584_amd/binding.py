"""Thin ctypes binding of the C ABI in ``include/mi355am.h``.

Argument marshalling only: every function takes torch tensors that already
live on the GPU, passes their device pointers and the current HIP stream to
the native library, and raises ``AmError`` on a non-OK status.  All compute
happens in the library's HIP kernels.  If the library has not been built the
first call raises; there is no fallback path.
"""

import ctypes
import os
from dataclasses import dataclass

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmi355am.so")

F32, BF16 = 0, 1
MEAN_VALID, SUM = 0, 1
K_GEMM_FWD, K_GEMM_BWD_DATA, K_GEMM_BWD_WGT, K_LSTM_FWD, K_LSTM_BWD = 0, 1, 2, 3, 4
K_CE, K_ENCODE, K_DECODE, K_SGD, K_MISC, K_BMUF = 5, 6, 7, 8, 9, 10
K_GATED, K_NORM, K_ADAMW, K_Q8 = 11, 12, 13, 14
KERNEL_CLASSES = ["gemm_fwd", "gemm_bwd_data", "gemm_bwd_wgt", "lstm_fwd", "lstm_bwd",
                  "soft_ce", "encode", "decode", "sgd", "misc", "bmuf", "gated", "norm", "adamw", "q8"]


OK, EINVAL, ECAPACITY, EUNSUPPORTED, EHIP, EWORKSPACE, ETIMEOUT = 0, -1, -2, -3, -4, -5, -6
PATH_XCD, PATH_DEVICE, PATH_STEP, PATH_SOLO, PATH_PIPE = 1, 2, 3, 4, 5


class AmError(RuntimeError):
    """A non-OK am_status (``status``), with the library's message."""

    def __init__(self, msg, status=None):
        super().__init__(msg)
        self.status = status


class _Model(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("input_dim", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("classes", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


@dataclass(frozen=True)
class Model:
    layers: int
    input_dim: int
    hidden: int
    classes: int
    dtype: int = BF16

    def c(self):
        return _Model(self.layers, self.input_dim, self.hidden, self.classes, self.dtype)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == BF16 else torch.float32


_lib = None
_P, _I32, _I64, _F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_U32, _F64 = ctypes.c_uint32, ctypes.c_double
_PROTOS = {
    "am_param_count": (_I64, [_P]),
    "am_param_offsets": (_I32, [_P, _P]),
    "am_workspace_bytes": (_I64, [_P, _I32, _I32, _I64]),
    "am_ce_workspace_bytes": (_I64, [_I64]),
    "am_encode_workspace_bytes": (_I64, [_I64]),
    "am_status_string": (ctypes.c_char_p, [_I32]),
    "am_recurrence_path": (_I32, [_P, _I32, _I32, _I32, _I32]),
    "am_last_error": (ctypes.c_char_p, []),
    "lstm_am_forward": (_I32, [_P, _P, _P, _P, _P, _P, _I32, _I32, _P, _P, _P, _P, _I64, _P]),
    "sparse_soft_ce": (_I32, [_I64, _I32, _I32, _P, _P, _P, _P, _I32, _P, _P, _I32, _P, _I64, _P]),
    "lstm_am_backward": (_I32, [_P, _P, _P, _P, _I32, _I32, _P, _P, _I64, _P, _P]),
    "grad_threshold_encode": (_I32, [_I64, _P, _P, _F32, _P, _I64, _P, _P, _I64, _P]),
    "grad_threshold_encode_noalloc": (_I32, [_I64, _P, _P, _F32, _P, _I64, _P, _P]),
    "grad_threshold_decode": (_I32, [_P, _P, _I64, _F32, _I64, _P, _I32, _P]),
    "grad_threshold_decode_sgd": (_I32, [_P, _P, _I64, _F32, _I64, _F32, _P, _P, _P]),
    "sgd_apply": (_I32, [_I64, _P, _P, _P, _F32, _P]),
    "am_decode_multi_workspace_bytes": (_I64, [_I32, _I64]),
    "grad_threshold_decode_multi": (_I32, [_I32, _P, _I64, _P, _F32, _I64, _P, _I32, _P, _I64, _P]),
    "bmuf_block_update": (_I32, [_I64, _I32, _I32, _P, _I64, _P, _P, _F32, _F32, _F32, _P, _P, _P]),
    "am_lfr_frames": (_I32, [_I32, _I32, _I32, _I32]),
    "am_teacher_param_count": (_I64, [_P]),
    "am_teacher_param_offsets": (_I32, [_P, _P]),
    "am_teacher_workspace_bytes": (_I64, [_P, _I32, _I32, _I64]),
    "blstm_teacher_forward": (_I32, [_P, _P, _P, _P, _I32, _I32, _P, _P, _I64, _P]),
    "kbest_logits": (_I32, [_I64, _I32, _I32, _P, _P, _P, _P]),
    "kbest_posteriors": (_I32, [_I64, _I32, _P, _P, _P]),
    "lfr_features": (_I32, [_I32, _P, _P, _I32, _I32, _I32, _I32, _P, _P, _P, _I32, _P]),
    "delay_targets": (_I32, [_I32, _I32, _P, _I32, _I32, _P, _P, _P, _P, _P, _P]),
    "am_gated_recurrence_workspace_bytes": (_I64, [_I32, _I32, _I32, _I32, _I32]),
    "gated_recurrence_forward": (_I32, [_I32, _I32, _I32, _I32, _P, _P, _P, _P, _I64, _P, _F32, _P, _P,
                                        _P, _I32, _P, _I64, _P]),
    "gated_recurrence_backward": (_I32, [_I32, _I32, _I32, _I32, _P, _P, _P, _P, _I64, _P, _F32, _P, _I64,
                                         _P, _P, _P, _P, _I64, _P, _P, _P, _I64, _P]),
    "am_gated_delta_workspace_bytes": (_I64, [_I32] * 9),
    "gated_delta_forward": (_I32, [_I32] * 7 + [_P] + [_P, _I64] * 5 + [_P, _F32, _F32, _P, _P, _I64, _P, _I32, _P,
                                   _I64, _P]),
    "gated_delta_backward": (_I32, [_I32] * 7 + [_P] + [_P, _I64] * 5 + [_P, _F32, _F32, _P, _P, _I64, _P]
                             + [_P, _I64] * 5 + [_P, _P, _P, _I64, _P]),
    "am_gated_norm_workspace_bytes": (_I64, [_I64, _I32]),
    "gated_norm_forward": (_I32, [_I64, _I32, _I32, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _F32, _P,
                                  _P, _P, _P]),
    "gated_norm_backward": (_I32, [_I64, _I32, _I32, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _F32, _P,
                                   _P, _P, _P, _I64, _P, _I64, _P, _P, _P, _P, _P, _I64, _P]),
    "gated_norm_forward_q8": (_I32, [_I64, _I32, _I32, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _F32, _P,
                                     _P, _P, _P, _I64, _P, _I64, _P]),
    "q8_quantise": (_I32, [_I64, _I64, _I32, _P, _I64, _I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]),
    "am_q8_matmul_workspace_bytes": (_I64, [_I64, _I64, _I64]),
    "q8_matmul": (_I32, [_I64, _I64, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _I32, _P, _P, _I64, _I32,
                         _P, _I64, _P]),
    "adamw_apply": (_I32, [_I32, _P, _I32, _I32, _F64, _F64, _F64, _F64, _I64, _P, _U32, _P]),
    "am_cast_f32_to_bf16": (_I32, [_I64, _P, _P, _P]),
    "am_workspace_check": (_I32, [_P, _I64, _P]),
    "am_profile_begin": (_I32, [ctypes.c_uint32]),
    "am_profile_end": (_I32, []),
    "am_profile_sample_every": (_I32, [_I32]),
    "am_profile_get": (_I32, [_I32, _P, _P, _P, _P]),
}


def lib():
    """The loaded native library (loads it on first use)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise AmError(f"native library missing: {LIB_PATH} "
                          "(build it with `python -m paper_1904_10584_amd.build`)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _PROTOS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def exported_symbols():
    return list(_PROTOS)


def _check(status):
    if status != 0:
        L = lib()
        raise AmError(f"{L.am_status_string(status).decode()} ({status}): "
                      f"{L.am_last_error().decode()}", status)


def _dev(t, name, dtype=None):
    """Device pointer of a contiguous GPU tensor, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise AmError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise AmError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise AmError(f"{name} must be {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


# torch's own way to a stream's handle without making a Stream object (a microsecond,
# not three); a torch without it takes the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
        return _raw_stream(_raw_device())
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _host_i32(a):
    if a is None:
        return None, None
    import numpy as np
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return arr, arr.ctypes.data_as(ctypes.c_void_p)


# ----------------------------------------------------------------- queries --

def param_count(m: Model) -> int:
    n = lib().am_param_count(ctypes.byref(m.c()))
    if n < 0:
        _check(-1)
    return int(n)


def param_offsets(m: Model):
    out = (ctypes.c_int64 * (3 * m.layers + 2))()
    _check(lib().am_param_offsets(ctypes.byref(m.c()), out))
    return list(out)


def workspace_bytes(m: Model, T, B, N) -> int:
    n = lib().am_workspace_bytes(ctypes.byref(m.c()), T, B, N)
    if n < 0:
        raise AmError("invalid model or batch for workspace query")
    return int(n)


def recurrence_path(m: Model, T, B, varlen=False, forward=True) -> int:
    """PATH_SOLO, PATH_PIPE, PATH_XCD, PATH_DEVICE or PATH_STEP: the kernels the
    recurrence takes for this batch shape (see am_recurrence_path)."""
    p = lib().am_recurrence_path(ctypes.byref(m.c()), T, B, 1 if varlen else 0, 1 if forward else 0)
    if p < 0:
        raise AmError("invalid model or batch for the recurrence-path query", EINVAL)
    return int(p)


def ce_workspace_bytes(N) -> int:
    return int(lib().am_ce_workspace_bytes(N))


def encode_workspace_bytes(n) -> int:
    return int(lib().am_encode_workspace_bytes(n))


# ------------------------------------------------------------- entry points --

def lstm_am_forward(m: Model, params, x, T, B, logits, ws, lengths=None, h0=None, c0=None,
                    hT=None, cT=None, stream=None):
    dt = m.torch_dtype
    arr, lp = _host_i32(lengths)  # arr keeps the host array alive during the call
    _check(lib().lstm_am_forward(
        ctypes.byref(m.c()), _dev(params, "params", dt), _dev(x, "x", dt), lp,
        _dev(h0, "h0", torch.float32), _dev(c0, "c0", torch.float32), T, B,
        _dev(logits, "logits", torch.float32), _dev(hT, "hT", torch.float32),
        _dev(cT, "cT", torch.float32), _dev(ws, "ws"), ws.numel() * ws.element_size(),
        _stream(stream)))


def lstm_am_backward(m: Model, params, x, T, B, dlogits, ws, grads, lengths=None, stream=None):
    dt = m.torch_dtype
    arr, lp = _host_i32(lengths)
    _check(lib().lstm_am_backward(
        ctypes.byref(m.c()), _dev(params, "params", dt), _dev(x, "x", dt), lp, T, B,
        _dev(dlogits, "dlogits", dt), _dev(ws, "ws"), ws.numel() * ws.element_size(),
        _dev(grads, "grads", torch.float32), _stream(stream)))


def sparse_soft_ce(logits, idx, prob, loss, dlogits, ws, mask=None, reduction=MEAN_VALID,
                   stream=None):
    N, C = logits.shape
    K = idx.shape[1]
    dt = BF16 if dlogits.dtype == torch.bfloat16 else F32
    _check(lib().sparse_soft_ce(
        N, C, K, _dev(logits, "logits", torch.float32), _dev(idx, "idx", torch.int32),
        _dev(prob, "prob", torch.float32), _dev(mask, "mask", torch.uint8), reduction,
        _dev(loss, "loss", torch.float32), _dev(dlogits, "dlogits"), dt, _dev(ws, "ws"),
        ws.numel() * ws.element_size(), _stream(stream)))


def workspace_check(ws, stream=None):
    """Synchronise the stream; raise AmError if a wait of the last forward/backward
    pass on `ws` (the LSTM's, or a gated recurrence's that is not empty) timed out:
    its outputs are then invalid."""
    _check(lib().am_workspace_check(_dev(ws, "ws"), ws.numel() * ws.element_size(),
                                    _stream(stream)))


def grad_threshold_encode(grad, residual, tau, words, count, ws, stream=None):
    n = grad.numel()
    _check(lib().grad_threshold_encode(
        n, _dev(grad, "grad", torch.float32), _dev(residual, "residual", torch.float32),
        float(tau), _dev(words, "words", torch.int32), words.numel(),
        _dev(count, "count", torch.int64), _dev(ws, "ws"), ws.numel() * ws.element_size(),
        _stream(stream)))


ENCODE_NOALLOC_MAX_N = 1 << 25


def grad_threshold_encode_noalloc(grad, residual, tau, words, count, stream=None):
    """grad_threshold_encode without a workspace (library-owned scratch)."""
    n = grad.numel()
    _check(lib().grad_threshold_encode_noalloc(
        n, _dev(grad, "grad", torch.float32), _dev(residual, "residual", torch.float32),
        float(tau), _dev(words, "words", torch.int32), words.numel(),
        _dev(count, "count", torch.int64), _stream(stream)))


def grad_threshold_decode(words, count, tau, dense, accumulate=False, stream=None):
    _check(lib().grad_threshold_decode(
        _dev(words, "words", torch.int32), _dev(count, "count", torch.int64), words.numel(),
        float(tau), dense.numel(), _dev(dense, "dense", torch.float32), int(bool(accumulate)),
        _stream(stream)))


def grad_threshold_decode_sgd(words, count, tau, master, lr, weights_bf16=None, stream=None):
    """The decode of one stream and the SGD step on its update in one pass
    (the dense update is not materialised)."""
    _check(lib().grad_threshold_decode_sgd(
        _dev(words, "words", torch.int32), _dev(count, "count", torch.int64), words.numel(),
        float(tau), master.numel(), float(lr), _dev(master, "master", torch.float32),
        _dev(weights_bf16, "weights_bf16", torch.bfloat16), _stream(stream)))


def decode_multi_workspace_bytes(streams, n) -> int:
    return int(lib().am_decode_multi_workspace_bytes(streams, n))


def grad_threshold_decode_multi(words, counts, tau, dense, ws, accumulate=False, stream=None):
    """words: [streams][capacity] int32 GPU tensor; counts: [streams] int64."""
    if words.dim() != 2:
        raise AmError("words must be [streams][capacity]")
    S, cap = words.shape
    _check(lib().grad_threshold_decode_multi(
        S, _dev(words, "words", torch.int32), cap, _dev(counts, "counts", torch.int64),
        float(tau), dense.numel(), _dev(dense, "dense", torch.float32), int(bool(accumulate)),
        _dev(ws, "ws"), ws.numel() * ws.element_size(), _stream(stream)))


def bmuf_block_update(models, workers, global_model, delta, eta, eta_next, zeta,
                      local_master=None, local_bf16=None, stream=None):
    """models: [count][n] (or [n]) fp32 GPU tensor of the average's addends."""
    m2 = models if models.dim() == 2 else models.view(1, -1)
    count, n = m2.shape
    if global_model.numel() != n or delta.numel() != n:
        raise AmError("global_model and delta must hold n elements")
    _check(lib().bmuf_block_update(
        n, count, int(workers), _dev(m2, "models", torch.float32), n,
        _dev(global_model, "global_model", torch.float32), _dev(delta, "delta", torch.float32),
        float(eta), float(eta_next), float(zeta),
        _dev(local_master, "local_master", torch.float32),
        _dev(local_bf16, "local_bf16", torch.bfloat16), _stream(stream)))


def lfr_frames(raw_frames, stack=3, skip=3, offset=0) -> int:
    return int(lib().am_lfr_frames(raw_frames, stack, skip, offset))


def lfr_features(raw_lengths, raw, mean, std, x, stack=3, skip=3, offset=0, stream=None):
    """raw: [sum raw_lengths][raw_dim] fp32 GPU tensor; x: packed model input."""
    arr, lp = _host_i32(raw_lengths)
    dt = BF16 if x.dtype == torch.bfloat16 else F32
    _check(lib().lfr_features(
        len(raw_lengths), lp, _dev(raw, "raw", torch.float32), raw.shape[1], stack, skip, offset,
        _dev(mean, "mean", torch.float32), _dev(std, "std", torch.float32), _dev(x, "x"), dt,
        _stream(stream)))


def delay_targets(T, B, idx, prob, idx_out, prob_out, mask_out, delay, lengths=None, stream=None):
    arr, lp = _host_i32(lengths)
    _check(lib().delay_targets(
        T, B, lp, idx.shape[1], delay, _dev(idx, "idx", torch.int32), _dev(prob, "prob", torch.float32),
        _dev(idx_out, "idx_out", torch.int32), _dev(prob_out, "prob_out", torch.float32),
        _dev(mask_out, "mask_out", torch.uint8), _stream(stream)))


def teacher_param_count(m: Model) -> int:
    n = lib().am_teacher_param_count(ctypes.byref(m.c()))
    if n < 0:
        _check(-1)
    return int(n)


def teacher_param_offsets(m: Model):
    out = (ctypes.c_int64 * (6 * m.layers + 2))()
    _check(lib().am_teacher_param_offsets(ctypes.byref(m.c()), out))
    return list(out)


def teacher_workspace_bytes(m: Model, T, B, N) -> int:
    n = lib().am_teacher_workspace_bytes(ctypes.byref(m.c()), T, B, N)
    if n < 0:
        raise AmError("invalid model or batch for workspace query")
    return int(n)


def blstm_teacher_forward(m: Model, params, x, T, B, logits, ws, lengths=None, stream=None):
    dt = m.torch_dtype
    arr, lp = _host_i32(lengths)
    _check(lib().blstm_teacher_forward(
        ctypes.byref(m.c()), _dev(params, "params", dt), _dev(x, "x", dt), lp, T, B,
        _dev(logits, "logits", torch.float32), _dev(ws, "ws"), ws.numel() * ws.element_size(),
        _stream(stream)))


def kbest_logits(logits, idx, val, stream=None):
    N, C = logits.shape
    _check(lib().kbest_logits(N, C, idx.shape[1], _dev(logits, "logits", torch.float32),
                              _dev(idx, "idx", torch.int32), _dev(val, "val", torch.float32),
                              _stream(stream)))


def kbest_posteriors(val, prob, stream=None):
    N, K = val.shape
    _check(lib().kbest_posteriors(N, K, _dev(val, "val", torch.float32),
                                  _dev(prob, "prob", torch.float32), _stream(stream)))


def sgd_apply(master, update, lr, weights_bf16=None, stream=None):
    _check(lib().sgd_apply(
        master.numel(), _dev(master, "master", torch.float32),
        _dev(weights_bf16, "weights_bf16", torch.bfloat16),
        _dev(update, "update", torch.float32), float(lr), _stream(stream)))


def cast_f32_to_bf16(src, dst, stream=None):
    _check(lib().am_cast_f32_to_bf16(
        src.numel(), _dev(src, "src", torch.float32), _dev(dst, "dst", torch.bfloat16),
        _stream(stream)))


# ------------------------------------------- gated linear recurrences --

def _dtype(t, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.float32, torch.bfloat16):
        raise AmError(f"{name} must be a float32 or bfloat16 tensor")
    return BF16 if t.dtype == torch.bfloat16 else F32


def _refuse(t, name, shape, dtype, how):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise AmError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype or tuple(t.shape) != shape:
        raise AmError(f"{name} must be {dtype} of shape {shape}, got {t.dtype} of shape {tuple(t.shape)}")
    raise AmError(f"{name} must {how}")


def _shaped(t, name, shape, dtype=torch.float32):
    """Device pointer of a contiguous GPU tensor of this shape, or None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape
            and t.is_contiguous()):
        _refuse(t, name, shape, dtype, "be contiguous")
    return t.data_ptr()


def _row(t, name, N, H, dtype):
    """Device pointer and row stride of [N][H] rows, which may be columns of a
    wider matrix; (None, H) for None."""
    if t is None:
        return None, H
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == (N, H)):
        _refuse(t, name, (N, H), dtype, "")
    s0, s1 = t.stride()
    if s1 != 1 and H > 1 and N > 0:
        _refuse(t, name, (N, H), dtype, "have rows of unit stride")
    if N < 2:
        return t.data_ptr(), H
    if s0 < H:
        _refuse(t, name, (N, H), dtype, "have rows that do not overlap")
    return t.data_ptr(), s0


def _here(stream, names, *tensors):
    """Refuses tensors (of these names, or Nones) of another GPU than the one whose stream
    the call takes."""
    now = stream.device_index if stream is not None else _raw_device() if _raw_device else torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != now:
            name = next(n for n, x in zip(names.split(), tensors) if x is t)
            raise AmError(f"{name} is on GPU {t.get_device()}, the call on GPU {now}")


def _rows3(x, r, i, names, N, H, dtype):
    """Device pointers and the one row stride of three matrices."""
    (xp, ld), (rp, lr), (ip, li) = (_row(x, names[0], N, H, dtype), _row(r, names[1], N, H, dtype),
                                    _row(i, names[2], N, H, dtype))
    if lr != ld or li != ld:
        raise AmError(f"{', '.join(names)} must have one row stride, got {ld}, {lr} and {li}")
    return xp, rp, ip, ld


def _packed_rows(T, B, lengths):
    if lengths is None:
        return None, None, T * B
    arr, lp = _host_i32(lengths)
    if arr.shape != (B,):
        raise AmError(f"lengths must hold B = {B} values")
    return arr, lp, sum(lengths) if isinstance(lengths, list) else int(arr.sum())


def _workspace(ws):
    if ws is None:
        return None, 0
    if not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.is_contiguous()):
        raise AmError("ws must be a contiguous GPU tensor")
    return ws.data_ptr(), ws.nbytes


def gated_recurrence_workspace_bytes(T, B, H, lengths=None, train=False) -> int:
    n = lib().am_gated_recurrence_workspace_bytes(T, B, H, int(lengths is not None), int(bool(train)))
    if n < 0:
        raise AmError("invalid sizes for workspace query", EINVAL)
    return int(n)


def gated_recurrence_forward(x, r, i, lam, T, B, h, ws=None, lengths=None, h0=None, hT=None, c=8.0,
                             train=False, stream=None):
    """x, r, i: [N][H] rows of one stride (columns of one projection, say); h:
    [N][H]; lam: [H]; h0, hT: [B][H] fp32 (hT may be h0)."""
    dt, (N, H) = _dtype(x, "x"), h.shape
    arr, lp, rows = _packed_rows(T, B, lengths)
    if rows != N:
        raise AmError(f"h must have {rows} rows, got {N}")
    xp, rp, ip, ld = _rows3(x, r, i, "xri", N, H, x.dtype)
    wp, wn = _workspace(ws)
    st = (_lib or lib()).gated_recurrence_forward(
        T, B, H, dt, lp, xp, rp, ip, ld, _shaped(lam, "lam", (H,)), c, _shaped(h0, "h0", (B, H)),
        _shaped(h, "h", (N, H), x.dtype), _shaped(hT, "hT", (B, H)), 1 if train else 0, wp, wn,
        _stream(stream))
    if st:
        _check(st)


def gated_recurrence_backward(x, r, i, lam, T, B, dh, ws, dx, dr, di, dlam, lengths=None, dhT=None,
                              dh0=None, c=8.0, stream=None):
    """The gradient of the forward call (train=True) that filled `ws`; dx, dr, di:
    [N][H] rows of one stride."""
    dt, (N, H) = _dtype(x, "x"), x.shape
    arr, lp, rows = _packed_rows(T, B, lengths)
    if rows != N:
        raise AmError(f"x must have {rows} rows, got {N}")
    xp, rp, ip, ld = _rows3(x, r, i, "xri", N, H, x.dtype)
    dhp, lddh = _row(dh, "dh", N, H, x.dtype)
    dxp, drp, dip, ldd = _rows3(dx, dr, di, ("dx", "dr", "di"), N, H, x.dtype)
    wp, wn = _workspace(ws)
    st = (_lib or lib()).gated_recurrence_backward(
        T, B, H, dt, lp, xp, rp, ip, ld, _shaped(lam, "lam", (H,)), c, dhp, lddh,
        _shaped(dhT, "dhT", (B, H)), dxp, drp, dip, ldd, _shaped(dlam, "dlam", (H,)),
        _shaped(dh0, "dh0", (B, H)), wp, wn, _stream(stream))
    if st:
        _check(st)


def gated_delta_workspace_bytes(T, B, heads, dk, dv, key_heads=None, dtype=torch.bfloat16, lengths=None,
                                train=False) -> int:
    kinds = {torch.float32: F32, torch.bfloat16: BF16}
    n = lib().am_gated_delta_workspace_bytes(T, B, heads, heads if key_heads is None else key_heads, dk, dv,
                                             kinds.get(dtype, -1), int(lengths is not None), int(bool(train)))
    if n < 0:
        raise AmError("invalid sizes for workspace query", EINVAL)
    return int(n)


def _delta(q, k, v, r, b, T, B, heads, key_heads, lengths):
    """What both passes share: columns of q and v, frames, type, states' shape, what must
    live until the call, and its arguments up to b."""
    key_heads = heads if key_heads is None else key_heads
    arr, lp, N = _packed_rows(T, B, lengths)
    if heads < 1 or key_heads < 1 or heads % key_heads:
        raise AmError(f"key_heads = {key_heads} must divide heads = {heads}")
    dt, kind = _dtype(q, "q"), q.dtype
    for t, name, n in ((q, "q", key_heads), (v, "v", heads)):
        if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.shape[1] % n:
            raise AmError(f"{name} must be [{N}] rows of {n} heads")
    nq, nv = q.shape[1], v.shape[1]
    dk, dv = nq // key_heads, nv // heads
    args = (T, B, heads, key_heads, dk, dv, dt, lp, *_row(q, "q", N, nq, kind), *_row(k, "k", N, nq, kind),
            *_row(v, "v", N, nv, kind), *_row(r, "r", N, heads, kind), *_row(b, "b", N, heads, kind))
    return nq, nv, N, kind, (B, heads, dk, dv), arr, args


def gated_delta_forward(q, k, v, r, b, lam, T, B, o, ws=None, heads=1, key_heads=None, lengths=None, s0=None,
                        sT=None, c=8.0, eps=1e-6, train=False, stream=None):
    """q, k: [N][key_heads dk], v and o: [N][heads dv], r, b: [N][heads] rows (columns of
    one projection, say); lam: [heads]; s0, sT: [B][heads][dk][dv] fp32 (sT may be s0)."""
    nq, nv, N, kind, state, arr, args = _delta(q, k, v, r, b, T, B, heads, key_heads, lengths)
    wp, wn = _workspace(ws)
    call = (*args, _shaped(lam, "lam", (heads,)), c, eps, _shaped(s0, "s0", state), *_row(o, "o", N, nv, kind),
            _shaped(sT, "sT", state), 1 if train else 0, wp, wn)
    _here(stream, "q k v r b lam s0 o sT ws", q, k, v, r, b, lam, s0, o, sT, ws)
    st = (_lib or lib()).gated_delta_forward(*call, _stream(stream))
    if st:
        _check(st)


def gated_delta_backward(q, k, v, r, b, lam, T, B, do, ws, dq, dk, dv, dr, db, dlam, heads=1, key_heads=None,
                         lengths=None, s0=None, dsT=None, ds0=None, c=8.0, eps=1e-6, stream=None):
    """The gradient of the forward call (train=True) that filled `ws`, with the s0 that
    it had; dq, dk, dv, dr, db: rows as of q, k, v, r, b."""
    nq, nv, N, kind, state, arr, args = _delta(q, k, v, r, b, T, B, heads, key_heads, lengths)
    wp, wn = _workspace(ws)
    call = (*args, _shaped(lam, "lam", (heads,)), c, eps, _shaped(s0, "s0", state),
            *_row(do, "do", N, nv, kind), _shaped(dsT, "dsT", state), *_row(dq, "dq", N, nq, kind),
            *_row(dk, "dk", N, nq, kind), *_row(dv, "dv", N, nv, kind), *_row(dr, "dr", N, heads, kind),
            *_row(db, "db", N, heads, kind), _shaped(dlam, "dlam", (heads,)), _shaped(ds0, "ds0", state), wp, wn)
    _here(stream, "q k v r b lam s0 do dsT dq dk dv dr db dlam ds0 ws", q, k, v, r, b, lam, s0, do, dsT, dq, dk, dv, dr,
          db, dlam, ds0, ws)
    st = (_lib or lib()).gated_delta_backward(*call, _stream(stream))
    if st:
        _check(st)


def gated_norm_workspace_bytes(N, H) -> int:
    n = lib().am_gated_norm_workspace_bytes(N, H)
    if n < 0:
        raise AmError("invalid sizes for workspace query", EINVAL)
    return int(n)


def gated_norm_forward(res, o=None, gate=None, w_post=None, scale=None, w_next=None, res_out=None,
                       y=None, rstd=None, eps=1e-6, stream=None):
    """res, res_out: the residual stream, [N][H] fp32 or bf16; o, gate: [N][H]
    rows; y: [N][H] of their type.  Every part may be left out (see the C ABI)."""
    (N, H), act = res.shape, o if o is not None else y if y is not None else res
    (op, ldo), (gp, ldg) = _row(o, "o", N, H, act.dtype), _row(gate, "gate", N, H, act.dtype)
    st = (_lib or lib()).gated_norm_forward(
        N, H, _dtype(act, "o"), _dtype(res, "res"), op, ldo, gp, ldg, _shaped(w_post, "w_post", (H,)),
        _shaped(scale, "scale", (H,)), _shaped(res, "res", (N, H), res.dtype),
        _shaped(w_next, "w_next", (H,)), float(eps), _shaped(res_out, "res_out", (N, H), res.dtype),
        _shaped(y, "y", (N, H), act.dtype), _shaped(rstd, "rstd", (N, 2)), _stream(stream))
    if st:
        _check(st)


def gated_norm_backward(res, rstd, dres, ws, o=None, gate=None, w_post=None, scale=None, w_next=None,
                        dy=None, dres_out=None, do=None, dgate=None, dw_post=None, dscale=None,
                        dw_next=None, eps=1e-6, stream=None):
    """The gradient of gated_norm_forward with the same res (as it was before),
    o, gate and factors, and the rstd it wrote."""
    (N, H), act = res.shape, o if o is not None else dy if dy is not None else res
    (op, ldo), (gp, ldg) = _row(o, "o", N, H, act.dtype), _row(gate, "gate", N, H, act.dtype)
    (dop, lddo), (dgp, lddg) = _row(do, "do", N, H, act.dtype), _row(dgate, "dgate", N, H, act.dtype)
    wp, wn = _workspace(ws)
    st = (_lib or lib()).gated_norm_backward(
        N, H, _dtype(act, "o"), _dtype(res, "res"), op, ldo, gp, ldg, _shaped(w_post, "w_post", (H,)),
        _shaped(scale, "scale", (H,)), _shaped(res, "res", (N, H), res.dtype),
        _shaped(w_next, "w_next", (H,)), float(eps), _shaped(rstd, "rstd", (N, 2)),
        _shaped(dy, "dy", (N, H), act.dtype), _shaped(dres_out, "dres_out", (N, H), res.dtype),
        dop, lddo, dgp, lddg, _shaped(dres, "dres", (N, H), res.dtype),
        _shaped(dw_post, "dw_post", (H,)), _shaped(dscale, "dscale", (H,)),
        _shaped(dw_next, "dw_next", (H,)), wp, wn, _stream(stream))
    if st:
        _check(st)


# ------------------------------------------------------ matrices in 8 bits --

Q8_BLOCK = 128  # elements that share a scale
_CODES = (torch.float8_e4m3fn, torch.uint8)
_SCALES = (torch.float8_e8m0fnu, torch.uint8)


def q8_empty(rows, cols, tiles=False, device="cuda"):
    """Room for a matrix [rows][cols] in 8 bits: its codes, a view [rows][cols] of rows
    that start on 16 bytes, and its scales, in rows of a multiple of 4 (unused ones are
    zeros).  `tiles`: a scale for each 128 x 128, else for each 128 of a row."""
    codes = torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=device)
    scales = torch.zeros((-(-rows // Q8_BLOCK) if tiles else rows, -(-cols // (4 * Q8_BLOCK)) * 4),
                         dtype=torch.uint8, device=device)
    return codes.view(torch.float8_e4m3fn)[:, :cols], scales.view(torch.float8_e8m0fnu)


def _q8(codes, scales, name, rows, cols, tiles=False):
    """Pointers and row strides of a matrix in 8 bits; Nones for None."""
    if codes is None and scales is None:
        return None, 0, None, 0
    if cols % 16 == 0 and codes is not None and scales is not None:  # (most calls)
        (ldc, one), (lds, unit), (n, room) = codes.stride(), scales.stride(), scales.shape
        if (one == 1 and unit == 1 and rows > 1 and n > 1 and n == (-(-rows // Q8_BLOCK) if tiles else rows)
                and 128 * room >= cols and room % 4 == 0 and codes.shape == (rows, cols) and codes.is_cuda
                and scales.is_cuda and codes.dtype in _CODES and scales.dtype in _SCALES):
            return codes.data_ptr(), ldc, scales.data_ptr(), lds
    for t, what, kinds, n, least in (
            (codes, "codes", _CODES, rows, cols),
            (scales, "scales", _SCALES, -(-rows // Q8_BLOCK) if tiles else rows, -(-cols // (4 * Q8_BLOCK)) * 4)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise AmError(f"{what} of {name} must be a GPU tensor")
        if t.dtype not in kinds:
            raise AmError(f"{what} of {name} must be {kinds[0]} or uint8, got {t.dtype}")
        if t.dim() != 2 or t.shape[0] != n or (t.shape[1] != cols if what == "codes" else t.shape[1] < least):
            raise AmError(f"{what} of {name} must be of shape ({n}, {least}), got {tuple(t.shape)}")
        if t.stride(1) != 1 and t.shape[1] > 1:
            raise AmError(f"{what} of {name} must have rows of unit stride")
    # (a row's end: what is allocated behind the last one too)
    ldc = codes.stride(0) if rows > 1 else max(codes.stride(0), -(-cols // 16) * 16)
    behind = codes.untyped_storage().nbytes() - codes.storage_offset() - (rows - 1) * ldc
    if rows and cols and behind < -(-cols // 16) * 16:
        raise AmError(f"codes of {name} must have room for a multiple of 16 codes in every row")
    lds = scales.stride(0) if scales.shape[0] > 1 else max(scales.stride(0), scales.shape[1])
    return codes.data_ptr(), ldc, scales.data_ptr(), lds


def q8_quantise(x, codes=None, scales=None, codes_t=None, scales_t=None, tiles=False, stream=None):
    """x [rows][cols] fp32 or bf16 (rows may be columns of a wider matrix) in 8 bits, as
    it lies and, with codes_t and scales_t, transposed; see q8_empty."""
    dt, (rows, cols) = _dtype(x, "x"), x.shape
    xp, ld = _row(x, "x", rows, cols, x.dtype)
    call = (rows, cols, dt, xp, ld, 1 if tiles else 0, *_q8(codes, scales, "x", rows, cols, tiles),
            *_q8(codes_t, scales_t, "x transposed", cols, rows, tiles))
    _here(stream, "x codes scales codes_t scales_t", x, codes, scales, codes_t, scales_t)
    st = (_lib or lib()).q8_quantise(*call, _stream(stream))
    if st:
        _check(st)


def q8_matmul_workspace_bytes(M, N, K) -> int:
    n = lib().am_q8_matmul_workspace_bytes(M, N, K)
    if n < 0:
        raise AmError("invalid sizes for workspace query", EINVAL)
    return int(n)


def q8_matmul(a, a_scales, b, b_scales, out, tiles=False, bias=None, accumulate=False, ws=None, stream=None):
    """out [M][N] bf16 = a [M][K] b [N][K]^T of matrices in 8 bits (+ bias [N] fp32) (+
    out); tiles: b has a scale for each 128 x 128."""
    if a.dim() != 2 or b.dim() != 2 or a.shape[1] != b.shape[1]:
        raise AmError(f"a and b must be [M][K] and [N][K], got {tuple(a.shape)} and {tuple(b.shape)}")
    (M, K), N = a.shape, b.shape[0]
    op, ldo = _row(out, "out", M, N, torch.bfloat16)
    wp, wn = _workspace(ws)
    call = (M, N, K, *_q8(a, a_scales, "a", M, K), *_q8(b, b_scales, "b", N, K, tiles), 1 if tiles else 0,
            _shaped(bias, "bias", (N,)), op, ldo, 1 if accumulate else 0, wp, wn)
    _here(stream, "a a_scales b b_scales bias out ws", a, a_scales, b, b_scales, bias, out, ws)
    st = (_lib or lib()).q8_matmul(*call, _stream(stream))
    if st:
        _check(st)


def gated_norm_forward_q8(res, codes, scales, o=None, gate=None, w_post=None, scale=None, w_next=None,
                          res_out=None, y=None, rstd=None, eps=1e-6, stream=None):
    """gated_norm_forward whose norm leaves in 8 bits, and in y if that is given."""
    (N, H), act = res.shape, o if o is not None else y if y is not None else res
    (op, ldo), (gp, ldg) = _row(o, "o", N, H, act.dtype), _row(gate, "gate", N, H, act.dtype)
    call = (N, H, _dtype(act, "o"), _dtype(res, "res"), op, ldo, gp, ldg, _shaped(w_post, "w_post", (H,)),
            _shaped(scale, "scale", (H,)), _shaped(res, "res", (N, H), res.dtype),
            _shaped(w_next, "w_next", (H,)), float(eps), _shaped(res_out, "res_out", (N, H), res.dtype),
            _shaped(y, "y", (N, H), act.dtype), _shaped(rstd, "rstd", (N, 2)),
            *_q8(codes, scales, "y", N, H))
    _here(stream, "res o gate w_post scale w_next res_out y rstd codes scales", res, o, gate, w_post, scale, w_next,
          res_out, y, rstd, codes, scales)
    st = (_lib or lib()).gated_norm_forward_q8(*call, _stream(stream))
    if st:
        _check(st)


class _AdamWTensor(ctypes.Structure):
    _fields_ = [("n", _I64)] + [(k, _P) for k in ("master", "weights_bf16", "grad", "m", "v", "m_scale",
                                                  "v_scale")] + [("weight_decay", _F64)]


ADAMW_BLOCK = 256  # elements that share a scale of 8-bit moments


def adamw_scales(n) -> int:
    """Scales of each 8-bit moment of a tensor of n elements."""
    return -(-n // ADAMW_BLOCK)


class AdamWTensors:
    """The tensors of an optimizer step, as adamw_apply takes them: a list of
    dicts of contiguous GPU tensors `master` (fp32), `grad` (fp32 or bf16, alike
    in all of them), `m` and `v` (fp32, or 8-bit: torch.float8_e4m3fn or uint8,
    then with fp32 `m_scale` and `v_scale` of adamw_scales(n) elements),
    optionally `weights_bf16`, and a number `weight_decay`.  The list keeps the
    tensors alive and passes the addresses that they have when it is made; it holds
    nothing of a step.  Making it costs some microseconds a tensor, more than a small
    step itself, so a program makes it once and writes its gradients into the same
    tensors each step; gradients allocated anew need a new list."""

    def __init__(self, tensors):
        self.tensors = [dict(t) for t in tensors]
        self.array = (_AdamWTensor * max(1, len(self.tensors)))()
        for k, t in enumerate(self.tensors):
            for name in ("master", "grad", "m", "v"):
                if not isinstance(t.get(name), torch.Tensor):
                    raise AmError(f"tensor {k} has no {name}")
        first = self.tensors[0] if self.tensors else None
        self.grad_dtype = _dtype(first["grad"], "grad") if first else F32
        self.state_bits = 32 if first is None or first["m"].dtype == torch.float32 else 8
        codes = (torch.float8_e4m3fn, torch.uint8)
        for k, t in enumerate(self.tensors):
            n, out = t["master"].numel(), self.array[k]
            out.n, out.weight_decay = n, float(t.get("weight_decay", 0.0))
            kinds = {"master": torch.float32, "weights_bf16": torch.bfloat16, "grad": first["grad"].dtype,
                     "m": torch.float32, "v": torch.float32, "m_scale": torch.float32,
                     "v_scale": torch.float32}
            for name, kind in kinds.items():
                v = t.get(name)
                if v is None:
                    if self.state_bits == 8 and "scale" in name:
                        raise AmError(f"tensor {k} has no {name}")
                    continue
                if name in ("m", "v") and self.state_bits == 8:
                    if v.dtype not in codes:
                        raise AmError(f"tensor {k}: {name} must be torch.float8_e4m3fn or uint8")
                    kind = v.dtype
                if "scale" in name and self.state_bits == 32:
                    raise AmError(f"tensor {k}: {name} with 32-bit moments")
                if v.numel() != (adamw_scales(n) if "scale" in name else n):
                    raise AmError(f"tensor {k}: {name} has {v.numel()} elements")
                setattr(out, name, _dev(v, f"tensor {k}: {name}", kind))

    def __len__(self):
        return len(self.tensors)


def adamw_apply(tensors, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, seed=0,
                stream=None):
    """One AdamW step of an AdamWTensors; grad_scale: [1] fp32 GPU tensor that the
    gradients are multiplied by; seed: of the rounding of 8-bit moments."""
    st = (_lib or lib()).adamw_apply(
        len(tensors), tensors.array, tensors.grad_dtype, tensors.state_bits, float(lr), float(beta1),
        float(beta2), float(eps), int(step), _shaped(grad_scale, "grad_scale", (1,)),
        int(seed) & 0xFFFFFFFF, _stream(stream))
    if st:
        _check(st)


# ------------------------------------------------------------------ timing --

def profile_begin(classes, every=1):
    """Brackets the launches of `classes` with HIP events; with every > 1
    only every n-th launch of each class is bracketed."""
    mask = 0
    for k in classes:
        mask |= 1 << k
    _check(lib().am_profile_sample_every(int(every)))
    _check(lib().am_profile_begin(mask))


def profile_end():
    _check(lib().am_profile_end())


def profile_get(kernel_class):
    n = ctypes.c_int64()
    ms, fl, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    _check(lib().am_profile_get(kernel_class, ctypes.byref(n), ctypes.byref(ms),
                                ctypes.byref(fl), ctypes.byref(by)))
    return {"launches": n.value, "ms": ms.value, "flops": fl.value, "bytes": by.value}
