"""Thin ctypes binding of the LM head's other objectives (include/mst_objective.h, in libmst_lmhead.so): argument checks and
marshalling only.

Cross-entropy of capped logits with token weights (wce) and distillation from a teacher's largest logits run in the HIP kernels
behind the C ABI.  PyTorch appears here only as the owner of device memory and of the stream.  There is no CPU fallback.

A C call takes addresses and cannot see what they are of; the functions here refuse tensors whose shape, type, layout or device
is not what the call reads or writes (MstError, with the C call's status).
"""
from __future__ import annotations

import ctypes

import torch

from .binding import MST_OK, MstError, load_library
from .norm_binding import BAD_ARGUMENT, BAD_SHAPE, NO_DEVICE, TYPE_BF16, TYPE_FP32, _raw_stream, _refuse, _stream_handle

_BF16, _FP32, _INT32, _INT64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
NULL_POINTER = -1                                    # MST_ERR_NULL_POINTER
MAX_ENTRIES = 256                                    # MST_MAX_ENTRIES

_ready = False


def _lib():
    global _ready
    lib = load_library()
    if not _ready:
        c = ctypes
        p, i32, i64, f32, size = c.c_void_p, c.c_int32, c.c_int64, c.c_float, c.c_size_t
        lib.mst_objective_bytes.argtypes = [i64, i64, i64, i32, i32] + [c.POINTER(size)] * 3
        lib.mst_lmhead_wce_fwd.argtypes = [p] * 4 + [i64] * 3 + [i32, i32, f32, f32, i64, p, size, p, size] + [p] * 5
        lib.mst_lmhead_wce_bwd.argtypes = [p, p, i64, i64, i64, i32, f32, p, size, p, size, p, p, p]
        lib.mst_lmhead_distill_fwd.argtypes = ([p] * 6 + [i32, p] + [i64] * 3 + [i32] * 3 + [f32] * 4 + [i64, p, size, p, size] + [p] * 5)
        lib.mst_lmhead_distill_bwd.argtypes = [p, p, i64, i64, i64, i32, i32, f32, p, size, p, size, p, p, p]
        for name in ("mst_objective_bytes", "mst_lmhead_wce_fwd", "mst_lmhead_wce_bwd", "mst_lmhead_distill_fwd", "mst_lmhead_distill_bwd"):
            getattr(lib, name).restype = c.c_int
        _ready = True
    return lib


def _check(status: int) -> None:
    if status != MST_OK:
        raise MstError(status, load_library().mst_strerror(status).decode())


def _int(name: str, value: int, lo: int, hi: int) -> int:
    """ctypes keeps the low bits of what does not fit."""
    if not lo <= value <= hi:
        raise MstError(BAD_ARGUMENT, f"{name}: {value}")
    return value


def _int32(name: str, value: int) -> int:
    return _int(name, value, -(1 << 31), (1 << 31) - 1)


class _Head:
    """The tensors of one call: `at` checks each for what the call expects, `ready` that they are on the current GPU."""

    __slots__ = ("S", "d", "V", "device", "h", "w")

    def __init__(self, H, W):
        for name, t in (("H", H), ("W", W)):
            if t is None or t.dim() != 2:
                raise MstError(BAD_SHAPE, f"{name}: a matrix is needed")
        self.S, self.d = H.shape
        self.V = W.shape[0]
        self.device = H.get_device()
        self.h = self.at("H", H, _BF16, H.shape)
        self.w = self.at("W", W, _BF16, (self.V, self.d))

    def at(self, name: str, t, dtype, shape):
        """Address of t (None: NULL)."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self.device:
            _refuse(name, t, dtype, shape)
        return t.data_ptr()

    def rows(self, name: str, t, dtype=_FP32):
        return self.at(name, t, dtype, (self.S,))

    def scalar(self, name: str, t, dtype=_FP32):
        return self.at(name, t, dtype, (1,) if t is None or t.dim() else ())

    def room(self, name: str, t):
        if t is None:
            return None, 0
        if not t.is_contiguous() or t.get_device() != self.device:
            _refuse(name, t, t.dtype, t.shape)
        return t.data_ptr(), t.nbytes

    def ready(self, stream):
        """Handle of the stream to enqueue on."""
        if self.device < 0 or self.device != torch.cuda.current_device():
            raise MstError(NO_DEVICE, f"tensors on {f'GPU {self.device}' if self.device >= 0 else 'the CPU'}, expected the current GPU")
        if stream is not None and stream.device.index != self.device:
            raise MstError(NO_DEVICE, f"stream of {stream.device}, tensors on GPU {self.device}")
        return _raw_stream(self.device) if stream is None and _raw_stream else _stream_handle(stream)


def mst_objective_bytes(S: int, d: int, V: int, M: int, K: int = 0):
    """(forward workspace, backward workspace, saved) in bytes.  K: the teacher's entries of a row, 0 for wce."""
    n = [ctypes.c_size_t(0) for _ in range(3)]
    _check(_lib().mst_objective_bytes(S, d, V, _int32("M", M), _int32("K", K), *(ctypes.byref(x) for x in n)))
    return tuple(int(x.value) for x in n)


def mst_lmhead_wce_fwd(H, W, labels, ignore_index: int, M: int, workspace, loss, saved=None, weights=None, softcap: float = 0.0,
                       z_coef: float = 0.0, divisor: int = 0, nll=None, lse=None, n_valid=None, stream=None) -> None:
    """Enqueue the forward pass of the weighted cross-entropy of capped logits.  H bf16 [S,d], W bf16 [V,d], labels int32 [S],
    weights fp32 [S] or None; loss fp32 [1], nll and lse fp32 [S] or None, n_valid int64 [1] or None are overwritten, and saved
    (None without a backward pass)."""
    t = _Head(H, W)
    y, wt = t.rows("labels", labels, _INT32), t.rows("weights", weights)
    out, a, b, n = t.scalar("loss", loss), t.rows("nll", nll), t.rows("lse", lse), t.scalar("n_valid", n_valid, _INT64)
    (ws, size), (sv, sv_size) = t.room("workspace", workspace), t.room("saved", saved)
    if out is None or y is None:
        raise MstError(NULL_POINTER, "labels and loss are needed")
    _check(_lib().mst_lmhead_wce_fwd(t.h, t.w, y, wt, t.S, t.d, t.V, _int32("ignore_index", ignore_index), _int32("M", M), softcap, z_coef,
                                     _int("divisor", divisor, 0, (1 << 63) - 1), ws, size, sv, sv_size, out, a, b, n, t.ready(stream)))


def mst_lmhead_wce_bwd(H, W, M: int, grad_loss: float, saved, workspace, dH, dW, stream=None) -> None:
    """Enqueue the gradients of mst_lmhead_wce_fwd's loss, from what it left in saved.  dH bf16 [S,d] and dW fp32 [V,d] are fully
    overwritten."""
    t = _Head(H, W)
    dh, dw = t.at("dH", dH, _BF16, (t.S, t.d)), t.at("dW", dW, _FP32, (t.V, t.d))
    (ws, size), (sv, sv_size) = t.room("workspace", workspace), t.room("saved", saved)
    _check(_lib().mst_lmhead_wce_bwd(t.h, t.w, t.S, t.d, t.V, _int32("M", M), grad_loss, sv, sv_size, ws, size, dh, dw, t.ready(stream)))


def mst_lmhead_distill_fwd(H, W, teacher_index, teacher_logits, M: int, workspace, loss, saved=None, teacher_lse=None, labels=None,
                           ignore_index: int = -100, weights=None, softcap: float = 0.0, label_coef: float = 0.0, teacher_coef: float = 1.0,
                           temperature: float = 1.0, divisor: int = 0, nll=None, kd=None, n_valid=None, stream=None) -> None:
    """Enqueue the forward pass of the distillation loss.  teacher_index int32 [S,K], below 0 for no entry; teacher_logits bf16 or
    fp32 [S,K]; teacher_lse fp32 [S], the log-sum-exp of all the teacher's logits divided by the temperature, or None: its shares are
    those among its entries.  labels int32 [S] or None (label_coef 0).  loss fp32 [1], nll and kd fp32 [S] or None, n_valid int64 [1]
    or None are overwritten, and saved (None without a backward pass)."""
    t = _Head(H, W)
    if teacher_index is None or teacher_logits is None or teacher_index.dim() != 2:
        raise MstError(BAD_SHAPE, "teacher_index and teacher_logits: matrices [S, K] are needed")
    K = teacher_index.shape[1]
    index = t.at("teacher_index", teacher_index, _INT32, (t.S, K))
    bf16 = teacher_logits.dtype is _BF16
    logits = t.at("teacher_logits", teacher_logits, _BF16 if bf16 else _FP32, (t.S, K))
    y, wt, tl = t.rows("labels", labels, _INT32), t.rows("weights", weights), t.rows("teacher_lse", teacher_lse)
    out, a, b, n = t.scalar("loss", loss), t.rows("nll", nll), t.rows("kd", kd), t.scalar("n_valid", n_valid, _INT64)
    (ws, size), (sv, sv_size) = t.room("workspace", workspace), t.room("saved", saved)
    if out is None:
        raise MstError(NULL_POINTER, "loss is needed")
    _check(_lib().mst_lmhead_distill_fwd(t.h, t.w, y, wt, index, logits, TYPE_BF16 if bf16 else TYPE_FP32, tl, t.S, t.d, t.V, _int32("K", K),
                                         _int32("ignore_index", ignore_index), _int32("M", M), softcap, label_coef, teacher_coef, temperature,
                                         _int("divisor", divisor, 0, (1 << 63) - 1), ws, size, sv, sv_size, out, a, b, n, t.ready(stream)))


def mst_lmhead_distill_bwd(H, W, K: int, M: int, grad_loss: float, saved, workspace, dH, dW, stream=None) -> None:
    """Enqueue the gradients of mst_lmhead_distill_fwd's loss, from what it left in saved; K as there.  dH bf16 [S,d] and dW fp32
    [V,d] are fully overwritten."""
    t = _Head(H, W)
    dh, dw = t.at("dH", dH, _BF16, (t.S, t.d)), t.at("dW", dW, _FP32, (t.V, t.d))
    (ws, size), (sv, sv_size) = t.room("workspace", workspace), t.room("saved", saved)
    _check(_lib().mst_lmhead_distill_bwd(t.h, t.w, t.S, t.d, t.V, _int32("K", K), _int32("M", M), grad_loss, sv, sv_size, ws, size, dh, dw,
                                         t.ready(stream)))
