"""Thin ctypes binding of libmst_norm.so: argument checks and marshalling only.

The norms, residuals, their gradients and the 8-bit checkpoints run in the HIP kernels behind the C ABI declared in
include/mst_norm.h.  PyTorch appears here only as the owner of device memory and of the stream.  There is no CPU fallback:
without the built library the calls fail loudly.

A C call takes addresses and cannot see what they are of; the functions here refuse tensors whose shape, type, layout or device
is not what the call reads or writes (MstError, with the C call's status).
"""
from __future__ import annotations

import ctypes
import os

import torch

from .binding import MST_OK, MstError, _stream_handle
from .binding import load_library as _load_lmhead_library

HERE = os.path.dirname(os.path.abspath(__file__))
NORM_LIB_PATH = os.path.join(HERE, "libmst_norm.so")

BAD_SHAPE, BAD_ARGUMENT, NO_DEVICE = -2, -8, -7      # MST_ERR_* of include/mst_lmhead.h
TYPE_BF16, TYPE_FP32 = 0, 1                          # MST_TYPE_*

_lib = None


def load_norm_library() -> ctypes.CDLL:
    """Load the in-tree library (built by paper_2407_15892_amd.build.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(NORM_LIB_PATH):
        raise RuntimeError(
            f"{NORM_LIB_PATH} is missing: build it first (python -m paper_2407_15892_amd.build); "
            "there is no fallback path")
    _load_lmhead_library()      # loads PyTorch's HIP runtime globally first; also provides mst_strerror
    lib = ctypes.CDLL(NORM_LIB_PATH)
    c = ctypes
    p, i32, i64, f32, size = c.c_void_p, c.c_int32, c.c_int64, c.c_float, c.c_size_t
    lib.mst_norm_version.restype = c.c_char_p
    lib.mst_norm_version.argtypes = []
    lib.mst_norm_workspace_bytes.argtypes = [i64, i64, i64, c.POINTER(size)]
    lib.mst_norm_bwd_info.argtypes = [i64, i64, i64, i32, c.POINTER(i64)]
    lib.mst_ckpt_pack.argtypes = [p, i32, i64, i64, p, p, p]
    lib.mst_ckpt_unpack.argtypes = [p, p, i64, i64, p, i32, p]
    lib.mst_prenorm_fwd.argtypes = [p, i32, p, f32, f32, i64, i64, p, p, p, p]
    lib.mst_prenorm_rebuild.argtypes = [p, p, p, f32, f32, i64, i64, p, p]
    lib.mst_prenorm_bwd.argtypes = [p] * 5 + [i32, p, f32, f32, i64, i64, p, size, p, p, p]
    lib.mst_residual_fwd.argtypes = [p, p, i32, i32, p, f32, f32, p, i64, f32, i64, i64, p, p, p, p]
    lib.mst_residual_bwd.argtypes = [p, i32, p, p, p, i32, p, f32, f32, p, i64, f32, i64, i64, p, size, p, p, p, p]
    lib.mst_residual_prenorm_fwd.argtypes = [p, p, i32, i32, p, p, i64, f32, p, f32, f32, i64, i64] + [p] * 7
    lib.mst_residual_prenorm_bwd.argtypes = ([p, p, i32] + [p] * 6 + [i32, p, p, i64, f32, p, f32, f32, i64, i64, p, size] + [p] * 6)
    for name in ("mst_norm_workspace_bytes", "mst_norm_bwd_info", "mst_ckpt_pack", "mst_ckpt_unpack", "mst_prenorm_fwd",
                 "mst_prenorm_rebuild", "mst_prenorm_bwd", "mst_residual_fwd", "mst_residual_bwd", "mst_residual_prenorm_fwd",
                 "mst_residual_prenorm_bwd"):
        getattr(lib, name).restype = c.c_int
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != MST_OK:
        raise MstError(status, _load_lmhead_library().mst_strerror(status).decode())


_BF16, _FP32, _INT8, _UINT8 = torch.bfloat16, torch.float32, torch.int8, torch.uint8

# A short call on the GPU takes less time than its checks here would if they were written without care: one pass over
# each tensor's attributes, texts only where something is refused.


def _refuse(name, t, dtype, shape):
    if t.dtype is not dtype:
        raise MstError(BAD_ARGUMENT, f"{name}: {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise MstError(BAD_SHAPE, f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise MstError(BAD_ARGUMENT, f"{name}: not contiguous (strides {t.stride()})")
    raise MstError(NO_DEVICE, f"{name}: on {t.device}, not on the device of the other tensors")


class _Tensors:
    """The tensors of one call: `at` checks each for what the call expects, `ready` that they are on the current GPU."""

    __slots__ = ("S", "d", "shape", "stream_dtype", "stream_type", "device")

    def __init__(self, name: str, t):
        """t: the [S, d] tensor of the residual stream (or H) that sets the sizes, the type and the device of the others."""
        if t is None or t.dim() != 2:
            raise MstError(BAD_SHAPE, f"{name}: a tensor [S, d] is needed")
        self.shape = t.shape
        self.S, self.d = t.shape
        self.stream_dtype = t.dtype
        self.device = t.get_device()
        self.stream_type = TYPE_BF16
        if t.dtype is _FP32:
            self.stream_type = TYPE_FP32
        elif t.dtype is not _BF16:
            raise MstError(BAD_ARGUMENT, f"{name}: {t.dtype}, expected {_BF16} or {_FP32}")

    def at(self, name: str, t, dtype, shape):
        """Address of t (None: NULL)."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self.device:
            _refuse(name, t, dtype, shape)
        return t.data_ptr()

    def stream_rows(self, name: str, t):
        return self.at(name, t, self.stream_dtype, self.shape)

    def rows(self, name: str, t):
        return self.at(name, t, _BF16, self.shape)

    def weight(self, name: str, t, dtype=_BF16):
        return self.at(name, t, dtype, (self.d,))

    def checkpoint(self, codes, exps, which: str = ""):
        if codes is None and exps is None:
            return None, None
        return self.at("codes" + which, codes, _INT8, self.shape), self.at("exps" + which, exps, _UINT8, (self.S, (self.d + 31) // 32))

    def gate(self, name: str, t, gate_rows: int, dtype=_BF16):
        if t is None:
            return None
        if not 1 <= gate_rows < 1 << 63:      # ctypes keeps the low 64 bits
            raise MstError(BAD_ARGUMENT, f"{name}: gate_rows is {gate_rows}")
        return self.at(name, t, dtype, (-(-self.S // gate_rows), self.d))

    def workspace(self, t):
        if t is None:
            return None, 0
        if not t.is_contiguous() or t.get_device() != self.device:
            _refuse("workspace", t, t.dtype, t.shape)
        return t.data_ptr(), t.nbytes

    def ready(self, stream):
        """Handle of the stream to enqueue on."""
        if self.device < 0 or self.device != torch.cuda.current_device():
            raise MstError(NO_DEVICE, f"tensors on {f'GPU {self.device}' if self.device >= 0 else 'the CPU'}, expected the current GPU")
        if stream is not None and stream.device.index != self.device:
            raise MstError(NO_DEVICE, f"stream of {stream.device}, tensors on GPU {self.device}")
        return _raw_stream(self.device) if stream is None and _raw_stream else _stream_handle(stream)


# PyTorch's current stream as an integer (0: the default one), without a Stream object around it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def mst_norm_version() -> str:
    return load_norm_library().mst_norm_version().decode()


def mst_norm_workspace_bytes(S: int, d: int, gate_rows: int = 0) -> int:
    """Bytes of workspace of the backward calls; gate_rows as in the call, 0 without a gate."""
    n = ctypes.c_size_t(0)
    _check(load_norm_library().mst_norm_workspace_bytes(S, d, gate_rows, ctypes.byref(n)))
    return int(n.value)


def mst_norm_bwd_info(S: int, d: int, gate_rows: int = 0, prenorm: bool = True) -> dict:
    """How a backward call goes over the rows: threads of a workgroup, teams in it, rows of a team, workgroups, whether a team
    takes whole rows of the gate.  prenorm: False for mst_residual_bwd."""
    info = (ctypes.c_int64 * 5)()
    _check(load_norm_library().mst_norm_bwd_info(S, d, gate_rows, int(prenorm), info))
    return dict(zip(("threads", "teams", "rows", "workgroups", "whole"), (int(x) for x in info)))


def mst_ckpt_pack(X, codes, exps, stream=None) -> None:
    """Enqueue the 8-bit checkpoint of X (bf16 or fp32 [S,d]): codes int8 [S,d], exps uint8 [S,ceil(d/32)]."""
    t = _Tensors("X", X)
    x, (c, e) = t.stream_rows("X", X), t.checkpoint(codes, exps)
    _check(load_norm_library().mst_ckpt_pack(x, t.stream_type, t.S, t.d, c, e, t.ready(stream)))


def mst_ckpt_unpack(codes, exps, X, stream=None) -> None:
    """Enqueue the tensor that a checkpoint stands for, into X (bf16 or fp32 [S,d]; the same values in either)."""
    t = _Tensors("X", X)
    x, (c, e) = t.stream_rows("X", X), t.checkpoint(codes, exps)
    _check(load_norm_library().mst_ckpt_unpack(c, e, t.S, t.d, x, t.stream_type, t.ready(stream)))


def mst_prenorm_fwd(X, w_pre, H, eps: float, w_offset: float = 0.0, codes=None, exps=None, stream=None) -> None:
    """Enqueue the norm before a block.  X bf16 or fp32 [S,d], w_pre bf16 [d] or None (ones); H bf16 [S,d] is overwritten, and
    the checkpoint of X where codes and exps are given."""
    t = _Tensors("X", X)
    x, w, h = t.stream_rows("X", X), t.weight("w_pre", w_pre), t.rows("H", H)
    c, e = t.checkpoint(codes, exps)
    _check(load_norm_library().mst_prenorm_fwd(x, t.stream_type, w, w_offset, eps, t.S, t.d, h, c, e, t.ready(stream)))


def mst_prenorm_rebuild(codes, exps, w_pre, H, eps: float, w_offset: float = 0.0, stream=None) -> None:
    """Enqueue H = norm of the tensor that a checkpoint stands for: a block's input again, for its backward pass."""
    t = _Tensors("H", H)
    w, h, (c, e) = t.weight("w_pre", w_pre), t.rows("H", H), t.checkpoint(codes, exps)
    _check(load_norm_library().mst_prenorm_rebuild(c, e, w, w_offset, eps, t.S, t.d, h, t.ready(stream)))


def mst_prenorm_bwd(dH, w_pre, dX, dw_pre, workspace, eps: float, w_offset: float = 0.0, X=None, codes=None, exps=None, dres=None,
                    stream=None) -> None:
    """Enqueue the gradients of the norm before a block.  dH bf16 [S,d]; X (the type of dX) or its checkpoint; dres (the type of
    dX) or None: what reaches X around the block.  dX bf16 or fp32 [S,d] and dw_pre fp32 [d] (None with w_pre None) are overwritten."""
    t = _Tensors("dX", dX)
    dx = t.stream_rows("dX", dX)
    dh, x, r = t.rows("dH", dH), t.stream_rows("X", X), t.stream_rows("dres", dres)
    w, dw, (c, e) = t.weight("w_pre", w_pre), t.weight("dw_pre", dw_pre, _FP32), t.checkpoint(codes, exps)
    ws, size = t.workspace(workspace)
    _check(load_norm_library().mst_prenorm_bwd(dh, x, c, e, r, t.stream_type, w, w_offset, eps, t.S, t.d, ws, size, dx, dw,
                                               t.ready(stream)))


def mst_residual_fwd(O, X, Y, w=None, gate=None, gate_rows: int = 0, scale: float = 1.0, normalize: bool = True, eps: float = 1e-5,
                     w_offset: float = 0.0, codes=None, exps=None, stream=None) -> None:
    """Enqueue Y = X + scale * gate * norm(O) (or O, normalize False).  O bf16 [S,d], X bf16 or fp32 [S,d], w bf16 [d] or None
    (ones), gate bf16 [ceil(S/gate_rows),d] or None; Y (the type of X) is overwritten, and the checkpoint of O where codes and exps
    are given."""
    t = _Tensors("X", X)
    x = t.stream_rows("X", X)
    o, y, (c, e) = t.rows("O", O), t.stream_rows("Y", Y), t.checkpoint(codes, exps)
    w_, g = t.weight("w", w), t.gate("gate", gate, gate_rows)
    _check(load_norm_library().mst_residual_fwd(o, x, t.stream_type, int(normalize), w_, w_offset, eps, g, gate_rows, scale, t.S, t.d, y, c, e,
                                                t.ready(stream)))


def mst_residual_bwd(dY, dO, workspace, w=None, dw=None, gate=None, gate_rows: int = 0, dgate=None, scale: float = 1.0,
                     normalize: bool = True, eps: float = 1e-5, w_offset: float = 0.0, O=None, codes=None, exps=None, stream=None) -> None:
    """Enqueue the gradients of the residual.  dY bf16 or fp32 [S,d]; O bf16 or its checkpoint (neither is needed without norm and
    gate).  dO bf16 [S,d], dw fp32 [d] (with w) and dgate fp32 (the shape of gate, with it) are overwritten."""
    t = _Tensors("dY", dY)
    dy, do, o = t.stream_rows("dY", dY), t.rows("dO", dO), t.rows("O", O)
    c, e = t.checkpoint(codes, exps)
    w_, dw_ = t.weight("w", w), t.weight("dw", dw, _FP32)
    g, dg = t.gate("gate", gate, gate_rows), t.gate("dgate", dgate, gate_rows, _FP32)
    ws, size = t.workspace(workspace)
    _check(load_norm_library().mst_residual_bwd(dy, t.stream_type, o, c, e, int(normalize), w_, w_offset, eps, g, gate_rows, scale, t.S, t.d,
                                                ws, size, do, dw_, dg, t.ready(stream)))


def mst_residual_prenorm_fwd(O, X, Y, H, w_pre, w_post=None, gate=None, gate_rows: int = 0, scale: float = 1.0, normalize: bool = True,
                             eps: float = 1e-5, w_offset: float = 0.0, codes_o=None, exps_o=None, codes_y=None, exps_y=None,
                             stream=None) -> None:
    """Enqueue mst_residual_fwd and, from its Y, mst_prenorm_fwd, in one pass."""
    t = _Tensors("X", X)
    x = t.stream_rows("X", X)
    o, y, h = t.rows("O", O), t.stream_rows("Y", Y), t.rows("H", H)
    (co, eo), (cy, ey) = t.checkpoint(codes_o, exps_o, "_o"), t.checkpoint(codes_y, exps_y, "_y")
    wo, wp = t.weight("w_post", w_post), t.weight("w_pre", w_pre)
    g = t.gate("gate", gate, gate_rows)
    _check(load_norm_library().mst_residual_prenorm_fwd(o, x, t.stream_type, int(normalize), wo, g, gate_rows, scale, wp, w_offset, eps, t.S, t.d,
                                                        y, h, co, eo, cy, ey, t.ready(stream)))


def mst_residual_prenorm_bwd(dH, dres, dY, dO, workspace, w_pre, dw_pre, w_post=None, dw_post=None, gate=None, gate_rows: int = 0,
                             dgate=None, scale: float = 1.0, normalize: bool = True, eps: float = 1e-5, w_offset: float = 0.0,
                             Y=None, O=None, codes_o=None, exps_o=None, codes_y=None, exps_y=None, stream=None) -> None:
    """Enqueue mst_prenorm_bwd, whose dX is dY, and mst_residual_bwd of that dY, in one pass.  Y (the type of dY) and O (bf16):
    each itself or its checkpoint."""
    t = _Tensors("dY", dY)
    dy = t.stream_rows("dY", dY)
    dh, r, y, o = t.rows("dH", dH), t.stream_rows("dres", dres), t.stream_rows("Y", Y), t.rows("O", O)
    do, (co, eo), (cy, ey) = t.rows("dO", dO), t.checkpoint(codes_o, exps_o, "_o"), t.checkpoint(codes_y, exps_y, "_y")
    wo, wp = t.weight("w_post", w_post), t.weight("w_pre", w_pre)
    dwo, dwp = t.weight("dw_post", dw_post, _FP32), t.weight("dw_pre", dw_pre, _FP32)
    g, dg = t.gate("gate", gate, gate_rows), t.gate("dgate", dgate, gate_rows, _FP32)
    ws, size = t.workspace(workspace)
    _check(load_norm_library().mst_residual_prenorm_bwd(dh, r, t.stream_type, y, cy, ey, o, co, eo, int(normalize), wo, g, gate_rows, scale,
                                                        wp, w_offset, eps, t.S, t.d, ws, size, dy, do, dwp, dwo, dg, t.ready(stream)))
