"""Binding of the block-scaled operands (fp4_mx_* of include/fp4_linear.h): argument marshalling only.

Tensors may have any row stride (their last dimension is contiguous); the calls run on the context's device,
on the stream that is current there.
"""
from __future__ import annotations

import ctypes as C
from struct import Struct

import torch

from .binding import Context, _check, _ptr, load_library

FP4_MX_E2M1 = 0
FP4_MX_NVFP4 = 1
FP4_MX_E4M3 = 2
FP4_DTYPE_BF16 = 0
FP4_DTYPE_FP16 = 1
FP4_DTYPE_FP32 = 2
FP4_MX_AMAX_GIVEN = 1
FP4_MX_A_T = 1
FP4_MX_B_T = 2
FP4_MX_ACCUMULATE = 4
FP4_MX_ACCUMULATE_DX = 1
FP4_MX_ACCUMULATE_DW = 2
FP4_REUSE_W = 1
FP4_REUSE_X = 2


class _Dtypes(dict):
    def __missing__(self, dtype):
        raise AssertionError(f"{dtype}: a matrix is of torch.bfloat16, torch.float16 or torch.float32")


_DTYPES = _Dtypes({torch.bfloat16: FP4_DTYPE_BF16, torch.float16: FP4_DTYPE_FP16, torch.float32: FP4_DTYPE_FP32})


class fp4_mx_matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ld", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class fp4_mx_tensor(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("codes", C.c_void_p), ("scales", C.c_void_p),
                ("codes_t", C.c_void_p), ("scales_t", C.c_void_p), ("amax", C.c_void_p), ("format", C.c_int32),
                ("flags", C.c_int32)]


def declare(lib: C.CDLL):
    """Prototypes of the fp4_mx_* functions."""
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    mat, ten = vp, C.POINTER(fp4_mx_tensor)          # (an fp4_mx_matrix by reference, or its bytes)
    lib.fp4_mx_pitch.argtypes, lib.fp4_mx_pitch.restype = [i64, i32], i64
    lib.fp4_mx_scale_bytes.argtypes, lib.fp4_mx_scale_bytes.restype = [i64, i64, i32], i64
    lib.fp4_mx_workspace_bytes.argtypes, lib.fp4_mx_workspace_bytes.restype = [i64, i64, i64], C.c_size_t
    for name, args in (("quantize", [mat, ten, vp]), ("dequantize", [ten, i32, mat, vp]), ("gemm", [ten, ten, i32, mat, vp]),
                       ("linear_fwd", [mat, mat, i64, i64, i64, i32, mat, ten, ten, vp]),
                       ("linear_bwd", [mat, ten, ten, i64, i64, i64, i32, mat, mat, vp]),
                       ("swiglu_fwd", [mat, mat, i64, i64, mat, ten, ten, ten, vp]),
                       ("swiglu_bwd", [mat, ten, ten, i64, i64, mat, mat, mat, ten, vp])):
        f = getattr(lib, "fp4_mx_" + name)
        f.argtypes, f.restype = [vp, vp] + args, i32


_stream_of = torch._C._cuda_getCurrentRawStream
_pack = Struct("@Pqii").pack               # the bytes of an fp4_mx_matrix: a ctypes structure takes three times as long to make
assert Struct("@Pqii").size == C.sizeof(fp4_mx_matrix)


def _matrix(ctx: Context, t):
    """Structure of a matrix (None: of none)."""
    if t is None:
        return None
    rows, cols = t.stride()
    assert t.get_device() == ctx.device and (cols == 1 or t.shape[1] <= 1)
    return _pack(t.data_ptr(), rows, _DTYPES[t.dtype], 0)


def _tensor(ctx: Context, q):
    """Reference to an operand's structure (None: of none)."""
    if q is None:
        return None
    assert q.device == ctx.device, f"an operand on device {q.device}, the context on device {ctx.device}"
    return q.ref


def _new(ctx: Context, rows: int, cols: int, dtype):
    return torch.empty((rows, cols), dtype=dtype, device=f"cuda:{ctx.device}")


class MXTensor:
    """Caller-owned buffers of a block-scaled tensor (struct fp4_mx_tensor).  `codes`: blocks along the columns;
    `codes_t`: blocks along the rows, one row of codes per column."""

    def __init__(self, rows: int, cols: int, device, fmt: int = FP4_MX_E2M1, codes: bool = True, codes_t: bool = False):
        lib = load_library()
        byte = lambda n: torch.empty(n, dtype=torch.uint8, device=device)                     # noqa: E731
        self.rows, self.cols, self.fmt = rows, cols, fmt
        side = lambda r, c: (byte((r, int(lib.fp4_mx_pitch(c, fmt)))), byte(int(lib.fp4_mx_scale_bytes(r, c, fmt))))   # noqa: E731
        self.codes, self.scales = side(rows, cols) if codes else (None, None)
        self.codes_t, self.scales_t = side(cols, rows) if codes_t else (None, None)
        self.amax = torch.zeros(1, dtype=torch.float32, device=device) if fmt == FP4_MX_NVFP4 else None
        # (an empty tensor has no address; a direction is there all the same)
        where = lambda t: None if t is None else (t.data_ptr() or 16)                         # noqa: E731
        self.struct = fp4_mx_tensor(rows, cols, where(self.codes), where(self.scales), where(self.codes_t), where(self.scales_t),
                                    _ptr(self.amax), fmt, 0)
        self.ref = C.byref(self.struct)
        self.device = (self.codes if codes else self.codes_t).get_device() if codes or codes_t else -1


class SwigluCheckpoint:
    """gate and up of a SwiGLU in 8 bits (FP4_MX_E4M3), for its backward pass."""

    def __init__(self, rows: int, cols: int, device):
        self.gate = MXTensor(rows, cols, device, fmt=FP4_MX_E4M3)
        self.up = MXTensor(rows, cols, device, fmt=FP4_MX_E4M3)


def fp4_mx_quantize(ctx: Context, x: torch.Tensor, fmt: int = FP4_MX_E2M1, codes: bool = True, codes_t: bool = False,
                    out: MXTensor | None = None, amax: torch.Tensor | None = None) -> MXTensor:
    """`x` in blocks along its columns (`codes`) and / or its rows (`codes_t`).  `amax` (FP4_MX_NVFP4; one float on the
    device) is taken for the tensor's largest magnitude instead of looking for it."""
    if out is None:
        out = MXTensor(*x.shape, x.device, fmt, codes, codes_t)
    assert x.shape == (out.rows, out.cols)
    given = amax is not None and out.amax is not None
    if given:
        out.amax.copy_(amax.reshape(1))
        out.struct.flags = FP4_MX_AMAX_GIVEN
    rc = ctx.lib.fp4_mx_quantize(ctx.handle, _stream_of(ctx.device), _matrix(ctx, x), _tensor(ctx, out), ctx.status.data_ptr())
    if given:
        out.struct.flags = 0
    _check(rc)
    return out


def fp4_mx_dequantize(ctx: Context, q: MXTensor, transposed: bool = False, dtype=torch.bfloat16,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """The values of `q.codes` [rows x cols], or of `q.codes_t` [cols x rows]."""
    shape = (q.cols, q.rows) if transposed else (q.rows, q.cols)
    if out is None:
        out = _new(ctx, *shape, dtype)
    assert out.shape == shape
    _check(ctx.lib.fp4_mx_dequantize(ctx.handle, _stream_of(ctx.device), _tensor(ctx, q), int(transposed), _matrix(ctx, out),
                                     ctx.status.data_ptr()))
    return out


def fp4_mx_gemm(ctx: Context, a: MXTensor, b: MXTensor, a_t: bool = False, b_t: bool = False, dtype=torch.bfloat16,
                out: torch.Tensor | None = None, accumulate: bool = False) -> torch.Tensor:
    """out (+)= a b^T over the rows' blocks of each operand: of `codes`, or with a_t / b_t of `codes_t`."""
    shape = (a.cols if a_t else a.rows, b.cols if b_t else b.rows)
    if out is None:
        assert not accumulate
        out = _new(ctx, *shape, dtype)
    assert out.shape == shape
    flags = (FP4_MX_A_T if a_t else 0) | (FP4_MX_B_T if b_t else 0) | (FP4_MX_ACCUMULATE if accumulate else 0)
    _check(ctx.lib.fp4_mx_gemm(ctx.handle, _stream_of(ctx.device), _tensor(ctx, a), _tensor(ctx, b), flags, _matrix(ctx, out), ctx.status.data_ptr()))
    return out


def fp4_mx_linear_fwd(ctx: Context, X: torch.Tensor | None, W: torch.Tensor | None, fmt: int = FP4_MX_E2M1,
                      saved_x: MXTensor | None = None, saved_w: MXTensor | None = None, reuse_x: bool = False,
                      reuse_w: bool = False, dtype=None, out: torch.Tensor | None = None):
    """Y = Q(X) Q(W) and the operands for the backward pass.  Without `saved_x` / `saved_w` both are made in both
    directions; buffers without the backward's direction (serving) leave that one out."""
    M, K = (saved_x.rows, saved_x.cols) if reuse_x else X.shape
    N = saved_w.cols if reuse_w else W.shape[1]
    assert K == (saved_w.rows if reuse_w else W.shape[0])
    if saved_x is None:
        saved_x = MXTensor(M, K, X.device, fmt, True, True)
    if saved_w is None:
        saved_w = MXTensor(K, N, W.device, fmt, True, True)
    if not reuse_x:
        assert (saved_x.rows, saved_x.cols) == (M, K)
    if not reuse_w:
        assert (saved_w.rows, saved_w.cols) == (K, N)
    if out is None:
        out = _new(ctx, M, N, dtype or (X.dtype if X is not None else torch.bfloat16))
    assert out.shape == (M, N)
    reuse = (FP4_REUSE_X if reuse_x else 0) | (FP4_REUSE_W if reuse_w else 0)
    _check(ctx.lib.fp4_mx_linear_fwd(ctx.handle, _stream_of(ctx.device), None if reuse_x else _matrix(ctx, X),
                                     None if reuse_w else _matrix(ctx, W), M, K, N, reuse, _matrix(ctx, out),
                                     _tensor(ctx, saved_x), _tensor(ctx, saved_w), ctx.status.data_ptr()))
    return out, saved_x, saved_w


def fp4_mx_linear_bwd(ctx: Context, dY: torch.Tensor, saved_x: MXTensor, saved_w: MXTensor, dtype=None,
                      dX: torch.Tensor | None = None, dW: torch.Tensor | None = None, want_dx: bool = True,
                      want_dw: bool = True, accumulate_dx: bool = False, accumulate_dw: bool = False):
    """dX = Q(dY) Q(W)^T and dW = Q(X)^T Q(dY)."""
    M, N = dY.shape
    K = saved_x.cols if want_dw or dW is not None else saved_w.rows
    if dX is None and want_dx:
        assert not accumulate_dx
        dX = _new(ctx, M, K, dtype or dY.dtype)
    if dW is None and want_dw:
        assert not accumulate_dw
        dW = _new(ctx, K, N, dtype or dY.dtype)
    assert (dX is None or dX.shape == (M, K)) and (dW is None or dW.shape == (K, N))
    flags = (FP4_MX_ACCUMULATE_DX if accumulate_dx else 0) | (FP4_MX_ACCUMULATE_DW if accumulate_dw else 0)
    _check(ctx.lib.fp4_mx_linear_bwd(ctx.handle, _stream_of(ctx.device), _matrix(ctx, dY), _tensor(ctx, saved_x), _tensor(ctx, saved_w), M, K, N,
                                     flags, _matrix(ctx, dX), _matrix(ctx, dW), ctx.status.data_ptr()))
    return dX, dW


def fp4_mx_swiglu_fwd(ctx: Context, gate: torch.Tensor, up: torch.Tensor, out: torch.Tensor | None = None,
                      checkpoint: SwigluCheckpoint | None = None, quantized: MXTensor | None = None, want_h: bool = True):
    """h = gate * sigmoid(gate) * up, the inputs in 8 bits into `checkpoint`, h as an operand into `quantized`."""
    shape = rows, cols = gate.shape
    if out is None and want_h:
        out = _new(ctx, rows, cols, gate.dtype)
    assert up.shape == shape and (out is None or out.shape == shape)
    g = u = q = None
    if checkpoint is not None:
        assert (checkpoint.gate.rows, checkpoint.gate.cols) == shape
        g, u = _tensor(ctx, checkpoint.gate), _tensor(ctx, checkpoint.up)
    if quantized is not None:
        assert (quantized.rows, quantized.cols) == shape
        q = _tensor(ctx, quantized)
    _check(ctx.lib.fp4_mx_swiglu_fwd(ctx.handle, _stream_of(ctx.device), _matrix(ctx, gate), _matrix(ctx, up), rows, cols,
                                     _matrix(ctx, out), g, u, q, ctx.status.data_ptr()))
    return out, checkpoint, quantized


def fp4_mx_swiglu_bwd(ctx: Context, dh: torch.Tensor, checkpoint: SwigluCheckpoint, dgate: torch.Tensor | None = None,
                      dup: torch.Tensor | None = None, h: torch.Tensor | None = None, quantized: MXTensor | None = None):
    """d_gate and d_up from the checkpoint; h made again into `h` and / or, as an operand, into `quantized`."""
    shape = rows, cols = dh.shape
    dgate = _new(ctx, rows, cols, dh.dtype) if dgate is None else dgate
    dup = _new(ctx, rows, cols, dh.dtype) if dup is None else dup
    assert dgate.shape == shape and dup.shape == shape and (h is None or h.shape == shape)
    q = None
    if quantized is not None:
        assert (quantized.rows, quantized.cols) == shape
        q = _tensor(ctx, quantized)
    _check(ctx.lib.fp4_mx_swiglu_bwd(ctx.handle, _stream_of(ctx.device), _matrix(ctx, dh), _tensor(ctx, checkpoint.gate),
                                     _tensor(ctx, checkpoint.up), rows, cols,
                                     _matrix(ctx, dgate), _matrix(ctx, dup), _matrix(ctx, h), q, ctx.status.data_ptr()))
    return dgate, dup
