"""Binding of the block-scaled operands (fp4_mx_* of include/fp4_linear.h): argument marshalling only, the tensors' part of it in
csrc/mx_call.cpp.

Tensors may have any row stride (their last dimension is contiguous); the calls run on the context's device,
on the stream that is current there.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
import sys

import torch

from .binding import Context, _check, _ptr, load_library
from .build import call_path

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


class fp4_mx_matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ld", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class fp4_mx_tensor(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("codes", C.c_void_p), ("scales", C.c_void_p),
                ("codes_t", C.c_void_p), ("scales_t", C.c_void_p), ("amax", C.c_void_p), ("format", C.c_int32),
                ("flags", C.c_int32)]


ENTRIES = ("quantize", "dequantize", "gemm", "linear_fwd", "linear_bwd", "swiglu_fwd", "swiglu_bwd")
QUANTIZE, DEQUANTIZE, GEMM, LINEAR_FWD, LINEAR_BWD, SWIGLU_FWD, SWIGLU_BWD = range(7)


class _Calls:
    """The functions of the module _mx_call, which is loaded when the first of them is asked for: the library's other calls need no
    part of it."""

    def __getattr__(self, name: str):
        module = _load_call()
        self.__dict__.update({f: getattr(module, f) for f in ENTRIES})
        return getattr(module, name)


def _load_call():
    """The module of this torch and this interpreter (build.call_path); one that was built for others is not looked at."""
    name = __package__ + "._mx_call"
    if name not in sys.modules:
        path = call_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with `python -m paper_2501_17116_b200.build`", name=name, path=path)
        spec = importlib.util.spec_from_file_location(name, path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        sys.modules[name] = module
    if sys.modules[name] is None:
        raise ImportError(f"import of {name} halted; None in sys.modules", name=name)
    return sys.modules[name]


_call = _Calls()


def declare(lib: C.CDLL):
    """Prototypes of the fp4_mx_* functions, and the addresses that _mx_call takes."""
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    mat, ten = C.POINTER(fp4_mx_matrix), C.POINTER(fp4_mx_tensor)
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
    lib.mx_entries = tuple(C.cast(getattr(lib, "fp4_mx_" + name), vp).value for name in ENTRIES)


_stream_of = torch._C._cuda_getCurrentRawStream


def _head(ctx: Context, entry: int):
    """What every call begins with."""
    return ctx.lib.mx_entries[entry], ctx.handle.value, _stream_of(ctx.device), ctx.status.data_ptr(), ctx.device


def _tensor(ctx: Context, q):
    """Address of an operand's structure (None: of none)."""
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
        self.ref = C.addressof(self.struct)
        self.device = (self.codes if codes else self.codes_t).get_device() if codes or codes_t else -1


class SwigluCheckpoint:
    """gate and up of a SwiGLU in 8 bits (FP4_MX_E4M3), for its backward pass."""

    def __init__(self, rows: int, cols: int, device):
        self.gate = MXTensor(rows, cols, device, fmt=FP4_MX_E4M3)
        self.up = MXTensor(rows, cols, device, fmt=FP4_MX_E4M3)


def fp4_mx_quantize(ctx: Context, x: torch.Tensor, fmt: int = FP4_MX_E2M1, codes: bool = True, codes_t: bool = False,
                    out: MXTensor | None = None, amax: torch.Tensor | None = None) -> MXTensor:
    """`x` in blocks along its columns (`codes`) and / or its rows (`codes_t`).  `amax` (FP4_MX_NVFP4, the other formats have no
    use for it; one finite float) is taken for the tensor's largest magnitude instead of looking for it."""
    if out is None:
        out = MXTensor(*x.shape, x.device, fmt, codes, codes_t)
    at = _tensor(ctx, out)
    given = amax is not None and out.amax is not None
    if given:
        # (in a structure of the call's own: a call that is refused leaves the operand, its amax and its flags as they were)
        amax = amax.detach().to(out.amax.device, torch.float32).reshape(1)
        struct = fp4_mx_tensor.from_buffer_copy(out.struct)
        struct.amax, struct.flags, at = amax.data_ptr(), struct.flags | FP4_MX_AMAX_GIVEN, C.addressof(struct)
    _check(_call.quantize(*_head(ctx, QUANTIZE), x, at))
    if given:
        out.amax.copy_(amax)
    return out


def fp4_mx_dequantize(ctx: Context, q: MXTensor, transposed: bool = False, dtype=torch.bfloat16,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """The values of `q.codes` [rows x cols], or of `q.codes_t` [cols x rows]."""
    if out is None:
        out = _new(ctx, *((q.cols, q.rows) if transposed else (q.rows, q.cols)), dtype)
    _check(_call.dequantize(*_head(ctx, DEQUANTIZE), _tensor(ctx, q), int(transposed), out))
    return out


def fp4_mx_gemm(ctx: Context, a: MXTensor, b: MXTensor, a_t: bool = False, b_t: bool = False, dtype=torch.bfloat16,
                out: torch.Tensor | None = None, accumulate: bool = False) -> torch.Tensor:
    """out (+)= a b^T over the rows' blocks of each operand: of `codes`, or with a_t / b_t of `codes_t`."""
    if out is None:
        assert not accumulate
        out = _new(ctx, a.cols if a_t else a.rows, b.cols if b_t else b.rows, dtype)
    flags = (FP4_MX_A_T if a_t else 0) | (FP4_MX_B_T if b_t else 0) | (FP4_MX_ACCUMULATE if accumulate else 0)
    _check(_call.gemm(*_head(ctx, GEMM), _tensor(ctx, a), _tensor(ctx, b), flags, out))
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
    reuse = (FP4_REUSE_X if reuse_x else 0) | (FP4_REUSE_W if reuse_w else 0)
    _check(_call.linear_fwd(*_head(ctx, LINEAR_FWD), None if reuse_x else X, None if reuse_w else W, M, K, N, reuse, out, _tensor(ctx, saved_x),
                            _tensor(ctx, saved_w)))
    return out, saved_x, saved_w


def fp4_mx_linear_bwd(ctx: Context, dY: torch.Tensor, saved_x: MXTensor | None, saved_w: MXTensor | None, dtype=None,
                      dX: torch.Tensor | None = None, dW: torch.Tensor | None = None, want_dx: bool = True,
                      want_dw: bool = True, accumulate_dx: bool = False, accumulate_dw: bool = False):
    """dX = Q(dY) Q(W)^T and dW = Q(X)^T Q(dY).  `saved_x` may be None where dW is not wanted, `saved_w` where dX is not."""
    M, N = dY.shape
    K = saved_x.cols if want_dw or dW is not None else saved_w.rows
    if dX is None and want_dx:
        assert not accumulate_dx
        dX = _new(ctx, M, K, dtype or dY.dtype)
    if dW is None and want_dw:
        assert not accumulate_dw
        dW = _new(ctx, K, N, dtype or dY.dtype)
    flags = (FP4_MX_ACCUMULATE_DX if accumulate_dx else 0) | (FP4_MX_ACCUMULATE_DW if accumulate_dw else 0)
    _check(_call.linear_bwd(*_head(ctx, LINEAR_BWD), dY, _tensor(ctx, saved_x), _tensor(ctx, saved_w), M, K, N, flags, dX, dW))
    return dX, dW


def fp4_mx_swiglu_fwd(ctx: Context, gate: torch.Tensor, up: torch.Tensor, out: torch.Tensor | None = None,
                      checkpoint: SwigluCheckpoint | None = None, quantized: MXTensor | None = None, want_h: bool = True):
    """h = gate * sigmoid(gate) * up, the inputs in 8 bits into `checkpoint`, h as an operand into `quantized`."""
    shape = rows, cols = gate.shape
    if out is None and want_h:
        out = _new(ctx, rows, cols, gate.dtype)
    g = u = q = None
    if checkpoint is not None:
        assert (checkpoint.gate.rows, checkpoint.gate.cols) == shape
        g, u = _tensor(ctx, checkpoint.gate), _tensor(ctx, checkpoint.up)
    if quantized is not None:
        assert (quantized.rows, quantized.cols) == shape
        q = _tensor(ctx, quantized)
    _check(_call.swiglu_fwd(*_head(ctx, SWIGLU_FWD), gate, up, rows, cols, out, g, u, q))
    return out, checkpoint, quantized


def fp4_mx_swiglu_bwd(ctx: Context, dh: torch.Tensor, checkpoint: SwigluCheckpoint, dgate: torch.Tensor | None = None,
                      dup: torch.Tensor | None = None, h: torch.Tensor | None = None, quantized: MXTensor | None = None):
    """d_gate and d_up from the checkpoint; h made again into `h` and / or, as an operand, into `quantized`."""
    shape = rows, cols = dh.shape
    dgate = _new(ctx, rows, cols, dh.dtype) if dgate is None else dgate
    dup = _new(ctx, rows, cols, dh.dtype) if dup is None else dup
    q = None
    if quantized is not None:
        assert (quantized.rows, quantized.cols) == shape
        q = _tensor(ctx, quantized)
    _check(_call.swiglu_bwd(*_head(ctx, SWIGLU_BWD), dh, _tensor(ctx, checkpoint.gate), _tensor(ctx, checkpoint.up), rows, cols, dgate, dup, h, q))
    return dgate, dup
