"""CPU-only checks of the block-scaled entry points: sizes, and every refusal.  The calls validate their arguments before
they touch the device, and read nothing of the context before but its mutex: zeroed bytes stand in for one, and a call that
passes all checks ends with the error of the missing device (or, on a GPU machine, is not made)."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

from paper_2501_17116_b200 import build as fp4_build
import paper_2501_17116_b200 as fp4
from paper_2501_17116_b200.mx import fp4_mx_matrix, fp4_mx_tensor

NULL, ALIGN, CUDA, ARG, RANGE, WORKSPACE = -1, -4, -6, -7, -10, -5
P = 0x10000                                   # an address that is never read


@pytest.fixture(scope="module")
def lib():
    fp4_build.build()
    return fp4.load_library()


@pytest.fixture(scope="module")
def ctx():
    buf = C.create_string_buffer(8192)
    yield C.cast(buf, C.c_void_p)


def mat(ld=64, dtype=0, data=P, reserved=0):
    return fp4_mx_matrix(data, ld, dtype, reserved)


def ten(rows=8, cols=64, fmt=0, codes=True, codes_t=True, amax=None, flags=0, **kw):
    q = fp4_mx_tensor(rows, cols, P if codes else None, P if codes else None, P if codes_t else None, P if codes_t else None,
                      amax if amax is not None else (P if fmt == 1 else None), fmt, flags)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def ref(x):
    return None if x is None else C.byref(x)


def passes(rc):
    """The arguments were accepted: only the device is missing."""
    return rc == CUDA


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would run on made-up addresses")


def test_sizes(lib):
    assert lib.fp4_mx_pitch(1, 0) == 64 and lib.fp4_mx_pitch(128, 1) == 64 and lib.fp4_mx_pitch(129, 2) == 256
    assert lib.fp4_mx_pitch(0, 0) == 0 and lib.fp4_mx_pitch(-1, 0) == -1 and lib.fp4_mx_pitch(1, 3) == -1
    assert lib.fp4_mx_scale_bytes(1, 1, 0) == 512 and lib.fp4_mx_scale_bytes(129, 128, 1) == 2048
    assert lib.fp4_mx_scale_bytes(0, 5, 0) == 0 and lib.fp4_mx_scale_bytes(1 << 31, 5, 0) == -1
    assert lib.fp4_mx_scale_bytes((1 << 31) - 1, (1 << 31) - 1, 0) == -1                      # too many tiles
    M, K, N = 100, 300, 500
    assert lib.fp4_mx_workspace_bytes(M, K, N) >= M * 256 + N * 64 + 2 * 4 * 1024
    assert lib.fp4_mx_workspace_bytes(-1, 1, 1) == 0 and lib.fp4_mx_workspace_bytes(0, 0, 0) > 0


def test_status_string(lib):
    assert b"stride" in lib.fp4_status_string(RANGE)


@no_gpu
def test_quantize_refusals(lib, ctx):
    call = lambda x, q, c=ctx, st=P: lib.fp4_mx_quantize(c, None, ref(x), ref(q), st)          # noqa: E731
    assert passes(call(mat(), ten())) and passes(call(mat(dtype=2), ten(fmt=1))) and passes(call(mat(dtype=1), ten(fmt=2)))
    assert call(mat(), ten(), c=None) == NULL and call(None, ten()) == NULL and call(mat(), None) == NULL
    assert call(mat(), ten(), st=None) == NULL and call(mat(data=None), ten()) == NULL
    assert call(mat(), ten(codes=False, codes_t=False)) == NULL
    assert call(mat(), ten(scales=None)) == NULL and call(mat(), ten(scales_t=None)) == NULL     # a direction that is not complete
    assert call(mat(), ten(fmt=1, amax=0)) == NULL
    assert call(mat(ld=63), ten()) == RANGE and passes(call(mat(ld=0), ten(rows=1)))            # one row: any stride
    assert call(mat(), ten(rows=-1)) == RANGE and call(mat(), ten(cols=1 << 31)) == RANGE
    assert call(mat(dtype=3), ten()) == ARG and call(mat(dtype=-1), ten()) == ARG and call(mat(reserved=1), ten()) == ARG
    assert call(mat(), ten(fmt=3)) == ARG and call(mat(), ten(flags=2)) == ARG
    assert call(mat(data=P + 1), ten()) == ALIGN and call(mat(data=P + 2, dtype=2), ten()) == ALIGN and passes(call(mat(data=P + 2), ten()))
    assert call(mat(), ten(scales=P + 8)) == ALIGN and call(mat(), ten(scales_t=P + 4)) == ALIGN
    assert call(mat(), ten(fmt=1, amax=P + 2)) == ALIGN


@no_gpu
def test_dequantize_refusals(lib, ctx):
    call = lambda q, t, o, c=ctx, st=P: lib.fp4_mx_dequantize(c, None, ref(q), t, ref(o), st)   # noqa: E731
    assert passes(call(ten(), 0, mat())) and passes(call(ten(), 1, mat(ld=8)))
    assert call(ten(), 0, None) == NULL and call(None, 0, mat()) == NULL and call(ten(), 0, mat(), c=None) == NULL and call(ten(), 0, mat(), st=None) == NULL
    assert call(ten(codes_t=False), 1, mat()) == NULL and call(ten(codes=False), 0, mat()) == NULL
    assert call(ten(), 1, mat(ld=7)) == RANGE and call(ten(), 0, mat(ld=63)) == RANGE
    assert call(ten(), 0, mat(data=None)) == NULL and call(ten(rows=0), 0, mat(data=None)) == 0


@no_gpu
def test_gemm_refusals(lib, ctx):
    call = lambda a, b, f, o, c=ctx, st=P: lib.fp4_mx_gemm(c, None, ref(a), ref(b), f, ref(o), st)   # noqa: E731
    assert passes(call(ten(), ten(rows=16), 0, mat(ld=16))) and passes(call(ten(fmt=1), ten(rows=16, fmt=1), 4, mat(ld=16)))
    assert passes(call(ten(), ten(), 3, mat()))                                                # both by columns: C = 8
    assert call(ten(), ten(cols=32), 0, mat()) == RANGE                                        # contractions differ
    assert call(ten(), ten(), 1, mat()) == RANGE
    assert call(ten(), ten(fmt=1), 0, mat()) == ARG and call(ten(fmt=2), ten(fmt=2), 0, mat()) == ARG
    assert call(ten(), ten(), 8, mat()) == ARG
    assert call(ten(codes=False), ten(), 0, mat()) == NULL and call(ten(), ten(codes_t=False, rows=64, cols=64), 2, mat()) == NULL
    assert call(ten(), ten(), 0, mat(ld=7)) == RANGE and call(ten(), ten(), 0, mat(data=None)) == NULL
    assert call(ten(), ten(), 0, mat(), st=None) == NULL and call(None, ten(), 0, mat()) == NULL
    big = (1 << 31) - 1
    assert call(ten(rows=big), ten(rows=big), 0, mat(ld=big)) == RANGE


@no_gpu
def test_linear_refusals(lib, ctx):
    M, K, N = 8, 64, 32
    fwd = lambda x, w, y, sx, sw, reuse=0, c=ctx: lib.fp4_mx_linear_fwd(c, None, ref(x), ref(w), M, K, N, reuse, ref(y), ref(sx), ref(sw), P)  # noqa: E731
    sx, sw = ten(M, K), ten(K, N)
    assert passes(fwd(mat(), mat(ld=32), mat(ld=32), sx, sw))
    assert passes(fwd(mat(), None, mat(ld=32), ten(M, K, codes_t=False), ten(K, N, codes=False), reuse=1))    # serving
    assert passes(fwd(None, None, mat(ld=32), sx, sw, reuse=3))
    assert fwd(mat(), None, mat(ld=32), sx, sw) == NULL and fwd(None, mat(ld=32), mat(ld=32), sx, sw) == NULL
    assert fwd(mat(), mat(ld=32), mat(ld=32), ten(M, K, codes=False), sw) == NULL
    assert fwd(mat(), mat(ld=32), mat(ld=32), sx, ten(K, N, codes_t=False)) == NULL
    assert fwd(mat(), mat(ld=32), mat(ld=32), sx, ten(K, N, fmt=1)) == ARG
    assert fwd(mat(), mat(ld=32), mat(ld=32), sx, sw, reuse=4) == ARG
    assert fwd(mat(), mat(ld=32), mat(ld=32), sx, ten(K, N + 1), reuse=1) == RANGE              # a saved operand of another shape
    assert fwd(mat(), mat(ld=31), mat(ld=32), sx, sw) == RANGE
    bwd = lambda dy, sx, sw, dx, dw, flags=0, c=ctx: lib.fp4_mx_linear_bwd(c, None, ref(dy), ref(sx), ref(sw), M, K, N, flags, ref(dx), ref(dw), P)  # noqa: E731
    dy, dx, dw = mat(ld=32), mat(), mat(ld=32)
    sx, sw = ten(M, K), ten(K, N)
    assert bwd(dy, sx, sw, dx, dw) == WORKSPACE                                                # the stand-in has none
    assert bwd(dy, sx, sw, None, None) == 0 and bwd(dy, sx, sw, dx, dw, flags=4) == ARG
    assert bwd(dy, ten(M, K, codes_t=False), sw, dx, dw) == NULL and bwd(dy, sx, ten(K, N, codes=False), dx, dw) == NULL
    assert bwd(dy, ten(M, K, codes_t=False), sw, dx, None) == WORKSPACE                        # not needed for dX
    assert bwd(dy, ten(M + 1, K), sw, dx, dw) == RANGE and bwd(dy, sx, ten(K, N, fmt=1), dx, dw) == ARG
    assert bwd(mat(ld=31), sx, sw, dx, dw) == RANGE and bwd(dy, sx, sw, mat(ld=63), dw) == RANGE


@no_gpu
def test_swiglu_refusals(lib, ctx):
    R, K = 8, 64
    ck = lambda cols=K: ten(R, cols, fmt=2, codes_t=False)                                  # noqa: E731
    fwd = lambda g, u, h, a, b, q, c=ctx: lib.fp4_mx_swiglu_fwd(c, None, ref(g), ref(u), R, K, ref(h), ref(a), ref(b), ref(q), P)   # noqa: E731
    assert passes(fwd(mat(), mat(ld=128), mat(), ck(), ck(), ten())) and passes(fwd(mat(), mat(), None, None, None, ten(codes_t=False)))
    assert fwd(mat(), mat(), None, None, None, None) == NULL and fwd(mat(), mat(), mat(), ck(), None, None) == NULL
    assert fwd(mat(), mat(dtype=1), mat(), None, None, None) == ARG and fwd(mat(), mat(), mat(dtype=2), None, None, None) == ARG
    assert fwd(mat(), mat(), mat(), ck(), ten(), None) == ARG                                   # a checkpoint is E4M3
    assert fwd(mat(), mat(), mat(), None, None, ten(fmt=1)) == ARG and fwd(mat(), mat(), mat(), None, None, ck()) == ARG
    assert fwd(mat(ld=10), mat(), mat(), None, None, None) == RANGE and fwd(mat(data=None), mat(), mat(), None, None, None) == NULL
    bwd = lambda dh, a, b, dg, du, h=None, q=None, c=ctx: lib.fp4_mx_swiglu_bwd(c, None, ref(dh), ref(a), ref(b), R, K, ref(dg), ref(du), ref(h), ref(q), P)   # noqa: E731
    assert passes(bwd(mat(), ck(), ck(), mat(), mat(), mat(), ten()))
    assert bwd(mat(), ck(), None, mat(), mat()) == NULL and bwd(mat(), ck(), ck(), mat(), None) == NULL
    assert bwd(mat(), ck(), ck(cols=65), mat(), mat()) == RANGE and bwd(mat(), ck(), ck(), mat(ld=1), mat()) == RANGE
    assert bwd(mat(), ck(), ck(), mat(dtype=1), mat()) == ARG and bwd(mat(), ck(), ck(), mat(), mat(), h=mat(dtype=1)) == ARG
    assert bwd(mat(), ck(), ten(R, K), mat(), mat()) == ARG


@no_gpu
def test_one_tensor_in_two_places_is_refused(lib, ctx):
    """What a call writes twice: the second size would not fit the first one's buffers."""
    fwd = lambda x, w, sx, sw, reuse: lib.fp4_mx_linear_fwd(ctx, None, ref(x), ref(w), 64, 64, 64, reuse, ref(mat()), ref(sx), ref(sw), P)   # noqa: E731
    q = ten(64, 64)
    assert passes(fwd(mat(), mat(), q, ten(64, 64), 0)) and passes(fwd(None, None, q, q, 3))
    assert fwd(mat(), mat(), q, q, 0) == ARG and fwd(mat(), None, q, q, 1) == ARG and fwd(None, mat(), q, q, 2) == ARG
    one, other = ten(64, 64, fmt=1), ten(64, 64, fmt=1)
    assert fwd(mat(), mat(), one, other, 0) == ARG and fwd(mat(), None, one, other, 1) == ARG      # one amax for both
    other.amax = P + 4
    assert passes(fwd(mat(), mat(), one, other, 0))
    ck = ten(8, 64, fmt=2, codes_t=False)
    assert lib.fp4_mx_swiglu_fwd(ctx, None, ref(mat()), ref(mat()), 8, 64, None, ref(ck), ref(ck), None, P) == ARG
    gemm = lambda a, b: lib.fp4_mx_gemm(ctx, None, ref(a), ref(b), 0, ref(mat()), P)              # noqa: E731
    assert passes(gemm(q, q))                                                                  # (only read: as good as two)


def test_binding_refuses_an_operand_of_another_device(lib):
    q = fp4.MXTensor(4, 64, "cpu")
    with pytest.raises(AssertionError, match="device"):
        fp4.mx._tensor(SimpleNamespace(device=0), q)
    assert fp4.mx._tensor(SimpleNamespace(device=-1), q) is q.ref                               # (torch's number for the CPU)
    assert fp4.mx._tensor(SimpleNamespace(device=0), None) is None


def test_binding_refuses_what_is_no_matrix_of_the_call(lib):
    """Each is refused ahead of the call (whose address here is of no function)."""
    call, head = fp4.mx._call, (16, None, 0, P, 0)
    q = ten(4, 64)
    at = C.addressof(q)
    for bad in (torch.zeros(4, 64), torch.zeros(4, 63), torch.zeros(64), torch.zeros(2, 2, 64), "a tensor", 7,
                torch.zeros(4, 64, device="meta"), torch.zeros(4, 64).to_sparse()):
        with pytest.raises(AssertionError):
            call.quantize(*head, bad, at)
    with pytest.raises(TypeError):
        call.quantize(*head, None)
    with pytest.raises(TypeError):
        call.gemm(*head, at, at, "flags", None)
    with pytest.raises(ValueError):
        call.quantize(None, None, 0, P, 0, None, at)
