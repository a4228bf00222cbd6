"""Products of block-scaled operands whose values are far from 1.

The allowance of test_gpu_mx, 2^-22 (C / 64 + 1) sum |products|, and half a step of the output's type; below its normal range half of its
smallest number, and half of fp32's, in which the result is scaled before it is rounded."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as O
from test_gpu_mx import DT, fmt_of, half_step, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context.for_mx(1024, 1024, 1024)
    yield c
    c.close()


def check_in_range(got, a, b, fmt, before=0.0):
    """Of operands' values a [I x C] and b [J x C]: what is finite comes out finite, what is beyond the type an infinity of its sign.
    (Blocks of 32 are summed at their own magnitude: a sum whose parts leave fp32's range may leave it too, and parts below its normal range
    may count as nothing.  Blocks of 16 are summed without the tensors' powers of two, far inside of it.)"""
    info, steps = torch.finfo(got.dtype), -(-a.shape[1] // 64) + 1
    y, terms = a @ b.T + before, np.abs(a) @ np.abs(b).T
    room = 2.0 ** -22 * steps * terms + 2.0 ** -24 * np.abs(before) + (steps * 2.0 ** -126 if fmt == "mxfp4" else 0.0)
    room = room + half_step(got.dtype) * (np.abs(y) + room) + info.smallest_normal * info.eps / 2 + 2.0 ** -150
    out = host(got)
    summed = terms < info.max if fmt == "mxfp4" else np.ones_like(y, dtype=bool)
    inside = (np.abs(y) + room < info.max) & summed
    assert (inside.any() or fmt == "mxfp4") and np.isfinite(out[inside]).all()
    err = np.abs(np.where(inside, out, 0.0) - np.where(inside, y, 0.0))
    assert (err <= room).all(), f"{(err / room).max():.3g} of the allowance"
    beyond = (np.abs(y) - room > info.max * (1 + info.eps)) & summed
    assert (np.isinf(out) & (np.sign(out) == np.sign(y)))[beyond].all()


def filled(rows, cols, most, seed):
    """Values of either sign up to `most`, which one of them is."""
    x = (2 * torch.rand((rows, cols), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) - 1) * most
    x[rows - 1, cols // 2] = most
    return x


# magnitudes of the operands; the largest ones leave the result inside of fp32's range, or around its end
MAGNITUDES = [(1e-30, 0.02), (1.0, 1.0), (1e35, 0.02), (1e36, 0.02), (3.3e38, 0.005), (3.3e38, 1.0), (3.3e38, 1e-35), (1e20, 1e17), (1e-25, 1e-18), (1e-30, 1e-30)]


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("large,small", MAGNITUDES)
@pytest.mark.parametrize("I", [3, 300])
def test_product_far_from_one(lib, ctx, fmt, large, small, I):
    """The large values on either side, through the kernel of few rows and through tiles."""
    f, J, C = fmt_of(lib, fmt), 260, 512
    for p, q in ((large, small), (small, large)):
        for dt in ("bf16", "fp32"):
            x, w = filled(I, C, p, 1).to(DT[dt]).cuda(), filled(J, C, q, 2).to(DT[dt]).cuda()
            a, b = lib.fp4_mx_quantize(ctx, x, f), lib.fp4_mx_quantize(ctx, w, f)
            av, bv = O.quantize(host(x), fmt).values, O.quantize(host(w), fmt).values
            check_in_range(lib.fp4_mx_gemm(ctx, a, b, dtype=DT[dt]), av, bv, fmt)
            out = torch.full((I, J), 2.0, dtype=DT[dt], device="cuda")
            check_in_range(lib.fp4_mx_gemm(ctx, a, b, out=out, accumulate=True), av, bv, fmt, 2.0)


@pytest.mark.parametrize("large,small", MAGNITUDES)
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("M", [1, 5])
def test_few_tokens_far_from_one(lib, ctx, large, small, given, M):
    """The kernel that makes the tokens' operand itself (blocks of 16: one token, or a given amax)."""
    f, K, N = lib.FP4_MX_NVFP4, 700, 260
    for p, q in ((large, small), (small, large)):
        x, w = filled(M, K, p, 3).float().cuda(), filled(K, N, q, 4).float().cuda()
        wq, saved = lib.fp4_mx_quantize(ctx, w, f, codes=False, codes_t=True), lib.MXTensor(M, K, "cuda", f)
        if given:
            saved.amax.copy_(x.abs().max())
            saved.struct.flags = 1
        y, _, _ = lib.fp4_mx_linear_fwd(ctx, x, None, f, saved, wq, reuse_w=True)
        check_in_range(y, O.quantize(host(x), "nvfp4").values, O.quantize(host(w).T, "nvfp4").values, "nvfp4")
