"""A tile's copy that never comes: the kernels that quantise, give values back and make SwiGLU return, say so and write nothing beside their outputs; the
next call is sound.  (The copy is left out by a switch, and nothing is in flight; products: test_gpu_mx.)"""
import pytest
import torch

from test_gpu_mx import check_quantized, draw

pytestmark = pytest.mark.gpu
R, K = 300, 264


def calls(lib, c, fmt):
    """(call into a matrix or None, its reference afterwards) of every kernel that waits for a tile."""
    x, y, dh = draw(R, K, "bf16", 1, 3.0), draw(R, K, "bf16", 2, 3.0), draw(R, K, "bf16", 3, 3.0)
    q, ckpt = lib.MXTensor(R, K, "cuda", fmt, True, True), lib.SwigluCheckpoint(R, K, "cuda")
    lib.fp4_mx_quantize(c, x, fmt, out=q)
    lib.fp4_mx_swiglu_fwd(c, x, y, checkpoint=ckpt, want_h=False)
    other = lib.MXTensor(R, K, "cuda", fmt, True, True)
    rest = torch.empty_like(dh)
    yield lambda out: lib.fp4_mx_quantize(c, x, fmt, out=other)
    yield lambda out: lib.fp4_mx_dequantize(c, q, out=out)
    yield lambda out: lib.fp4_mx_swiglu_fwd(c, x, y, out=out)
    yield lambda out: lib.fp4_mx_swiglu_bwd(c, dh, ckpt, dgate=out, dup=rest)
    yield lambda out: lib.fp4_mx_swiglu_bwd(c, dh, ckpt, dgate=rest, dup=torch.empty_like(dh), h=out)
    check_quantized(other, x, {lib.FP4_MX_E2M1: "mxfp4", lib.FP4_MX_NVFP4: "nvfp4", lib.FP4_MX_E4M3: "mxfp8"}[fmt])


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_a_tile_that_never_comes_ends_the_kernel(lib, fmt):
    c = lib.Context(0, 0)
    for call in calls(lib, c, fmt):
        want = torch.zeros((R, K), dtype=torch.bfloat16, device="cuda")
        call(want)
        torch.cuda.synchronize()
        assert c.read_status() == 0
        c.debug_set(lib.binding.FP4_DEBUG_WAIT_LIMIT_US, 1000)
        c.debug_set(lib.binding.FP4_DEBUG_SKIP_FILL, 0)
        guard = torch.full((R + 2, K + 16), 7.0, dtype=torch.bfloat16, device="cuda")
        call(guard[1:-1, 8:-8])
        torch.cuda.synchronize()
        assert c.read_status() & lib.FP4_DEV_TIMEOUT
        assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (guard[:, :8] == 7).all() and (guard[:, -8:] == 7).all()
        c.debug_set(lib.binding.FP4_DEBUG_SKIP_FILL, -1)
        c.debug_set(lib.binding.FP4_DEBUG_WAIT_LIMIT_US, 0)
        c.status.zero_()
        again = torch.zeros_like(want)
        call(again)
        torch.cuda.synchronize()
        assert c.read_status() == 0 and torch.equal(again, want)
    c.close()
