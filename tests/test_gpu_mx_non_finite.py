"""Infinities and NaNs in a tensor that is quantised: they spoil their blocks, and nothing else of it."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as O
from test_gpu_mx import DT, check_quantized, check_side, draw, fmt_of, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context.for_mx(1024, 1024, 1024)
    yield c
    c.close()


# sizes by how the amax is found: by every block for itself, in parts, joined by the block that ends last; rows of any alignment
SIZES = [(1, 1), (1, 40), (3, 33), (40, 200), (200, 1000), (90, 1111), (1300, 1024), (1100, 1031)]
BAD = [float("inf"), float("-inf"), float("nan")]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("R,K", SIZES)
def test_what_is_not_finite_leaves_the_tensors_scale_alone(lib, ctx, dt, R, K):
    """Blocks of 16: every block without an infinity or a NaN has the codes and the scale that it has without them in the tensor."""
    f = lib.FP4_MX_NVFP4
    for apart in (0, 5):
        x = draw(R, K, dt, R + K, 3.0)
        bad, zeros = (torch.zeros((R, K + apart), dtype=DT[dt], device="cuda")[:, :K].copy_(x) for _ in range(2))
        at = [(0, 0), (R - 1, K - 1), (R // 2, K // 3), (R // 3, K // 2), (R // 4, min(K - 1, 8)), (R - 1, max(0, K - 9))]
        for i, p in enumerate(at):
            bad[p], zeros[p] = BAD[i % 3], 0.0
        ctx.status.zero_()
        q = lib.fp4_mx_quantize(ctx, bad, f, True, True)
        assert ctx.read_status() == lib.FP4_DEV_NONFINITE
        ctx.status.zero_()
        without = lib.fp4_mx_quantize(ctx, zeros, f, True, True)
        assert torch.equal(q.amax, without.amax)
        check_quantized(without, zeros, "nvfp4")
        check_side(q.codes, q.scales, O.quantize(host(bad), "nvfp4"))
        check_side(q.codes_t, q.scales_t, O.quantize(host(bad).T, "nvfp4"))
        for t in (False, True):
            spoilt = ~np.isfinite(O.quantize(host(bad).T if t else host(bad), "nvfp4").values)
            got, want = (host(lib.fp4_mx_dequantize(ctx, p, transposed=t, dtype=torch.float32)) for p in (q, without))
            np.testing.assert_array_equal(np.isnan(got), spoilt)
            np.testing.assert_array_equal(got[~spoilt], want[~spoilt])


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
def test_nothing_finite_at_all(lib, ctx, dt):
    for R, K in ((1, 17), (70, 900), (1300, 1024)):
        for bad in BAD:
            x = torch.full((R, K), bad, dtype=DT[dt], device="cuda")
            q = lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_NVFP4, True, True)
            assert float(q.amax.item()) == 0.0 and torch.isnan(lib.fp4_mx_dequantize(ctx, q)).all()
            check_side(q.codes, q.scales, O.quantize(host(x), "nvfp4"))
    ctx.status.zero_()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("M", [1, 4, 200])
def test_a_bad_token_leaves_the_others_their_results(lib, ctx, fmt, M):
    """The whole layer: a row that is not finite, the other rows as they are without it; one token by itself: its NaN, and its amax."""
    f, K, N = fmt_of(lib, fmt), 700, 260
    x, w, dy = draw(M, K, "bf16", 5, 3.0), draw(K, N, "bf16", 6, 3.0), draw(M, N, "bf16", 7, 3.0)
    dy[M // 2] = 1.0
    bad, zero = x.clone(), x.clone()
    bad[M // 2, 555], zero[M // 2, 555] = float("inf"), 0.0
    wq = lib.fp4_mx_quantize(ctx, w, f, True, True)
    saved = [lib.MXTensor(M, K, "cuda", f) for _ in range(2)]
    y, want = (lib.fp4_mx_linear_fwd(ctx, t, None, f, s, wq, reuse_w=True)[0] for t, s in zip((bad, zero), saved))
    assert torch.isnan(y[M // 2]).all()
    assert fmt == "mxfp4" or torch.equal(saved[0].amax, saved[1].amax)
    others = [i for i in range(M) if i != M // 2]
    assert torch.equal(y[others], want[others]) and (M == 1 or float(want[others].abs().max()) > 0)
    badg, zerog = dy.clone(), dy.clone()
    badg[M // 2, 200], zerog[M // 2, 200] = float("nan"), 0.0
    dx, wantx = (lib.fp4_mx_linear_bwd(ctx, t, lib.fp4_mx_quantize(ctx, x, f, True, True), wq, want_dw=False)[0] for t in (badg, zerog))
    assert torch.isnan(dx[M // 2]).all() and torch.equal(dx[others], wantx[others])
    ctx.status.zero_()
