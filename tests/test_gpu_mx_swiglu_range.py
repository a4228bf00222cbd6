"""SwiGLU where sigmoid(gate) is far below fp32's normal range and the factor beside it far above 1: the results are ordinary numbers.

Allowance, relative: the exponential's root to 2^-22, twice (it is squared), the reciprocal to 2^-23, six roundings to 2^-24: 16 units of 2^-24; the root's
exponent is off by a rounding of the product and the constant's own (0.22 of a unit), which is at most 1.23 |gate| units of the square: less than (1 + |gate| / 8) 2^-20.
Where 1 + gate (1 - sigmoid) cancels, the same of the terms.  Half a step of the output's type, and of its smallest numbers one."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as O
from test_gpu_mx import DT, check_quantized, half_step, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context.for_mx(1, 1, 1)
    yield c
    c.close()


def check(got, want, terms, g):
    info = torch.finfo(got.dtype)
    room = 2.0 ** -20 * (1 + np.abs(g) / 8) * terms
    room = room + half_step(got.dtype) * (np.abs(want) + room) + info.smallest_normal * info.eps + 2.0 ** -149
    err = np.abs(host(got) - want)
    assert (err <= room).all(), f"{(err / room).max():.3g} of the allowance"


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [256, 131])
def test_far_gates_with_large_factors(lib, ctx, dt, K):
    R = 96
    gate = torch.linspace(-160.0, 100.0, R * K, dtype=torch.float64).reshape(R, K)
    gate[::3] = torch.linspace(-110.0, -84.0, 32 * K, dtype=torch.float64).reshape(32, K)
    # factors with which the result stays inside of the type: 3e38 for gates below -8 (silu and its derivative are at most 1/300 there)
    factor = torch.where(gate < -8, 3e38, 1e30) * (1 - 2 * (torch.arange(K) % 2))
    gate, factor = gate.to(DT[dt]).cuda(), factor.to(DT[dt]).cuda()
    one = torch.ones_like(factor)
    ctx.status.zero_()
    g, f = host(gate), host(factor)
    h, _, q = lib.fp4_mx_swiglu_fwd(ctx, gate, factor, quantized=lib.MXTensor(R, K, "cuda"))
    check(h, O.swiglu(g, f), np.abs(O.swiglu(g, f)), g)
    check_quantized(q, h, "mxfp4")
    for up, dh in ((factor, one), (one, factor)):
        c = lib.SwigluCheckpoint(R, K, "cuda")
        lib.fp4_mx_swiglu_fwd(ctx, gate, up, checkpoint=c, want_h=False)
        again = torch.empty_like(gate)
        dg, du = lib.fp4_mx_swiglu_bwd(ctx, dh, c, h=again)
        gv, uv, d = O.quantize(g, "mxfp8").values, O.quantize(host(up), "mxfp8").values, host(dh)
        wg, wu = O.swiglu_grad(gv, uv, d)
        s = np.where(gv < 0, np.exp(-np.abs(gv)), 1.0) / (1 + np.exp(-np.abs(gv)))
        check(du, wu, np.abs(wu), gv)
        check(dg, wg, np.abs(d * uv) * s * (1 + np.abs(gv)), gv)
        check(again, O.swiglu(gv, uv), np.abs(O.swiglu(gv, uv)), gv)
        plain = lib.fp4_mx_swiglu_bwd(ctx, dh, c)
        assert torch.equal(plain[0], dg) and torch.equal(plain[1], du)
    assert ctx.read_status() == 0
