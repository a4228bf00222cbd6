"""Randomised parity of the block-scaled operands: sizes, types, strides, offsets and the parts of a call drawn from a seed, against the
double-precision oracle with the allowances of test_gpu_mx.  FP4_RANDOM_DRAWS in the environment sets how many are made (default 16),
FP4_RANDOM_SEED moves the generator to another sequence."""
import os

import numpy as np
import pytest
import torch

from oracle import mx_oracle as O
from test_gpu_mx import DT, check_product, check_quantized, check_side, draw, fmt_of, host, near

pytestmark = pytest.mark.gpu
SEED = 100003 * int(os.environ.get("FP4_RANDOM_SEED", "0"))
DRAWS = range(int(os.environ.get("FP4_RANDOM_DRAWS", "16")))
GUARD = 5.0


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context.for_mx(1024, 1536, 1024)
    yield c
    c.close()


class Drawer:
    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)

    def size(self, most):
        """Log-uniform, now and then a neighbour of a multiple of 64."""
        n = int(round(np.exp(self.rng.uniform(0, np.log(most)))))
        if self.rng.random() < 0.4:
            n = (n + 63) // 64 * 64 + int(self.rng.integers(-1, 2))
        return max(1, min(n, most))

    def one(self, *of):
        return of[int(self.rng.integers(len(of)))]

    def seed(self):
        return int(self.rng.integers(1 << 30))

    def place(self, rows, cols, dt):
        """(buffer full of the guard, a matrix in it, dense, with rows apart or at any offset)."""
        before, behind = self.one((0, 0), (0, 8), (8, 8), (int(self.rng.integers(9)), int(self.rng.integers(9))))
        buf = torch.full((rows + 2, before + cols + behind), GUARD, dtype=DT[dt], device="cuda")
        return buf, buf[1:rows + 1, before:before + cols]

    def matrix(self, rows, cols, dt, spread=3.0):
        _, m = self.place(rows, cols, dt)
        return m.copy_(draw(rows, cols, dt, self.seed(), spread))


def untouched(buf, m):
    m.fill_(GUARD)
    return bool((buf == GUARD).all())


@pytest.mark.parametrize("i", DRAWS)
def test_quantise_and_back(lib, ctx, i):
    d = Drawer(SEED + 7001 + i)
    fmt, dt, rows, cols = d.one("mxfp4", "nvfp4", "mxfp8"), d.one(*DT), d.size(700), d.size(1500)
    x = d.matrix(rows, cols, dt, spread=float(d.one(0.0, 3.0, 9.0)))
    both = d.one((True, False), (False, True), (True, True))
    ctx.status.zero_()
    q = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), *both)
    check_quantized(q, x, fmt)
    for t in (False, True):
        if both[t]:
            want = torch.from_numpy(O.quantize(host(x).T if t else host(x), fmt).values).float()
            odt = d.one(*DT)
            buf, out = d.place(*want.shape, odt)
            lib.fp4_mx_dequantize(ctx, q, transposed=t, out=out)
            assert torch.equal(out.cpu(), want.to(DT[odt])) and untouched(buf, out)
    assert ctx.read_status() == 0


@pytest.mark.parametrize("i", DRAWS)
def test_products(lib, ctx, i):
    d = Drawer(SEED + 7002 + i)
    fmt, dt, I, J, C = d.one("mxfp4", "nvfp4"), d.one(*DT), d.size(900), d.size(900), d.size(3000)
    a, b, ta, tb = d.matrix(I, C, "bf16"), d.matrix(J, C, "bf16"), bool(d.one(0, 1)), bool(d.one(0, 1))
    quantised = lambda x, t: lib.fp4_mx_quantize(ctx, x.T.contiguous() if t else x, fmt_of(lib, fmt), not t, t)     # noqa: E731
    buf, out = d.place(I, J, dt)
    before = draw(I, J, dt, d.seed()) if d.one(0, 1) else None
    if before is not None:
        out.copy_(before)
    ctx.status.zero_()
    lib.fp4_mx_gemm(ctx, quantised(a, ta), quantised(b, tb), ta, tb, out=out, accumulate=before is not None)
    check_product(out, O.quantize(host(a), fmt).values, O.quantize(host(b), fmt).values, None if before is None else host(before))
    assert untouched(buf, out) and ctx.read_status() == 0


@pytest.mark.parametrize("i", DRAWS)
def test_layers(lib, ctx, i):
    d = Drawer(SEED + 7003 + i)
    fmt, dt, M, K, N = d.one("mxfp4", "nvfp4"), d.one(*DT), d.one(d.size(20), d.size(500)), d.size(1500), d.size(700)
    f, X, W, dY = fmt_of(lib, fmt), d.matrix(M, K, dt), d.matrix(K, N, d.one(dt, "bf16")), d.matrix(M, N, dt)
    value = lambda x: O.quantize(host(x), fmt).values                                          # noqa: E731
    buf, y = d.place(M, N, d.one(*DT))
    ctx.status.zero_()
    if d.one(0, 1):                                            # serving: W is there, X in one direction
        sx, sw = lib.MXTensor(M, K, "cuda", f), lib.fp4_mx_quantize(ctx, W, f, False, True)
        sx.codes.fill_(0xAA), sx.scales.fill_(0xAA)
        lib.fp4_mx_linear_fwd(ctx, X, None, f, sx, sw, reuse_w=True, out=y)
        check_product(y, value(X), value(W.T))
        check_side(sx.codes, sx.scales, O.quantize(host(X), fmt))
        assert fmt == "mxfp4" or float(sx.amax.item()) == float(X.abs().max())
    else:
        _, sx, sw = lib.fp4_mx_linear_fwd(ctx, X, W, f, out=y)
        check_product(y, value(X), value(W.T))
        which = d.one((True, True), (True, False), (False, True))
        bx, dx = d.place(M, K, d.one(*DT))
        bw, dw = d.place(K, N, d.one(*DT))
        lib.fp4_mx_linear_bwd(ctx, dY, sx, sw, dX=dx if which[0] else None, dW=dw if which[1] else None, want_dx=which[0], want_dw=which[1])
        if which[0]:
            check_product(dx, value(dY), value(W))
        if which[1]:
            check_product(dw, value(X.T), value(dY.T))
        assert untouched(bx, dx) and untouched(bw, dw)
    assert untouched(buf, y) and ctx.read_status() == 0


@pytest.mark.parametrize("i", DRAWS)
def test_swiglu(lib, ctx, i):
    d = Drawer(SEED + 7004 + i)
    dt, R, K = d.one(*DT), d.size(400), d.size(1200)
    gate, up, dh = (d.matrix(R, K, dt, 1.0) for _ in range(3))
    sides = d.one((True, False), (False, True), (True, True))
    q = lambda: lib.MXTensor(R, K, "cuda", codes=sides[0], codes_t=sides[1])                   # noqa: E731
    kept, q1, q2 = lib.SwigluCheckpoint(R, K, "cuda"), q(), q()
    bh, h = d.place(R, K, dt)
    ctx.status.zero_()
    lib.fp4_mx_swiglu_fwd(ctx, gate, up, out=h, checkpoint=kept, quantized=q1)
    g, u, s = host(gate), host(up), host(dh)
    near(h, O.swiglu(g, u), np.abs(O.swiglu(g, u)) * (1 + np.abs(g) / 16))
    check_quantized(q1, h, "mxfp4")
    rg, ru = O.quantize(g, "mxfp8"), O.quantize(u, "mxfp8")
    check_side(kept.gate.codes, kept.gate.scales, rg)
    check_side(kept.up.codes, kept.up.scales, ru)
    (bg, dg), (bu, du), (b2, h2) = (d.place(R, K, dt) for _ in range(3))
    lib.fp4_mx_swiglu_bwd(ctx, dh, kept, dgate=dg, dup=du, h=h2, quantized=q2)
    wg, wu = O.swiglu_grad(rg.values, ru.values, s)
    slack = 1 + np.abs(rg.values) / 16
    near(dg, wg, np.abs(s * ru.values) / (1 + np.exp(-rg.values)) * (1 + np.abs(rg.values)) * slack)
    near(du, wu, np.abs(wu) * slack)
    near(h2, O.swiglu(rg.values, ru.values), np.abs(O.swiglu(rg.values, ru.values)) * slack)
    check_quantized(q2, h2, "mxfp4")
    assert all(untouched(b, m) for b, m in ((bh, h), (bg, dg), (bu, du), (b2, h2))) and ctx.read_status() == 0
