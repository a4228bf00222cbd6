"""GPU parity of the block-scaled operands against the double-precision oracle.

Codes, scales and their padding, and the checkpoints are compared bit for bit.  Products: the oracle's codes multiplied in
float64; the GPU's may be off by 2^-22 (C / 64 + 1) sum |products| (one addition of 64 products into the fp32 accumulator rounds
toward zero twice at most) and half a step of the output's type.  SwiGLU: fp32 arithmetic, a few units in the last place of
every factor (sigmoid through two approximate instructions: 2^-20 with room), and half a step of the output's type; where a
factor cancels (1 - s), the same relative to the terms."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as O

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
FMTS = ("mxfp4", "nvfp4", "mxfp8")


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context.for_mx(4096, 2048, 4096)
    yield c
    c.close()


def fmt_of(lib, fmt):
    return {"mxfp4": lib.FP4_MX_E2M1, "nvfp4": lib.FP4_MX_NVFP4, "mxfp8": lib.FP4_MX_E4M3}[fmt]


def host(t):
    return t.detach().cpu().double().numpy()


def half_step(dt):
    return torch.finfo(dt).eps / 2


def draw(rows, cols, dt, seed, spread=6.0):
    """Normal values whose blocks differ in size by powers of two, with zeros, negative zeros and a zero row."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    x *= torch.exp2(torch.round(torch.randn((rows, (cols + 7) // 8), generator=g) * spread / 3)).repeat_interleave(8, 1)[:, :cols]
    x[torch.rand((rows, cols), generator=g) < 0.05] = 0.0
    x[torch.rand((rows, cols), generator=g) < 0.02] = -0.0
    if rows > 3:
        x[rows // 2] = 0.0
    return x.to(DT[dt]).cuda()


def check_side(q_codes, q_scales, ref):
    np.testing.assert_array_equal(q_codes.cpu().numpy(), O.packed_codes(ref))
    np.testing.assert_array_equal(q_scales.cpu().numpy(), O.packed_scales(ref))


def check_quantized(q, x, fmt, amax=None):
    xs = host(x)
    if q.codes is not None:
        check_side(q.codes, q.scales, O.quantize(xs, fmt, amax))
    if q.codes_t is not None:
        check_side(q.codes_t, q.scales_t, O.quantize(xs.T, fmt, amax))
    if fmt == "nvfp4" and amax is None and x.numel():
        assert float(q.amax.item()) == np.abs(xs).max()


SHAPES = [(1, 1), (1, 16), (1, 33), (1, 4096), (33, 1), (3, 31), (31, 130), (128, 128), (129, 257), (256, 384), (77, 1000), (500, 17)]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize(lib, ctx, fmt, dt, shape):
    x = draw(*shape, dt, seed=shape[0] + 7 * shape[1])
    ctx.status.zero_()
    for codes, codes_t in ((True, True), (True, False), (False, True)):
        q = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), codes, codes_t)
        check_quantized(q, x, fmt)
    assert ctx.read_status() == 0


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [1, 7, 8, 128, 137, 393])
def test_every_alignment_of_rows(lib, ctx, dt, cols):
    """Rows that begin at each place within 16 bytes, read and written, in matrices that begin and end where their memory does."""
    E = torch.finfo(DT[dt]).bits // 8
    for ld in range(cols, cols + 16 // E):
        for first in range(0, 16 // E, 3):
            rows = 131
            flat = draw(1, first + (rows - 1) * ld + cols, dt, seed=ld + first)[0]
            x = torch.as_strided(flat, (rows, cols), (ld, 1), first)
            q = lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_NVFP4, True, True)
            check_quantized(q, x, "nvfp4")
            before = flat.clone()
            out = torch.as_strided(flat, (rows, cols), (ld, 1), first)
            lib.fp4_mx_dequantize(ctx, q, out=out)
            want = torch.from_numpy(O.quantize(host(torch.as_strided(before, (rows, cols), (ld, 1), first)), "nvfp4").values).to(DT[dt])
            assert torch.equal(out.cpu(), want)
            torch.as_strided(before, (rows, cols), (ld, 1), first).copy_(out)
            assert torch.equal(before, flat)                          # nothing beside the matrix was written


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_quantize_strided_input(lib, ctx, fmt, dt):
    """A slice of a wider matrix: rows 16-byte aligned or not, elements beside it untouched."""
    wide = draw(70, 600, dt, seed=5)
    for c0, c1 in ((0, 256), (8, 264), (3, 260), (5, 6), (599, 600)):
        x = wide[:, c0:c1]
        check_quantized(lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), True, True), x, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_every_bf16_value_under_every_kind_of_maximum(lib, ctx, fmt):
    """All finite BF16 patterns, sorted by magnitude (each block spans few exponents), and beside a maximum drawn for them."""
    bits = np.arange(65536, dtype=np.uint32)
    bits = bits[(bits & 0x7F80) != 0x7F80].astype(np.uint16)
    order = np.argsort(bits & 0x7FFF, kind="stable")
    a = torch.from_numpy(bits[order].view(np.int16).copy()).cuda().view(torch.bfloat16).reshape(-1, 32 * 5)
    check_quantized(lib.fp4_mx_quantize(ctx, a, fmt_of(lib, fmt), True, True), a, fmt)
    # values within the formats' range of a maximum whose mantissa takes every value
    rng = np.random.default_rng(3)
    x = (rng.integers(-512, 513, (512, 160)) * 2.0 ** rng.integers(-12, -6, (512, 160))).astype(np.float32)
    x[:, ::16] = ((128 + np.arange(512) % 128) * 2.0 ** (np.arange(512) // 128 - 6))[:, None] * (1 - 2 * (np.arange(10) % 2))
    x = torch.from_numpy(x).cuda().to(torch.bfloat16)
    check_quantized(lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), True, True), x, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_extreme_magnitudes(lib, ctx, fmt, dt):
    """Blocks of the largest and of subnormal values, alone and mixed."""
    x = torch.zeros((8, 160))
    x[0] = torch.finfo(DT[dt]).max
    x[1] = torch.finfo(DT[dt]).tiny * 0.5
    x[2, ::2], x[2, 1::2] = torch.finfo(DT[dt]).max, 1e-38
    x[3] = -torch.finfo(DT[dt]).tiny
    x[4] = torch.linspace(-1, 1, 160) * 3e38
    x[5] = 2.0 ** -126 * torch.arange(160)
    x[6, 5] = 1.0
    for part in (x, x[1:2], x[3:4] * 2.0 ** 20, x[5:7]):
        t = part.to(DT[dt]).cuda()
        ctx.status.zero_()
        check_quantized(lib.fp4_mx_quantize(ctx, t, fmt_of(lib, fmt), True, True), t, fmt)
        assert ctx.read_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_non_finite_value_spoils_its_block_alone(lib, ctx, fmt, dt, bad):
    x = draw(40, 200, dt, seed=9)
    x[17, 75] = bad
    ctx.status.zero_()
    q = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), True, True)
    assert ctx.read_status() == lib.FP4_DEV_NONFINITE
    xs = host(x)
    check_side(q.codes, q.scales, O.quantize(xs, fmt))
    check_side(q.codes_t, q.scales_t, O.quantize(xs.T, fmt))
    n = O.BLOCK[fmt]
    back = lib.fp4_mx_dequantize(ctx, q, dtype=torch.float32)
    nan = torch.zeros((40, 200), dtype=torch.bool)
    nan[17, 75 // n * n:75 // n * n + n] = True
    assert torch.equal(torch.isnan(back).cpu(), nan)
    ctx.status.zero_()


def test_given_amax(lib, ctx):
    x = draw(60, 100, "bf16", seed=11)
    for a in (0.0, 0.01, 3.0, 1e6):
        q = lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_NVFP4, True, True, amax=torch.tensor([a], device="cuda"))
        assert float(q.amax.item()) == np.float32(a)
        check_quantized(q, x, "nvfp4", amax=float(np.float32(a)))


def test_given_amax_far_below_the_values(lib, ctx):
    """Saturation, with the values' signs, however far beyond: quotients that overflow fp32 among them."""
    x = draw(40, 96, "bf16", seed=12)
    x[3, 10], x[3, 11], x[20, 40], x[21, 41] = 3e38, -3e38, 1e30, -1e20
    for a in (0.0, 1e-37, 1e-20, 1.0):
        q = lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_NVFP4, True, True, amax=torch.tensor([a], device="cuda"))
        check_quantized(q, x, "nvfp4", amax=float(np.float32(a)))


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("k", [-100, -37, 0, 40, 110])
def test_every_tie_of_blocks_of_16(lib, ctx, dt, k):
    """Every E4M3 scale with every value that lies on a tie of E2M1 under it, and its neighbours in the type, at several scales of the tensor."""
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    s = O.E4M3[1:]                                                    # every scale but 0
    x = np.zeros((2 * len(s), 32))
    for i, v in enumerate(s):
        ties = mids * v * 2.0 ** k
        x[2 * i, :7], x[2 * i, 7:14] = ties, -ties
        x[2 * i, 14] = x[2 * i + 1, 14] = 6.0 * v * 2.0 ** k          # the block's amax: its scale is v
        t = torch.tensor(ties).to(DT[dt])
        inf = torch.tensor(float("inf"), dtype=DT[dt])
        x[2 * i + 1, :7], x[2 * i + 1, 7:14] = torch.nextafter(t, inf).double(), -torch.nextafter(t, -inf).double()
    t = torch.tensor(x).to(DT[dt]).cuda()
    if dt == "fp32" or k > -90:
        assert np.array_equal(host(t)[::2], x[::2])                   # the ties are values of the type
    q = lib.fp4_mx_quantize(ctx, t, lib.FP4_MX_NVFP4, True, True, amax=torch.tensor([2688.0 * 2.0 ** k], device="cuda"))
    check_quantized(q, t, "nvfp4", amax=2688.0 * 2.0 ** k)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
def test_dequantize(lib, ctx, fmt, dt):
    for shape in ((1, 1), (5, 33), (130, 259), (64, 512)):
        x = draw(*shape, "fp32", seed=sum(shape))
        q = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), True, True)
        for t in (False, True):
            ref = O.quantize(host(x).T if t else host(x), fmt).values
            want = torch.from_numpy(ref).to(torch.float32).to(DT[dt])            # (exact in fp32)
            assert torch.equal(lib.fp4_mx_dequantize(ctx, q, transposed=t, dtype=DT[dt]).cpu(), want)
        buf = torch.full((shape[0] + 1, shape[1] + 3), 7.0, dtype=DT[dt], device="cuda")
        lib.fp4_mx_dequantize(ctx, q, out=buf[:shape[0], 1:shape[1] + 1])
        assert torch.equal(buf[:shape[0], 1:shape[1] + 1], lib.fp4_mx_dequantize(ctx, q, dtype=DT[dt]))
        buf[:shape[0], 1:shape[1] + 1] = 7.0
        assert (buf == 7.0).all()


# ------------------------------------------------------------------------------- product ------
def product(a, b, dt, before=None):
    """(exact result, allowance) of quantised operands a [I x C] and b [J x C]."""
    C = a.shape[1]
    y = a @ b.T + (0.0 if before is None else before)
    terms = np.abs(a) @ np.abs(b).T
    room = 2.0 ** -22 * (-(-C // 64) + 1) * terms + (0 if before is None else 2.0 ** -24 * np.abs(y))
    return y, room + half_step(dt) * (np.abs(y) + room)


def check_product(got, a, b, before=None):
    y, room = product(a, b, got.dtype, before)
    err = np.abs(host(got) - y)
    # fp16: what lies below its normal range is rounded to multiples of 2^-24
    room = room + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    assert (err <= room).all(), f"{(err / np.maximum(room, 1e-300)).max():.3g} of the allowance"


GEMMS = [(1, 1, 1), (1, 64, 16), (1, 300, 4096), (2, 128, 257), (16, 129, 300), (17, 1000, 1111), (64, 256, 640), (100, 4096, 512),
         (128, 77, 2048), (129, 1, 64), (130, 64, 128), (200, 63, 1000), (256, 256, 256), (300, 520, 31), (385, 449, 777),
         (1000, 1032, 512), (640, 2500, 128)]


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("shape", GEMMS)
def test_gemm(lib, ctx, fmt, shape):
    I, J, C = shape
    x, w = draw(I, C, "bf16", seed=I + C, spread=3.0), draw(J, C, "bf16", seed=J + C + 1, spread=3.0)
    a, b = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, w, fmt_of(lib, fmt))
    av, bv = O.quantize(host(x), fmt).values, O.quantize(host(w), fmt).values
    ctx.status.zero_()
    for dt in DT.values():
        out = torch.full((I + 1, J + 5), 3.0, dtype=dt, device="cuda")           # rows off any alignment, and what lies beside
        lib.fp4_mx_gemm(ctx, a, b, out=out[:I, 2:J + 2])
        got = out[:I, 2:J + 2].clone()
        check_product(got, av, bv)
        out[:I, 2:J + 2] = 3.0
        assert (out == 3.0).all()
        assert torch.equal(lib.fp4_mx_gemm(ctx, a, b, dtype=dt), got)             # dense: aligned or not, the same values
        wide = torch.full((I, (J + 15) // 8 * 8), 3.0, dtype=dt, device="cuda")   # aligned rows with room behind them
        lib.fp4_mx_gemm(ctx, a, b, out=wide[:, :J])
        assert torch.equal(wide[:, :J], got) and (wide[:, J:] == 3.0).all()
        before = torch.randn((I, J), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(dt)
        acc = before.clone()
        lib.fp4_mx_gemm(ctx, a, b, out=acc, accumulate=True)
        check_product(acc, av, bv, before=host(before))
    assert ctx.read_status() == 0


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("shape", [(2048, 1920, 4096), (2300, 2500, 2304), (4096, 520, 8192), (900, 4100, 5000), (128, 13824, 5120),
                                   (1, 11008, 4096), (300, 128, 13824)])
def test_gemm_large(lib, ctx, fmt, shape):
    """Sizes that take every form of the kernels, against a product in 64 bits of the dequantised operands."""
    I, J, C = shape
    g = torch.Generator("cuda").manual_seed(I)
    x, w = (torch.randn((r, C), device="cuda", generator=g).bfloat16() for r in (I, J))
    a, b = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, w, fmt_of(lib, fmt))
    av, bv = (lib.fp4_mx_dequantize(ctx, q, dtype=torch.float32).double() for q in (a, b))
    y, terms = av @ bv.T, av.abs() @ bv.abs().T
    room = 2.0 ** -22 * (-(-C // 64) + 1) * terms
    ctx.status.zero_()
    for dt in DT.values():
        got = lib.fp4_mx_gemm(ctx, a, b, dtype=dt).double()
        assert ((got - y).abs() <= room + half_step(dt) * (y.abs() + room)).all()
        off = torch.full((I, J + 1), 2.0, dtype=dt, device="cuda")
        lib.fp4_mx_gemm(ctx, a, b, out=off[:, 1:])
        assert torch.equal(off[:, 1:].double(), got) and (off[:, 0] == 2.0).all()
    assert ctx.read_status() == 0


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("shape", [(5, 200, 300), (300, 200, 150), (128, 512, 640)])
def test_gemm_by_columns(lib, ctx, fmt, shape):
    """Operands quantised along their rows' blocks or their columns' (what linear's three products take)."""
    I, J, C = shape
    x, w = draw(I, C, "bf16", 1, 3.0), draw(J, C, "bf16", 2, 3.0)
    qa = lib.fp4_mx_quantize(ctx, x.t().contiguous(), fmt_of(lib, fmt), False, True)
    qb = lib.fp4_mx_quantize(ctx, w.t().contiguous(), fmt_of(lib, fmt), False, True)
    ra, rb = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, w, fmt_of(lib, fmt))
    want = lib.fp4_mx_gemm(ctx, ra, rb, dtype=torch.float32)
    for a, at, b, bt in ((qa, True, qb, True), (ra, False, qb, True), (qa, True, rb, False)):
        assert torch.equal(lib.fp4_mx_gemm(ctx, a, b, a_t=at, b_t=bt, dtype=torch.float32), want)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("I", [100, 256])
def test_every_scale_reaches_its_block(lib, ctx, fmt, I):
    """Elements of one magnitude, scales that differ from block to block and row to row by powers of two: an operand against one
    whose only non-zero block moves along the contraction gives that block's scale exactly."""
    n, blocks, J = O.BLOCK[fmt], 40, 200
    C = n * blocks
    rng = np.random.default_rng(4)
    ea, eb = rng.integers(-4, 5, (I, blocks)), rng.integers(-3, 4, (J, blocks))
    a = np.repeat(2.0 ** ea, n, axis=1)
    b = np.repeat(2.0 ** eb, n, axis=1) * (np.arange(C) // n % blocks == (np.arange(J) % blocks)[:, None])
    ta, tb = torch.from_numpy(a).cuda().bfloat16(), torch.from_numpy(b).cuda().bfloat16()
    got = lib.fp4_mx_gemm(ctx, lib.fp4_mx_quantize(ctx, ta, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, tb, fmt_of(lib, fmt)), dtype=torch.float32)
    va, vb = O.quantize(a, fmt).values, O.quantize(b, fmt).values
    np.testing.assert_array_equal(host(got), va @ vb.T)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_accumulation_stays_inside_its_allowance(lib, ctx, fmt):
    """Sums that cancel, at a long contraction: the error is held to a half of what the header allows."""
    I, J, C = 130, 192, 16384
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.randn((I, C), device="cuda", generator=g).abs().bfloat16()
    w = torch.randn((J, C), device="cuda", generator=g).abs()
    w[:, ::2] *= -1
    w = w.bfloat16()
    a, b = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, w, fmt_of(lib, fmt))
    av, bv = O.quantize(host(x), fmt).values, O.quantize(host(w), fmt).values
    for rows in (I, 3):
        got = lib.fp4_mx_gemm(ctx, a, b, dtype=torch.float32) if rows == I else lib.fp4_mx_gemm(
            ctx, lib.fp4_mx_quantize(ctx, x[:rows], fmt_of(lib, fmt), amax=a.amax), b, dtype=torch.float32)
        y, terms = av[:rows] @ bv.T, np.abs(av[:rows]) @ np.abs(bv).T
        assert np.median(np.abs(y) / terms) < 0.05
        err = np.abs(host(got) - y) - 2.0 ** -23 * np.abs(y)
        assert (err <= 0.5 * 2.0 ** -22 * (C // 64 + 1) * terms).all(), f"{(err / terms).max() * 2 ** 22 / (C // 64 + 1):.3f}"


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_non_finite_blocks_spoil_their_rows_alone(lib, ctx, fmt):
    for I in (7, 300):
        x, w = draw(I, 320, "bf16", 1, 3.0), draw(150, 320, "bf16", 2, 3.0)
        x[3, 40] = float("nan")
        w[9, 300] = float("inf")
        a, b = lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, w, fmt_of(lib, fmt))
        got = host(lib.fp4_mx_gemm(ctx, a, b, dtype=torch.float32))
        nan = np.zeros((I, 150), dtype=bool)
        nan[3], nan[:, 9] = True, True
        np.testing.assert_array_equal(np.isnan(got), nan)
    ctx.status.zero_()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_empty_sizes(lib, ctx, fmt):
    f = fmt_of(lib, fmt)
    empty = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    q0, q = lib.fp4_mx_quantize(ctx, empty, f, True, True), lib.fp4_mx_quantize(ctx, draw(32, 64, "bf16", 1), f, True, True)
    assert lib.fp4_mx_dequantize(ctx, q0).shape == (0, 64)
    assert lib.fp4_mx_gemm(ctx, q0, q).shape == (0, 32) and lib.fp4_mx_gemm(ctx, q, q0).shape == (32, 0)
    out = torch.full((64, 64), 5.0, device="cuda")
    assert (lib.fp4_mx_gemm(ctx, q0, q0, a_t=True, b_t=True, out=out, accumulate=True) == 5.0).all()
    out = torch.full((64, 70), 5.0, device="cuda")
    lib.fp4_mx_gemm(ctx, q0, q0, a_t=True, b_t=True, out=out[:, 3:67])           # a contraction of length 0
    assert (out[:, 3:67] == 0).all() and (out[:, :3] == 5).all() and (out[:, 67:] == 5).all()
    W = draw(64, 48, "bf16", 2)
    y, sx, sw = lib.fp4_mx_linear_fwd(ctx, empty, W, fmt=f)
    dx, dw = lib.fp4_mx_linear_bwd(ctx, y, sx, sw)
    assert y.shape == (0, 48) and dx.shape == (0, 64) and (dw == 0).all() and dw.shape == (64, 48)
    h, c, _ = lib.fp4_mx_swiglu_fwd(ctx, empty, empty, checkpoint=lib.SwigluCheckpoint(0, 64, "cuda"))
    assert lib.fp4_mx_swiglu_bwd(ctx, h, c)[0].shape == (0, 64)


# ------------------------------------------------------------------------------- linear -------
@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 64, 96), (37, 200, 130), (256, 384, 192), (300, 129, 515)])
def test_linear(lib, ctx, fmt, dt, shape):
    M, K, N = shape
    X, W, dY = draw(M, K, dt, 1, 3.0), draw(K, N, dt, 2, 3.0), draw(M, N, dt, 3, 3.0)
    xs, ws, ds = host(X), host(W), host(dY)
    q = lambda x: O.quantize(x, fmt).values                                       # noqa: E731
    y, sx, sw = lib.fp4_mx_linear_fwd(ctx, X, W, fmt=fmt_of(lib, fmt), dtype=torch.float32)
    check_product(y, q(xs), q(ws.T))
    dx, dw = lib.fp4_mx_linear_bwd(ctx, dY, sx, sw, dtype=torch.float32)
    check_product(dx, q(ds), q(ws))
    check_product(dw, q(xs.T), q(ds.T))
    # operands that are there, one gradient alone, sums
    again, _, _ = lib.fp4_mx_linear_fwd(ctx, None, None, saved_x=sx, saved_w=sw, reuse_x=True, reuse_w=True, dtype=torch.float32)
    assert torch.equal(again, y)
    assert torch.equal(lib.fp4_mx_linear_bwd(ctx, dY, sx, sw, dtype=torch.float32, want_dw=False)[0], dx)
    assert torch.equal(lib.fp4_mx_linear_bwd(ctx, dY, sx, sw, dtype=torch.float32, want_dx=False)[1], dw)
    a, b = torch.ones_like(dx), torch.ones_like(dw)
    lib.fp4_mx_linear_bwd(ctx, dY, sx, sw, dX=a, dW=b, accumulate_dx=True, accumulate_dw=True)
    assert torch.equal(a, dx + 1) and torch.equal(b, dw + 1)
    # serving: the forward's directions alone
    lean = lib.MXTensor(M, K, "cuda", fmt=fmt_of(lib, fmt))
    served, _, _ = lib.fp4_mx_linear_fwd(ctx, X, None, saved_x=lean, saved_w=lib.fp4_mx_quantize(ctx, W, fmt_of(lib, fmt), False, True),
                                         reuse_w=True, dtype=torch.float32)
    assert torch.equal(served, y)


def test_linear_gradients_against_differences(lib, ctx):
    """Values on the format's grid in blocks of one scale are not changed by quantisation, nor by a step to a neighbour:
    there the layer is linear, and the gradients are its differences (the loss <Y, dY>)."""
    M, K, N = 64, 96, 128
    g = torch.Generator("cuda").manual_seed(3)
    grid = torch.tensor([-4.0, -2.0, -1.0, 0.0, 1.0, 2.0, 4.0], device="cuda")
    pick = lambda r, c: grid[torch.randint(0, 7, (r, c), generator=g, device="cuda")].bfloat16()     # noqa: E731
    X, W, dY = pick(M, K), pick(K, N), pick(M, N)
    for t in (X, W, dY):                             # a 6 in every block, either way: one scale for all
        t[::16, :] = 6.0
        t[:, ::16] = 6.0
    y, sx, sw = lib.fp4_mx_linear_fwd(ctx, X, W, dtype=torch.float32)
    dx, dw = lib.fp4_mx_linear_bwd(ctx, dY, sx, sw, dtype=torch.float32)
    loss = lambda X, W: float((lib.fp4_mx_linear_fwd(ctx, X, W, dtype=torch.float32)[0].double() * dY.double()).sum())   # noqa: E731
    base = loss(X, W)
    for m, k in ((1, 1), (17, 33), (63, 95)):
        P = X.clone()
        P[m, k] = 3.0
        assert loss(P, W) - base == float(dx[m, k].double() * (3.0 - X[m, k].double()))
    for k, n in ((1, 1), (50, 100), (95, 127)):
        P = W.clone()
        P[k, n] = -3.0
        assert loss(X, P) - base == float(dw[k, n].double() * (-3.0 - W[k, n].double()))


# ------------------------------------------------------------------------------- SwiGLU -------
def gate_up(R, K, dt, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    mk = lambda s: (torch.randn((R, K), device="cuda", generator=g) * s).to(DT[dt])                   # noqa: E731
    gate, up, dh = mk(3.0), mk(1.0), mk(0.5)
    gate[torch.rand((R, K), device="cuda", generator=g) < 0.02] = -90.0
    gate[torch.rand((R, K), device="cuda", generator=g) < 0.02] = 60.0
    up[torch.rand((R, K), device="cuda", generator=g) < 0.02] = 0.0
    return gate, up, dh


def near(got, want, terms):
    room = 2.0 ** -20 * terms
    room = room + half_step(got.dtype) * (np.abs(want) + room) + (2.0 ** -25 if got.dtype == torch.float16 else 2.0 ** -126)
    err = np.abs(host(got) - want)
    assert (err <= room).all(), f"{(err / room).max():.3g}"


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 2000), (3, 33), (129, 260), (256, 512), (40, 1111)])
def test_swiglu(lib, ctx, dt, shape):
    R, K = shape
    gate, up, dh = gate_up(R, K, dt, R + K)
    g, u, d = host(gate), host(up), host(dh)
    ctx.status.zero_()
    c, q = lib.SwigluCheckpoint(R, K, "cuda"), lib.MXTensor(R, K, "cuda", codes_t=True)
    h, _, _ = lib.fp4_mx_swiglu_fwd(ctx, gate, up, checkpoint=c, quantized=q)
    near(h, O.swiglu(g, u), np.abs(O.swiglu(g, u)) * (1 + np.abs(g) / 16))
    rg, ru = O.quantize(g, "mxfp8"), O.quantize(u, "mxfp8")
    check_side(c.gate.codes, c.gate.scales, rg)
    check_side(c.up.codes, c.up.scales, ru)
    check_quantized(q, h, "mxfp4")
    # each output alone gives the same
    assert torch.equal(lib.fp4_mx_swiglu_fwd(ctx, gate, up)[0], h)
    for kw in (dict(), dict(codes=False, codes_t=True), dict(codes_t=True)):
        lone = lib.MXTensor(R, K, "cuda", **kw)
        lib.fp4_mx_swiglu_fwd(ctx, gate, up, quantized=lone, want_h=False)
        check_quantized(lone, h, "mxfp4")
    # backward from the checkpoint
    dg, du = lib.fp4_mx_swiglu_bwd(ctx, dh, c)
    wg, wu = O.swiglu_grad(rg.values, ru.values, d)
    s = 1 / (1 + np.exp(-rg.values))
    slack = 1 + np.abs(rg.values) / 16
    near(dg, wg, np.abs(d * ru.values) * s * (1 + np.abs(rg.values)) * slack)
    near(du, wu, np.abs(wu) * slack)
    h2, q2 = torch.empty_like(h), lib.MXTensor(R, K, "cuda", codes_t=True)
    e, f = lib.fp4_mx_swiglu_bwd(ctx, dh, c, h=h2, quantized=q2)
    assert torch.equal(e, dg) and torch.equal(f, du)
    near(h2, O.swiglu(rg.values, ru.values), np.abs(O.swiglu(rg.values, ru.values)) * slack)
    check_quantized(q2, h2, "mxfp4")
    assert ctx.read_status() == 0


def test_swiglu_gradient_against_differences(lib, ctx):
    """Gate and up on the checkpoint's grid (it keeps them exactly), fp32: the gradients against differences of the oracle's h."""
    R, K = 4, 64
    g = torch.Generator("cuda").manual_seed(7)
    gate = torch.randint(-15, 16, (R, K), generator=g, device="cuda").float() / 4
    up = torch.randint(-15, 16, (R, K), generator=g, device="cuda").float() / 4
    dh = torch.randn((R, K), generator=g, device="cuda")
    c = lib.SwigluCheckpoint(R, K, "cuda")
    lib.fp4_mx_swiglu_fwd(ctx, gate, up, checkpoint=c)
    assert torch.equal(lib.fp4_mx_dequantize(ctx, c.gate, dtype=torch.float32), gate)
    dg, du = lib.fp4_mx_swiglu_bwd(ctx, dh, c)
    e, (gs, us, ds) = 1e-5, (host(t) for t in (gate, up, dh))
    np.testing.assert_allclose(host(dg), ds * (O.swiglu(gs + e, us) - O.swiglu(gs - e, us)) / (2 * e), rtol=1e-5, atol=1e-6)
    np.testing.assert_allclose(host(du), ds * (O.swiglu(gs, us + e) - O.swiglu(gs, us - e)) / (2 * e), rtol=1e-5, atol=1e-6)


def test_swiglu_halves_of_one_matrix(lib, ctx):
    """gate and up as the halves of one projection's output, gradients into the halves of another, odd widths too."""
    for K in (256, 131):
        both, dh = torch.randn((50, 2 * K), device="cuda").bfloat16(), torch.randn((50, K), device="cuda").bfloat16()
        c, c2 = lib.SwigluCheckpoint(50, K, "cuda"), lib.SwigluCheckpoint(50, K, "cuda")
        h, _, _ = lib.fp4_mx_swiglu_fwd(ctx, both[:, :K], both[:, K:], checkpoint=c)
        assert torch.equal(h, lib.fp4_mx_swiglu_fwd(ctx, both[:, :K].contiguous(), both[:, K:].contiguous(), checkpoint=c2)[0])
        assert torch.equal(c.up.codes, c2.up.codes) and torch.equal(c.gate.scales, c2.gate.scales)
        grad = torch.empty_like(both)
        lib.fp4_mx_swiglu_bwd(ctx, dh, c, dgate=grad[:, :K], dup=grad[:, K:])
        dg, du = lib.fp4_mx_swiglu_bwd(ctx, dh, c2)
        assert torch.equal(grad[:, :K], dg) and torch.equal(grad[:, K:], du)


def test_swiglu_non_finite(lib, ctx):
    gate, up, dh = gate_up(40, 200, "bf16", 1)
    gate[5, 7] = float("nan")
    up[9, 100] = float("inf")
    c = lib.SwigluCheckpoint(40, 200, "cuda")
    ctx.status.zero_()
    h, _, _ = lib.fp4_mx_swiglu_fwd(ctx, gate, up, checkpoint=c)
    assert ctx.read_status() == lib.FP4_DEV_NONFINITE
    ctx.status.zero_()
    bad = torch.zeros((40, 200), dtype=torch.bool, device="cuda")
    bad[5, 7] = bad[9, 100] = True
    assert torch.equal(~torch.isfinite(h), bad)
    dg, du = lib.fp4_mx_swiglu_bwd(ctx, dh, c)
    bad[5, :32] = bad[9, 96:128] = True                                          # the checkpoint's blocks
    assert not (~torch.isfinite(dg) & ~bad).any() and not (~torch.isfinite(du) & ~bad).any()
    assert torch.isnan(dg[5, :32]).all() and torch.isnan(dg[9, 96:128]).all()


# ------------------------------------------------------------------------- together -----------
def mlp(lib, ctx, x, wg, wu, wd, dy, fmt):
    """Forward and backward of a gated MLP, as a training step calls it."""
    f, M, F = fmt_of(lib, fmt), x.shape[0], wg.shape[1]
    gate, sx, sg = lib.fp4_mx_linear_fwd(ctx, x, wg, fmt=f)
    up, _, su = lib.fp4_mx_linear_fwd(ctx, x, wu, fmt=f, saved_x=sx, reuse_x=True)
    ck = lib.SwigluCheckpoint(M, F, x.device)
    if fmt == "mxfp4":                                # h as an operand in either pass, never in memory itself
        hq, hqt = lib.MXTensor(M, F, x.device), lib.MXTensor(M, F, x.device, codes=False, codes_t=True)
        lib.fp4_mx_swiglu_fwd(ctx, gate, up, checkpoint=ck, quantized=hq, want_h=False)
    else:
        hq = lib.fp4_mx_quantize(ctx, lib.fp4_mx_swiglu_fwd(ctx, gate, up, checkpoint=ck)[0], f)
    sd = lib.fp4_mx_quantize(ctx, wd, f, True, True)
    y = lib.fp4_mx_gemm(ctx, hq, sd, b_t=True, dtype=x.dtype)
    dyq = lib.fp4_mx_quantize(ctx, dy, f, True, True)
    dh = lib.fp4_mx_gemm(ctx, dyq, sd, dtype=x.dtype)
    if fmt == "mxfp4":
        dgate, dup = lib.fp4_mx_swiglu_bwd(ctx, dh, ck, quantized=hqt)
    else:
        h = torch.empty_like(gate)
        dgate, dup = lib.fp4_mx_swiglu_bwd(ctx, dh, ck, h=h)
        hqt = lib.fp4_mx_quantize(ctx, h, f, False, True)
    dwd = lib.fp4_mx_gemm(ctx, hqt, dyq, a_t=True, b_t=True, dtype=x.dtype)
    dx, dwg = lib.fp4_mx_linear_bwd(ctx, dgate, sx, sg)
    dx, dwu = lib.fp4_mx_linear_bwd(ctx, dup, sx, su, dX=dx, accumulate_dx=True)
    return dict(gate=gate, up=up, y=y, dh=dh, dgate=dgate, dup=dup, dwd=dwd, dwg=dwg, dwu=dwu, dx=dx)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("M", [1, 200])
def test_mlp_forward_and_backward(lib, ctx, fmt, M):
    """Every product of the run against the oracle, each from the tensors that the run itself handed on."""
    K, F = 160, 300
    g = torch.Generator("cuda").manual_seed(M)
    mk = lambda r, c, s: (torch.randn((r, c), device="cuda", generator=g) * s).bfloat16()             # noqa: E731
    x, wg, wu, wd, dy = mk(M, K, 1.0), mk(K, F, 0.1), mk(K, F, 0.1), mk(F, K, 0.1), mk(M, K, 0.1)
    ctx.status.zero_()
    r = mlp(lib, ctx, x, wg, wu, wd, dy, fmt)
    assert ctx.read_status() == 0
    q = lambda t: O.quantize(host(t), fmt).values                                                     # noqa: E731
    qt = lambda t: O.quantize(host(t).T, fmt).values                                                  # noqa: E731
    check_product(r["gate"], q(x), qt(wg))
    check_product(r["up"], q(x), qt(wu))
    h = lib.fp4_mx_swiglu_fwd(ctx, r["gate"], r["up"])[0]
    check_product(r["y"], q(h), qt(wd))
    check_product(r["dh"], q(dy), q(wd))
    rg, ru = O.quantize(host(r["gate"]), "mxfp8").values, O.quantize(host(r["up"]), "mxfp8").values
    near(r["dgate"], O.swiglu_grad(rg, ru, host(r["dh"]))[0], np.abs(host(r["dh"]) * ru) * (1 + np.abs(rg)))
    near(r["dup"], O.swiglu_grad(rg, ru, host(r["dh"]))[1], np.abs(host(r["dh"]) * rg))
    ck = lib.SwigluCheckpoint(M, F, "cuda")
    lib.fp4_mx_swiglu_fwd(ctx, r["gate"], r["up"], checkpoint=ck)
    h2 = torch.empty_like(h)
    lib.fp4_mx_swiglu_bwd(ctx, r["dh"], ck, h=h2)
    check_product(r["dwd"], qt(h2), qt(dy))
    check_product(r["dwg"], qt(x), qt(r["dgate"]))
    check_product(r["dwu"], qt(x), qt(r["dup"]))
    part = lib.fp4_mx_gemm(ctx, lib.fp4_mx_quantize(ctx, r["dgate"], fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, wg, fmt_of(lib, fmt)))
    check_product(r["dx"], q(r["dup"]), q(wu), before=host(part))


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_captured_replayed_and_on_other_streams(lib, ctx, fmt):
    """A captured step gives the eager one's bits when replayed, also on new inputs written in place, beside another context's
    graph; nothing of a call depends on the one before."""
    M, K, F = 150, 256, 384
    mk = lambda r, c: (torch.randn((r, c), device="cuda") * 0.2).bfloat16()                            # noqa: E731
    ins = [mk(M, K), mk(K, F), mk(K, F), mk(F, K), mk(M, K)]
    other = lib.Context.for_mx(M, 512, 512)
    static = [t.clone() for t in ins]
    first = mlp(lib, ctx, *ins, fmt)
    graphs, outs = [], []
    for c in (ctx, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(mlp(lib, c, *static, fmt))
        graphs.append(graph)
    for trial in range(3):
        fresh = ins if trial == 0 else [mk(*t.shape) for t in ins]
        want = mlp(lib, ctx, *fresh, fmt)
        for s, t in zip(static, fresh):
            s.copy_(t)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(o[k], want[k]) for k in want)
        if trial == 0:
            assert all(torch.equal(first[k], want[k]) for k in want)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        again = mlp(lib, other, *fresh, fmt)
    st.synchronize()
    assert all(torch.equal(again[k], want[k]) for k in want)
    other.close()


def test_workspace_too_small_is_refused(lib):
    c = lib.Context(0, 1024)
    X, W = draw(64, 128, "bf16", 1), draw(128, 96, "bf16", 2)
    y, sx, sw = lib.fp4_mx_linear_fwd(c, X, W)
    with pytest.raises(lib.Fp4Error) as e:
        lib.fp4_mx_linear_bwd(c, y, sx, sw)
    assert e.value.code == -5
    c.close()


def test_offsets_beyond_32_bits(lib, ctx):
    """A tensor of more than 2^31 elements, whose last rows are checked, and a matrix whose rows lie 2^31 elements apart."""
    rows, cols = 262400, 8192
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = draw(130, cols, "bf16", 3)
    x[-130:] = tail
    x[0, 0] = 1.0
    q = lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_NVFP4, amax=torch.tensor([100.0], device="cuda"))
    ref = O.quantize(host(tail), "nvfp4", amax=100.0)
    np.testing.assert_array_equal(q.codes[-130:].cpu().numpy(), O.packed_codes(ref))
    back = lib.fp4_mx_dequantize(ctx, q)
    assert torch.equal(back[-130:].cpu(), torch.from_numpy(ref.values).bfloat16())
    assert float(back[0, 0]) == O.quantize(np.eye(1, 16), "nvfp4", amax=100.0).values[0, 0]
    del back
    w = lib.fp4_mx_quantize(ctx, draw(16, cols, "bf16", 4), lib.FP4_MX_NVFP4)
    y = lib.fp4_mx_gemm(ctx, q, w, dtype=torch.float32)
    assert (y[1:-130] == 0).all()
    flat = x.view(-1)
    del y
    two = torch.as_strided(flat, (2, 300), (2 ** 31 - 512 * 8192, 1))
    two.copy_(draw(2, 300, "bf16", 5))
    check_quantized(lib.fp4_mx_quantize(ctx, two, lib.FP4_MX_E2M1, True, True), two.contiguous(), "mxfp4")


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("I,J,C,fill", [(5, 640, 4096, 2), (5, 640, 512, 0), (256, 384, 512, 1), (1024, 1024, 4096, 9), (2048, 1920, 4096, 3),
                                        (4096, 1920, 4096, 20)])
def test_a_copy_that_never_comes_ends_the_kernel(lib, fmt, I, J, C, fill):
    """A copy is left out, so that every role's wait runs out: the kernel returns and says so, and the next call is sound.  Few rows, tiles of
    one CTA (a tile's first copies, which go ahead, and later ones) and of pairs."""
    c = lib.Context(0, 0)
    a = lib.fp4_mx_quantize(c, draw(I, C, "bf16", 1), fmt_of(lib, fmt))
    b = lib.fp4_mx_quantize(c, draw(J, C, "bf16", 2), fmt_of(lib, fmt))
    want = lib.fp4_mx_gemm(c, a, b)
    torch.cuda.synchronize()
    assert c.read_status() == 0
    c.debug_set(lib.binding.FP4_DEBUG_WAIT_LIMIT_US, 1000)
    c.debug_set(lib.binding.FP4_DEBUG_SKIP_FILL, fill)
    guard = torch.full((I + 2, J + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.fp4_mx_gemm(c, a, b, out=guard[1:-1, :J])
    torch.cuda.synchronize()
    assert c.read_status() & lib.FP4_DEV_TIMEOUT
    assert (guard[0] == 7).all() and (guard[-1] == 7).all() and (guard[:, J:] == 7).all()
    c.debug_set(lib.binding.FP4_DEBUG_SKIP_FILL, -1)
    c.debug_set(lib.binding.FP4_DEBUG_WAIT_LIMIT_US, 0)
    c.status.zero_()
    again = lib.fp4_mx_gemm(c, a, b)
    torch.cuda.synchronize()
    assert c.read_status() == 0 and torch.equal(again, want)
    c.close()


def test_empty_contraction_over_rows_far_apart(lib, ctx):
    """Zeros in rows 2^32 bytes apart, and nothing else touched."""
    a, b = (lib.fp4_mx_quantize(ctx, torch.empty((r, 0), dtype=torch.bfloat16, device="cuda")) for r in (2, 5))
    flat = torch.full(((1 << 30) + 16,), 3.0, device="cuda")
    lib.fp4_mx_gemm(ctx, a, b, out=torch.as_strided(flat, (2, 5), (1 << 30, 1)))
    assert (flat[:5] == 0).all() and (flat[5:64] == 3).all() and (flat[(1 << 30) - 64:1 << 30] == 3).all()
    assert (flat[1 << 30:(1 << 30) + 5] == 0).all() and (flat[(1 << 30) + 5:] == 3).all()


def test_operands_of_another_device_are_refused(lib, ctx):
    on_cpu, x = lib.MXTensor(64, 128, "cpu", codes_t=True), draw(64, 128, "bf16", 1)
    here = lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_E2M1, True, True)
    y, g = torch.empty((64, 64), device="cuda"), draw(64, 128, "bf16", 2)
    kept = lib.SwigluCheckpoint(64, 128, "cpu")
    for call in (lambda: lib.fp4_mx_quantize(ctx, x, out=on_cpu), lambda: lib.fp4_mx_dequantize(ctx, on_cpu),
                 lambda: lib.fp4_mx_gemm(ctx, here, on_cpu, out=y), lambda: lib.fp4_mx_gemm(ctx, on_cpu, here, out=y),
                 lambda: lib.fp4_mx_linear_fwd(ctx, x, x.T.contiguous(), saved_x=on_cpu),
                 lambda: lib.fp4_mx_linear_fwd(ctx, x, x.T.contiguous(), saved_w=lib.MXTensor(128, 64, "cpu", codes_t=True)),
                 lambda: lib.fp4_mx_linear_bwd(ctx, y, on_cpu, here), lambda: lib.fp4_mx_linear_bwd(ctx, y, here, on_cpu),
                 lambda: lib.fp4_mx_swiglu_fwd(ctx, x, g, checkpoint=kept), lambda: lib.fp4_mx_swiglu_fwd(ctx, x, g, quantized=on_cpu),
                 lambda: lib.fp4_mx_swiglu_bwd(ctx, x, kept)):
        with pytest.raises(AssertionError, match="device"):
            call()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_capture_that_forks_and_joins(lib, ctx, fmt):
    """Two contexts quantise on two captured streams, which join ahead of the product; replayed twice, on new inputs."""
    other, side = lib.Context(0, 0), torch.cuda.Stream()
    x, w = draw(300, 640, "bf16", 1), draw(260, 640, "bf16", 2)
    one = lambda: lib.MXTensor(300, 640, "cuda", fmt_of(lib, fmt))                            # noqa: E731
    qx, qw, y = one(), lib.MXTensor(260, 640, "cuda", fmt_of(lib, fmt)), torch.empty((300, 260), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            lib.fp4_mx_quantize(other, w, out=qw)
        lib.fp4_mx_quantize(ctx, x, out=qx)
        main.wait_stream(side)
        lib.fp4_mx_gemm(ctx, qx, qw, out=y)
    for trial in range(2):
        x.copy_(draw(300, 640, "bf16", 3 + trial))
        w.copy_(draw(260, 640, "bf16", 5 + trial))
        graph.replay()
        want = lib.fp4_mx_gemm(ctx, lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt)), lib.fp4_mx_quantize(ctx, w, fmt_of(lib, fmt)), dtype=torch.float32)
        assert torch.equal(y, want)
    other.close()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("rows", [3, 300])
def test_a_tensor_times_itself(lib, ctx, fmt, rows):
    """x x^T from one tensor, and x^T x from its other direction."""
    x = draw(rows, 200, "bf16", 1)
    q, r = (lib.fp4_mx_quantize(ctx, x, fmt_of(lib, fmt), True, True) for _ in range(2))
    for t in (False, True):
        assert torch.equal(lib.fp4_mx_gemm(ctx, q, q, t, t, dtype=torch.float32), lib.fp4_mx_gemm(ctx, q, r, t, t, dtype=torch.float32))


def test_host_threads_take_turns(lib, ctx):
    """Four threads, one context, one stream: each has its own result."""
    import threading
    ins = [(draw(100 + 30 * i, 384, "bf16", 10 + i), draw(200, 384, "bf16", 20 + i)) for i in range(4)]
    work = lambda x, w: lib.fp4_mx_gemm(ctx, lib.fp4_mx_quantize(ctx, x, lib.FP4_MX_NVFP4), lib.fp4_mx_quantize(ctx, w, lib.FP4_MX_NVFP4))   # noqa: E731
    want, got = [work(x, w) for x, w in ins], [None] * 4
    torch.cuda.synchronize()

    def run(i):
        for _ in range(20):
            got[i] = work(*ins[i])

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("M,K,N", [(1, 1, 5), (1, 40, 130), (1, 4096, 700), (3, 1000, 129), (5, 2051, 640), (16, 384, 256), (16, 8192, 512), (17, 512, 300),
                                   (2, 13824, 4096), (1, 33000, 200)])
def test_few_tokens_onto_weights_that_are_there(lib, ctx, fmt, dt, M, K, N):
    """Serving: the tokens' operand is made beside the product, or ahead of it; both give the codes, scales, amax and results of the two calls."""
    f = fmt_of(lib, fmt)
    w = lib.fp4_mx_quantize(ctx, draw(K, N, "bf16", K + N), f, codes=False, codes_t=True)
    for seed, (ld, skip) in enumerate(((K, 0), (K + 8, 8), (K + 3, 1))):
        x = torch.zeros((M, ld), dtype=DT[dt], device="cuda")[:, skip:]
        x = x[:, :K] if x.shape[1] >= K else torch.zeros((M, ld + skip), dtype=DT[dt], device="cuda")[:, skip:skip + K]
        x.copy_(draw(M, K, dt, 7 * seed + M))
        want = lib.fp4_mx_quantize(ctx, x, f)
        saved = lib.MXTensor(M, K, "cuda", f)
        for t in (saved.codes, saved.scales):
            t.fill_(0xAA)
        ctx.status.zero_()
        y, _, _ = lib.fp4_mx_linear_fwd(ctx, x, None, f, saved, w, reuse_w=True, dtype=torch.float32)
        assert torch.equal(saved.codes, want.codes) and torch.equal(saved.scales, want.scales)
        assert fmt == "mxfp4" or torch.equal(saved.amax, want.amax)
        assert torch.equal(y, lib.fp4_mx_gemm(ctx, want, w, b_t=True, dtype=torch.float32))
        assert ctx.read_status() == 0
    out = torch.full((M, N + 5), 9.0, dtype=torch.bfloat16, device="cuda")                      # results off 16-byte boundaries
    lib.fp4_mx_linear_fwd(ctx, x, None, f, saved, w, reuse_w=True, out=out[:, 1:N + 1])
    assert torch.equal(out[:, 1:N + 1], y.bfloat16()) and (out[:, 0] == 9).all() and (out[:, N + 1:] == 9).all()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_few_tokens_with_a_non_finite_value(lib, ctx, fmt, bad):
    f, M, K, N = fmt_of(lib, fmt), 4, 700, 260
    w = lib.fp4_mx_quantize(ctx, draw(K, N, "bf16", 1), f, codes=False, codes_t=True)
    x = draw(M, K, "bf16", 2)
    x[2, 555] = bad
    want, saved = lib.fp4_mx_quantize(ctx, x, f), lib.MXTensor(M, K, "cuda", f)
    ctx.status.zero_()
    y, _, _ = lib.fp4_mx_linear_fwd(ctx, x, None, f, saved, w, reuse_w=True)
    assert ctx.read_status() == lib.FP4_DEV_NONFINITE
    ctx.status.zero_()
    assert torch.equal(saved.codes, want.codes) and torch.equal(saved.scales, want.scales)
    assert y[2].isnan().all() and y[[0, 1, 3]].isfinite().all()


def test_few_tokens_with_a_given_amax(lib, ctx):
    f, M, K, N = lib.FP4_MX_NVFP4, 16, 3000, 512
    w = lib.fp4_mx_quantize(ctx, draw(K, N, "bf16", 1), f, codes=False, codes_t=True)
    x = draw(M, K, "bf16", 2)
    for a in (1e-20, 2.0, 1000.0):
        amax = torch.tensor([a], device="cuda")
        want, saved = lib.fp4_mx_quantize(ctx, x, f, amax=amax), lib.MXTensor(M, K, "cuda", f)
        saved.amax.copy_(amax)
        saved.struct.flags = 1
        y, _, _ = lib.fp4_mx_linear_fwd(ctx, x, None, f, saved, w, reuse_w=True)
        assert torch.equal(saved.codes, want.codes) and torch.equal(saved.scales, want.scales) and torch.equal(saved.amax, amax)
        assert torch.equal(y, lib.fp4_mx_gemm(ctx, want, w, b_t=True))


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_few_tokens_captured_and_with_a_copy_that_never_comes(lib, fmt):
    """The serving call in a graph, replayed on new tokens; and the wait that runs out in the kernel that makes the operand itself."""
    c, f, M, K, N = lib.Context(0, 0), fmt_of(lib, fmt), 1, 2000, 640
    w = lib.fp4_mx_quantize(c, draw(K, N, "bf16", 1), f, codes=False, codes_t=True)
    x, y, saved = draw(M, K, "bf16", 2), torch.empty((M, N), device="cuda"), lib.MXTensor(M, K, "cuda", f)
    call = lambda out: lib.fp4_mx_linear_fwd(c, x, None, f, saved, w, reuse_w=True, out=out)     # noqa: E731
    call(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y)
        call(y)                                              # back to back: the second one starts while the first drains
    for seed in (3, 4):
        x.copy_(draw(M, K, "bf16", seed))
        graph.replay()
        assert torch.equal(y, lib.fp4_mx_gemm(c, lib.fp4_mx_quantize(c, x, f), w, b_t=True, dtype=torch.float32))
    torch.cuda.synchronize()
    c.debug_set(lib.binding.FP4_DEBUG_WAIT_LIMIT_US, 1000)
    c.debug_set(lib.binding.FP4_DEBUG_SKIP_FILL, 1)
    call(torch.empty_like(y))
    torch.cuda.synchronize()
    assert c.read_status() & lib.FP4_DEV_TIMEOUT
    c.debug_set(lib.binding.FP4_DEBUG_SKIP_FILL, -1)
    c.debug_set(lib.binding.FP4_DEBUG_WAIT_LIMIT_US, 0)
    c.status.zero_()
    again = torch.empty_like(y)
    call(again)
    assert torch.equal(again, y) and c.read_status() == 0
    c.close()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("M", [1, 12, 100, 700])
def test_calls_back_to_back_keep_their_order(lib, ctx, fmt, M):
    """A chain of calls that each read what the one before wrote and write what it read, without a wait between them (each kernel starts while the
    one before drains): the bits of the same chain with a wait behind every call."""
    f, K, F = fmt_of(lib, fmt), 520, 640
    wu = lib.fp4_mx_quantize(ctx, draw(K, 2 * F, "bf16", 1, 0.0), f, True, True)
    wd = lib.fp4_mx_quantize(ctx, draw(F, K, "bf16", 2, 0.0), f, True, True)
    start = draw(M, K, "bf16", 3, 0.0)

    def chain(pause):
        new = lambda r, c: torch.empty((r, c), dtype=torch.bfloat16, device="cuda")            # noqa: E731
        x, gu, h, products = start.clone(), new(M, 2 * F), new(M, F), [new(M, M) for _ in range(12)]
        sx, sh, kept, q8 = lib.MXTensor(M, K, "cuda", f), lib.MXTensor(M, F, "cuda", f), lib.SwigluCheckpoint(M, F, "cuda"), lib.MXTensor(M, F, "cuda")
        for product in products:
            for call in (lambda: lib.fp4_mx_linear_fwd(ctx, x, None, f, sx, wu, reuse_w=True, out=gu),
                         lambda: lib.fp4_mx_swiglu_fwd(ctx, gu[:, :F], gu[:, F:], out=h, checkpoint=kept),
                         lambda: lib.fp4_mx_linear_fwd(ctx, h, None, f, sh, wd, reuse_w=True, out=x),
                         lambda: lib.fp4_mx_swiglu_bwd(ctx, h, kept, dgate=gu[:, :F], dup=gu[:, F:], quantized=q8),
                         lambda: lib.fp4_mx_dequantize(ctx, q8, out=h),
                         lambda: lib.fp4_mx_gemm(ctx, sx, sx, out=product),
                         lambda: lib.fp4_mx_dequantize(ctx, sx, out=x)):
                call()
                if pause:
                    torch.cuda.synchronize()
        return [x, gu, h, q8.codes, sh.codes] + products

    assert all(torch.equal(a, b) for a, b in zip(chain(False), chain(True)))
