"""Pins of the block-scaled oracle: grids, ties, scale rules and layout by brute force on small inputs."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import fp4_oracle as F
from oracle import mx_oracle as O


def test_grids():
    assert O.E2M1.tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert O.E4M3[0x7E] == 448 and O.E4M3[1] == 2.0 ** -9 and O.E4M3[0x38] == 1.0 and (np.diff(O.E4M3) > 0).all()


@pytest.mark.parametrize("grid", [O.E2M1, O.E4M3])
def test_nearest_code_by_brute_force(grid):
    mids = (grid[1:] + grid[:-1]) / 2
    a = np.unique(np.concatenate([grid, mids, np.nextafter(mids, 0), np.nextafter(mids, 1e9), [grid[-1] * 2]]))
    for v, c in zip(a, O.nearest_code(a, grid)):
        d = [abs(Fraction(float(g)) - Fraction(float(v))) for g in grid]
        best = [i for i in range(len(grid)) if d[i] == min(d)]
        assert c == (best[0] if len(best) == 1 else [i for i in best if i % 2 == 0][0])


@pytest.mark.parametrize("most,fmt", [(6, "mxfp4"), (448, "mxfp8")])
def test_power_of_two_scale_is_the_least_that_fits(most, fmt):
    tops = [most * 2.0 ** k * f for k in (-140, -127, -20, 0, 50, 120) for f in (1.0, 1 - 2.0 ** -24, 1 + 2.0 ** -23)] + [0.0, 2.0 ** -149]
    for t in tops:
        x = np.zeros((1, 32))
        x[0, 7] = -t
        e = int(O.quantize(x, fmt).scales[0, 0]) - 127
        assert Fraction(t) <= most * Fraction(2) ** e
        assert e == -127 or Fraction(t) > most * Fraction(2) ** (e - 1)


def test_tensor_scale_of_blocks_of_16():
    for t in (2688.0, np.nextafter(2688.0, 1e9), 2.0 ** -140, 1.0, 3.0e38):
        x = np.zeros((2, 16))
        x[1, 3] = t
        q = O.quantize(x, "nvfp4")
        k = max(-100, next(k for k in range(-150, 130) if Fraction(t) <= 2688 * Fraction(2) ** k))
        assert q.scales[0, 0] == 0 and (q.codes[0] == 0).all()
        assert O.E4M3[q.scales[1, 0]] == O.E4M3[O.nearest_code(np.array([t / 2.0 ** k / 6]), O.E4M3)[0]]


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "mxfp8"])
def test_values_are_near_their_inputs(fmt):
    rng = np.random.default_rng(1)
    x = np.float64(np.float32(rng.standard_normal((5, 75))))
    q = O.quantize(x, fmt)
    assert q.values.shape == x.shape and np.isfinite(q.values).all()
    # half a step of the format's coarsest interval, of the block's largest value (4 to 6, 416 to 448), plus half a step of an E4M3 scale
    n = O.BLOCK[fmt]
    for r in range(5):
        for b in range(0, 75, n):
            top = np.abs(x[r, b:b + n]).max()
            step = {"mxfp4": 1 / 3, "nvfp4": 1 / 6 + 1 / 16, "mxfp8": 1 / 14}[fmt]
            assert (np.abs(q.values[r, b:b + n] - x[r, b:b + n]) <= step * top).all()


def test_a_block_with_a_nan_is_nan_and_alone():
    x = np.ones((1, 96))
    x[0, 40] = np.nan
    q = O.quantize(x, "mxfp4")
    assert q.scales.tolist() == [[125, 255, 125]] and np.isnan(q.values[0, 32:64]).all()
    assert (q.values[0, :32] == 1).all() and (q.values[0, 64:] == 1).all() and (q.codes[0, 32:64] == 0).all()


def test_layout_by_hand():
    q = O.Quantized("mxfp4", np.arange(130 * 160, dtype=np.int64).reshape(130, 160).astype(np.uint8) % 16,
                    (np.arange(130 * 5).reshape(130, 5) % 251).astype(np.uint8), 0.0, None)
    c, s = O.packed_codes(q), O.packed_scales(q)
    assert c.shape == (130, 128) and c[3, 5] == q.codes[3, 10] | q.codes[3, 11] << 4 and (c[:, 80:] == 0).all()
    assert s.shape == (2 * 2 * 512,)
    assert s[33 % 32 * 16 + 4 + 2] == q.scales[33, 2]                 # row 33, block 2: first tile
    assert s[3 * 512 + 16] == q.scales[129, 4]                        # row 129, block 4: last tile, its row 1, its block 0


def test_swiglu_gradient_against_differences():
    rng = np.random.default_rng(2)
    g, u, dh = rng.standard_normal((3, 40)) * 3
    h = 1e-6
    dg, du = O.swiglu_grad(g, u, dh)
    assert np.allclose(dg, dh * (O.swiglu(g + h, u) - O.swiglu(g - h, u)) / (2 * h), rtol=1e-6, atol=1e-8)
    assert np.allclose(du, dh * (O.swiglu(g, u + h) - O.swiglu(g, u - h)) / (2 * h), rtol=1e-6, atol=1e-8)


def test_e4m3_grid_is_the_other_oracles():
    codes = np.arange(0x7F, dtype=np.uint8)
    assert np.array_equal(F.e4m3_decode(codes) if hasattr(F, "e4m3_decode") else O.E4M3, O.E4M3)


def test_the_tensors_scale_leaves_out_what_is_not_finite():
    """Blocks of 16: the blocks without an infinity or a NaN are what they are with zeros in its place."""
    x = np.random.default_rng(4).standard_normal((5, 64))
    bad, zeros = x.copy(), x.copy()
    for p, v in (((0, 3), np.inf), ((2, 40), np.nan), ((4, 63), -np.inf)):
        bad[p], zeros[p] = v, 0.0
    q, without = O.quantize(bad, "nvfp4"), O.quantize(zeros, "nvfp4")
    nan = np.isnan(q.values)
    assert q.amax == without.amax == np.abs(zeros).max() and nan.sum() == 3 * 16 and (q.codes[nan] == 0).all()
    assert np.array_equal(q.codes[~nan], without.codes[~nan]) and np.array_equal(q.values[~nan], without.values[~nan]) and (q.codes[~nan] != 0).any()
    assert O.quantize(np.full((1, 16), np.nan), "nvfp4").amax == 0.0
