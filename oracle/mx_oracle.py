"""Plain double-precision oracle of the block-scaled operands, their product and SwiGLU (fp4_mx_*).

TEST INFRASTRUCTURE, like fp4_oracle: the yardstick of the CUDA library, never reached from the product path,
and without a table or helper in common with it.  NumPy, float64; written from the definitions:

* E2M1 values 0, 1/2, 1, 3/2, 2, 3, 4, 6 (codes 0..7, sign in bit 3), E4M3 as in OCP's 8-bit formats
  (bias 7, subnormals, no infinity, 448 the largest); nearest value, a tie to the even code;
* "mxfp4": blocks of 32, scale 2^e, e the least integer in [-127, 127] with amax <= 6 * 2^e; "mxfp8": E4M3
  elements, 448 in place of 6; "nvfp4": blocks of 16, g = 2^k with k >= -100 the least integer with
  amax(tensor) <= 2688 * 2^k (infinities and NaNs left out), s = E4M3(amax(block) / g / 6), elements E2M1(x / g / s), 0 where s is 0.
  The two quotients are float32 numbers (RN32).
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

BLOCK = {"mxfp4": 32, "nvfp4": 16, "mxfp8": 32}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# the finite non-negative E4M3 values by code 0x00 .. 0x7E
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(0x7F)])


def rn32(v: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore"):                     # (beyond its range: infinity)
        return v.astype(np.float32).astype(np.float64)


def nearest_code(a: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Code of the value of `grid` nearest to each a >= 0, a tie to the even code, saturating."""
    hi = np.clip(np.searchsorted(grid, a, side="left"), 1, len(grid) - 1)
    lo = hi - 1
    up, down = grid[hi] - a, a - grid[lo]
    return np.where(up < down, hi, np.where(down < up, lo, np.where(lo % 2 == 0, lo, hi)))


def least_exponent(amax: np.ndarray, most: float, lowest: int) -> np.ndarray:
    """The least integer e >= lowest with amax <= most * 2^e."""
    e = np.full(amax.shape, lowest, dtype=np.int64)
    pos = amax > 0
    guess = np.zeros(amax.shape, dtype=np.int64)
    guess[pos] = np.ceil(np.log2(amax[pos] / most)).astype(np.int64)
    for step in (1, 0, -1):                              # the logarithm may be off by a rounding
        cand = guess + step
        fits = pos & (amax <= np.ldexp(np.full(amax.shape, most), cand))
        e = np.where(fits, np.maximum(cand, lowest), e)
    return e


@dataclass
class Quantized:
    fmt: str
    codes: np.ndarray          # [rows, cols] E2M1 nibbles or E4M3 bytes (sign included)
    scales: np.ndarray         # [rows, blocks] bytes
    amax: float
    values: np.ndarray         # [rows, cols] what the codes stand for


def quantize(x: np.ndarray, fmt: str, amax: float | None = None) -> Quantized:
    """Blocks along the columns of x (float64, holding values of the input type)."""
    rows, cols = x.shape
    n = BLOCK[fmt]
    nb = -(-cols // n)
    wide = np.zeros((rows, nb * n))
    wide[:, :cols] = x
    b = wide.reshape(rows, nb, n)
    finite = np.isfinite(b).all(axis=2)
    b = np.where(finite[:, :, None], b, 0.0)
    top = np.abs(b).max(axis=2) if b.size else np.zeros((rows, nb))
    tensor = float(np.abs(x[np.isfinite(x)]).max(initial=0.0)) if amax is None else float(amax)
    if fmt == "nvfp4":
        k = int(least_exponent(np.array([tensor]), 2688.0, -100)[0])
        s_code = nearest_code(rn32(np.ldexp(top, -k) / 6.0), E4M3)
        s = E4M3[s_code]
        with np.errstate(divide="ignore", invalid="ignore"):
            v = np.where(s[:, :, None] > 0, rn32(np.ldexp(b, -k) / s[:, :, None]), 0.0)
        scales, unit = np.where(finite, s_code, 0x7F), np.ldexp(s, k)
    else:
        e = least_exponent(top, 6.0 if fmt == "mxfp4" else 448.0, -127)
        v = np.ldexp(b, -e[:, :, None])
        scales, unit = np.where(finite, e + 127, 0xFF), np.ldexp(1.0, e)
    grid = E4M3 if fmt == "mxfp8" else E2M1
    mag = nearest_code(np.abs(v), grid)
    sign = np.signbit(v)
    if fmt == "mxfp8":
        codes = mag | (sign << 7)
    else:
        codes = mag | ((sign & (mag > 0)) << 3)
    codes = np.where(finite[:, :, None], codes, 0)
    values = np.where(sign, -1.0, 1.0) * grid[mag] * unit[:, :, None]
    values = np.where(finite[:, :, None], values, np.nan)
    flat = lambda a: a.reshape(rows, nb * n)[:, :cols]                               # noqa: E731
    return Quantized(fmt, flat(codes).astype(np.uint8), scales.astype(np.uint8), tensor, flat(values))


def pitch(cols: int, fmt: str) -> int:
    return -(-cols // 128) * (128 if fmt == "mxfp8" else 64)


def packed_codes(q: Quantized) -> np.ndarray:
    rows, cols = q.codes.shape
    wide = np.zeros((rows, -(-cols // 128) * 128), dtype=np.uint8)
    wide[:, :cols] = q.codes
    return wide if q.fmt == "mxfp8" else (wide[:, 0::2] | (wide[:, 1::2] << 4))


def packed_scales(q: Quantized) -> np.ndarray:
    """Scales in the order of the header: tiles of 128 rows x 4 blocks, written out entry by entry."""
    rows, nb = q.scales.shape
    cols = q.codes.shape[1]
    T = -(-cols // 128) * (2 if q.fmt == "nvfp4" else 1)
    out = np.zeros(-(-rows // 128) * T * 512, dtype=np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    out[(r // 128 * T + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4] = q.scales
    return out


def swiglu(g: np.ndarray, u: np.ndarray) -> np.ndarray:
    return g * u * _sigmoid(g)


def _sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def swiglu_grad(g: np.ndarray, u: np.ndarray, dh: np.ndarray):
    s = _sigmoid(g)
    return dh * u * (s + g * s * _sigmoid(-g)), dh * g * s
