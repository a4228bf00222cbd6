// Scales and codes of blocks: what the kernels that quantise share.  Internal.
#pragma once

#include <cuda_fp16.h>

#include "mx.cuh"

namespace mx_codes {

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// ------------------------------------------------------------------------- element types ---
// `most(m, w)`: the larger magnitude in each half (of fp32: of the word), a NaN if either is one; the sign bits mean nothing.
template <class T> struct TypeOf;
template <> struct TypeOf<__nv_bfloat16> {
  static constexpr uint32_t INF = 0x7F80;
  __device__ static uint32_t most(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static float value(uint32_t bits) { return __uint_as_float(bits << 16); }
  __device__ static float lo(uint32_t w) { return __uint_as_float(w << 16); }
  __device__ static float hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
  __device__ static uint32_t word(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <> struct TypeOf<__half> {
  static constexpr uint32_t INF = 0x7C00;
  __device__ static uint32_t most(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static float value(uint32_t bits) { return __half2float(__ushort_as_half(static_cast<unsigned short>(bits))); }
  __device__ static float lo(uint32_t w) { return __low2float(*reinterpret_cast<const __half2*>(&w)); }
  __device__ static float hi(uint32_t w) { return __high2float(*reinterpret_cast<const __half2*>(&w)); }
  __device__ static uint32_t word(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <> struct TypeOf<float> {
  static constexpr uint32_t INF = 0x7F800000;
  __device__ static uint32_t most(uint32_t a, uint32_t b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(__uint_as_float(a))), "f"(fabsf(__uint_as_float(b))));
    return __float_as_uint(r);
  }
  __device__ static float value(uint32_t bits) { return __uint_as_float(bits); }
};
// The larger of a pattern and the finite magnitudes in a word (two of 16 bits, or one).
template <class T>
__device__ __forceinline__ uint32_t most_finite(uint32_t m, uint32_t w) {
  constexpr uint32_t MAGNITUDE = sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFFu;
  const uint32_t lo = w & MAGNITUDE, hi = sizeof(T) == 4 ? 0u : (w >> 16) & MAGNITUDE;
  return max(m, max(lo < TypeOf<T>::INF ? lo : 0u, hi < TypeOf<T>::INF ? hi : 0u));
}
// -------------------------------------------------------------------------------- codes ----
__device__ __forceinline__ uint32_t e2m1_word(const f32x2 (&v)[4]) {      // eight elements, the first in the low nibble
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  // nibbles 1000 become 0000: the sum has a nibble's top bit set where its magnitude is not 0
  return r & (((r & 0x77777777u) + 0x77777777u) | 0x77777777u);
}
__device__ __forceinline__ uint32_t e4m3_word(f32x2 v0, f32x2 v1) {       // four elements, the first in the low byte
  float a, b, c, d;
  unpack2(v0, a, b);
  unpack2(v1, c, d);
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 y, %4, %3;\n\tmov.b32 %0, {x, y};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {              // finite
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<unsigned short>(byte)));
  return __half2float(__ushort_as_half(static_cast<unsigned short>(h)));
}
__device__ __forceinline__ float pow2_byte(uint32_t e8) { return __uint_as_float(e8 ? e8 << 23 : 0x400000u); }   // 2^(e8 - 127)
__device__ __forceinline__ float pow2_int(int k) { return __uint_as_float(uint32_t(k + 127) << 23); }            // -126 <= k <= 127

#define NO_TENSOR_SCALE make_float2(1.0f, 1.0f)

// Scale of a block: its byte, and what its elements are scaled with.
struct Scale {
  uint32_t byte;
  float mul;                 // 2^-e; NVFP4: 1 / s rounded, times 2^-k
  float s;                   // NVFP4 of fp32: s 2^k
  bool far;                  // NVFP4 of fp32: far beyond the given amax
  bool finite;
};
template <class T, int FMT>
__device__ __forceinline__ Scale scale_of(uint32_t amax_pattern, float2 tensor) {
  Scale r;
  r.finite = amax_pattern < TypeOf<T>::INF;                 // patterns of infinities and NaNs lie above all others
  const float amax = TypeOf<T>::value(amax_pattern);
  if constexpr (FMT == FP4_MX_NVFP4) {
    // The quotient by 6, and in fp32 later those by s, rounded correctly from the correctly rounded reciprocal (Markstein 1990:
    // q + (a - q s) inv in two fused steps); a value that lies on a tie of the format then comes out on it.
    const float a = fminf(amax * tensor.y, 1e30f), sixth = 1.0f / 6.0f;
    const float q = a * sixth;
    const float v = fmaf(fmaf(-q, 6.0f, a), sixth, q);
    r.byte = e4m3_word(pack2(v, 0.0f), pack2(0.0f, 0.0f)) & 0xFFu;
    // 1 / s from the special-function unit's approximation by a Newton step
    const float s = e4m3_value(r.byte);
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    inv = fmaf(inv, fmaf(-s, inv, 1.0f), inv);
    r.mul = r.byte ? inv * tensor.y : 0.0f;
    r.s = s * tensor.x;
    r.far = v > 1e6f;
    if (!r.finite) r.byte = 0x7Fu;
  } else {
    // 6 = 1.5 * 2^2 and 448 = 1.75 * 2^8: the sum carries into the exponent where the mantissa is larger
    const uint32_t over = FMT == FP4_MX_E2M1 ? 0x7FFFFFu - 0x400000u : 0x7FFFFFu - 0x600000u;
    const int e8 = max(0, int((__float_as_uint(amax) + over) >> 23) - (FMT == FP4_MX_E2M1 ? 2 : 8));
    r.byte = uint32_t(e8);
    r.mul = __uint_as_float(uint32_t(254 - e8) << 23);
    if (!r.finite) r.byte = 0xFFu;
  }
  return r;
}
template <class T, int FMT>
__device__ __forceinline__ f32x2 scaled(f32x2 x, const Scale& s) {
  const f32x2 mul = pack2(s.mul, s.mul);
  if constexpr (FMT != FP4_MX_NVFP4) return mul2(x, mul);
  if constexpr (sizeof(T) == 2) {
    // The quotient to the nearest multiple of 2^-15 (384 + q has no finer bits): on a tie of E2M1, a multiple of 1/4, it is the tie again, since
    // q = x mul is off by less than 2^-19.  Off a tie t, x differs from t s 2^k by a part in 2^11 at least (x has 11 bits and t s has 7), which is
    // 2^-13, so the multiple is on q's side of t.  Two steps; the quotient rounded correctly takes three: 16384 x 13824 both ways, amax found, 234 -> 210 us.
    return add2(fma2(x, mul, pack2(384.0f, 384.0f)), pack2(-384.0f, -384.0f));
  } else {
    // (the powers of two are kept out of nothing's range: k from -100 to 117, s from 2^-9 to 448; the remainder of a value that a code other
    // than 0 stands for is at least 2^-139)
    const f32x2 q = mul2(x, mul);
    return fma2(fma2(q, pack2(-s.s, -s.s), x), mul, q);
  }
}
__device__ __forceinline__ f32x2 within(f32x2 v, float most) {
  float a, b;
  unpack2(v, a, b);
  return pack2(fminf(fmaxf(a, -most), most), fminf(fmaxf(b, -most), most));
}
// Codes of one block of N elements, pair(i) being elements 2 i and 2 i + 1.  (A block with an infinity or a NaN: 0.)
template <class T, int FMT, int N, class Pair>
__device__ __forceinline__ void encode_block(const Scale& s, Pair pair, uint32_t* out) {
  if constexpr (FMT == FP4_MX_E4M3) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) out[i] = e4m3_word(scaled<T, FMT>(pair(2 * i), s), scaled<T, FMT>(pair(2 * i + 1), s));
  } else {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const f32x2 v[4] = {scaled<T, FMT>(pair(4 * i), s), scaled<T, FMT>(pair(4 * i + 1), s), scaled<T, FMT>(pair(4 * i + 2), s), scaled<T, FMT>(pair(4 * i + 3), s)};
      out[i] = e2m1_word(v);
    }
  }
  if (FMT == FP4_MX_NVFP4 && sizeof(T) == 4 && s.far) {
    // quotients that could overflow, and their remainders with them: from values that saturate all the same (without a remainder they do by themselves)
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      f32x2 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = scaled<T, FMT>(within(pair(4 * i + k), 8.0f * s.s), s);
      out[i] = e2m1_word(v);
    }
  }
  if (!s.finite)
#pragma unroll
    for (int i = 0; i < N / (FMT == FP4_MX_E4M3 ? 4 : 8); ++i) out[i] = 0;
}
__host__ __device__ constexpr int code_words(int fmt) { return fmt == FP4_MX_E4M3 ? 8 : 4; }               // of 32 elements
__host__ __device__ constexpr int code_row_bytes(int fmt) { return fmt == FP4_MX_E4M3 ? 128 : 64; }        // of 128 elements

// Where the scale byte of row r (0..127), block b of the tile of 128 elements goes among the tile's bytes.
__device__ __forceinline__ int scale_at(int r, int b) { return (b >> 2) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (b & 3); }
__host__ __device__ constexpr int scale_tile_bytes(int fmt) { return fmt == FP4_MX_NVFP4 ? 1024 : 512; }

}  // namespace mx_codes
