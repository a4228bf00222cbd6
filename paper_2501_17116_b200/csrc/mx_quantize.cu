// Quantisation to block-scaled operands and back, and SwiGLU, whose inputs are kept for the backward pass as such operands.
//
// A block of B elements has amax = max |x| and
//   E2M1, B = 32   scale 2^e, e the least integer in [-127, 127] with amax <= 6 * 2^e;   code = E2M1(x 2^-e)
//   E2M1, B = 16   (NVFP4) with the tensor's 2^k (mx_tensor_exponent): s = E4M3(amax 2^-k / 6), code = E2M1(x 2^-k / s),
//                  0 where s = 0
//   E4M3, B = 32   scale 2^e with amax <= 448 * 2^e;   code = E4M3(x 2^-e)
// rounded to the nearest code, ties to even; a code of -0 in E2M1 is written as 0.  With powers of two nothing saturates
// and the scaled value is exact: the only rounding is the one to the code.
//
// All kernels walk the tensor in tiles of 128 x 128 elements, one block of 256 threads each: 128 elements are the scale tile's
// four blocks of 32 (two tiles of blocks of 16) along either side, so both directions' codes and scales of a tile belong to one
// block, and leave as 64-byte pieces (codes) and whole 512-byte tiles (scales).  A lane holds eight neighbours of a row; the four
// (two) lanes of a block agree on its amax by shuffles.  Blocks along the columns are read back from a copy of the tile in
// shared memory, 32 rows of two neighbouring columns a thread.
#include <cuda_fp16.h>

#include "mx.cuh"

namespace {

constexpr int THREADS = 256;
constexpr int WARP_ROWS = MX_TILE / (THREADS / 32);      // rows of a warp
constexpr int STEPS = WARP_ROWS / 2;                     // it takes two at a time, 16 lanes each

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
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// ------------------------------------------------------------------------- element types ---
// Eight neighbours of a row as they lie in memory.
template <class T>
struct Vec8 {
  static constexpr int WORDS = int(sizeof(T)) * 2;
  uint32_t w[WORDS];
};
template <class T> struct TypeOf;
template <> struct TypeOf<__nv_bfloat16> {
  static constexpr uint32_t INF = 0x7F80;
  __device__ static float value(uint32_t bits) { return __uint_as_float(bits << 16); }
  __device__ static f32x2 pair(uint32_t w) { return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
  __device__ static uint32_t word(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <> struct TypeOf<__half> {
  static constexpr uint32_t INF = 0x7C00;
  __device__ static float value(uint32_t bits) { return __half2float(__ushort_as_half(static_cast<unsigned short>(bits))); }
  __device__ static f32x2 pair(uint32_t w) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pack2(f.x, f.y);
  }
  __device__ static uint32_t word(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <> struct TypeOf<float> { static constexpr uint32_t INF = 0x7F800000; };

template <class T>
__device__ __forceinline__ f32x2 pair_of(const Vec8<T>& v, int i) {       // elements 2 i and 2 i + 1
  if constexpr (sizeof(T) == 4) return pack2(__uint_as_float(v.w[2 * i]), __uint_as_float(v.w[2 * i + 1]));
  else return TypeOf<T>::pair(v.w[i]);
}
template <class T>
__device__ __forceinline__ void set_pair(Vec8<T>& v, int i, float a, float b) {
  if constexpr (sizeof(T) == 4) { v.w[2 * i] = __float_as_uint(a); v.w[2 * i + 1] = __float_as_uint(b); }
  else v.w[i] = TypeOf<T>::word(a, b);
}
// Bit patterns of magnitudes grow with the magnitude, and those of infinities and NaNs lie above all others: maxima are taken
// over patterns, pairs of 16-bit types at a time.
template <class T>
__device__ __forceinline__ uint32_t max_patterns(uint32_t a, uint32_t b) {
  if constexpr (sizeof(T) == 4) return max(a, b & 0x7FFFFFFFu);
  else return __vmaxu2(a, b & 0x7FFF7FFFu);
}
template <class T>
__device__ __forceinline__ uint32_t amax_word(const Vec8<T>& v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < Vec8<T>::WORDS; ++i) m = max_patterns<T>(m, v.w[i]);
  return m;
}
template <class T>
__device__ __forceinline__ uint32_t join_halves(uint32_t m) {             // pattern of the larger half
  if constexpr (sizeof(T) == 4) return m;
  else return max(m & 0xFFFFu, m >> 16);
}
template <class T>
__device__ __forceinline__ float pattern_value(uint32_t m) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(m);
  else return TypeOf<T>::value(m);
}

// `wide`: the matrix's rows all start on 16-byte boundaries.
template <class T>
__device__ __forceinline__ Vec8<T> load8(const void* base, int64_t ld, int64_t row, int64_t col, int64_t cols, bool wide) {
  Vec8<T> v;
  const T* p = static_cast<const T*>(base) + row * ld + col;
  if (wide && col + 8 <= cols) {
#pragma unroll
    for (int i = 0; i < Vec8<T>::WORDS / 4; ++i) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(p) + i);
      v.w[4 * i] = q.x; v.w[4 * i + 1] = q.y; v.w[4 * i + 2] = q.z; v.w[4 * i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t bits = 0;
      if (col + i < cols) {
        if constexpr (sizeof(T) == 4) bits = __ldg(reinterpret_cast<const uint32_t*>(p) + i);
        else bits = __ldg(reinterpret_cast<const unsigned short*>(p) + i);
      }
      if constexpr (sizeof(T) == 4) v.w[i] = bits;
      else v.w[i / 2] = i % 2 ? v.w[i / 2] | (bits << 16) : bits;
    }
  }
  return v;
}
template <class T>
__device__ __forceinline__ void store8(void* base, int64_t ld, int64_t row, int64_t col, int64_t cols, bool wide, const Vec8<T>& v) {
  T* p = static_cast<T*>(base) + row * ld + col;
  if (wide && col + 8 <= cols) {
#pragma unroll
    for (int i = 0; i < Vec8<T>::WORDS / 4; ++i)
      reinterpret_cast<uint4*>(p)[i] = make_uint4(v.w[4 * i], v.w[4 * i + 1], v.w[4 * i + 2], v.w[4 * i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i < cols) {
        if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p)[i] = v.w[i];
        else reinterpret_cast<unsigned short*>(p)[i] = static_cast<unsigned short>(i % 2 ? v.w[i / 2] >> 16 : v.w[i / 2]);
      }
  }
}

// -------------------------------------------------------------------------------- codes ----
__device__ __forceinline__ uint32_t e2m1_pair(f32x2 v) {                  // element 0 in the low nibble
  float a, b;
  unpack2(v, a, b);
  uint32_t r;
  asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t e4m3_pair(f32x2 v) {                  // element 0 in the low byte
  float a, b;
  unpack2(v, a, b);
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(a), "f"(b));
  return r;
}
// Nibbles 1000 become 0000: the sum has a nibble's top bit set where its magnitude is not 0.
__device__ __forceinline__ uint32_t clear_negative_zeros(uint32_t w) {
  return w & (((w & 0x77777777u) + 0x77777777u) | 0x77777777u);
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {              // finite
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<unsigned short>(byte)));
  return __half2float(__ushort_as_half(static_cast<unsigned short>(h)));
}
__device__ __forceinline__ float pow2_byte(uint32_t e8) { return __uint_as_float(e8 ? e8 << 23 : 0x400000u); }   // 2^(e8 - 127)
__device__ __forceinline__ float pow2_int(int k) { return __uint_as_float(uint32_t(k + 127) << 23); }            // -126 <= k <= 127

// Scale of a block: its byte, and what its elements are scaled with.
struct Scale {
  uint32_t byte;
  float mul;                 // 2^-e; NVFP4: 2^-k
  float s, inv;              // NVFP4: s and 1 / s rounded
  bool finite;
};
template <class T, int FMT>
__device__ __forceinline__ Scale scale_of(uint32_t amax_pattern, float inv_tensor) {
  Scale r;
  r.finite = amax_pattern < TypeOf<T>::INF;
  const float amax = pattern_value<T>(amax_pattern);
  if constexpr (FMT == FP4_MX_NVFP4) {
    // The quotient by 6, and later those by s, rounded correctly from the correctly rounded reciprocal (Markstein 1990:
    // q + (a - q s) inv in two fused steps); a value that lies on a tie of the format then comes out on it.
    const float a = amax * inv_tensor, sixth = 1.0f / 6.0f;
    const float q = a * sixth;
    const float v = fmaf(fmaf(-q, 6.0f, a), sixth, q);
    r.byte = e4m3_pair(pack2(v, 0.0f)) & 0xFFu;
    r.s = e4m3_value(r.byte);
    r.inv = r.byte ? __frcp_rn(r.s) : 0.0f;
    r.mul = inv_tensor;
    if (!r.finite) { r.byte = 0x7Fu; r.mul = r.inv = r.s = 0.0f; }
  } else {
    // 6 = 1.5 * 2^2 and 448 = 1.75 * 2^8: the sum carries into the exponent where the mantissa is larger
    const uint32_t over = FMT == FP4_MX_E2M1 ? 0x7FFFFFu - 0x400000u : 0x7FFFFFu - 0x600000u;
    const int e8 = max(0, int((__float_as_uint(amax) + over) >> 23) - (FMT == FP4_MX_E2M1 ? 2 : 8));
    r.byte = uint32_t(e8);
    r.mul = __uint_as_float(uint32_t(254 - e8) << 23);
    if (!r.finite) { r.byte = 0xFFu; r.mul = 0.0f; }
  }
  return r;
}
template <int FMT>
__device__ __forceinline__ f32x2 scaled(f32x2 x, const Scale& s) {
  const f32x2 v = mul2(x, pack2(s.mul, s.mul));
  if constexpr (FMT != FP4_MX_NVFP4) return v;
  const f32x2 inv = pack2(s.inv, s.inv), neg = pack2(-s.s, -s.s);
  const f32x2 q = mul2(v, inv);
  return fma2(fma2(q, neg, v), inv, q);
}
// Codes of eight elements: one word of nibbles or two of bytes.  (A block with an infinity or a NaN: 0.)
template <class T, int FMT>
__device__ __forceinline__ void encode8(const Vec8<T>& v, const Scale& s, uint32_t (&out)[FMT == FP4_MX_E4M3 ? 2 : 1]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = FMT == FP4_MX_E4M3 ? e4m3_pair(scaled<FMT>(pair_of(v, i), s)) : e2m1_pair(scaled<FMT>(pair_of(v, i), s));
  if constexpr (FMT == FP4_MX_E4M3) {
    out[0] = s.finite ? __byte_perm(r[0], r[1], 0x5410) : 0u;
    out[1] = s.finite ? __byte_perm(r[2], r[3], 0x5410) : 0u;
  } else {
    const uint32_t w = __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
    out[0] = s.finite ? clear_negative_zeros(w) : 0u;
  }
}

// Where the scale byte of row r (0..127), block b of the tile of 128 elements goes among the tile's bytes.
__device__ __forceinline__ int scale_at(int r, int b) { return (b >> 2) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (b & 3); }
__host__ __device__ constexpr int scale_tile_bytes(int fmt) { return fmt == FP4_MX_NVFP4 ? 1024 : 512; }

// What the kernels write of one direction.
struct Codes {
  uint8_t* codes;
  uint8_t* scales;
  int64_t pitch;               // bytes of a row of codes
  int64_t tiles;               // 128-element tiles of a row
};
__device__ __forceinline__ void copy_out_scales(const uint8_t* smem, const Codes& c, int64_t row_tile, int64_t col_tile, int bytes) {
  uint32_t* dst = reinterpret_cast<uint32_t*>(c.scales + (row_tile * c.tiles + col_tile) * bytes);
  for (int i = threadIdx.x; i < bytes / 4; i += THREADS) dst[i] = reinterpret_cast<const uint32_t*>(smem)[i];
}

// Row `r` of the tile, eight elements of lane (lane & 15): the codes go out, the scale byte to shared memory.  All lanes call.
template <class T, int FMT>
__device__ __forceinline__ void encode_rows(const Vec8<T>& v, int r, int lane, bool row_there, int64_t row, int64_t col_tile,
                                            float inv_tensor, const Codes& out, uint8_t* s_scale, bool& bad) {
  uint32_t m = amax_word(v);
  m = max_patterns<T>(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  if (mx_block(FMT) == 32) m = max_patterns<T>(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
  const Scale s = scale_of<T, FMT>(join_halves<T>(m), inv_tensor);
  bad |= !s.finite;
  uint32_t w[FMT == FP4_MX_E4M3 ? 2 : 1];
  encode8<T, FMT>(v, s, w);
  const int piece = lane & 15;
  if (piece % (mx_block(FMT) / 8) == 0) s_scale[scale_at(r, piece / (mx_block(FMT) / 8))] = uint8_t(s.byte);
  if (row_there) {
    uint8_t* p = out.codes + row * out.pitch + col_tile * (FMT == FP4_MX_E4M3 ? 128 : 64);
    if constexpr (FMT == FP4_MX_E4M3) reinterpret_cast<uint2*>(p)[piece] = make_uint2(w[0], w[1]);
    else reinterpret_cast<uint32_t*>(p)[piece] = w[0];
  }
}

// The tile in shared memory: row r's 16-byte units, exchanged so that a thread's 32 rows and its neighbours' lie in other banks
// (lanes of a quarter read the same two columns of rows 32 apart).
template <class T>
__device__ __forceinline__ void tile_store(uint8_t* tile, int r, int piece, const Vec8<T>& v) {
  constexpr int ROW = MX_TILE * int(sizeof(T));
#pragma unroll
  for (int i = 0; i < Vec8<T>::WORDS / 4; ++i) {
    const int unit = (piece * (Vec8<T>::WORDS / 4) + i) ^ ((r >> 5) << (sizeof(T) == 4 ? 2 : 1));
    *reinterpret_cast<uint4*>(tile + r * ROW + unit * 16) = make_uint4(v.w[4 * i], v.w[4 * i + 1], v.w[4 * i + 2], v.w[4 * i + 3]);
  }
}
// Blocks along the columns: thread t takes columns 2 p and 2 p + 1 (p = warp * 8 + lane / 4) of rows 32 b .. 32 b + 31
// (b = lane % 4); four neighbouring lanes write 64 (E4M3: 128) contiguous bytes of a column's codes.
template <class T, int FMT>
__device__ __forceinline__ void encode_cols(const uint8_t* tile, int64_t row_tile, int64_t col_tile, int64_t cols,
                                            float inv_tensor, const Codes& out, uint8_t* s_scale, bool& bad) {
  constexpr int ROW = MX_TILE * int(sizeof(T)), N = mx_block(FMT);
  const int lane = threadIdx.x & 31, p = (threadIdx.x >> 5) * 8 + (lane >> 2), b = lane & 3;
#pragma unroll 1
  for (int part = 0; part < 32 / N; ++part) {
    uint32_t lo[N], hi[N];                   // fp32: the two columns; 16 bits: both in lo
    uint32_t ma = 0, mb = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint8_t* row = tile + (32 * b + part * N + i) * ROW;
      if constexpr (sizeof(T) == 4) {
        const uint2 q = *reinterpret_cast<const uint2*>(row + ((p * 8) ^ (b << 6)));
        lo[i] = q.x; hi[i] = q.y;
        ma = max_patterns<T>(ma, q.x); mb = max_patterns<T>(mb, q.y);
      } else {
        lo[i] = *reinterpret_cast<const uint32_t*>(row + ((p * 4) ^ (b << 5)));
        ma = max_patterns<T>(ma, lo[i]);
      }
    }
    if constexpr (sizeof(T) == 2) { mb = ma >> 16; ma &= 0xFFFFu; }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const Scale s = scale_of<T, FMT>(c ? mb : ma, inv_tensor);
      bad |= !s.finite;
      const int col = 2 * p + c;
      s_scale[scale_at(col, b * (32 / N) + part)] = uint8_t(s.byte);
      uint32_t w[N / 8][FMT == FP4_MX_E4M3 ? 2 : 1];
#pragma unroll
      for (int k = 0; k < N / 8; ++k) {
        Vec8<T> v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 8 * k + 2 * i;
          if constexpr (sizeof(T) == 4) { v.w[2 * i] = c ? hi[e] : lo[e]; v.w[2 * i + 1] = c ? hi[e + 1] : lo[e + 1]; }
          else v.w[i] = __byte_perm(lo[e], lo[e + 1], c ? 0x7632 : 0x5410);
        }
        encode8<T, FMT>(v, s, w[k]);
      }
      const int64_t gcol = col_tile * MX_TILE + col;
      if (gcol < cols) {
        if constexpr (FMT == FP4_MX_E4M3) {
          uint4* dst = reinterpret_cast<uint4*>(out.codes + gcol * out.pitch + row_tile * 128 + b * 32);
          dst[0] = make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
          dst[1] = make_uint4(w[2][0], w[2][1], w[3][0], w[3][1]);
        } else if constexpr (N == 32) {
          *reinterpret_cast<uint4*>(out.codes + gcol * out.pitch + row_tile * 64 + b * 16) = make_uint4(w[0][0], w[1][0], w[2][0], w[3][0]);
        } else {
          *reinterpret_cast<uint2*>(out.codes + gcol * out.pitch + row_tile * 64 + b * 16 + part * 8) = make_uint2(w[0][0], w[1][0]);
        }
      }
    }
  }
}

struct TileAt {
  int64_t row, col;            // tile coordinates
};
__device__ __forceinline__ TileAt tile_at(int64_t col_tiles) {
  const int64_t t = blockIdx.x;
  return {t / col_tiles, t % col_tiles};
}
__device__ __forceinline__ void report(bool bad, int32_t* status) {
  if (__syncthreads_or(bad) && threadIdx.x == 0) atomicOr(status, FP4_DEV_NONFINITE);
}

// -------------------------------------------------------------------------- quantisation ---
struct QuantArgs {
  const void* x;
  int64_t rows, cols, ld;
  bool wide;
  Codes along, across;         // blocks along the rows, along the columns (codes null: not wanted)
  const uint32_t* amax;        // NVFP4
  int32_t* status;
};
template <class T, int FMT, bool ROWS, bool COLS>
__global__ void __launch_bounds__(THREADS) mx_quantize_kernel(const QuantArgs a) {
  extern __shared__ __align__(16) uint8_t tile[];
  __shared__ __align__(16) uint8_t s_scale[2][1024];
  const TileAt at = tile_at(mx_tiles(a.cols));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t col = at.col * MX_TILE + (lane & 15) * 8;
  const float inv_tensor = FMT == FP4_MX_NVFP4 ? pow2_int(-mx_tensor_exponent(__ldg(a.amax))) : 1.0f;
  bool bad = false;
  Vec8<T> v[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int64_t row = at.row * MX_TILE + warp * WARP_ROWS + 2 * i + (lane >> 4);
    if (row < a.rows && col < a.cols) v[i] = load8<T>(a.x, a.ld, row, col, a.cols, a.wide);
    else
#pragma unroll
      for (int j = 0; j < Vec8<T>::WORDS; ++j) v[i].w[j] = 0;
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int r = warp * WARP_ROWS + 2 * i + (lane >> 4);
    const int64_t row = at.row * MX_TILE + r;
    if (COLS) tile_store(tile, r, lane & 15, v[i]);
    if (ROWS) encode_rows<T, FMT>(v[i], r, lane, row < a.rows, row, at.col, inv_tensor, a.along, s_scale[0], bad);
  }
  __syncthreads();
  if (COLS) {
    encode_cols<T, FMT>(tile, at.row, at.col, a.cols, inv_tensor, a.across, s_scale[1], bad);
    __syncthreads();
    copy_out_scales(s_scale[1], a.across, at.col, at.row, scale_tile_bytes(FMT));
  }
  if (ROWS) copy_out_scales(s_scale[0], a.along, at.row, at.col, scale_tile_bytes(FMT));
  report(bad, a.status);
}

// Largest magnitude of a tensor as a pattern of fp32 (integer maxima: the order of the blocks does not matter).
template <class T>
__global__ void __launch_bounds__(THREADS) mx_amax_kernel(const void* x, int64_t rows, int64_t cols, int64_t ld, bool wide, uint32_t* amax) {
  const int64_t per_row = (cols + 7) / 8, n = rows * per_row, step = int64_t(gridDim.x) * THREADS;
  uint32_t m = 0;
  for (int64_t i = int64_t(blockIdx.x) * THREADS + threadIdx.x; i < n; i += 4 * step) {
    Vec8<T> v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t k = i + j * step;
      if (k < n) v[j] = load8<T>(x, ld, k / per_row, k % per_row * 8, cols, wide);
      else
#pragma unroll
        for (int w = 0; w < Vec8<T>::WORDS; ++w) v[j].w[w] = 0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max_patterns<T>(m, amax_word(v[j]));
  }
  m = __reduce_max_sync(0xFFFFFFFFu, join_halves<T>(m));
  __shared__ uint32_t s[THREADS / 32];
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = m;
  __syncthreads();
  if (threadIdx.x < 32) {
    m = __reduce_max_sync(0xFFFFFFFFu, threadIdx.x < THREADS / 32 ? s[threadIdx.x] : 0u);
    if (threadIdx.x == 0 && m) atomicMax(amax, __float_as_uint(pattern_value<T>(m)));
  }
}

// ------------------------------------------------------------------------ dequantisation ---
__device__ __forceinline__ void decode8_e4m3(uint2 w, float s, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned short h = static_cast<unsigned short>((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
    uint32_t t;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(t) : "h"(h));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&t));
    f[2 * i] = v.x * s;
    f[2 * i + 1] = v.y * s;
  }
}
__device__ __forceinline__ void decode8_e2m1(uint32_t w, float s, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t t;
    asm("{\n\t.reg .b8 b;\n\tcvt.u8.u32 b, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(t) : "r"((w >> (8 * i)) & 0xFFu));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&t));
    f[2 * i] = v.x * s;
    f[2 * i + 1] = v.y * s;
  }
}
// Value of a scale byte; a NaN's is NaN.
template <int FMT>
__device__ __forceinline__ float scale_value(uint32_t byte) {
  if (FMT == FP4_MX_NVFP4) return byte == 0x7Fu ? __uint_as_float(0x7FC00000u) : e4m3_value(byte);
  return byte == 0xFFu ? __uint_as_float(0x7FC00000u) : pow2_byte(byte);
}
template <class T>
__device__ __forceinline__ Vec8<T> vec_of(const float (&f)[8]) {
  Vec8<T> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) set_pair(v, i, f[2 * i], f[2 * i + 1]);
  return v;
}

struct DequantArgs {
  const uint8_t *codes, *scales;
  const uint32_t* amax;
  int64_t rows, cols;
  void* out;
  int64_t ld;
  bool wide;
};
template <class T, int FMT>
__global__ void __launch_bounds__(THREADS) mx_dequantize_kernel(const DequantArgs a) {
  constexpr int BYTES = scale_tile_bytes(FMT);
  __shared__ __align__(16) uint8_t s_scale[BYTES];
  const int64_t col_tiles = mx_tiles(a.cols);
  const TileAt at = tile_at(col_tiles);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane & 15;
  const uint8_t* src = a.scales + (at.row * col_tiles + at.col) * BYTES;
  for (int i = threadIdx.x; i < BYTES / 4; i += THREADS)
    reinterpret_cast<uint32_t*>(s_scale)[i] = __ldg(reinterpret_cast<const uint32_t*>(src) + i);
  const float tensor = FMT == FP4_MX_NVFP4 ? pow2_int(mx_tensor_exponent(__ldg(a.amax))) : 1.0f;
  const int64_t pitch = mx_pitch(a.cols, FMT);
  uint2 w[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int64_t row = at.row * MX_TILE + warp * WARP_ROWS + 2 * i + (lane >> 4);
    w[i] = make_uint2(0, 0);
    if (row < a.rows) {
      const uint8_t* p = a.codes + row * pitch + at.col * (FMT == FP4_MX_E4M3 ? 128 : 64);
      if (FMT == FP4_MX_E4M3) w[i] = __ldg(reinterpret_cast<const uint2*>(p) + piece);
      else w[i].x = __ldg(reinterpret_cast<const uint32_t*>(p) + piece);
    }
  }
  __syncthreads();
  const int64_t col = at.col * MX_TILE + piece * 8;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int r = warp * WARP_ROWS + 2 * i + (lane >> 4);
    const int64_t row = at.row * MX_TILE + r;
    // (a product of a code, its scale and the tensor's power of two is exact until the last step, which may round or overflow)
    const float s = scale_value<FMT>(s_scale[scale_at(r, piece * 8 / mx_block(FMT))]);
    float f[8];
    if (FMT == FP4_MX_E4M3) decode8_e4m3(w[i], s, f);
    else decode8_e2m1(w[i].x, s, f);
    if (FMT == FP4_MX_NVFP4)
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] *= tensor;
    if (row < a.rows && col < a.cols) store8<T>(a.out, a.ld, row, col, a.cols, a.wide, vec_of<T>(f));
  }
}

// -------------------------------------------------------------------------------- SwiGLU ---
// h = g sigmoid(g) u in fp32, rounded once.  sigmoid(g) and 1 - sigmoid(g) = sigmoid(-g) from exp(-|g|), which cannot overflow:
// neither loses its digits where it is small.
struct Sigmoid {
  float s, rest;               // sigmoid(g), sigmoid(-g)
};
__device__ __forceinline__ Sigmoid sigmoid(float g) {
  const float e = __expf(-fabsf(g)), r = __fdividef(1.0f, 1.0f + e), small = e * r;
  return {g < 0.0f ? small : r, g < 0.0f ? r : small};
}

struct SwigluArgs {
  const void *gate, *up;       // forward
  int64_t ld_gate, ld_up;
  Codes ckpt_gate, ckpt_up;    // forward: written (codes null: not wanted); backward: read
  const void* dh;              // backward
  void *dgate, *dup;
  int64_t ld_dh, ld_dgate, ld_dup;
  void* h;                     // either (null: not wanted)
  int64_t ld_h;
  Codes along, across;
  int64_t rows, cols;
  bool wide;                   // every matrix of the caller's has rows on 16-byte boundaries
  int32_t* status;
};
template <class T, bool BWD, bool KEEP, bool COLS>
__global__ void __launch_bounds__(THREADS) mx_swiglu_kernel(const SwigluArgs a) {
  extern __shared__ __align__(16) uint8_t tile[];
  __shared__ __align__(16) uint8_t s_scale[4][512];        // along, across, gate, up
  const TileAt at = tile_at(mx_tiles(a.cols));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane & 15;
  const int64_t col = at.col * MX_TILE + piece * 8;
  bool bad = false;
  if (BWD) {
    const int64_t tile_no = (at.row * a.ckpt_gate.tiles + at.col) * 512;
    if (threadIdx.x < 128)
      reinterpret_cast<uint32_t*>(s_scale[2])[threadIdx.x] = __ldg(reinterpret_cast<const uint32_t*>(a.ckpt_gate.scales + tile_no) + threadIdx.x);
    else
      reinterpret_cast<uint32_t*>(s_scale[3])[threadIdx.x - 128] = __ldg(reinterpret_cast<const uint32_t*>(a.ckpt_up.scales + tile_no) + threadIdx.x - 128);
    __syncthreads();
  }
  constexpr int AT_ONCE = 4;
#pragma unroll 1
  for (int i0 = 0; i0 < STEPS; i0 += AT_ONCE) {
    Vec8<T> x[AT_ONCE], y[AT_ONCE];            // forward: gate and up; backward: dh
    uint2 cg[AT_ONCE], cu[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int64_t row = at.row * MX_TILE + warp * WARP_ROWS + 2 * (i0 + i) + (lane >> 4);
      const bool there = row < a.rows && col < a.cols;
#pragma unroll
      for (int j = 0; j < Vec8<T>::WORDS; ++j) x[i].w[j] = y[i].w[j] = 0;
      cg[i] = cu[i] = make_uint2(0, 0);
      if (there) {
        if (BWD) {
          x[i] = load8<T>(a.dh, a.ld_dh, row, col, a.cols, a.wide);
          cg[i] = __ldg(reinterpret_cast<const uint2*>(a.ckpt_gate.codes + row * a.ckpt_gate.pitch + at.col * 128) + piece);
          cu[i] = __ldg(reinterpret_cast<const uint2*>(a.ckpt_up.codes + row * a.ckpt_up.pitch + at.col * 128) + piece);
        } else {
          x[i] = load8<T>(a.gate, a.ld_gate, row, col, a.cols, a.wide);
          y[i] = load8<T>(a.up, a.ld_up, row, col, a.cols, a.wide);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int r = warp * WARP_ROWS + 2 * (i0 + i) + (lane >> 4);
      const int64_t row = at.row * MX_TILE + r;
      const bool there = row < a.rows && col < a.cols;
      float g[8], u[8], h[8];
      if (BWD) {
        decode8_e4m3(cg[i], scale_value<FP4_MX_E4M3>(s_scale[2][scale_at(r, piece / 4)]), g);
        decode8_e4m3(cu[i], scale_value<FP4_MX_E4M3>(s_scale[3][scale_at(r, piece / 4)]), u);
        float dg[8], du[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float d[2];
          unpack2(pair_of(x[i], j), d[0], d[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int k = 2 * j + e;
            const Sigmoid s = sigmoid(g[k]);
            const float gs = g[k] * s.s;
            h[k] = gs * u[k];
            du[k] = d[e] * gs;
            // d/dg g s = s (1 + g (1 - s)) = s + g s (1 - s)
            dg[k] = d[e] * u[k] * fmaf(gs, s.rest, s.s);
          }
        }
        if (there) {
          store8<T>(a.dgate, a.ld_dgate, row, col, a.cols, a.wide, vec_of<T>(dg));
          store8<T>(a.dup, a.ld_dup, row, col, a.cols, a.wide, vec_of<T>(du));
        }
        // (dh: no block of it is scaled here, so its infinities and NaNs pass on to the gradients as they are)
      } else {
        if (KEEP) {
          encode_rows<T, FP4_MX_E4M3>(x[i], r, lane, row < a.rows, row, at.col, 1.0f, a.ckpt_gate, s_scale[2], bad);
          encode_rows<T, FP4_MX_E4M3>(y[i], r, lane, row < a.rows, row, at.col, 1.0f, a.ckpt_up, s_scale[3], bad);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          unpack2(pair_of(x[i], j), g[2 * j], g[2 * j + 1]);
          unpack2(pair_of(y[i], j), u[2 * j], u[2 * j + 1]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) h[k] = g[k] * sigmoid(g[k]).s * u[k];
      }
      const Vec8<T> hv = vec_of<T>(h);
      if (a.h && there) store8<T>(a.h, a.ld_h, row, col, a.cols, a.wide, hv);
      if (a.along.codes) encode_rows<T, FP4_MX_E2M1>(hv, r, lane, row < a.rows, row, at.col, 1.0f, a.along, s_scale[0], bad);
      if (COLS) tile_store(tile, r, piece, hv);
    }
  }
  __syncthreads();
  if (COLS) {
    encode_cols<T, FP4_MX_E2M1>(tile, at.row, at.col, a.cols, 1.0f, a.across, s_scale[1], bad);
    __syncthreads();
    copy_out_scales(s_scale[1], a.across, at.col, at.row, 512);
  }
  if (a.along.codes) copy_out_scales(s_scale[0], a.along, at.row, at.col, 512);
  if (!BWD && KEEP) {
    copy_out_scales(s_scale[2], a.ckpt_gate, at.row, at.col, 512);
    copy_out_scales(s_scale[3], a.ckpt_up, at.row, at.col, 512);
  }
  report(bad, a.status);
}

// ------------------------------------------------------------------------------ launches ---
bool rows_aligned(const void* p, int64_t ld, int dtype) {
  const int64_t elt = dtype == FP4_DTYPE_FP32 ? 4 : 2;
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * elt) % 16 == 0;
}
Codes codes_along(const fp4_mx_tensor& q, int64_t rows, int64_t cols) {
  (void)rows;
  return {q.codes, q.scales, mx_pitch(cols, q.format), mx_tiles(cols)};
}
Codes codes_across(const fp4_mx_tensor& q, int64_t rows, int64_t cols) {
  (void)cols;
  return {q.codes_t, q.scales_t, mx_pitch(rows, q.format), mx_tiles(rows)};
}
template <auto KERNEL, class A>
int launch_tiles(int device, int64_t rows, int64_t cols, size_t smem, cudaStream_t stream, const A& args) {
  const int64_t n = mx_tiles(rows) * mx_tiles(cols);
  if (n > 0x7FFFFFFF) return FP4_ERR_SHAPE;
  if (smem > 40 * 1024)
    FP4_CUDA_TRY(mx_allow_smem<KERNEL>(device, int(smem)));
  KERNEL<<<unsigned(n), THREADS, smem, stream>>>(args);
  FP4_CUDA_TRY(cudaGetLastError());
  return FP4_OK;
}

template <class T, int FMT>
int quantize_as(int device, cudaStream_t stream, const QuantArgs& a) {
  const size_t smem = MX_TILE * MX_TILE * sizeof(T);
  if (a.along.codes && a.across.codes) return launch_tiles<mx_quantize_kernel<T, FMT, true, true>>(device, a.rows, a.cols, smem, stream, a);
  if (a.across.codes) return launch_tiles<mx_quantize_kernel<T, FMT, false, true>>(device, a.rows, a.cols, smem, stream, a);
  return launch_tiles<mx_quantize_kernel<T, FMT, true, false>>(device, a.rows, a.cols, 0, stream, a);
}
template <class T>
int quantize_from(fp4_ctx* ctx, cudaStream_t stream, const QuantArgs& a, const fp4_mx_tensor& q) {
  if (q.format == FP4_MX_NVFP4 && !(q.flags & FP4_MX_AMAX_GIVEN)) {
    FP4_CUDA_TRY(cudaMemsetAsync(q.amax, 0, sizeof(float), stream));
    const int64_t n = (a.rows * ((a.cols + 7) / 8) + 4 * THREADS - 1) / (4 * THREADS), most = int64_t(ctx->num_sms) * 8;
    KernelScope scope(ctx, stream, KC_ABSMAX, 1);
    mx_amax_kernel<T><<<unsigned(n < most ? n : most), THREADS, 0, stream>>>(a.x, a.rows, a.cols, a.ld, a.wide, reinterpret_cast<uint32_t*>(q.amax));
    FP4_CUDA_TRY(cudaGetLastError());
  }
  KernelScope scope(ctx, stream, KC_ENCODE, 1);
  if (q.format == FP4_MX_E2M1) return quantize_as<T, FP4_MX_E2M1>(ctx->device, stream, a);
  if (q.format == FP4_MX_NVFP4) return quantize_as<T, FP4_MX_NVFP4>(ctx->device, stream, a);
  return quantize_as<T, FP4_MX_E4M3>(ctx->device, stream, a);
}

template <class T>
int dequantize_to(int device, cudaStream_t stream, const DequantArgs& a, int format) {
  if (format == FP4_MX_E2M1) return launch_tiles<mx_dequantize_kernel<T, FP4_MX_E2M1>>(device, a.rows, a.cols, 0, stream, a);
  if (format == FP4_MX_NVFP4) return launch_tiles<mx_dequantize_kernel<T, FP4_MX_NVFP4>>(device, a.rows, a.cols, 0, stream, a);
  return launch_tiles<mx_dequantize_kernel<T, FP4_MX_E4M3>>(device, a.rows, a.cols, 0, stream, a);
}

template <class T>
int swiglu_as(int device, cudaStream_t stream, const SwigluArgs& a, bool bwd, bool keep) {
  const size_t smem = a.across.codes ? MX_TILE * MX_TILE * sizeof(T) : 0;
  if (bwd)
    return smem ? launch_tiles<mx_swiglu_kernel<T, true, false, true>>(device, a.rows, a.cols, smem, stream, a)
                : launch_tiles<mx_swiglu_kernel<T, true, false, false>>(device, a.rows, a.cols, 0, stream, a);
  if (keep)
    return smem ? launch_tiles<mx_swiglu_kernel<T, false, true, true>>(device, a.rows, a.cols, smem, stream, a)
                : launch_tiles<mx_swiglu_kernel<T, false, true, false>>(device, a.rows, a.cols, 0, stream, a);
  return smem ? launch_tiles<mx_swiglu_kernel<T, false, false, true>>(device, a.rows, a.cols, smem, stream, a)
              : launch_tiles<mx_swiglu_kernel<T, false, false, false>>(device, a.rows, a.cols, 0, stream, a);
}
int swiglu(fp4_ctx* ctx, cudaStream_t stream, const SwigluArgs& a, int dtype, bool bwd, bool keep) {
  KernelScope scope(ctx, stream, KC_ENCODE, 1);
  if (dtype == FP4_DTYPE_BF16) return swiglu_as<__nv_bfloat16>(ctx->device, stream, a, bwd, keep);
  if (dtype == FP4_DTYPE_FP16) return swiglu_as<__half>(ctx->device, stream, a, bwd, keep);
  return swiglu_as<float>(ctx->device, stream, a, bwd, keep);
}

}  // namespace

int launch_mx_quantize(fp4_ctx* ctx, cudaStream_t stream, MxMatrix x, int dtype, const fp4_mx_tensor& q, int32_t* status) {
  QuantArgs a = {};
  a.x = x.p;
  a.rows = q.rows;
  a.cols = q.cols;
  a.ld = x.ld;
  a.wide = rows_aligned(x.p, x.ld, dtype);
  a.along = codes_along(q, q.rows, q.cols);
  a.across = codes_across(q, q.rows, q.cols);
  a.amax = reinterpret_cast<const uint32_t*>(q.amax);
  a.status = status;
  if (dtype == FP4_DTYPE_BF16) return quantize_from<__nv_bfloat16>(ctx, stream, a, q);
  if (dtype == FP4_DTYPE_FP16) return quantize_from<__half>(ctx, stream, a, q);
  return quantize_from<float>(ctx, stream, a, q);
}

int launch_mx_dequantize(fp4_ctx* ctx, cudaStream_t stream, const uint8_t* codes, const uint8_t* scales, const float* amax,
                         int64_t rows, int64_t cols, int format, void* out, int64_t ld, int dtype) {
  const DequantArgs a = {codes, scales, reinterpret_cast<const uint32_t*>(amax), rows, cols, out, ld, rows_aligned(out, ld, dtype)};
  KernelScope scope(ctx, stream, KC_ENCODE, 1);
  if (dtype == FP4_DTYPE_BF16) return dequantize_to<__nv_bfloat16>(ctx->device, stream, a, format);
  if (dtype == FP4_DTYPE_FP16) return dequantize_to<__half>(ctx->device, stream, a, format);
  return dequantize_to<float>(ctx->device, stream, a, format);
}

int launch_mx_swiglu_fwd(fp4_ctx* ctx, cudaStream_t stream, MxMatrix gate, MxMatrix up, int64_t rows, int64_t cols, int dtype,
                         MxMatrix h, const fp4_mx_tensor* ckpt_gate, const fp4_mx_tensor* ckpt_up, const fp4_mx_tensor* q,
                         int32_t* status) {
  SwigluArgs a = {};
  a.gate = gate.p;
  a.up = up.p;
  a.ld_gate = gate.ld;
  a.ld_up = up.ld;
  if (ckpt_gate) {
    a.ckpt_gate = codes_along(*ckpt_gate, rows, cols);
    a.ckpt_up = codes_along(*ckpt_up, rows, cols);
  }
  a.h = const_cast<void*>(h.p);
  a.ld_h = h.ld;
  if (q) {
    a.along = codes_along(*q, rows, cols);
    a.across = codes_across(*q, rows, cols);
  }
  a.rows = rows;
  a.cols = cols;
  a.wide = rows_aligned(gate.p, gate.ld, dtype) && rows_aligned(up.p, up.ld, dtype) && (!h.p || rows_aligned(h.p, h.ld, dtype));
  a.status = status;
  return swiglu(ctx, stream, a, dtype, false, ckpt_gate != nullptr);
}

int launch_mx_swiglu_bwd(fp4_ctx* ctx, cudaStream_t stream, MxMatrix dh, const fp4_mx_tensor& gate, const fp4_mx_tensor& up,
                         int64_t rows, int64_t cols, int dtype, MxMatrix dgate, MxMatrix dup, MxMatrix h,
                         const fp4_mx_tensor* q, int32_t* status) {
  SwigluArgs a = {};
  a.dh = dh.p;
  a.ld_dh = dh.ld;
  a.ckpt_gate = codes_along(gate, rows, cols);
  a.ckpt_up = codes_along(up, rows, cols);
  a.dgate = const_cast<void*>(dgate.p);
  a.dup = const_cast<void*>(dup.p);
  a.ld_dgate = dgate.ld;
  a.ld_dup = dup.ld;
  a.h = const_cast<void*>(h.p);
  a.ld_h = h.ld;
  if (q) {
    a.along = codes_along(*q, rows, cols);
    a.across = codes_across(*q, rows, cols);
  }
  a.rows = rows;
  a.cols = cols;
  a.wide = rows_aligned(dh.p, dh.ld, dtype) && rows_aligned(dgate.p, dgate.ld, dtype) && rows_aligned(dup.p, dup.ld, dtype) &&
           (!h.p || rows_aligned(h.p, h.ld, dtype));
  a.status = status;
  return swiglu(ctx, stream, a, dtype, true, false);
}
