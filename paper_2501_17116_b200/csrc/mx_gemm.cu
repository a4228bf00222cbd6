// Product of two block-scaled E2M1 operands on the 5th-generation tensor cores (tcgen05.mma with block scales), sm_100a.
//
//   out[i, j] (+)= g_a g_b sum_c (a[i, c] s_a[i, c / B]) (b[j, c] s_b[j, c / B])
//
// kind::mxf4 (B = 32, powers of two) and kind::mxf4nvf4 (B = 16, E4M3) multiply 64 elements of the contraction per
// instruction with the blocks' scales, which the instruction reads from tensor memory.  A k-block is 256 elements: 128 bytes
// of codes a row (one swizzled row of shared memory) and 2 (4) scale tiles of 128 rows x 4 blocks.  The scale tiles lie in
// global memory in the order that tcgen05.cp hands to tensor memory, so they travel like the codes: TMA into the ring's
// stage, from there by one tcgen05.cp of 512 bytes each, issued by the thread that issues the MMAs, ahead of them (the
// tensor core carries out one thread's copies and MMAs in order).  The tensor maps fill with zeros what lies behind the
// operand, rows and blocks alike, so no tile is a special case until the results are stored.
//
// Two kernels.  `mx_gemm_kernel`: persistent, 128 x BN tiles by single CTAs or 256 x BN by pairs (cta_group::2: the accumulators,
// A and its scales are split by rows, B's codes in halves, B's scales are needed whole in both tensor memories); two accumulator
// stages, so that the results of a tile leave under the next one's MMAs.  `mx_gemm_few_kernel`: few rows (tokens), where the
// weight's bytes and the latency count: the operands change places, so that 128 rows of the weight fill the instruction's rows
// and the tokens its columns, and the CTAs of a cluster split the contraction and add their parts through distributed shared
// memory in order of rank.  Of very few tokens it takes the values themselves (a layer's forward pass onto weights that are there): each CTA
// quantises what its k-blocks need while the weights travel, which saves the quantiser's launch and the wait for it.
//
// What bounds it: at 8192^3 (173 us in blocks of 32, 181 in blocks of 16, 6.4 and 6.1 PFLOP/s; the power cap in a long run: 206) the operands' way from L2: a
// pair's k-block of 256 x 256 is 35 KB a CTA, 60 bytes a clock at the tensor cores' rate, where L2 gives 64; a 256 x 256 x 2048 tile takes 4650 cycles alone
// and 6000 beside 73 others.  Few rows: a launch and the weight's bytes; tokens x contraction x weight rows back to back, the tokens an operand already and
// the weights from HBM: 1 x 4096 x 11008 7.8 us, 8 x 8192 x 28672 21.8 (5.7 TB/s).
// Every wait is bounded: on a timeout a CTA raises FP4_DEV_TIMEOUT, drains its copies, frees its tensor memory and returns.
#include <cuda.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "mx.cuh"
#include "mx_codes.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int BM = 128;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int A_BYTES = BM * 128;                 // codes of a k-block of 128 rows
constexpr int TMEM_COLS = 512;
// Widths are multiples of 64: a tile's columns then begin at a half of a scale tile at least.  Tensor memory holds 192 columns twice
// beside the scales; of 256 columns the second accumulator stage shares its first columns with the first stage's last.
constexpr int BN_TWICE = 192, BN_MAX = 256;
constexpr int MAX_STAGES = 6;
constexpr int STAGE_OUT = 4096;                   // of an epilogue warp
constexpr int MISC_BYTES = 256;
constexpr int MOST_SMEM = 227 * 1024;

__host__ __device__ constexpr int scale_tiles(int fmt) { return fmt == FP4_MX_NVFP4 ? 4 : 2; }      // of a k-block
__host__ __device__ constexpr int scale_bytes(int fmt) { return scale_tiles(fmt) * 512; }           // of 128 rows
// Tensor memory: accumulators at 0 and acc_offset, then the scales: A's, 4 columns a tile, and B's, 8; two sets of them, which
// k-blocks take in turn, where there is room.
__host__ __device__ constexpr int sf_cols(int fmt) { return scale_tiles(fmt) * 12; }
__host__ __device__ constexpr int sf_offset_wide(int fmt) { return fmt == FP4_MX_NVFP4 ? 448 : 480; }
__host__ __device__ constexpr int acc_offset(int fmt, bool wide) { return wide ? sf_offset_wide(fmt) - BN_MAX : BN_TWICE; }

constexpr uint32_t idesc_mx(int fmt, int m, int n) {
  return (1u << 7) | (1u << 10) | (uint32_t(n >> 3) << 17) | (fmt == FP4_MX_NVFP4 ? 0u : 1u << 23) | (uint32_t(m >> 4) << 24);
}

template <int FMT, int CTAS>
__device__ __forceinline__ void mma_mx(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa,
                                       uint32_t sfb, uint32_t accumulate) {
  if constexpr (FMT == FP4_MX_E2M1) {
    mma_mxf4<CTAS>(d_tmem, a_desc, b_desc, idesc, sfa, sfb, accumulate);
  } else if constexpr (CTAS == 2) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
  }
}
// 512 bytes of scales (32 rows of 16 bytes in shared memory) to four columns of tensor memory, the same in every lane quarter.
template <int CTAS>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if constexpr (CTAS == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// No swizzle: groups of eight 16-byte rows, 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem_addr) {
  return uint64_t((smem_addr & 0x3FFFFu) >> 4) | (uint64_t(128 >> 4) << 32) | (uint64_t(1) << 46);
}

// Arrives on a barrier of the pair's even CTA.  What it says (these accumulators have been read) is no data in memory, and the arrival
// needs no release at cluster scope, which takes 1200 cycles more, in the path from one tile to the next.
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// The last copies of a ring's producer have landed (or were given a millisecond each): a CTA must not leave ahead of them, whoever of it gave up.
// In the ordinary course they have when the last MMA is issued.
__device__ __forceinline__ void await_fills(uint64_t* full_bar, int stages, uint32_t fills) {
  for (uint32_t f = fills < uint32_t(stages) ? 0u : fills - uint32_t(stages); f < fills; ++f) {
    const uint64_t t0 = global_timer_ns();
    while (!mbar_try_wait(&full_bar[f % uint32_t(stages)], (f / uint32_t(stages)) & 1u))
      if (global_timer_ns() - t0 > 1000000ull) break;
  }
}

// One k-block: its scales to tensor memory, then four MMAs.  `sfb_cols`: columns of B's scales per tile; `sfb_shift`: 2 where the
// tile's columns begin with the second half of a scale tile.
template <int FMT, int CTAS>
__device__ __forceinline__ void issue_k_block(uint32_t a, uint32_t b, uint32_t sa, uint32_t sb, int b_tiles, uint32_t d_tmem,
                                              uint32_t sf_tmem, int sfb_shift, uint32_t idesc, bool first) {
  constexpr int T = scale_tiles(FMT);
  const uint32_t sfa = sf_tmem, sfb = sf_tmem + 4 * T;
#pragma unroll
  for (int t = 0; t < T; ++t) copy_scales<CTAS>(sfa + 4 * t, scale_desc(sa + 512 * t));
  for (int c = 0; c < b_tiles; ++c)
#pragma unroll
    for (int t = 0; t < T; ++t) copy_scales<CTAS>(sfb + 8 * t + 4 * c, scale_desc(sb + scale_bytes(FMT) * c + 512 * t));
  const uint64_t a_desc = make_smem_desc(a), b_desc = make_smem_desc(b);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    // blocks of 32: an instruction takes two of a tile's four scales, named by the descriptor
    const int t = FMT == FP4_MX_NVFP4 ? k : k >> 1;
    const uint32_t id = FMT == FP4_MX_NVFP4 ? 0u : uint32_t(k & 1) * 2;
    mma_mx<FMT, CTAS>(d_tmem, a_desc + uint64_t(2 * k), b_desc + uint64_t(2 * k), idesc | (id << 4) | (id << 29), sfa + 4 * t,
                      sfb + 8 * t + sfb_shift, first && k == 0 ? 0u : 1u);
  }
}

// --------------------------------------------------------------------------------- results --
template <int DT> struct OutOf;
template <> struct OutOf<FP4_DTYPE_BF16> {
  typedef __nv_bfloat16 type;
  __device__ static float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  __device__ static __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct OutOf<FP4_DTYPE_FP16> {
  typedef __half type;
  __device__ static float get(__half v) { return __half2float(v); }
  __device__ static __half put(float v) { return __float2half_rn(v); }
};
template <> struct OutOf<FP4_DTYPE_FP32> {
  typedef float type;
  __device__ static float get(float v) { return v; }
  __device__ static float put(float v) { return v; }
};
struct OutArgs {
  void* p;
  int64_t ld;
  int I, J, dtype;
  bool accumulate;
  bool bulk;                   // rows begin and end on 16-byte boundaries: bulk stores
};
// The tensors' powers of two (none without them).  Their product 2^k, k from -200 to 236, is applied in two halves of one sign: the first step never
// leaves fp32's range where the result stays inside (2^ka, then 2^kb does: values near 1e35 times weights of 0.02 came out infinite), and, the sums
// being multiples of 2^-20, never rounds.
struct Powers {
  const uint32_t *a, *b;
};
__device__ __forceinline__ float2 tensor_scales(uint32_t amax_a, uint32_t amax_b) {
  const int k = mx_tensor_exponent(amax_a) + mx_tensor_exponent(amax_b);
  return make_float2(mx_codes::pow2_int(k / 2), mx_codes::pow2_int(k - k / 2));
}
__device__ __forceinline__ float2 tensor_scales(const Powers& p) {
  return p.a ? tensor_scales(*p.a, *p.b) : make_float2(1.0f, 1.0f);
}

// 32 rows x 32 columns (the last ones: fewer) of a warp, row `lane` in y.  Ways out:
//   BULK      boxes of 32 rows x 64 bytes through shared memory to the copy engine
//   BULK_ADD  the same, what is there added first: every lane reads its row's 64 (fp32: 128) bytes
//   ANY       any alignment: rows through shared memory, from there in aligned pieces of 16 bytes
//   ANY_ADD   the same, in fp32 to the last, with what is there added
enum Way { BULK = 0, BULK_ADD = 1, ANY = 2, ANY_ADD = 3 };
template <int DT>
__device__ __forceinline__ uint32_t two_values(float a, float b) {
  if constexpr (DT == FP4_DTYPE_BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
template <int DT>
__device__ __forceinline__ float2 two_floats(uint32_t w) {
  if constexpr (DT == FP4_DTYPE_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <int DT>
struct Old {                   // what is there of a lane's row, as it lies in memory
  uint4 q[DT == FP4_DTYPE_FP32 ? 8 : 4];
};
template <int DT>
__device__ __forceinline__ void load_old(Old<DT>& old, const OutArgs& o, int row, int col0) {
  constexpr int PER = DT == FP4_DTYPE_FP32 ? 4 : 8;      // values in 16 bytes; a row has whole ones (OutArgs::bulk)
  const typename OutOf<DT>::type* p = static_cast<const typename OutOf<DT>::type*>(o.p) + int64_t(row) * o.ld + col0;
#pragma unroll
  for (int i = 0; i < 32 / PER; ++i) {
    old.q[i] = make_uint4(0, 0, 0, 0);
    if (row < o.I && col0 + i * PER < o.J) old.q[i] = *reinterpret_cast<const uint4*>(p + i * PER);
  }
}
template <int DT>
__device__ __forceinline__ void add_old(float (&y)[32], const Old<DT>& old) {
#pragma unroll
  for (int i = 0; i < (DT == FP4_DTYPE_FP32 ? 8 : 4); ++i) {
    const uint32_t w[4] = {old.q[i].x, old.q[i].y, old.q[i].z, old.q[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (DT == FP4_DTYPE_FP32) {
        y[4 * i + k] += __uint_as_float(w[k]);
      } else {
        const float2 f = two_floats<DT>(w[k]);
        y[8 * i + 2 * k] += f.x;
        y[8 * i + 2 * k + 1] += f.y;
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ void store_bulk(const float (&y)[32], uint8_t* stage, const OutArgs& o, const CUtensorMap* map, int row0,
                                           int col0, int lane, uint32_t& seq) {
  // two 2 KB buffers in turn; with the 64-byte swizzle 16-byte slot s of row r sits at s ^ ((r >> 1) & 3), so the rows' writes touch
  // every bank once
  const int fx = (lane >> 1) & 3;
#pragma unroll
  for (int u = 0; u < (DT == FP4_DTYPE_FP32 ? 2 : 1); ++u) {
    if (u && col0 + 16 >= o.J) break;
    uint8_t* buf = stage + (seq & 1u) * 2048;
    ++seq;
    if (elect_one()) tma_store_wait_read_1();
    __syncwarp();
    uint8_t* my_row = buf + lane * 64;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint4 q;
      if constexpr (DT == FP4_DTYPE_FP32) {
        const float* v = y + 16 * u + 4 * j;
        q = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      } else {
        const float* v = y + 8 * j;
        q = make_uint4(two_values<DT>(v[0], v[1]), two_values<DT>(v[2], v[3]), two_values<DT>(v[4], v[5]), two_values<DT>(v[6], v[7]));
      }
      *reinterpret_cast<uint4*>(my_row + ((j ^ fx) * 16)) = q;
    }
    fence_async_smem();
    __syncwarp();
    if (elect_one()) tma_store_2d(map, buf, col0 + 16 * u, row0);
  }
}
// Staged rows (32 of 128 bytes, 16-byte unit u of row r at u ^ (r & 7)) to rows of any alignment: whole aligned pieces of 16 bytes from where in
// the staged row they lie, then what is left of a row at either end.  Several rows' loads are on their way together: two warps a scheduler
// hide little else.  (A bulk copy of the aligned part of each row instead: 4096 x 5505 x 2048 48 us; element by element 71.)
__device__ __forceinline__ uint32_t at_stage(int r, int byte) { return uint32_t(r * 128 + (byte ^ ((r & 7) << 4))); }
template <int DT>
__device__ __forceinline__ void send_rows(const uint8_t* stage, const OutArgs& o, int row0, int col0, int cols, int lane) {
  typedef typename OutOf<DT>::type T;
  constexpr int E = int(sizeof(T)), AT_ONCE = 2;
  const int rows = min(32, o.I - row0), width = min(cols, o.J - col0) * E;
  uint8_t* out = reinterpret_cast<uint8_t*>(static_cast<T*>(o.p) + int64_t(row0) * o.ld + col0);
  const uint32_t low = uint32_t(reinterpret_cast<uintptr_t>(out)), low_pitch = uint32_t(o.ld * E);      // (the low bits tell a row's place)
  const int64_t pitch = o.ld * E;
  uint8_t* p = out + (lane >> 3) * pitch;
#pragma unroll 1
  for (int i = 0; i < 8; i += AT_ONCE) {
    uint32_t w[AT_ONCE][5];
    int at[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = 4 * (i + j) + (lane >> 3);
      at[j] = int((0u - low - uint32_t(r) * low_pitch) & 15u) + 16 * (lane & 7);
      if (r >= rows || at[j] + 16 > width) at[j] = -1;
      const int word = at[j] < 0 ? 0 : at[j] & ~3;
#pragma unroll
      for (int k = 0; k < 5; ++k)                          // (the fifth, of a row's last piece, may lie in the next row: it is shifted out then)
        if (k < 4 || E == 2) w[j][k] = *reinterpret_cast<const uint32_t*>(stage + at_stage(r, (word + 4 * k) & 127));
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      if (E == 2)
#pragma unroll
        for (int k = 0; k < 4; ++k) w[j][k] = __funnelshift_r(w[j][k], w[j][k + 1], (at[j] & 3) * 8);
      if (at[j] >= 0) *reinterpret_cast<uint4*>(p + at[j]) = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
      p += 4 * pitch;
    }
  }
  // elements [0, head) and behind the last piece: of 128 bytes 16 / E together, else fewer than twice that
  const int lanes = width == 128 ? 16 / E : 16, e = lane % lanes * E, per = 32 / lanes;
  p = out + (lane / lanes) * pitch;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += AT_ONCE * per) {
    T v[AT_ONCE];
    int at[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = r0 + j * per + lane / lanes;
      const int head = min(int((0u - low - uint32_t(r) * low_pitch) & 15u), width), body = (width - head) & ~15;
      at[j] = e < head ? e : e + body;
      if (r >= rows || e >= width - body) at[j] = -1;
      v[j] = *reinterpret_cast<const T*>(stage + at_stage(r & 31, at[j] < 0 ? 0 : at[j]));
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      if (at[j] >= 0) *reinterpret_cast<T*>(p + at[j]) = v[j];
      p += per * pitch;
    }
  }
}
// Staged rows of 32 fp32 values (16-byte unit u of row r at u ^ (r & 7)), added to rows of any alignment.
template <int DT>
__device__ __forceinline__ void add_rows(const uint8_t* stage, const OutArgs& o, int row0, int col0, int lane) {
  typedef typename OutOf<DT>::type T;
  constexpr int E = int(sizeof(T)), PER = 16 / E, UNITS = 32 / PER, AT_ONCE = 4;
  const int rows = min(32, o.I - row0), width = min(32, o.J - col0);
  T* out = static_cast<T*>(o.p) + int64_t(row0) * o.ld + col0;
  const uint32_t low = uint32_t(reinterpret_cast<uintptr_t>(out)), low_pitch = uint32_t(o.ld * E);
#pragma unroll 1
  for (int i = 0; i < UNITS; i += AT_ONCE) {
    uint4 q[AT_ONCE];
    int at[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = (i + j) * (32 / UNITS) + lane / UNITS;
      at[j] = int((0u - low - uint32_t(r) * low_pitch) & 15u) / E + PER * (lane % UNITS);
      if (r >= rows || at[j] + PER > width) at[j] = -1;
      if (at[j] >= 0) q[j] = *reinterpret_cast<const uint4*>(out + int64_t(r) * o.ld + at[j]);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = (i + j) * (32 / UNITS) + lane / UNITS;
      if (at[j] < 0) continue;
      uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
      float v[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) v[k] = *reinterpret_cast<const float*>(stage + at_stage(r, 4 * (at[j] + k)));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (PER == 4) {
          w[k] = __float_as_uint(v[k] + __uint_as_float(w[k]));
        } else {
          const float2 f = two_floats<DT>(w[k]);
          w[k] = two_values<DT>(v[2 * k] + f.x, v[2 * k + 1] + f.y);
        }
      }
      *reinterpret_cast<uint4*>(out + int64_t(r) * o.ld + at[j]) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  // elements [0, head) and behind the last piece: of 32 columns PER together, else fewer than twice that
  const int lanes = width == 32 ? PER : 16, e = lane % lanes, per = 32 / lanes;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += AT_ONCE * per) {
    T old[AT_ONCE];
    int at[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = r0 + j * per + lane / lanes;
      const int head = min(int((0u - low - uint32_t(r) * low_pitch) & 15u) / E, width), body = (width - head) / PER * PER;
      at[j] = e < head ? e : e + body;
      if (r >= rows || e >= width - body) at[j] = -1;
      if (at[j] >= 0) old[j] = out[int64_t(r) * o.ld + at[j]];
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = r0 + j * per + lane / lanes;
      if (at[j] >= 0) out[int64_t(r) * o.ld + at[j]] = OutOf<DT>::put(*reinterpret_cast<const float*>(stage + at_stage(r, 4 * at[j])) + OutOf<DT>::get(old[j]));
    }
  }
}

__device__ __forceinline__ void read_accumulators(float (&y)[32], uint32_t taddr, float2 scales) {
  uint32_t v[32];
  tmem_ld_32x32(taddr, v);
  tmem_ld_wait(v);
#pragma unroll
  for (int k = 0; k < 32; ++k) y[k] = __uint_as_float(v[k]) * scales.x * scales.y;
}
// One tile's accumulators (`bn` columns from `t_base` on) for one warp: the two warps of a lane quarter take pieces of 32 columns (ANY, 16-bit
// results: 64) in turn, those that the stages share (wide: the first stage's last ones, the second's first) ahead of the others.  `free_bar`:
// barrier that says the accumulators may be overwritten (0: not this lane's to say).
template <int DT, int WAY>
__device__ __forceinline__ uint32_t store_tile(uint32_t t_base, int bn, bool wide, bool first_stage, int group, int row0, int n0, const OutArgs& o,
                                               const CUtensorMap* map, uint8_t* stage, int lane, uint32_t seq, float2 scales,
                                               uint32_t free_bar) {
  constexpr int COLS = WAY == ANY && DT != FP4_DTYPE_FP32 ? 64 : 32;
  const int n_valid = min(bn, o.J - n0), pieces = bn / COLS;
  const auto release = [&] {
    tc_fence_before();
    __syncwarp();
    if (free_bar) mbar_arrive_remote(free_bar);
  };
  if (group >= pieces) release();
#pragma unroll 1
  for (int i = group; i < pieces; i += 2) {
    const int c = COLS * (wide && first_stage ? pieces - 1 - i : i);
    const bool some = c < n_valid && row0 < o.I;
    const bool last_read = wide ? i == group : i + 2 >= pieces;
    float y[32];
    if constexpr (COLS == 64) {
      __syncwarp();
#pragma unroll
      for (int h = 0; h < 2; ++h) {                        // two times 32 columns
        if (some) read_accumulators(y, t_base + uint32_t(c + 32 * h), scales);
        if (h == 1 && last_read) release();
        if (some)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float* v = y + 8 * j;
            *reinterpret_cast<uint4*>(stage + at_stage(lane, 64 * h + 16 * j)) =
                make_uint4(two_values<DT>(v[0], v[1]), two_values<DT>(v[2], v[3]), two_values<DT>(v[4], v[5]), two_values<DT>(v[6], v[7]));
          }
      }
      __syncwarp();
      if (some) send_rows<DT>(stage, o, row0, n0 + c, 64, lane);
    } else {
      Old<DT> old;
      constexpr bool EARLY = WAY == BULK_ADD && DT != FP4_DTYPE_FP32;      // (fp32: the accumulators need the registers)
      if (EARLY && some) load_old<DT>(old, o, row0 + lane, n0 + c);
      if (some) read_accumulators(y, t_base + uint32_t(c), scales);
      if (last_read) release();
      if (!some) continue;
      if (WAY == BULK_ADD) {
        if (!EARLY) load_old<DT>(old, o, row0 + lane, n0 + c);
        add_old<DT>(y, old);
      }
      if constexpr (WAY == BULK || WAY == BULK_ADD) {
        store_bulk<DT>(y, stage, o, map, row0, n0 + c, lane, seq);
      } else {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<float4*>(stage + at_stage(lane, 16 * j)) = make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
        __syncwarp();
        if constexpr (WAY == ANY) send_rows<DT>(stage, o, row0, n0 + c, 32, lane);
        else add_rows<DT>(stage, o, row0, n0 + c, lane);
      }
    }
  }
  return seq;
}

// One product of a launch, of one or two (a second without tiles: none).
struct Problem {
  CUtensorMap a, b, sa, sb, out;
  int num_k_blocks, num_m_blocks, num_n_blocks;
  OutArgs to;
  Powers powers;
};
struct GemmArgs {
  Problem p[2];
  int bn;
  int b_tiles;                 // scale tiles of 128 rows that a tile's columns touch
  int stages, stage_bytes;
  uint32_t tx_bytes, idesc;
  int32_t* status;
  uint64_t wait_limit_ns;
  int skip_fill;               // fp4_debug_set
};
constexpr int FIXED_SMEM = 1024 + MISC_BYTES + EPI_WARPS * STAGE_OUT;

template <int FMT, bool PAIR, int DT, bool ALIGNED>
__global__ void __launch_bounds__(THREADS, 1) mx_gemm_kernel(const __grid_constant__ GemmArgs args) {
  constexpr int CTAS = PAIR ? 2 : 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int STAGES = args.stages, STAGE_BYTES = args.stage_bytes;      // a stage: A, B, A's scales, B's scales
  const int b_bytes = args.bn * (128 / CTAS);
  uint8_t* s_out = smem + STAGES * STAGE_BYTES;
  uint8_t* misc = s_out + EPI_WARPS * STAGE_OUT;
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(misc);
  uint64_t* empty_bar = full_bar + MAX_STAGES;
  uint64_t* acc_full = empty_bar + MAX_STAGES;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* final_bar = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(final_bar + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  // The tiles of the first product come first.
  const int tiles_first = args.p[0].num_m_blocks * args.p[0].num_n_blocks;
  const int num_tiles = tiles_first + args.p[1].num_m_blocks * args.p[1].num_n_blocks;
  const int rank = PAIR ? int(cluster_ctarank()) : 0;
  const int worker = int(blockIdx.x) / CTAS, workers = int(gridDim.x) / CTAS;
  const bool wide = args.bn > BN_TWICE;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&acc_full[a], 1);
      mbar_init(&acc_empty[a], CTAS * EPI_WARPS);
    }
    mbar_init(final_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  const uint32_t full0 = PAIR ? cluster_address(full_bar, 0) : smem_u32(full_bar);      // (a pair's copies complete on the even CTA's)
  const auto request = [&](const Problem& q, int m_blk, int n0, int kb, int stage, uint32_t fill) {
    if (blockIdx.x == 0 && int(fill) == args.skip_fill) return;            // a left-out fill: no copy, no arrival
    uint8_t* p = smem + stage * STAGE_BYTES;
    const uint32_t bar = full0 + 8 * stage;
    if (rank == 0) mbar_arrive_expect_tx(&full_bar[stage], CTAS * args.tx_bytes);
    tma_load_2d_group<CTAS>(p, &q.a, bar, kb * 128, m_blk * BM);
    tma_load_2d_group<CTAS>(p + A_BYTES, &q.b, bar, kb * 128, n0 + rank * (args.bn / CTAS));
    tma_load_2d_group<CTAS>(p + A_BYTES + b_bytes, &q.sa, bar, kb * (scale_bytes(FMT) / 8), m_blk);
    tma_load_2d_group<CTAS>(p + A_BYTES + b_bytes + scale_bytes(FMT), &q.sb, bar, kb * (scale_bytes(FMT) / 8), n0 / 128);
  };
  if (warp == 1) tmem_alloc<CTAS>(tmem_slot, TMEM_COLS);
  mx_wait_for_inputs();
  // Single CTAs: the stages are empty and the barriers this thread's own work, so the first tile's first k-blocks travel while the
  // others meet.  (A pair's barriers have to be known to exist first.)
  if (!PAIR && threadIdx.x == 0 && worker < num_tiles) {
    const Problem& q = args.p[worker >= tiles_first];
    const int tt = worker - (worker >= tiles_first ? tiles_first : 0);
    for (int s = 0; s < STAGES && s < q.num_k_blocks; ++s) request(q, tt % q.num_m_blocks, tt / q.num_m_blocks * args.bn, s, s, uint32_t(s));
  }
  tc_fence_before();
  __syncthreads();
  mx_let_next_start();
  if (PAIR) cluster_sync_all();               // the peer's barriers exist
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer -------
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0, fills = 0;
      bool ok = true;
      for (int t = worker; t < num_tiles && ok; t += workers) {
        const Problem& q = args.p[t >= tiles_first];
        const int tt = t - (t >= tiles_first ? tiles_first : 0);
        const int m_blk = CTAS * (tt % q.num_m_blocks) + rank, n0 = (tt / q.num_m_blocks) * args.bn;
        for (int kb = 0; kb < q.num_k_blocks; ++kb) {
          if (PAIR || t != worker || kb >= STAGES) {            // (those are on their way)
            ok = mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, args.status, args.wait_limit_ns);
            if (!ok) break;
            request(q, m_blk, n0, kb, stage, fills);
          }
          ++fills;
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        // In a pair the even CTA's commits arrive on the empty barriers of both: a CTA leaves when the arrivals for its last fills
        // have come, which nobody else waits for.
        if (PAIR && t + workers >= num_tiles)
          for (int s = 0; s < STAGES && ok; ++s) {
            ok = mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, args.status, args.wait_limit_ns);
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          }
      }
      if (!ok && PAIR) {
        // Gave up: the peer's copies complete on the even CTA's barriers too, so the copies in flight are given time to land.
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 1000000ull) {}
      }
      if (!PAIR) await_fills(full_bar, STAGES, fills);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer ---------
    if (rank == 0 && elect_one()) {
      int stage = 0, n = 0;                     // n: tiles so far
      uint32_t phase = 0, sf = 0;
      bool ok = true;
      for (int t = worker; t < num_tiles && ok; t += workers, ++n) {
        const int acc = n & 1;
        const uint32_t d_tmem = tmem_base + uint32_t(acc * acc_offset(FMT, wide));
        const Problem& q = args.p[t >= tiles_first];
        const int shift = (t - (t >= tiles_first ? tiles_first : 0)) / q.num_m_blocks * args.bn % 128 ? 2 : 0;
        const int num_k_blocks = q.num_k_blocks;
        for (int kb = 0; kb < num_k_blocks; ++kb) {
          ok = mbar_wait(&full_bar[stage], phase, abort_flag, args.status, args.wait_limit_ns);
          if (!ok) break;
          if (kb == 0) {
            // A stage is free when the tile before the last has left it.  Wide: when the last has left the columns that both stages have, which
            // the tensor core waits for: nothing else is left to be done between that and the first MMA.
            const int back = wide ? 1 : 2;
            ok = n < back || mbar_wait(&acc_empty[(n - back) & 1], uint32_t((n - back) >> 1) & 1u, abort_flag, args.status, args.wait_limit_ns);
            if (!ok) break;
          }
          tc_fence_after();
          const uint32_t p = smem_u32(smem + stage * STAGE_BYTES);
          issue_k_block<FMT, CTAS>(p, p + A_BYTES, p + A_BYTES + b_bytes, p + A_BYTES + b_bytes + scale_bytes(FMT), args.b_tiles, d_tmem,
                                   tmem_base + (wide ? sf_offset_wide(FMT) : 2 * BN_TWICE + sf * sf_cols(FMT)), shift, args.idesc, kb == 0);
          sf ^= 1u;
          tc_commit_all<CTAS>(&empty_bar[stage]);
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        tc_commit_all<CTAS>(&acc_full[acc]);
      }
      // All that this thread issued must have retired before tensor memory is freed.
      tc_commit<CTAS>(final_bar);
      const uint64_t t0 = global_timer_ns();
      while (!mbar_try_wait(final_bar, 0)) {
        if (global_timer_ns() - t0 > args.wait_limit_ns) {
          atomicOr(args.status, FP4_DEV_TIMEOUT);
          break;
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue -----------
    const int quarter = warp & 3, group = (warp - 2) >> 2;
    uint8_t* stage = s_out + (warp - 2) * STAGE_OUT;
    int acc = 0;
    uint32_t acc_phase = 0, seq = 0;
    const uint32_t acc_empty0 = PAIR ? cluster_address(acc_empty, 0) : smem_u32(acc_empty);
    for (int t = worker; t < num_tiles; t += workers) {
      const Problem& q = args.p[t >= tiles_first];
      const int tt = t - (t >= tiles_first ? tiles_first : 0);
      const int m_blk = CTAS * (tt % q.num_m_blocks) + rank, n0 = (tt / q.num_m_blocks) * args.bn;
      const float2 scales = tensor_scales(q.powers);
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, args.status, args.wait_limit_ns))) break;
      tc_fence_after();
      const uint32_t t_base = tmem_base + (uint32_t(quarter * 32) << 16) + uint32_t(acc * acc_offset(FMT, wide));
      const int row0 = m_blk * BM + quarter * 32;
      const uint32_t free_bar = lane == 0 ? acc_empty0 + 8 * acc : 0u;
      const auto store = [&](auto the_way) {
        seq = store_tile<DT, decltype(the_way)::value>(t_base, args.bn, wide, acc == 0, group, row0, n0, q.to, &q.out, stage, lane, seq,
                                                       scales, free_bar);
      };
      if (q.to.accumulate) store(std::integral_constant<int, ALIGNED ? BULK_ADD : ANY_ADD>());
      else store(std::integral_constant<int, ALIGNED ? BULK : ANY>());
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
    if (elect_one()) tma_store_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();               // neither CTA leaves while the other's MMAs or arrivals may touch it
  if (warp == 1) tmem_dealloc<CTAS>(tmem_base, TMEM_COLS);
}

// ------------------------------------------------------------------------------ few rows ----
// CTA `rank` of a cluster of `splits` takes k-blocks rank, rank + splits, ... of 128 weight rows (the instruction's rows) and all
// tokens (its columns, `nt` of them, a multiple of 16).
constexpr int FEW_ROWS = 128;                     // tokens at most: one scale tile
constexpr int FEW_THREADS = 64 + 32 * 8;              // at most: 8 warps read the accumulators, 4 of up to 32 tokens that are an operand already
constexpr int FEW_MAX_STAGES = 8;
constexpr int FEW_LEAST_SMEM = 78 * 1024;
constexpr int FEW_MISC = 512;
constexpr int FEW_X_ROWS = 16;                    // tokens at most of which the kernel makes the operand itself, and a CTA's k-blocks then
constexpr int FEW_X_BLOCKS = 16;
constexpr int FEW_X_PARTS = 48;                   // tokens times k-blocks of a CTA
// Tokens that are an operand not yet: the CTAs make what they need of it, those of the first weight rows write it down.
struct FewX {
  const void* p;
  int64_t ld, cols;
  uint8_t *codes, *scales;
  uint32_t* amax;              // NVFP4
  bool find;                   // amax is not there: every CTA looks for it
  bool wide;                   // rows on 16-byte boundaries
};
__host__ __device__ constexpr int few_x_bytes(int fmt) { return FEW_X_ROWS * 128 + scale_bytes(fmt); }      // of a k-block
struct FewArgs {
  FewX x;
  int num_k_blocks, nt, splits;
  int stages, stage_bytes;
  uint32_t tx_bytes, idesc, tmem_cols;
  OutArgs out;                 // I tokens x J weight rows
  Powers powers;
  int32_t* status;
  uint64_t wait_limit_ns;
  int skip_fill;
};
__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
template <int DT>
__device__ __forceinline__ void put_four_as(const OutArgs& o, int row, int col, const float (&f)[4]) {
  typedef typename OutOf<DT>::type T;
  T* p = static_cast<T*>(o.p) + int64_t(row) * o.ld + col;
  if (o.bulk && !o.accumulate && col + 4 <= o.J) {           // (rows on 16-byte boundaries)
    if constexpr (DT == FP4_DTYPE_FP32) *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(two_values<DT>(f[0], f[1]), two_values<DT>(f[2], f[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < o.J) p[i] = OutOf<DT>::put(o.accumulate ? f[i] + OutOf<DT>::get(p[i]) : f[i]);
  }
}
__device__ __forceinline__ void put_four(const OutArgs& o, int row, int col, const float (&f)[4]) {
  if (o.dtype == FP4_DTYPE_BF16) put_four_as<FP4_DTYPE_BF16>(o, row, col, f);
  else if (o.dtype == FP4_DTYPE_FP16) put_four_as<FP4_DTYPE_FP16>(o, row, col, f);
  else put_four_as<FP4_DTYPE_FP32>(o, row, col, f);
}
// Eight elements of a row, those behind its end 0.
template <class T>
__device__ __forceinline__ void load_eight(const FewX& x, int row, int64_t col, uint32_t (&w)[2 * sizeof(T)]) {
  const T* p = static_cast<const T*>(x.p) + row * x.ld + col;
  if (x.wide && col + 8 <= x.cols) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) {
      const uint4 q = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t v = 0;
      if (col + i < x.cols) {
        if constexpr (sizeof(T) == 4) v = reinterpret_cast<const uint32_t*>(p)[i];
        else v = reinterpret_cast<const unsigned short*>(p)[i];
      }
      if constexpr (sizeof(T) == 4) w[i] = v;
      else w[i / 2] = i % 2 ? w[i / 2] | (v << 16) : v;
    }
  }
}
template <class T>
__device__ __forceinline__ uint32_t amax_of_eight(const uint32_t (&w)[2 * sizeof(T)]) {
  uint32_t m = w[0];
#pragma unroll
  for (int i = 1; i < 2 * int(sizeof(T)); ++i) m = mx_codes::TypeOf<T>::most(m, w[i]);
  if constexpr (sizeof(T) == 4) return m & 0x7FFFFFFFu;
  else return max(m & 0x7FFFu, (m >> 16) & 0x7FFFu);
}
// Largest finite magnitude of the token, as a pattern of fp32, in every thread of warps 2 and up (`s_max`: a word for each).
template <class T>
__device__ __forceinline__ uint32_t few_amax(const FewX& x, uint32_t* s_max) {
  const int threads = int(blockDim.x) - 64, t = int(threadIdx.x) - 64;
  const int64_t pieces = (x.cols + 7) / 8;
  uint32_t m = 0;
  for (int64_t c = t; c < pieces; c += 4 * threads) {
    uint32_t w[4][2 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < 4; ++i) load_eight<T>(x, 0, (c + i * threads < pieces ? c + i * threads : c) * 8, w[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, amax_of_eight<T>(w[i]));
  }
  if (m >= mx_codes::TypeOf<T>::INF) {                       // (the thread met something that is not finite: once more, without it)
    m = 0;
#pragma unroll 1
    for (int64_t c = t; c < pieces; c += threads) {
      uint32_t w[2 * sizeof(T)];
      load_eight<T>(x, 0, c * 8, w);
#pragma unroll
      for (int i = 0; i < 2 * int(sizeof(T)); ++i) m = mx_codes::most_finite<T>(m, w[i]);
    }
  }
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) s_max[(threadIdx.x >> 5) - 2] = m;
  asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory");
  for (int i = 0; i < threads / 32; ++i) m = max(m, s_max[i]);
  return __float_as_uint(mx_codes::TypeOf<T>::value(m));
}
// The tokens' operand by warps 2 and up, a token's part of a k-block at a time, eight elements a lane: codes as TMA would have brought them
// (128-byte rows, swizzled), behind them the scales.  What stands for nothing is 0 already.  `note`: also to where the caller wants it.
template <class T, int FMT>
__device__ __forceinline__ void make_operand(const FewX& x, int rows, int blocks, int rank, int splits, float2 tensor, uint8_t* made, uint64_t* x_bar, bool note,
                                             bool& bad) {
  constexpr int LANES = mx_block(FMT) / 8, AT_ONCE = 4;      // lanes of a scale's block; parts on their way together
  const int lane = threadIdx.x & 31, warps = int(blockDim.x) / 32 - 2, parts = blocks * rows;
  const int64_t pitch = mx_pitch(x.cols, FMT), tiles = mx_scale_tiles(x.cols, FMT);
#pragma unroll 1
  for (int p0 = int(threadIdx.x >> 5) - 2; p0 < parts; p0 += AT_ONCE * warps) {
    uint32_t w[AT_ONCE][2 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int p = p0 + i * warps, n = p / rows;
      if (p < parts) load_eight<T>(x, p - n * rows, int64_t(rank + n * splits) * 256 + lane * 8, w[i]);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int p = p0 + i * warps, n = p / rows, r = p - n * rows, kb = rank + n * splits;
      if (p >= parts) break;
      uint8_t* to = made + n * few_x_bytes(FMT);
      uint32_t m = amax_of_eight<T>(w[i]);
#pragma unroll
      for (int k = 1; k < LANES; k *= 2) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, k));
      const mx_codes::Scale s = mx_codes::scale_of<T, FMT>(m, tensor);
      bad |= !s.finite;
      uint32_t codes;
      const auto value = [&](int k) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i][k]);
        else return k % 2 ? mx_codes::TypeOf<T>::hi(w[i][k / 2]) : mx_codes::TypeOf<T>::lo(w[i][k / 2]);
      };
      mx_codes::encode_block<T, FMT, 8>(s, [&](int k) { return mx_codes::pack2(value(2 * k), value(2 * k + 1)); }, &codes);
      const int at = mx_codes::scale_at(r, lane / LANES);
      *reinterpret_cast<uint32_t*>(to + r * 128 + ((lane * 4) ^ ((r & 7) << 4))) = codes;
      if (lane % LANES == 0) to[FEW_X_ROWS * 128 + at] = uint8_t(s.byte);
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&x_bar[n]);
      if (note) {
        if (kb * 128 + lane * 4 < pitch) *reinterpret_cast<uint32_t*>(x.codes + r * pitch + kb * 128 + lane * 4) = codes;
        if (lane % LANES == 0 && kb * scale_tiles(FMT) + at / 512 < tiles) x.scales[int64_t(kb) * scale_bytes(FMT) + at] = uint8_t(s.byte);
      }
    }
  }
}

// T: type of the tokens where they are no operand yet, else void.
template <int FMT, class T>
__global__ void __launch_bounds__(FEW_THREADS)
mx_gemm_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                   const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_sx,
                   const __grid_constant__ FewArgs args) {
  constexpr bool MAKE = !std::is_void_v<T>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  // a stage: weights, tokens, the scales of either; or tokens and their scales, by k-block, behind the ring
  const int STAGES = args.stages, STAGE_BYTES = args.stage_bytes, x_bytes = MAKE ? 0 : args.nt * 128;
  uint8_t* x_made = smem + STAGES * STAGE_BYTES;
  uint8_t* misc = x_made + (MAKE ? (args.num_k_blocks + args.splits - 1) / args.splits * few_x_bytes(FMT) : 0);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(misc);
  uint64_t* empty_bar = full_bar + FEW_MAX_STAGES;
  uint64_t* final_bar = empty_bar + FEW_MAX_STAGES;
  uint64_t* x_bar = final_bar + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(x_bar + FEW_X_BLOCKS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* s_amax = tmem_slot + 2;                        // the tokens' amax, then one word a warp
  const int warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const int rank = args.splits > 1 ? int(cluster_ctarank()) : 0;
  const int j_blk = int(blockIdx.x) / args.splits;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    mbar_init(final_bar, 1);
    if (MAKE)
      for (int i = 0; i < FEW_X_BLOCKS; ++i) mbar_init(&x_bar[i], uint32_t(args.out.I));
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  const auto request = [&](int kb, int stage, uint32_t fill) {
    if (blockIdx.x == 0 && int(fill) == args.skip_fill) return;
    uint8_t* p = smem + stage * STAGE_BYTES;
    mbar_arrive_expect_tx(&full_bar[stage], args.tx_bytes);
    tma_load_2d(p, &map_w, &full_bar[stage], kb * 128, j_blk * BM);
    tma_load_2d(p + A_BYTES + x_bytes, &map_sw, &full_bar[stage], kb * (scale_bytes(FMT) / 8), j_blk);
    if (!MAKE) {
      tma_load_2d(p + A_BYTES, &map_x, &full_bar[stage], kb * 128, 0);
      tma_load_2d(p + A_BYTES + x_bytes + scale_bytes(FMT), &map_sx, &full_bar[stage], kb * (scale_bytes(FMT) / 8), 0);
    }
  };
  if (warp == 1) tmem_alloc<1>(tmem_slot, args.tmem_cols);
  if (MAKE) {
    for (int i = threadIdx.x; i < int(misc - x_made) / 16; i += int(blockDim.x)) reinterpret_cast<uint4*>(x_made)[i] = make_uint4(0, 0, 0, 0);
    fence_async_smem();
  }
  mx_wait_for_inputs();
  if (MAKE && j_blk == 0) {
    // scales that stand for no token
    const int64_t words = mx_scale_tiles(args.x.cols, FMT) * 128;
    for (int64_t i = rank * int(blockDim.x) + int(threadIdx.x); i < words; i += args.splits * int(blockDim.x)) {
      const int row = int(i % 4) * 32 + int(i / 4) % 32;
      if (row >= args.out.I) reinterpret_cast<uint32_t*>(args.x.scales)[i] = 0;
    }
  }
  // The stages are empty and the barriers this thread's own work: the first k-blocks travel while the others meet.
  if (threadIdx.x == 0)
    for (int s = 0, kb = rank; s < STAGES && kb < args.num_k_blocks; ++s, kb += args.splits) request(kb, s, uint32_t(s));
  tc_fence_before();
  __syncthreads();
  mx_let_next_start();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0, fills = 0;
      bool ok = true;
      for (int kb = rank; kb < args.num_k_blocks; kb += args.splits) {
        if (fills >= uint32_t(STAGES)) {
          ok = mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, args.status, args.wait_limit_ns);
          if (!ok) break;
          request(kb, stage, fills);
        }
        ++fills;
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
      await_fills(full_bar, STAGES, fills);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      int stage = 0, n = 0;
      uint32_t phase = 0, sf = 0;
      bool ok = true;
      for (int kb = rank; kb < args.num_k_blocks; kb += args.splits, ++n) {
        if (MAKE) ok = mbar_wait(&x_bar[n], 0, abort_flag, args.status, args.wait_limit_ns);
        ok = ok && mbar_wait(&full_bar[stage], phase, abort_flag, args.status, args.wait_limit_ns);
        if (!ok) break;
        tc_fence_after();
        const uint32_t p = smem_u32(smem + stage * STAGE_BYTES), x = MAKE ? smem_u32(x_made + n * few_x_bytes(FMT)) : p + A_BYTES;
        issue_k_block<FMT, 1>(p, x, p + A_BYTES + x_bytes, MAKE ? x + FEW_X_ROWS * 128 : p + A_BYTES + x_bytes + scale_bytes(FMT), 1, tmem_base,
                              tmem_base + FEW_ROWS + sf * sf_cols(FMT), 0, args.idesc, kb == rank);
        sf ^= 1u;
        tc_commit<1>(&empty_bar[stage]);
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
      tc_commit<1>(final_bar);
    }
    __syncwarp();
  } else if constexpr (MAKE) {
    // ------------------------------------------------------------------ the tokens' operand ----
    const FewX& x = args.x;
    float2 tensor = make_float2(1.0f, 1.0f);
    if (FMT == FP4_MX_NVFP4) {
      const uint32_t m = x.find ? few_amax<T>(x, s_amax + 1) : *x.amax;
      const int k = mx_tensor_exponent(m);
      tensor = make_float2(mx_codes::pow2_int(k), mx_codes::pow2_int(-k));
      if (threadIdx.x == 64) {
        *s_amax = m;
        if (x.find && blockIdx.x == 0) *x.amax = m;
      }
    }
    bool bad = false;
    make_operand<T, FMT>(x, args.out.I, (args.num_k_blocks - rank + args.splits - 1) / args.splits, rank, args.splits, tensor, x_made, x_bar, j_blk == 0, bad);
    if (__any_sync(0xFFFFFFFFu, bad) && j_blk == 0 && lane == 0) atomicOr(args.status, FP4_DEV_NONFINITE);
  }
  // Every thread awaits the last MMA (of a CTA without a k-block: at once).
  const bool done = __all_sync(0xFFFFFFFFu, mbar_wait(final_bar, 0, abort_flag, args.status, args.wait_limit_ns));
  tc_fence_after();
  // The accumulators go to shared memory, token by token, over the first stages: their copies have landed and been read.
  float* part = reinterpret_cast<float*>(smem);
  if (done && warp >= 2) {
    const int quarter = warp & 3;
    const bool any = rank < args.num_k_blocks;             // a CTA without a k-block adds nothing
    for (int c = 16 * ((warp - 2) >> 2); c < args.nt; c += 4 * (int(blockDim.x) / 32 - 2)) {
      uint32_t v[32];
      tmem_ld_32x16(tmem_base + (uint32_t(quarter * 32) << 16) + uint32_t(c), v);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (c + i < args.out.I) part[(c + i) * BM + quarter * 32 + lane] = any ? __uint_as_float(v[i]) : 0.0f;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (args.splits > 1) cluster_sync_all();
  const float2 scales = MAKE && FMT == FP4_MX_NVFP4 ? tensor_scales(*s_amax, *args.powers.b) : tensor_scales(args.powers);
  // four neighbouring columns of a token at a time, and four such fours on their way together
  constexpr int AT_ONCE = 4;
  const int step = args.splits * int(blockDim.x), n = args.out.I * (BM / 4);
  for (int e0 = rank * int(blockDim.x) + int(threadIdx.x); e0 < n; e0 += AT_ONCE * step) {
    float4 sum[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) sum[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < args.splits; ++s) {
      const uint32_t from = args.splits > 1 ? cluster_address(part, uint32_t(s)) : smem_u32(part);
      float4 v[AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (e0 + i * step < n) v[i] = load_cluster(from + 16 * uint32_t(e0 + i * step));
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (e0 + i * step < n) { sum[i].x += v[i].x; sum[i].y += v[i].y; sum[i].z += v[i].z; sum[i].w += v[i].w; }
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int e = e0 + i * step;
      if (e >= n) break;
      const float f[4] = {sum[i].x * scales.x * scales.y, sum[i].y * scales.x * scales.y, sum[i].z * scales.x * scales.y,
                          sum[i].w * scales.x * scales.y};
      put_four(args.out, e / (BM / 4), j_blk * BM + e % (BM / 4) * 4, f);
    }
  }
  if (args.splits > 1) cluster_sync_all();                 // nobody leaves while others read its part
  if (warp == 1) tmem_dealloc<1>(tmem_base, args.tmem_cols);
}

// -------------------------------------------------------------------------------- launches --
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int make_map(fp4_ctx* ctx, CUtensorMap* map, CUtensorMapDataType type, const void* p, uint64_t inner, uint64_t outer, uint64_t stride,
             uint32_t box_inner, uint32_t box_outer, CUtensorMapSwizzle swizzle, CUtensorMapL2promotion l2) {
  const cuuint64_t dims[2] = {inner, outer}, strides[1] = {stride};
  const cuuint32_t box[2] = {box_inner, box_outer}, elem_strides[2] = {1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(map, type, 2, const_cast<void*>(p), dims, strides, box, elem_strides,
                                                                        CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, l2, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? FP4_OK : FP4_ERR_CUDA;
}
int make_codes_map(fp4_ctx* ctx, CUtensorMap* map, const uint8_t* codes, int64_t rows, int64_t C, int box_rows) {
  const uint64_t pitch = uint64_t(mx_pitch(C, FP4_MX_E2M1));
  return make_map(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, pitch, uint64_t(rows), pitch, 128, uint32_t(box_rows),
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}
// Scales, by row of scale tiles, in 8-byte elements (a box of all the tiles of a k-block stays within 256 of them).
int make_scales_map(fp4_ctx* ctx, CUtensorMap* map, const uint8_t* scales, int64_t rows, int64_t C, int format, int box_tiles) {
  const uint64_t bytes = uint64_t(mx_scale_tiles(C, format)) * 512;
  return make_map(ctx, map, CU_TENSOR_MAP_DATA_TYPE_INT64, scales, bytes / 8, uint64_t(mx_tiles(rows)), bytes,
                  uint32_t(scale_bytes(format) / 8), uint32_t(box_tiles), CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

OutArgs out_args(const MxGemm& g) {
  const int64_t elt = g.dtype == FP4_DTYPE_FP32 ? 4 : 2;
  OutArgs o = {g.out, g.ld, int(g.I), int(g.J), g.dtype, g.accumulate, false};
  // (a bulk store clips a row at its map's end to whole 16 bytes: a row that ends inside such a piece would take its neighbours' bytes along)
  o.bulk = (reinterpret_cast<uintptr_t>(g.out) & 15) == 0 && (g.ld * elt) % 16 == 0 && (g.J * elt) % 16 == 0;
  return o;
}
Powers powers_of(const MxGemm& g) {
  if (g.format != FP4_MX_NVFP4) return {nullptr, nullptr};
  return {reinterpret_cast<const uint32_t*>(g.a_amax), reinterpret_cast<const uint32_t*>(g.b_amax)};
}

// Times (ns) of the forms, as a model: a launch, then for each tile of the busiest worker a fixed part and one per k-block (blocks of 16 cost a tenth more
// of it).  It is there to order the forms.  Over 24 sizes from 129 x 128 x 256 to 8192 x 5120 x 13824 in either kind of blocks its times are off by 15 % by
// root mean square and 46 % at worst, while the form that it takes is the best of the seven or within 1.5 % of it in 40 of the 48 and 11 % behind at worst
// (1024 x 1024 x 4096: 128 x 64 8.5 us, pairs 128 wide 7.7).  One thread issues a k-block's copies of scales and MMAs in 250 ns, whatever the width, so narrow
// tiles pay only where they fill SMs that would idle: 1024^3 4.6 us by 128 x 64 against 5.7 by pairs 256 wide, 4096 x 2048 x 5504 47.8 against 19.3.
struct TileForm {
  int bn;
  bool pair;
  int64_t cost;
};
struct FormCost {
  int bn;
  bool pair;
  int launch, tile, k_block;
};
constexpr FormCost FORMS[] = {{64, false, 3400, 460, 251},  {128, false, 3400, 650, 270},  {192, false, 3400, 1030, 296}, {256, false, 3400, 1640, 344},
                              {128, true, 4000, 700, 228}, {192, true, 4000, 1030, 239}, {256, true, 4000, 1460, 279}};
TileForm choose_form(const fp4_ctx* ctx, const MxGemm* g, int n) {
  TileForm best = {64, false, -1};
  for (const FormCost& f : FORMS) {
    const int64_t rows = f.pair ? 2 * BM : BM, workers = f.pair ? ctx->num_sms / 2 : ctx->num_sms;
    if (!workers) continue;
    int64_t tiles[2] = {0, 0}, each[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
      tiles[i] = (g[i].I + rows - 1) / rows * ((g[i].J + f.bn - 1) / f.bn);
      each[i] = f.tile + (g[i].C + 255) / 256 * f.k_block * (g[i].format == FP4_MX_NVFP4 ? 11 : 10) / 10;
    }
    // worker r takes tiles r, r + workers, ...: the busiest is the first one, or the first one that begins with the second product
    int64_t busiest = 0;
    for (const int64_t r : {int64_t(0), tiles[0] % workers}) {
      const int64_t first = (tiles[0] - r + workers - 1) / workers, all = (tiles[0] + tiles[1] - r + workers - 1) / workers;
      const int64_t t = first * each[0] + (all - first) * each[1];
      if (t > busiest) busiest = t;
    }
    if (best.cost < 0 || f.launch + busiest < best.cost) best = {f.bn, f.pair, f.launch + busiest};
  }
  return best;
}

// Few rows: into how many parts a cluster splits the contraction, and the time by the same kind of model.  As a rule no more than four parts, and no more
// CTAs than SMs (24 tokens x contraction x weight rows, back to back with weights from HBM, 1 / 2 / 3 / 4 / 5 / 6 parts: 5504 x 2048 8.7 / 6.9 / 6.3 / 5.7 / 6.0 /
// 6.2; 4096 x 4096 7.2 / 5.9 / 6.4 / 6.1 / 6.7 / 6.8; 100 tokens 8.3 / 7.8 / 7.9 / 8.2 / 10.8 / 10.9).
struct FewForm {
  int splits;
  int64_t cost;
};
FewForm choose_few(const fp4_ctx* ctx, const MxGemm& g) {
  const int64_t kbs = (g.C + 255) / 256, tiles = (g.J + BM - 1) / BM;
  int64_t splits = ctx->num_sms / tiles;
  if (splits > (kbs + 1) / 2) splits = (kbs + 1) / 2;
  splits = splits < 1 ? 1 : (splits > 4 ? 4 : splits);
  // Two CTAs an SM, where each still has eight k-blocks, and the tokens take little room.  It hides latency, which pays where the weights are in L2, and
  // fills the SMs unevenly, which costs where they come from HBM and the parts are few: 24 tokens x contraction x weight rows, us without / with it, from L2
  // 4096 x 11008 7.2 / 6.4, 11008 x 4096 7.8 / 7.4, 13824 x 5120 9.3 / 7.9, 20000 x 1000 9.6 / 8.5; from HBM 7.8 / 8.3, 8.9 / 9.0, 10.4 / 10.5, 9.6 / 8.6.
  int64_t more = 2 * ctx->num_sms / tiles;
  if (more > kbs / 8) more = kbs / 8;
  if (more > 6) more = 6;
  if (g.I <= 32 && more > splits) splits = more;
  const int64_t rounds = (tiles + 2 * ctx->num_sms - 1) / (2 * ctx->num_sms);
  const int64_t one = (kbs + splits - 1) / splits * (g.format == FP4_MX_NVFP4 ? 200 : 150) + 15 * ((g.I + 15) / 16 * 16);
  return {int(splits), 4100 + (splits > 1 ? 300 : 0) + rounds * one};
}

template <int FMT, bool PAIR, int DT, bool ALIGNED>
int launch_tiles_as(fp4_ctx* ctx, cudaStream_t stream, const MxGemm* g, int n, int bn, int32_t* status) {
  constexpr int CTAS = PAIR ? 2 : 1;
  GemmArgs args = {};
  args.bn = bn;
  args.b_tiles = (bn + 127) / 128;
  args.stage_bytes = A_BYTES + bn * 128 / CTAS + scale_bytes(FMT) * (1 + args.b_tiles);
  args.tx_bytes = uint32_t(args.stage_bytes);
  args.stages = (MOST_SMEM - FIXED_SMEM) / args.stage_bytes;
  if (args.stages > MAX_STAGES) args.stages = MAX_STAGES;
  args.idesc = idesc_mx(FMT, CTAS * BM, bn);
  args.status = status;
  args.wait_limit_ns = mx_wait_limit(ctx);
  args.skip_fill = ctx->debug_skip_fill;
  int64_t tiles = 0;
  for (int i = 0; i < n; ++i) {
    Problem& p = args.p[i];
    const MxGemm& q = g[i];
    p.num_k_blocks = int((q.C + 255) / 256);
    p.num_m_blocks = int((q.I + CTAS * BM - 1) / (CTAS * BM));
    p.num_n_blocks = int((q.J + bn - 1) / bn);
    tiles += int64_t(p.num_m_blocks) * p.num_n_blocks;
    p.to = out_args(q);
    p.powers = powers_of(q);
    int rc = make_codes_map(ctx, &p.a, q.a, q.I, q.C, BM);
    if (rc == FP4_OK) rc = make_codes_map(ctx, &p.b, q.b, q.J, q.C, bn / CTAS);
    if (rc == FP4_OK) rc = make_scales_map(ctx, &p.sa, q.a_scales, q.I, q.C, FMT, 1);
    if (rc == FP4_OK) rc = make_scales_map(ctx, &p.sb, q.b_scales, q.J, q.C, FMT, args.b_tiles);
    if (rc == FP4_OK && ALIGNED) {
      const CUtensorMapDataType type = DT == FP4_DTYPE_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                       : DT == FP4_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                              : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
      constexpr uint32_t elt = DT == FP4_DTYPE_FP32 ? 4 : 2;
      rc = make_map(ctx, &p.out, type, q.out, uint64_t(q.J), uint64_t(q.I), uint64_t(q.ld) * elt, 64 / elt, 32, CU_TENSOR_MAP_SWIZZLE_64B,
                    CU_TENSOR_MAP_L2_PROMOTION_NONE);
    }
    if (rc != FP4_OK) return rc;
  }
  constexpr auto kernel = mx_gemm_kernel<FMT, PAIR, DT, ALIGNED>;
  FP4_CUDA_TRY(mx_allow_smem<kernel>(ctx->device, MOST_SMEM));
  const int64_t most = ctx->num_sms / CTAS;
  KernelScope scope(ctx, stream, KC_GEMM, 1);
  return mx_launch<kernel>(dim3(unsigned(CTAS * (tiles < most ? tiles : most))), THREADS, FIXED_SMEM + args.stages * args.stage_bytes, CTAS, stream, args);
}
template <int FMT>
int launch_tiles(fp4_ctx* ctx, cudaStream_t stream, const MxGemm* g, int n, const TileForm& f, int32_t* status) {
  const bool aligned = out_args(g[0]).bulk && (n == 1 || out_args(g[1]).bulk);
#define AS(PAIR, DT) \
  (aligned ? launch_tiles_as<FMT, PAIR, DT, true>(ctx, stream, g, n, f.bn, status) : launch_tiles_as<FMT, PAIR, DT, false>(ctx, stream, g, n, f.bn, status))
  if (g->dtype == FP4_DTYPE_BF16) return f.pair ? AS(true, FP4_DTYPE_BF16) : AS(false, FP4_DTYPE_BF16);
  if (g->dtype == FP4_DTYPE_FP16) return f.pair ? AS(true, FP4_DTYPE_FP16) : AS(false, FP4_DTYPE_FP16);
  return f.pair ? AS(true, FP4_DTYPE_FP32) : AS(false, FP4_DTYPE_FP32);
#undef AS
}

template <int FMT, class T = void>
int launch_few(fp4_ctx* ctx, cudaStream_t stream, const MxGemm& g, int splits, int32_t* status, const FewX* from = nullptr) {
  constexpr bool MAKE = !std::is_void_v<T>;
  CUtensorMap w, x = {}, sw, sx = {};
  FewArgs args = {};
  args.num_k_blocks = int((g.C + 255) / 256);
  args.nt = int((g.I + 15) / 16 * 16);
  const int tiles = int((g.J + BM - 1) / BM);
  args.splits = splits;
  const int per_cta = (args.num_k_blocks + args.splits - 1) / args.splits;
  args.stage_bytes = A_BYTES + (MAKE ? scale_bytes(FMT) : args.nt * 128 + 2 * scale_bytes(FMT));
  const int fixed = 1024 + FEW_MISC + (MAKE ? per_cta * few_x_bytes(FMT) : 0);
  // (more CTAs than SMs: two on each)
  args.stages = ((tiles * splits > ctx->num_sms ? 113 * 1024 : MOST_SMEM) - fixed) / args.stage_bytes;
  if (args.stages > FEW_MAX_STAGES) args.stages = FEW_MAX_STAGES;
  if (args.stages > per_cta) args.stages = per_cta;
  // (the parts of the result, 512 bytes a token, go over the ring)
  while (args.stages * args.stage_bytes < args.nt * BM * 4) ++args.stages;
  args.tx_bytes = uint32_t(args.stage_bytes);
  args.idesc = idesc_mx(FMT, BM, args.nt);
  args.tmem_cols = 256;
  args.out = out_args(g);
  args.powers = powers_of(g);
  args.status = status;
  args.wait_limit_ns = mx_wait_limit(ctx);
  args.skip_fill = ctx->debug_skip_fill;
  if (MAKE) args.x = *from;
  int rc = make_codes_map(ctx, &w, g.b, g.J, g.C, BM);
  if (rc == FP4_OK) rc = make_scales_map(ctx, &sw, g.b_scales, g.J, g.C, FMT, 1);
  if (rc == FP4_OK && !MAKE) rc = make_codes_map(ctx, &x, g.a, g.I, g.C, args.nt);
  if (rc == FP4_OK && !MAKE) rc = make_scales_map(ctx, &sx, g.a_scales, g.I, g.C, FMT, 1);
  if (rc != FP4_OK) return rc;
  constexpr auto kernel = mx_gemm_few_kernel<FMT, T>;
  FP4_CUDA_TRY(mx_allow_smem<kernel>(ctx->device, MOST_SMEM));
  // At least a third of an SM's shared memory: two CTAs an SM find their 256 columns of tensor memory, a third one would wait for
  // theirs, and CTAs of clusters that wait so for one another would wait for good.
  int smem = fixed + args.stages * args.stage_bytes;
  if (smem < FEW_LEAST_SMEM) smem = FEW_LEAST_SMEM;
  KernelScope scope(ctx, stream, KC_GEMM, 1);
  return mx_launch<kernel>(dim3(unsigned(tiles * args.splits)), args.nt <= 32 && !MAKE ? FEW_THREADS - 128 : FEW_THREADS, smem, args.splits, stream, w, x, sw, sx, args);
}

}  // namespace

int launch_mx_gemm(fp4_ctx* ctx, cudaStream_t stream, const MxGemm* g, int n, int32_t* status) {
  const bool nv = g->format == FP4_MX_NVFP4;
  // Two products in one launch: of one type, and neither with so few rows that it has a kernel of its own.  The one whose tiles take longer
  // comes first.
  if (n == 2) {
    bool apart = g[0].dtype != g[1].dtype;
    for (int i = 0; i < 2; ++i) apart = apart || (g[i].I <= FEW_ROWS && choose_few(ctx, g[i]).cost <= choose_form(ctx, g + i, 1).cost);
    if (apart) {
      const int rc = launch_mx_gemm(ctx, stream, g, 1, status);
      return rc != FP4_OK ? rc : launch_mx_gemm(ctx, stream, g + 1, 1, status);
    }
    const MxGemm in_order[2] = {g[g[1].C > g[0].C], g[g[1].C <= g[0].C]};
    const TileForm o = choose_form(ctx, in_order, 2);
    return nv ? launch_tiles<FP4_MX_NVFP4>(ctx, stream, in_order, 2, o, status) : launch_tiles<FP4_MX_E2M1>(ctx, stream, in_order, 2, o, status);
  }
  const TileForm f = choose_form(ctx, g, 1);
  if (g->I <= FEW_ROWS) {
    const FewForm few = choose_few(ctx, *g);
    if (few.cost <= f.cost) return nv ? launch_few<FP4_MX_NVFP4>(ctx, stream, *g, few.splits, status) : launch_few<FP4_MX_E2M1>(ctx, stream, *g, few.splits, status);
  }
  return nv ? launch_tiles<FP4_MX_NVFP4>(ctx, stream, g, 1, f, status) : launch_tiles<FP4_MX_E2M1>(ctx, stream, g, 1, f, status);
}

int launch_mx_linear_few(fp4_ctx* ctx, cudaStream_t stream, const MxQuantize& x, const MxGemm& g, int32_t* status, bool* done) {
  const bool nv = g.format == FP4_MX_NVFP4;
  const int elt = x.dtype == FP4_DTYPE_FP32 ? 4 : 2;
  *done = false;
  if (g.I > FEW_X_ROWS || x.q->codes_t) return FP4_OK;
  const FewForm few = choose_few(ctx, g);
  // A launch and its wait (1200 ns) against what every CTA does again (40 a part).  Tokens x contraction x weight rows, us back to back with the weights from
  // HBM, made by the kernel / by the quantiser: 1 x 4096 x 11008 8.8 / 9.1, 4 x 11008 x 4096 9.8 / 10.8 (44 parts), 6 x 4096 x 11008 9.7 / 10.1 (48), 8 x 4096 x 11008
  // 10.3 / 9.3 (64); beside tiles, which few tokens take where the contraction is short, 8 x 1024 x 1024 5.0 / 5.8 (16), 16 x 1024 x 512 6.0 / 5.7 (32).
  const int64_t per_cta = ((g.C + 255) / 256 + few.splits - 1) / few.splits, parts = g.I * per_cta;
  if (per_cta > FEW_X_BLOCKS || parts > FEW_X_PARTS || few.cost + 40 * parts > choose_form(ctx, &g, 1).cost + 1200) return FP4_OK;
  // Where every CTA has to look for the amax first: 1 x 13824 x 5120 12.8 / 15.1, 1 x 4096 x 4096 7.6 / 8.6, 1 x 4096 x 11008 10.8 / 10.4; two tokens of the last,
  // in a kernel that looked at more than one, 11.5 / 10.5.
  const bool find = nv && !(x.q->flags & FP4_MX_AMAX_GIVEN);
  if (find && g.I > 1) return FP4_OK;
  *done = true;
  const FewX from = {x.x.p, x.x.ld, g.C, x.q->codes, x.q->scales, reinterpret_cast<uint32_t*>(x.q->amax), find,
                     (reinterpret_cast<uintptr_t>(x.x.p) & 15) == 0 && (x.x.ld * elt) % 16 == 0};
#define FROM(T) \
  (nv ? launch_few<FP4_MX_NVFP4, T>(ctx, stream, g, few.splits, status, &from) : launch_few<FP4_MX_E2M1, T>(ctx, stream, g, few.splits, status, &from))
  if (x.dtype == FP4_DTYPE_BF16) return FROM(__nv_bfloat16);
  if (x.dtype == FP4_DTYPE_FP16) return FROM(__half);
  return FROM(float);
#undef FROM
}
