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
// memory in order of rank.
// Every wait is bounded: on a timeout a CTA raises FP4_DEV_TIMEOUT, drains its copies, frees its tensor memory and returns.
#include <cuda.h>
#include <cuda_fp16.h>

#include "mx.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int BM = 128;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int A_BYTES = BM * 128;                 // codes of a k-block of 128 rows
constexpr int TMEM_COLS = 512;
constexpr int BN_MAX = 192;                       // 2 x 192 accumulator columns leave room for the scales; a multiple of 64, so that
                                                  // a tile's columns begin at a half of a scale tile at least
constexpr int MAX_STAGES = 6;
constexpr int STAGE_OUT = 4096;                   // of an epilogue warp
constexpr int MISC_BYTES = 256;
constexpr int MOST_SMEM = 227 * 1024;

__host__ __device__ constexpr int scale_tiles(int fmt) { return fmt == FP4_MX_NVFP4 ? 4 : 2; }      // of a k-block
__host__ __device__ constexpr int scale_bytes(int fmt) { return scale_tiles(fmt) * 512; }           // of 128 rows
// Tensor memory: accumulators at 0 and BN_MAX, then two sets of scales (k-blocks alternate): A's, 4 columns a tile, and B's, 8.
__host__ __device__ constexpr int sf_cols(int fmt) { return scale_tiles(fmt) * 12; }

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
template <int DT>
__device__ __forceinline__ void put_one(void* out, int64_t at, float v, bool accumulate) {
  typename OutOf<DT>::type* p = static_cast<typename OutOf<DT>::type*>(out) + at;
  *p = OutOf<DT>::put(accumulate ? v + OutOf<DT>::get(*p) : v);
}
__device__ __forceinline__ void put_any(void* out, int64_t at, float v, bool accumulate, int dtype) {
  if (dtype == FP4_DTYPE_BF16) put_one<FP4_DTYPE_BF16>(out, at, v, accumulate);
  else if (dtype == FP4_DTYPE_FP16) put_one<FP4_DTYPE_FP16>(out, at, v, accumulate);
  else put_one<FP4_DTYPE_FP32>(out, at, v, accumulate);
}

struct OutArgs {
  void* p;
  int64_t ld;
  int I, J, dtype;
  bool accumulate;
  bool bulk;                   // rows on 16-byte boundaries and nothing to add to: bulk stores
};
// The tensors' powers of two (1 without them).
struct Powers {
  const uint32_t *a, *b;
};
__device__ __forceinline__ float2 tensor_scales(const Powers& p) {
  float2 s = make_float2(1.0f, 1.0f);
  if (p.a) {
    s.x = __uint_as_float(uint32_t(mx_tensor_exponent(__ldg(p.a)) + 127) << 23);
    s.y = __uint_as_float(uint32_t(mx_tensor_exponent(__ldg(p.b)) + 127) << 23);
  }
  return s;
}

// 32 rows x 32 columns (the last chunk: fewer) of a warp, row `lane` in y.
__device__ __forceinline__ void store_chunk(const float (&y)[32], uint8_t* stage, const OutArgs& o, const CUtensorMap* map, int row0,
                                            int col0, int lane, uint32_t& seq) {
  if (o.bulk) {
    // boxes of 32 rows x 64 bytes through two 2 KB buffers in turn; with the 64-byte swizzle 16-byte slot s of row r sits at
    // s ^ ((r >> 1) & 3), so the rows' writes touch every bank once
    const int fx = (lane >> 1) & 3;
    const int boxes = o.dtype == FP4_DTYPE_FP32 ? 2 : 1;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u >= boxes || (u && col0 + 16 >= o.J)) break;
      uint8_t* buf = stage + (seq & 1u) * 2048;
      ++seq;
      if (elect_one()) tma_store_wait_read_1();
      __syncwarp();
      uint8_t* my_row = buf + lane * 64;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint4 q;
        if (o.dtype == FP4_DTYPE_FP32) {
          const float* v = y + 16 * u + 4 * j;
          q = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        } else {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (o.dtype == FP4_DTYPE_BF16) {
              const __nv_bfloat162 h = __floats2bfloat162_rn(y[8 * j + 2 * i], y[8 * j + 2 * i + 1]);
              w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
              const __half2 h = __floats2half2_rn(y[8 * j + 2 * i], y[8 * j + 2 * i + 1]);
              w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
          }
          q = make_uint4(w[0], w[1], w[2], w[3]);
        }
        *reinterpret_cast<uint4*>(my_row + ((j ^ fx) * 16)) = q;
      }
      fence_async_smem();
      __syncwarp();
      if (elect_one()) tma_store_2d(map, buf, col0 + 16 * u, row0);
    }
  } else {
    // any alignment, or results to be added to what is there: through shared memory, so that a row's values lie in a row of lanes
    float* buf = reinterpret_cast<float*>(stage);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<float4*>(buf + lane * 32 + ((j ^ (lane & 7)) * 4)) = make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
    __syncwarp();
    const int rows = min(32, o.I - row0);
    if (col0 + lane < o.J)
      for (int r = 0; r < rows; ++r)
        put_any(o.p, int64_t(row0 + r) * o.ld + col0 + lane, buf[r * 32 + (((lane >> 2) ^ (r & 7)) * 4) + (lane & 3)], o.accumulate, o.dtype);
  }
}

struct GemmArgs {
  int num_k_blocks, num_m_blocks, num_n_blocks, bn;
  int b_tiles;                 // scale tiles of 128 rows that a tile's columns touch
  int stages, stage_bytes;
  uint32_t tx_bytes, idesc;
  OutArgs out;
  Powers powers;
  int32_t* status;
  uint64_t wait_limit_ns;
};
constexpr int FIXED_SMEM = 1024 + MISC_BYTES + EPI_WARPS * STAGE_OUT;

template <int FMT, bool PAIR>
__global__ void __launch_bounds__(THREADS, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
               const __grid_constant__ CUtensorMap map_out, const __grid_constant__ GemmArgs args) {
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
  const int num_tiles = args.num_m_blocks * args.num_n_blocks;
  const int rank = PAIR ? int(cluster_ctarank()) : 0;
  const int worker = int(blockIdx.x) / CTAS, workers = int(gridDim.x) / CTAS;

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
  if (warp == 1) tmem_alloc<CTAS>(tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();               // the peer's barriers exist
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer -------
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0, fills = 0;
      bool ok = true;
      const uint32_t full0 = PAIR ? cluster_address(full_bar, 0) : smem_u32(full_bar);
      for (int t = worker; t < num_tiles && ok; t += workers) {
        const int m_blk = CTAS * (t % args.num_m_blocks) + rank, n0 = (t / args.num_m_blocks) * args.bn;
        const int b_row = n0 + rank * (args.bn / CTAS);
        for (int kb = 0; kb < args.num_k_blocks; ++kb) {
          ok = mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, args.status, args.wait_limit_ns);
          if (!ok) break;
          uint8_t* p = smem + stage * STAGE_BYTES;
          const uint32_t bar = full0 + 8 * stage;
          if (rank == 0) mbar_arrive_expect_tx(&full_bar[stage], CTAS * args.tx_bytes);
          tma_load_2d_group<CTAS>(p, &map_a, bar, kb * 128, m_blk * BM);
          tma_load_2d_group<CTAS>(p + A_BYTES, &map_b, bar, kb * 128, b_row);
          tma_load_2d_group<CTAS>(p + A_BYTES + b_bytes, &map_sa, bar, kb * (scale_bytes(FMT) / 8), m_blk);
          tma_load_2d_group<CTAS>(p + A_BYTES + b_bytes + scale_bytes(FMT), &map_sb, bar, kb * (scale_bytes(FMT) / 8), n0 / 128);
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
      } else if (!ok) {
        const uint32_t last = fills < uint32_t(STAGES) ? fills : uint32_t(STAGES);
        for (uint32_t back = 1; back <= last; ++back) {
          const uint32_t f = fills - back;
          const uint64_t t0 = global_timer_ns();
          while (!mbar_try_wait(&full_bar[f % STAGES], (f / STAGES) & 1u)) {
            if (global_timer_ns() - t0 > 1000000ull) break;
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer ---------
    if (rank == 0 && elect_one()) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0, sf = 0;
      bool ok = true;
      for (int t = worker; t < num_tiles && ok; t += workers) {
        ok = mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag, args.status, args.wait_limit_ns);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + uint32_t(acc * BN_MAX);
        const int shift = (t / args.num_m_blocks) * args.bn % 128 ? 2 : 0;
        for (int kb = 0; kb < args.num_k_blocks; ++kb) {
          ok = mbar_wait(&full_bar[stage], phase, abort_flag, args.status, args.wait_limit_ns);
          if (!ok) break;
          tc_fence_after();
          const uint32_t p = smem_u32(smem + stage * STAGE_BYTES);
          issue_k_block<FMT, CTAS>(p, p + A_BYTES, p + A_BYTES + b_bytes, p + A_BYTES + b_bytes + scale_bytes(FMT), args.b_tiles, d_tmem,
                                   tmem_base + 2 * BN_MAX + sf * sf_cols(FMT), shift, args.idesc, kb == 0);
          sf ^= 1u;
          tc_commit_all<CTAS>(&empty_bar[stage]);
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        tc_commit_all<CTAS>(&acc_full[acc]);
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
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
    const float2 scales = tensor_scales(args.powers);
    for (int t = worker; t < num_tiles; t += workers) {
      const int m_blk = CTAS * (t % args.num_m_blocks) + rank, n0 = (t / args.num_m_blocks) * args.bn;
      const bool ok = mbar_wait(&acc_full[acc], acc_phase, abort_flag, args.status, args.wait_limit_ns);
      if (epilogue_bar_any(!ok, 32 * EPI_WARPS)) break;
      tc_fence_after();
      const uint32_t t_base = tmem_base + (uint32_t(quarter * 32) << 16) + uint32_t(acc * BN_MAX);
      const int row0 = m_blk * BM + quarter * 32, n_valid = min(args.bn, args.out.J - n0);
      if (row0 < args.out.I)
        for (int c = 32 * group; c < n_valid; c += 64) {
          uint32_t v[32];
          tmem_ld_32x32(t_base + uint32_t(c), v);
          tmem_ld_wait(v);
          float y[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) y[i] = __uint_as_float(v[i]) * scales.x * scales.y;
          store_chunk(y, stage, args.out, &map_out, row0, n0 + c, lane, seq);
        }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) mbar_arrive_cluster(acc_empty0 + 8 * acc); else mbar_arrive(&acc_empty[acc]);
      }
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
constexpr int FEW_THREADS = 64 + 128;
constexpr int FEW_MAX_STAGES = 8;
struct FewArgs {
  int num_k_blocks, nt, splits;
  int stages, stage_bytes;
  uint32_t tx_bytes, idesc, tmem_cols;
  OutArgs out;                 // I tokens x J weight rows
  Powers powers;
  int32_t* status;
  uint64_t wait_limit_ns;
};
__device__ __forceinline__ float load_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
template <int FMT>
__global__ void __launch_bounds__(FEW_THREADS)
mx_gemm_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                   const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_sx,
                   const __grid_constant__ FewArgs args) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int STAGES = args.stages, STAGE_BYTES = args.stage_bytes, x_bytes = args.nt * 128;
  uint8_t* misc = smem + STAGES * STAGE_BYTES;
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(misc);
  uint64_t* empty_bar = full_bar + FEW_MAX_STAGES;
  uint64_t* final_bar = empty_bar + FEW_MAX_STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(final_bar + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
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
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 1) tmem_alloc<1>(tmem_slot, args.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0, fills = 0;
      bool ok = true;
      for (int kb = rank; kb < args.num_k_blocks; kb += args.splits) {
        ok = mbar_wait(&empty_bar[stage], phase ^ 1u, abort_flag, args.status, args.wait_limit_ns);
        if (!ok) break;
        uint8_t* p = smem + stage * STAGE_BYTES;
        mbar_arrive_expect_tx(&full_bar[stage], args.tx_bytes);
        tma_load_2d(p, &map_w, &full_bar[stage], kb * 128, j_blk * BM);
        tma_load_2d(p + A_BYTES + x_bytes, &map_sw, &full_bar[stage], kb * (scale_bytes(FMT) / 8), j_blk);
        tma_load_2d(p + A_BYTES, &map_x, &full_bar[stage], kb * 128, 0);
        tma_load_2d(p + A_BYTES + x_bytes + scale_bytes(FMT), &map_sx, &full_bar[stage], kb * (scale_bytes(FMT) / 8), 0);
        ++fills;
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
      if (!ok) {
        const uint32_t last = fills < uint32_t(STAGES) ? fills : uint32_t(STAGES);
        for (uint32_t back = 1; back <= last; ++back) {
          const uint32_t f = fills - back;
          const uint64_t t0 = global_timer_ns();
          while (!mbar_try_wait(&full_bar[f % STAGES], (f / STAGES) & 1u)) {
            if (global_timer_ns() - t0 > 1000000ull) break;
          }
        }
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0, sf = 0;
      bool ok = true;
      for (int kb = rank; kb < args.num_k_blocks; kb += args.splits) {
        ok = mbar_wait(&full_bar[stage], phase, abort_flag, args.status, args.wait_limit_ns);
        if (!ok) break;
        tc_fence_after();
        const uint32_t p = smem_u32(smem + stage * STAGE_BYTES);
        issue_k_block<FMT, 1>(p, p + A_BYTES, p + A_BYTES + x_bytes, p + A_BYTES + x_bytes + scale_bytes(FMT), 1, tmem_base,
                              tmem_base + FEW_ROWS + sf * sf_cols(FMT), 0, args.idesc, kb == rank);
        sf ^= 1u;
        tc_commit<1>(&empty_bar[stage]);
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
      tc_commit<1>(final_bar);
    }
    __syncwarp();
  }
  // Every thread awaits the last MMA (of a CTA without a k-block: at once).
  const bool done = __all_sync(0xFFFFFFFFu, mbar_wait(final_bar, 0, abort_flag, args.status, args.wait_limit_ns));
  tc_fence_after();
  // The accumulators go to shared memory, token by token, over the first stages: their copies have landed and been read.
  float* part = reinterpret_cast<float*>(smem);
  if (done && warp >= 2) {
    const int quarter = warp & 3;
    const bool any = rank < args.num_k_blocks;             // a CTA without a k-block adds nothing
    for (int c = 0; c < args.nt; c += 16) {
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
  const float2 scales = tensor_scales(args.powers);
  for (int e = rank * FEW_THREADS + int(threadIdx.x); e < args.out.I * BM; e += args.splits * FEW_THREADS) {
    const int token = e / BM, j = j_blk * BM + e % BM;
    float sum = 0.0f;
    if (args.splits > 1)
      for (int s = 0; s < args.splits; ++s) sum += load_cluster(cluster_address(part + e, uint32_t(s)));
    else
      sum = part[e];
    if (j < args.out.J) put_any(args.out.p, int64_t(token) * args.out.ld + j, sum * scales.x * scales.y, args.out.accumulate, args.out.dtype);
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
  o.bulk = !g.accumulate && (reinterpret_cast<uintptr_t>(g.out) & 15) == 0 && (g.ld * elt) % 16 == 0 && (g.J * elt) % 16 == 0;
  return o;
}
Powers powers_of(const MxGemm& g) {
  if (g.format != FP4_MX_NVFP4) return {nullptr, nullptr};
  return {reinterpret_cast<const uint32_t*>(g.a_amax), reinterpret_cast<const uint32_t*>(g.b_amax)};
}
uint64_t wait_limit(const fp4_ctx* ctx) { return ctx->debug_wait_limit_ns ? ctx->debug_wait_limit_ns : WAIT_LIMIT_NS; }

struct TileForm {
  int bn;
  bool pair;
};
// The form whose busiest worker ends first: tiles of a worker x (what a tile costs beside its k-blocks + k-blocks x time of one).
TileForm choose_form(const fp4_ctx* ctx, const MxGemm& g) {
  const int64_t kbs = (g.C + 255) / 256;
  TileForm best = {64, false};
  int64_t best_cost = -1;
  for (const bool pair : {false, true})
    for (const int bn : {64, 128, 192}) {
      if (pair && (bn == 64 || ctx->num_sms < 2)) continue;
      const int64_t rows = pair ? 2 * BM : BM, workers = pair ? ctx->num_sms / 2 : ctx->num_sms;
      const int64_t tiles = (g.I + rows - 1) / rows * ((g.J + bn - 1) / bn), rounds = (tiles + workers - 1) / workers;
      const int64_t mma = pair ? 1300 + kbs * (105 + (83 * bn) / 100) : 800 + kbs * (170 + (17 * bn) / 20), epi = 10 * bn + (pair ? 900 : 0);
      const int64_t cost = rounds * (mma > epi ? mma : epi) + (mma > epi ? epi : mma) + (pair ? 1000 : 0);
      if (best_cost < 0 || cost < best_cost) {
        best_cost = cost;
        best = {bn, pair};
      }
    }
  return best;
}

template <int FMT, bool PAIR>
int launch_tiles(fp4_ctx* ctx, cudaStream_t stream, const MxGemm& g, int bn, int32_t* status) {
  constexpr int CTAS = PAIR ? 2 : 1;
  CUtensorMap a, b, sa, sb, out = {};
  GemmArgs args = {};
  args.num_k_blocks = int((g.C + 255) / 256);
  args.num_m_blocks = int((g.I + CTAS * BM - 1) / (CTAS * BM));
  args.bn = bn;
  args.num_n_blocks = int((g.J + bn - 1) / bn);
  args.b_tiles = (bn + 127) / 128;
  args.stage_bytes = A_BYTES + bn * 128 / CTAS + scale_bytes(FMT) * (1 + args.b_tiles);
  args.tx_bytes = uint32_t(args.stage_bytes);
  args.stages = (MOST_SMEM - FIXED_SMEM) / args.stage_bytes;
  if (args.stages > MAX_STAGES) args.stages = MAX_STAGES;
  args.idesc = idesc_mx(FMT, CTAS * BM, bn);
  args.out = out_args(g);
  args.powers = powers_of(g);
  args.status = status;
  args.wait_limit_ns = wait_limit(ctx);
  int rc = make_codes_map(ctx, &a, g.a, g.I, g.C, BM);
  if (rc == FP4_OK) rc = make_codes_map(ctx, &b, g.b, g.J, g.C, bn / CTAS);
  if (rc == FP4_OK) rc = make_scales_map(ctx, &sa, g.a_scales, g.I, g.C, FMT, 1);
  if (rc == FP4_OK) rc = make_scales_map(ctx, &sb, g.b_scales, g.J, g.C, FMT, args.b_tiles);
  if (rc == FP4_OK && args.out.bulk) {
    const CUtensorMapDataType type = g.dtype == FP4_DTYPE_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : g.dtype == FP4_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const uint32_t elt = g.dtype == FP4_DTYPE_FP32 ? 4 : 2;
    rc = make_map(ctx, &out, type, g.out, uint64_t(g.J), uint64_t(g.I), uint64_t(g.ld) * elt, 64 / elt, 32, CU_TENSOR_MAP_SWIZZLE_64B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE);
  }
  if (rc != FP4_OK) return rc;
  const auto kernel = mx_gemm_kernel<FMT, PAIR>;
  FP4_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST_SMEM));
  const int64_t tiles = int64_t(args.num_m_blocks) * args.num_n_blocks, most = ctx->num_sms / CTAS;
  cudaLaunchAttribute cluster = {};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = 2;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(CTAS * (tiles < most ? tiles : most)));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = size_t(FIXED_SMEM + args.stages * args.stage_bytes);
  cfg.stream = stream;
  cfg.attrs = &cluster;
  cfg.numAttrs = PAIR ? 1 : 0;
  KernelScope scope(ctx, stream, KC_GEMM, 1);
  FP4_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, b, sa, sb, out, args));
  return FP4_OK;
}

template <int FMT>
int launch_few(fp4_ctx* ctx, cudaStream_t stream, const MxGemm& g, int32_t* status) {
  CUtensorMap w, x, sw, sx;
  FewArgs args = {};
  args.num_k_blocks = int((g.C + 255) / 256);
  args.nt = int((g.I + 15) / 16 * 16);
  const int tiles = int((g.J + BM - 1) / BM);
  // as many parts of the contraction as fill the SMs once, at most a portable cluster
  args.splits = ctx->num_sms / tiles;
  if (args.splits > args.num_k_blocks) args.splits = args.num_k_blocks;
  args.splits = args.splits < 1 ? 1 : (args.splits > 8 ? 8 : args.splits);
  args.stage_bytes = A_BYTES + args.nt * 128 + 2 * scale_bytes(FMT);
  args.stages = (MOST_SMEM - 1024 - MISC_BYTES) / args.stage_bytes;
  if (args.stages > FEW_MAX_STAGES) args.stages = FEW_MAX_STAGES;
  const int per_cta = (args.num_k_blocks + args.splits - 1) / args.splits;
  if (args.stages > per_cta) args.stages = per_cta;
  // (the parts of the result, 512 bytes a token, go over the ring)
  while (args.stages * args.stage_bytes < args.nt * BM * 4) ++args.stages;
  args.tx_bytes = uint32_t(args.stage_bytes);
  args.idesc = idesc_mx(FMT, BM, args.nt);
  args.tmem_cols = 256;
  args.out = out_args(g);
  args.powers = powers_of(g);
  args.status = status;
  args.wait_limit_ns = wait_limit(ctx);
  int rc = make_codes_map(ctx, &w, g.b, g.J, g.C, BM);
  if (rc == FP4_OK) rc = make_codes_map(ctx, &x, g.a, g.I, g.C, args.nt);
  if (rc == FP4_OK) rc = make_scales_map(ctx, &sw, g.b_scales, g.J, g.C, FMT, 1);
  if (rc == FP4_OK) rc = make_scales_map(ctx, &sx, g.a_scales, g.I, g.C, FMT, 1);
  if (rc != FP4_OK) return rc;
  const auto kernel = mx_gemm_few_kernel<FMT>;
  FP4_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST_SMEM));
  cudaLaunchAttribute cluster = {};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = unsigned(args.splits);
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tiles * args.splits));
  cfg.blockDim = dim3(FEW_THREADS);
  cfg.dynamicSmemBytes = size_t(1024 + MISC_BYTES + args.stages * args.stage_bytes);
  cfg.stream = stream;
  cfg.attrs = &cluster;
  cfg.numAttrs = args.splits > 1 ? 1 : 0;
  KernelScope scope(ctx, stream, KC_GEMM, 1);
  FP4_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, w, x, sw, sx, args));
  return FP4_OK;
}

}  // namespace

int launch_mx_gemm(fp4_ctx* ctx, cudaStream_t stream, const MxGemm& g, int32_t* status) {
  const bool nv = g.format == FP4_MX_NVFP4;
  if (g.I <= FEW_ROWS) return nv ? launch_few<FP4_MX_NVFP4>(ctx, stream, g, status) : launch_few<FP4_MX_E2M1>(ctx, stream, g, status);
  const TileForm f = choose_form(ctx, g);
  if (f.pair) return nv ? launch_tiles<FP4_MX_NVFP4, true>(ctx, stream, g, f.bn, status) : launch_tiles<FP4_MX_E2M1, true>(ctx, stream, g, f.bn, status);
  return nv ? launch_tiles<FP4_MX_NVFP4, false>(ctx, stream, g, f.bn, status) : launch_tiles<FP4_MX_E2M1, false>(ctx, stream, g, f.bn, status);
}
