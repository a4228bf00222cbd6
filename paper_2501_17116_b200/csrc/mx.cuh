// Block-scaled ("microscaled") operands: layout, scale arithmetic and internal launchers (the public ABI is
// include/fp4_linear.h).  Internal.
//
// An operand of `rows` vectors of `cols` elements, scaled in blocks along `cols`:
//   codes   [rows x pitch], pitch = ceil(cols / 128) * 64 bytes of E2M1 nibbles (even element low) or * 128 of
//           E4M3 bytes; what lies behind `cols` is zero
//   scales  one byte per block, in tiles of 128 rows x 4 blocks (512 bytes): row r, block b at
//             tile (r / 128) * T + b / 4, byte (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4,
//           T = ceil(cols / 128) (E2M1 in blocks of 16: twice that).  It is the order in which tcgen05.cp
//           (32x128b.warpx4) hands the scales of 128 rows to tensor memory: four columns, four lane quarters alike.
//           Bytes that stand for no block are zero.
#pragma once

#include <atomic>

#include "common.cuh"
#include "tc_ptx.cuh"

constexpr int MX_TILE = 128;

__host__ __device__ constexpr bool mx_known(int format) { return format >= FP4_MX_E2M1 && format <= FP4_MX_E4M3; }
__host__ __device__ constexpr int mx_block(int format) { return format == FP4_MX_NVFP4 ? 16 : 32; }
__host__ __device__ constexpr int64_t mx_tiles(int64_t n) { return (n + MX_TILE - 1) / MX_TILE; }
__host__ __device__ constexpr int64_t mx_pitch(int64_t cols, int format) {
  return mx_tiles(cols) * (format == FP4_MX_E4M3 ? 128 : 64);
}
__host__ __device__ constexpr int64_t mx_scale_tiles(int64_t cols, int format) {
  return mx_tiles(cols) * (format == FP4_MX_NVFP4 ? 2 : 1);
}
__host__ __device__ constexpr int64_t mx_scale_bytes(int64_t rows, int64_t cols, int format) {
  return mx_tiles(rows) * mx_scale_tiles(cols, format) * 512;
}

// Scale of an NVFP4 tensor: the least 2^k, k >= -100, with amax <= 6 * 448 * 2^k (2688 = 1.3125 * 2^11; the sum carries into
// the exponent where the mantissa is larger).  A power of two, so that dividing by it is exact: whether a value of a 16-bit
// type lies on a tie of its format is then decided without a rounding.
__host__ __device__ inline int mx_tensor_exponent(uint32_t amax_bits) {
  const int k = int(((amax_bits & 0x7FFFFFFFu) + (0x7FFFFFu - 0x280000u)) >> 23) - 127 - 11;
  return k < -100 ? -100 : k;
}

inline uint64_t mx_wait_limit(const fp4_ctx* ctx) { return ctx->debug_wait_limit_ns ? ctx->debug_wait_limit_ns : WAIT_LIMIT_NS; }

// More than 48 KB of shared memory for a kernel: asked for once per kernel and device (the call takes half a microsecond).
template <auto KERNEL>
cudaError_t mx_allow_smem(int device, int bytes) {
  static std::atomic<uint64_t> done{0};
  const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// The kernels are launched so that one may start while the one before it on the stream drains (programmatic dependent launch): it sets
// itself up and waits here, ahead of its first access to global memory, until everything before it is complete and visible.  Global memory is read by
// ordinary loads alone: non-coherent ones (ld.global's read-only form) promise that nothing changes while the kernel runs, and need not stay behind the wait.
__device__ __forceinline__ void mx_wait_for_inputs() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Behind that, when the block holds all that it needs of its SM (tensor memory!): the next kernel's blocks may come, and must not get hold of
// what a block that they wait for is still to be given.
__device__ __forceinline__ void mx_let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// `cluster` CTAs a cluster.
template <auto KERNEL, class... A>
int mx_launch(dim3 grid, int threads, int smem, int cluster, cudaStream_t stream, const A&... args) {
  cudaLaunchAttribute attrs[2] = {};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = unsigned(cluster);
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = size_t(smem);
  cfg.stream = stream;
  cfg.attrs = attrs;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  FP4_CUDA_TRY(cudaLaunchKernelEx(&cfg, KERNEL, args...));
  return FP4_OK;
}

struct MxMatrix {               // a matrix of the caller's: rows of `ld` elements
  const void* p;
  int64_t ld;
};

// One tensor or two, neither empty.
struct MxQuantize {
  MxMatrix x;
  int dtype;
  const fp4_mx_tensor* q;
};
int launch_mx_quantize(fp4_ctx* ctx, cudaStream_t stream, const MxQuantize* what, int n, int32_t* status);
int launch_mx_dequantize(fp4_ctx* ctx, cudaStream_t stream, const uint8_t* codes, const uint8_t* scales, const float* amax,
                         int64_t rows, int64_t cols, int format, MxMatrix out, int dtype, int32_t* status);
// `h` may have no pointer; `q` (may be null): E2M1 in blocks of 32.
int launch_mx_swiglu_fwd(fp4_ctx* ctx, cudaStream_t stream, MxMatrix gate, MxMatrix up, int64_t rows, int64_t cols, int dtype,
                         MxMatrix h, const fp4_mx_tensor* ckpt_gate, const fp4_mx_tensor* ckpt_up, const fp4_mx_tensor* q,
                         int32_t* status);
int launch_mx_swiglu_bwd(fp4_ctx* ctx, cudaStream_t stream, MxMatrix dh, const fp4_mx_tensor& gate, const fp4_mx_tensor& up,
                         int64_t rows, int64_t cols, int dtype, MxMatrix dgate, MxMatrix dup, MxMatrix h,
                         const fp4_mx_tensor* q, int32_t* status);

// out[i, j] (+)= g_a g_b sum_c a[i, c] b[j, c]
struct MxGemm {
  const uint8_t *a, *a_scales, *b, *b_scales;
  const float *a_amax, *b_amax;      // NVFP4: the operands' amax
  int64_t I, J, C;
  int format;
  void* out;
  int64_t ld;
  int dtype;
  bool accumulate;
};
// One product or two that do not depend on one another, none of them empty.
int launch_mx_gemm(fp4_ctx* ctx, cudaStream_t stream, const MxGemm* g, int n, int32_t* status);
// The product of few rows with an operand that is there, a's codes (one direction, and its amax) being made from `x` by the kernel itself.
// `done`: false where that is not the faster way (nothing was launched).
int launch_mx_linear_few(fp4_ctx* ctx, cudaStream_t stream, const MxQuantize& x, const MxGemm& g, int32_t* status, bool* done);
