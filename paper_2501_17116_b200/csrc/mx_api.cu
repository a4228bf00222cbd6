// C ABI of the block-scaled operands (fp4_mx_*): argument validation and kernel sequencing.
#include "mx.cuh"

namespace {

constexpr int64_t MOST = 0x7FFFFFFF;

// The calls work on the context's device; the caller's stays current.
struct OnDevice {
  int before = -1;
  bool ok;
  explicit OnDevice(const fp4_ctx* ctx) {
    ok = cudaGetDevice(&before) == cudaSuccess;
    if (ok && before != ctx->device) ok = cudaSetDevice(ctx->device) == cudaSuccess;
    else before = -1;
  }
  ~OnDevice() {
    if (before >= 0) cudaSetDevice(before);
  }
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool wanted(const fp4_mx_matrix* m) { return m && m->data; }

int check_sizes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > MOST || cols > MOST) return FP4_ERR_RANGE;
  return mx_tiles(rows) * mx_tiles(cols) > MOST ? FP4_ERR_RANGE : FP4_OK;
}
int check_matrix(const fp4_mx_matrix* m, int64_t rows, int64_t cols) {
  if (m->dtype < FP4_DTYPE_BF16 || m->dtype > FP4_DTYPE_FP32 || m->reserved) return FP4_ERR_ARG;
  if (rows > 1 && (m->ld < cols || m->ld > (int64_t(1) << 36))) return FP4_ERR_RANGE;
  if (reinterpret_cast<uintptr_t>(m->data) % (m->dtype == FP4_DTYPE_FP32 ? 4 : 2)) return FP4_ERR_ALIGN;
  return FP4_OK;
}
// (the stride of a single row means nothing, but decides how its neighbours would be aligned)
MxMatrix matrix(const fp4_mx_matrix* m, int64_t rows, int64_t cols) {
  if (!wanted(m)) return {nullptr, 0};
  return {m->data, rows > 1 ? m->ld : (cols + 7) / 8 * 8};
}
int check_side(const uint8_t* codes, const uint8_t* scales) {
  if (!codes || !scales) return FP4_ERR_NULL;
  return aligned16(codes) && aligned16(scales) ? FP4_OK : FP4_ERR_ALIGN;
}
// A tensor that is written or read: each direction it has is complete, one at least is there.
int check_tensor(const fp4_mx_tensor* q, bool e2m1_only) {
  if (!mx_known(q->format) || (e2m1_only && q->format == FP4_MX_E4M3)) return FP4_ERR_ARG;
  if (q->flags & ~FP4_MX_AMAX_GIVEN) return FP4_ERR_ARG;
  if (q->format == FP4_MX_NVFP4 && !q->amax) return FP4_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(q->amax) % 4) return FP4_ERR_ALIGN;
  if (!q->codes && !q->codes_t) return FP4_ERR_NULL;
  int rc = FP4_OK;
  if (q->codes || q->scales) rc = check_side(q->codes, q->scales);
  if (rc == FP4_OK && (q->codes_t || q->scales_t)) rc = check_side(q->codes_t, q->scales_t);
  return rc;
}

// Up to two tensors; what is empty takes no launch.
struct Quantize {
  const fp4_mx_matrix* x;
  const fp4_mx_tensor* q;
};
int quantize(fp4_ctx* ctx, cudaStream_t st, const Quantize* what, int n, int32_t* status) {
  MxQuantize todo[2];
  int some = 0;
  for (int i = 0; i < n; ++i) {
    const fp4_mx_tensor& q = *what[i].q;
    if (q.rows == 0 || q.cols == 0) {
      if (q.format == FP4_MX_NVFP4 && !(q.flags & FP4_MX_AMAX_GIVEN)) FP4_CUDA_TRY(cudaMemsetAsync(q.amax, 0, sizeof(float), st));
    } else {
      todo[some++] = {matrix(what[i].x, q.rows, q.cols), what[i].x->dtype, &q};
    }
  }
  return some ? launch_mx_quantize(ctx, st, todo, some, status) : FP4_OK;
}

// `rows` rows of `width` bytes; those further apart than a two-dimensional memset reaches (few, then) one by one.
int clear(cudaStream_t st, char* p, int64_t pitch, int64_t width, int64_t rows) {
  if (pitch <= MOST) {
    FP4_CUDA_TRY(cudaMemset2DAsync(p, size_t(pitch), 0, size_t(width), size_t(rows), st));
    return FP4_OK;
  }
  for (int64_t r = 0; r < rows; ++r) FP4_CUDA_TRY(cudaMemsetAsync(p + r * pitch, 0, size_t(width), st));
  return FP4_OK;
}

// a b^T over I x J results and a contraction of C, up to two.
struct Gemm {
  const fp4_mx_tensor* a;
  bool a_t;
  const fp4_mx_tensor* b;
  bool b_t;
  int64_t I, J, C;
  const fp4_mx_matrix* out;
  bool accumulate;
};
MxGemm mx_gemm(const Gemm& g) {
  return {g.a_t ? g.a->codes_t : g.a->codes, g.a_t ? g.a->scales_t : g.a->scales, g.b_t ? g.b->codes_t : g.b->codes,
          g.b_t ? g.b->scales_t : g.b->scales, g.a->amax, g.b->amax, g.I, g.J, g.C, g.a->format, g.out->data, matrix(g.out, g.I, g.J).ld,
          g.out->dtype, g.accumulate};
}
int gemm(fp4_ctx* ctx, cudaStream_t st, const Gemm* what, int n, int32_t* status) {
  MxGemm todo[2];
  int some = 0;
  for (int i = 0; i < n; ++i) {
    const Gemm& g = what[i];
    if (g.I == 0 || g.J == 0) continue;
    const MxMatrix o = matrix(g.out, g.I, g.J);
    const int64_t elt = g.out->dtype == FP4_DTYPE_FP32 ? 4 : 2;
    if (g.C == 0) {
      if (!g.accumulate) {
        const int rc = clear(st, static_cast<char*>(g.out->data), o.ld * elt, g.J * elt, g.I);
        if (rc != FP4_OK) return rc;
      }
      continue;
    }
    todo[some++] = mx_gemm(g);
  }
  return some ? launch_mx_gemm(ctx, st, todo, some, status) : FP4_OK;
}

int check_swiglu_quantized(const fp4_mx_tensor* q) {
  if (!q) return FP4_OK;
  const int rc = check_tensor(q, true);
  return rc != FP4_OK ? rc : (q->format == FP4_MX_E2M1 ? FP4_OK : FP4_ERR_ARG);
}
int check_checkpoint(const fp4_mx_tensor* q) {
  if (q->format != FP4_MX_E4M3) return FP4_ERR_ARG;
  return check_side(q->codes, q->scales);
}

}  // namespace

extern "C" {

int64_t fp4_mx_pitch(int64_t cols, int format) {
  if (cols < 0 || cols > MOST || !mx_known(format)) return -1;
  return mx_pitch(cols, format);
}
int64_t fp4_mx_scale_bytes(int64_t rows, int64_t cols, int format) {
  if (check_sizes(rows, cols) != FP4_OK || !mx_known(format)) return -1;
  return mx_scale_bytes(rows, cols, format);
}

size_t fp4_mx_workspace_bytes(int64_t M, int64_t K, int64_t N) {
  if (check_sizes(M, N) != FP4_OK || check_sizes(M, K) != FP4_OK || check_sizes(K, N) != FP4_OK) return 0;
  // dY in both directions (the scales of blocks of 16 are the larger ones), each buffer and the amax in a block of its own
  const size_t along = size_t(M * mx_pitch(N, FP4_MX_NVFP4) + mx_scale_bytes(M, N, FP4_MX_NVFP4));
  const size_t across = size_t(N * mx_pitch(M, FP4_MX_NVFP4) + mx_scale_bytes(N, M, FP4_MX_NVFP4));
  return along + across + 5 * 256;
}

int fp4_mx_quantize(fp4_ctx* ctx, void* stream, const fp4_mx_matrix* x, fp4_mx_tensor* out, int32_t* status) {
  if (!ctx || !x || !out || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  int rc = check_sizes(out->rows, out->cols);
  if (rc == FP4_OK && !x->data && out->rows && out->cols) rc = FP4_ERR_NULL;
  if (rc == FP4_OK) rc = check_matrix(x, out->rows, out->cols);
  if (rc == FP4_OK) rc = check_tensor(out, false);
  if (rc != FP4_OK) return rc;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  const Quantize one = {x, out};
  return quantize(ctx, static_cast<cudaStream_t>(stream), &one, 1, status);
}

int fp4_mx_dequantize(fp4_ctx* ctx, void* stream, const fp4_mx_tensor* q, int transposed, const fp4_mx_matrix* out, int32_t* status) {
  if (!ctx || !q || !out || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  const int64_t rows = transposed ? q->cols : q->rows, cols = transposed ? q->rows : q->cols;
  int rc = check_sizes(rows, cols);
  if (rc == FP4_OK) rc = check_tensor(q, false);
  if (rc == FP4_OK && (!(transposed ? q->codes_t : q->codes) || (!out->data && rows && cols))) rc = FP4_ERR_NULL;
  if (rc == FP4_OK) rc = check_matrix(out, rows, cols);
  if (rc != FP4_OK || rows == 0 || cols == 0) return rc;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  const MxMatrix o = matrix(out, rows, cols);
  return launch_mx_dequantize(ctx, static_cast<cudaStream_t>(stream), transposed ? q->codes_t : q->codes,
                              transposed ? q->scales_t : q->scales, q->amax, rows, cols, q->format, o, out->dtype, status);
}

int fp4_mx_gemm(fp4_ctx* ctx, void* stream, const fp4_mx_tensor* a, const fp4_mx_tensor* b, int flags,
                const fp4_mx_matrix* out, int32_t* status) {
  if (!ctx || !a || !b || !out || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  if (flags & ~(FP4_MX_A_T | FP4_MX_B_T | FP4_MX_ACCUMULATE)) return FP4_ERR_ARG;
  const bool a_t = flags & FP4_MX_A_T, b_t = flags & FP4_MX_B_T;
  int rc = check_tensor(a, true);
  if (rc == FP4_OK) rc = check_tensor(b, true);
  if (rc != FP4_OK) return rc;
  if (!(a_t ? a->codes_t : a->codes) || !(b_t ? b->codes_t : b->codes)) return FP4_ERR_NULL;
  const int64_t I = a_t ? a->cols : a->rows, C = a_t ? a->rows : a->cols, J = b_t ? b->cols : b->rows;
  if (a->format != b->format) return FP4_ERR_ARG;
  if (C != (b_t ? b->rows : b->cols)) return FP4_ERR_RANGE;
  rc = check_sizes(I, C);
  if (rc == FP4_OK) rc = check_sizes(J, C);
  if (rc == FP4_OK) rc = check_sizes(I, 2 * J);          // (tiles may be 64 columns wide)
  if (rc == FP4_OK && !out->data && I && J) rc = FP4_ERR_NULL;
  if (rc == FP4_OK) rc = check_matrix(out, I, J);
  if (rc != FP4_OK) return rc;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  const Gemm one = {a, a_t, b, b_t, I, J, C, out, bool(flags & FP4_MX_ACCUMULATE)};
  return gemm(ctx, static_cast<cudaStream_t>(stream), &one, 1, status);
}

int fp4_mx_linear_fwd(fp4_ctx* ctx, void* stream, const fp4_mx_matrix* x, const fp4_mx_matrix* w, int64_t M, int64_t K, int64_t N,
                      int reuse, const fp4_mx_matrix* y, fp4_mx_tensor* saved_x, fp4_mx_tensor* saved_w, int32_t* status) {
  if (!ctx || !y || !saved_x || !saved_w || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  if (reuse & ~(FP4_REUSE_X | FP4_REUSE_W)) return FP4_ERR_ARG;
  const bool reuse_x = reuse & FP4_REUSE_X, reuse_w = reuse & FP4_REUSE_W;
  int rc = check_sizes(M, K);
  if (rc == FP4_OK) rc = check_sizes(K, N);
  if (rc == FP4_OK) rc = check_sizes(M, 2 * N);
  if (rc == FP4_OK) rc = check_tensor(saved_x, true);
  if (rc == FP4_OK) rc = check_tensor(saved_w, true);
  if (rc != FP4_OK) return rc;
  if (!saved_x->codes || !saved_w->codes_t) return FP4_ERR_NULL;
  if ((!reuse_x && (!x || (!x->data && M && K))) || (!reuse_w && (!w || (!w->data && K && N))) || (!y->data && M && N)) return FP4_ERR_NULL;
  if (saved_x->format != saved_w->format) return FP4_ERR_ARG;
  // (one tensor, or one amax, for both: only where neither is written)
  if ((saved_x == saved_w || (saved_x->format == FP4_MX_NVFP4 && saved_x->amax == saved_w->amax)) && !(reuse_x && reuse_w)) return FP4_ERR_ARG;
  if ((reuse_x && (saved_x->rows != M || saved_x->cols != K)) || (reuse_w && (saved_w->rows != K || saved_w->cols != N))) return FP4_ERR_RANGE;
  if (!reuse_x) rc = check_matrix(x, M, K);
  if (rc == FP4_OK && !reuse_w) rc = check_matrix(w, K, N);
  if (rc == FP4_OK) rc = check_matrix(y, M, N);
  if (rc != FP4_OK) return rc;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  Quantize todo[2];
  int n = 0;
  if (!reuse_w) {
    saved_w->rows = K;
    saved_w->cols = N;
    todo[n++] = {w, saved_w};
  }
  if (!reuse_x) {
    saved_x->rows = M;
    saved_x->cols = K;
    todo[n++] = {x, saved_x};
  }
  const Gemm one = {saved_x, false, saved_w, true, M, N, K, y, false};
  if (reuse_w && !reuse_x && M && N && K) {
    bool done;
    rc = launch_mx_linear_few(ctx, st, {matrix(x, M, K), x->dtype, saved_x}, mx_gemm(one), status, &done);
    if (rc != FP4_OK || done) return rc;
  }
  if (n) rc = quantize(ctx, st, todo, n, status);
  if (rc != FP4_OK) return rc;
  return gemm(ctx, st, &one, 1, status);
}

int fp4_mx_linear_bwd(fp4_ctx* ctx, void* stream, const fp4_mx_matrix* dy, const fp4_mx_tensor* saved_x, const fp4_mx_tensor* saved_w,
                      int64_t M, int64_t K, int64_t N, int flags, const fp4_mx_matrix* dx, const fp4_mx_matrix* dw, int32_t* status) {
  if (!ctx || !dy || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  if (flags & ~(FP4_MX_ACCUMULATE_DX | FP4_MX_ACCUMULATE_DW)) return FP4_ERR_ARG;
  const bool want_dx = wanted(dx), want_dw = wanted(dw);
  if ((want_dw && !saved_x) || (want_dx && !saved_w)) return FP4_ERR_NULL;
  int rc = check_sizes(M, 2 * K);
  if (rc == FP4_OK) rc = check_sizes(K, 2 * N);
  if (rc == FP4_OK) rc = check_sizes(M, N);
  if (rc == FP4_OK && want_dw) rc = check_tensor(saved_x, true);
  if (rc == FP4_OK && want_dx) rc = check_tensor(saved_w, true);
  if (rc != FP4_OK) return rc;
  if (!want_dx && !want_dw) return FP4_OK;
  if ((want_dw && !saved_x->codes_t) || (want_dx && !saved_w->codes) || (!dy->data && M && N)) return FP4_ERR_NULL;
  if (want_dx && want_dw && saved_x->format != saved_w->format) return FP4_ERR_ARG;
  if ((want_dw && (saved_x->rows != M || saved_x->cols != K)) || (want_dx && (saved_w->rows != K || saved_w->cols != N))) return FP4_ERR_RANGE;
  rc = check_matrix(dy, M, N);
  if (rc == FP4_OK && want_dx) rc = check_matrix(dx, M, K);
  if (rc == FP4_OK && want_dw) rc = check_matrix(dw, K, N);
  if (rc != FP4_OK) return rc;
  const int format = want_dw ? saved_x->format : saved_w->format;
  Arena arena(ctx->workspace, ctx->workspace_bytes);
  fp4_mx_tensor q = {};
  q.rows = M;
  q.cols = N;
  q.format = format;
  if (want_dx) {
    q.codes = arena.take<uint8_t>(size_t(M * mx_pitch(N, format)));
    q.scales = arena.take<uint8_t>(size_t(mx_scale_bytes(M, N, format)));
  }
  if (want_dw) {
    q.codes_t = arena.take<uint8_t>(size_t(N * mx_pitch(M, format)));
    q.scales_t = arena.take<uint8_t>(size_t(mx_scale_bytes(N, M, format)));
  }
  if (format == FP4_MX_NVFP4) q.amax = arena.take<float>(1);
  if (!arena.ok) return FP4_ERR_WORKSPACE;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const Quantize one = {dy, &q};
  rc = quantize(ctx, st, &one, 1, status);
  if (rc != FP4_OK) return rc;
  Gemm todo[2];
  int n = 0;
  if (want_dx) todo[n++] = {&q, false, saved_w, false, M, K, N, dx, bool(flags & FP4_MX_ACCUMULATE_DX)};
  if (want_dw) todo[n++] = {saved_x, true, &q, true, K, N, M, dw, bool(flags & FP4_MX_ACCUMULATE_DW)};
  return gemm(ctx, st, todo, n, status);
}

int fp4_mx_swiglu_fwd(fp4_ctx* ctx, void* stream, const fp4_mx_matrix* gate, const fp4_mx_matrix* up, int64_t rows, int64_t cols,
                      const fp4_mx_matrix* h, fp4_mx_tensor* ckpt_gate, fp4_mx_tensor* ckpt_up, fp4_mx_tensor* quantized, int32_t* status) {
  if (!ctx || !gate || !up || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  if (!ckpt_gate != !ckpt_up) return FP4_ERR_NULL;
  if (!wanted(h) && !ckpt_gate && !quantized) return FP4_ERR_NULL;
  int rc = check_sizes(rows, cols);
  if (rc == FP4_OK && rows && cols && (!gate->data || !up->data)) rc = FP4_ERR_NULL;
  if (rc == FP4_OK) rc = check_matrix(gate, rows, cols);
  if (rc == FP4_OK) rc = check_matrix(up, rows, cols);
  if (rc == FP4_OK && wanted(h)) rc = check_matrix(h, rows, cols);
  if (rc == FP4_OK && (gate->dtype != up->dtype || (wanted(h) && h->dtype != gate->dtype))) rc = FP4_ERR_ARG;
  if (rc == FP4_OK && ckpt_gate) rc = check_checkpoint(ckpt_gate);
  if (rc == FP4_OK && ckpt_up) rc = check_checkpoint(ckpt_up);
  if (rc == FP4_OK && ckpt_gate && ckpt_gate == ckpt_up) rc = FP4_ERR_ARG;
  if (rc == FP4_OK) rc = check_swiglu_quantized(quantized);
  if (rc != FP4_OK) return rc;
  for (fp4_mx_tensor* q : {ckpt_gate, ckpt_up, quantized})
    if (q) { q->rows = rows; q->cols = cols; }
  if (rows == 0 || cols == 0) return FP4_OK;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  return launch_mx_swiglu_fwd(ctx, static_cast<cudaStream_t>(stream), matrix(gate, rows, cols), matrix(up, rows, cols), rows, cols,
                              gate->dtype, matrix(h, rows, cols), ckpt_gate, ckpt_up, quantized, status);
}

int fp4_mx_swiglu_bwd(fp4_ctx* ctx, void* stream, const fp4_mx_matrix* dh, const fp4_mx_tensor* ckpt_gate, const fp4_mx_tensor* ckpt_up,
                      int64_t rows, int64_t cols, const fp4_mx_matrix* dgate, const fp4_mx_matrix* dup, const fp4_mx_matrix* h,
                      fp4_mx_tensor* quantized, int32_t* status) {
  if (!ctx || !dh || !ckpt_gate || !ckpt_up || !dgate || !dup || !status) return FP4_ERR_NULL;
  std::lock_guard<std::mutex> turn(ctx->mutex);
  int rc = check_sizes(rows, cols);
  if (rc == FP4_OK && rows && cols && (!dh->data || !dgate->data || !dup->data)) rc = FP4_ERR_NULL;
  for (const fp4_mx_matrix* m : {dh, dgate, dup})
    if (rc == FP4_OK) rc = m->dtype != dh->dtype ? FP4_ERR_ARG : check_matrix(m, rows, cols);
  if (rc == FP4_OK && wanted(h)) rc = h->dtype != dh->dtype ? FP4_ERR_ARG : check_matrix(h, rows, cols);
  for (const fp4_mx_tensor* q : {ckpt_gate, ckpt_up}) {
    if (rc == FP4_OK) rc = check_checkpoint(q);
    if (rc == FP4_OK && (q->rows != rows || q->cols != cols)) rc = FP4_ERR_RANGE;
  }
  if (rc == FP4_OK) rc = check_swiglu_quantized(quantized);
  if (rc != FP4_OK) return rc;
  if (quantized) {
    quantized->rows = rows;
    quantized->cols = cols;
  }
  if (rows == 0 || cols == 0) return FP4_OK;
  OnDevice device(ctx);
  if (!device.ok) return FP4_ERR_CUDA;
  return launch_mx_swiglu_bwd(ctx, static_cast<cudaStream_t>(stream), matrix(dh, rows, cols), *ckpt_gate, *ckpt_up, rows, cols, dh->dtype,
                              matrix(dgate, rows, cols), matrix(dup, rows, cols), matrix(h, rows, cols), quantized, status);
}

}  // extern "C"
