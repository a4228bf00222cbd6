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
// block.  Tiles travel between global and shared memory by TMA (rows of 128 bytes, 128-byte swizzle), codes too; a matrix
// whose rows lie off 16-byte boundaries is copied by the threads, neighbouring lanes neighbouring elements.  In shared memory a
// thread takes 64 neighbours of one row (blocks along the rows) and then 32 rows of two neighbouring columns (blocks along
// the columns); either way it holds whole blocks and no two threads have to agree on an amax, and either access touches
// every bank once.
//
// What bounds it: the bytes, one way and back (16384 x 8192 BF16 to E2M1 51 us = 6.6 TB/s, back 55; to E4M3 59, back 65); both ways also the instructions, 11.5
// a value for blocks of 32 (70 us, 90 % of the copy rate; E4M3 93) and 15.4 for blocks of 16 (78 us, 79 % of the issue slots; the pass for the amax 43).  Rows off
// 16-byte boundaries: 129 us in blocks of 16 both ways, back 80, most of it shifting.  SwiGLU of the same size: forward 117 us, with the checkpoint 164
// (the copy rate: 165), with the checkpoint and h as an operand along its rows in place of h 179 (135), both ways 206 (146); backward 168 (165), with h as an
// operand along its columns 227 (176), both ways 403 (187), which takes 113 KB of shared memory, one block an SM.  (A first version kept the tile in registers, eight neighbours
// a lane, and found a block's amax by shuffles: 23 instructions for both directions, 75 % of the issue slots at 40 % of the DRAM's throughput.)
#include <cuda.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "mx.cuh"
#include "mx_codes.cuh"
#include "tc_ptx.cuh"

namespace {

using namespace mx_codes;

constexpr int THREADS = 256;
constexpr int BOX_BYTES = MX_TILE * 128;                 // 128 rows of 128 bytes
constexpr int64_t MX_SMALL_BYTES = 64 << 10;             // a tensor up to this size: its amax is found by every block for itself
// More parts than this are joined by the kernel that finds them: every block of the quantiser reading 592 of them cost 10 us of 16384 x 13824;
// the join's ticket costs a small tensor 1 us.
constexpr int MX_FEW_PARTS = 64;

// 32 neighbours of a row.
template <class T>
struct Run {
  static constexpr int WORDS = 8 * int(sizeof(T));
  uint32_t w[WORDS];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return i % 2 ? TypeOf<T>::hi(w[i / 2]) : TypeOf<T>::lo(w[i / 2]);
  }
  __device__ __forceinline__ f32x2 pair(int i) const { return pack2(get(2 * i), get(2 * i + 1)); }
  __device__ __forceinline__ void set_pair(int i, float a, float b) {
    if constexpr (sizeof(T) == 4) { w[2 * i] = __float_as_uint(a); w[2 * i + 1] = __float_as_uint(b); }
    else w[i] = TypeOf<T>::word(a, b);
  }
  // pattern of the largest magnitude of elements [first, first + n)
  __device__ __forceinline__ uint32_t amax(int first, int n) const {
    constexpr int PER = 4 / int(sizeof(T));
    uint32_t m = w[first / PER];
#pragma unroll
    for (int i = 1; i < n / PER; ++i) m = TypeOf<T>::most(m, w[first / PER + i]);
    if constexpr (sizeof(T) == 4) return m & 0x7FFFFFFFu;
    else return max(m & 0x7FFFu, (m >> 16) & 0x7FFFu);
  }
};

// ------------------------------------------------------------------------ tiles in shared memory ---
// A tile of T: boxes of 128 rows x 128 bytes, 16-byte unit u of row r at u ^ (r & 7).
template <class T> __host__ __device__ constexpr int tile_bytes() { return MX_TILE * MX_TILE * int(sizeof(T)); }
__device__ __forceinline__ uint32_t at128(int row, int byte) {                          // byte offset in a row of the tile
  return uint32_t((byte >> 7) * BOX_BYTES + row * 128 + ((byte & 127) ^ ((row & 7) << 4)));
}
// 64-byte rows (codes in E2M1), 64-byte swizzle: unit u of row r at u ^ ((r >> 1) & 3).
__device__ __forceinline__ uint32_t at64(int row, int byte) { return uint32_t(row * 64 + (byte ^ (((row >> 1) & 3) << 4))); }

template <class T>
__device__ __forceinline__ Run<T> load_run(const uint8_t* tile, int row, int run) {      // elements 32 run .. 32 run + 31
  Run<T> v;
#pragma unroll
  for (int i = 0; i < Run<T>::WORDS / 4; ++i) {
    const uint4 q = *reinterpret_cast<const uint4*>(tile + at128(row, run * 32 * int(sizeof(T)) + 16 * i));
    v.w[4 * i] = q.x; v.w[4 * i + 1] = q.y; v.w[4 * i + 2] = q.z; v.w[4 * i + 3] = q.w;
  }
  return v;
}
// What comes behind starts from these registers: the compiler does not spread several steps' values over more registers than three blocks
// an SM leave a thread (80).
template <class T>
__device__ __forceinline__ void in_order(Run<T>& v) {
#pragma unroll
  for (int i = 0; i < Run<T>::WORDS; ++i) asm volatile("" : "+r"(v.w[i]));
}
// The 32 E4M3 codes of a run.
struct Run8 {
  uint32_t w[8];
};
__device__ __forceinline__ Run8 load_run8(const uint8_t* codes, int row, int run) {
  const uint4 a = *reinterpret_cast<const uint4*>(codes + at128(row, run * 32)), b = *reinterpret_cast<const uint4*>(codes + at128(row, run * 32 + 16));
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
template <class T>
__device__ __forceinline__ void store_run(uint8_t* tile, int row, int run, const Run<T>& v) {
#pragma unroll
  for (int i = 0; i < Run<T>::WORDS / 4; ++i)
    *reinterpret_cast<uint4*>(tile + at128(row, run * 32 * int(sizeof(T)) + 16 * i)) =
        make_uint4(v.w[4 * i], v.w[4 * i + 1], v.w[4 * i + 2], v.w[4 * i + 3]);
}

// Codes of a run of 32 elements into the staged codes of the tile (row r of 64 or 128 bytes), its scales among the tile's.
template <class T, int FMT, class Pair, class Amax>
__device__ __forceinline__ void encode_run(int r, int run, float2 tensor, Pair pair, Amax amax, uint8_t* s_codes, uint8_t* s_scale, bool& bad) {
  constexpr int N = mx_block(FMT), BLOCKS = 32 / N;
  uint32_t w[code_words(FMT)];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const Scale s = scale_of<T, FMT>(amax(b * N, N), tensor);
    bad |= !s.finite;
    s_scale[scale_at(r, run * BLOCKS + b)] = uint8_t(s.byte);
    encode_block<T, FMT, N>(s, [&](int i) { return pair(b * (N / 2) + i); }, w + b * (code_words(FMT) / BLOCKS));
  }
  if constexpr (FMT == FP4_MX_E4M3) {
    *reinterpret_cast<uint4*>(s_codes + at128(r, run * 32)) = make_uint4(w[0], w[1], w[2], w[3]);
    *reinterpret_cast<uint4*>(s_codes + at128(r, run * 32 + 16)) = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
    *reinterpret_cast<uint4*>(s_codes + at64(r, run * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// E4M3 codes of a run into staged codes of 64 columns (two runs), 64-byte rows.
template <class T>
__device__ __forceinline__ void keep_run(const Run<T>& v, int r, int run, uint8_t* s_codes, uint8_t* s_scale, bool& bad) {
  const Scale s = scale_of<T, FP4_MX_E4M3>(v.amax(0, 32), NO_TENSOR_SCALE);
  bad |= !s.finite;
  s_scale[scale_at(r, run)] = uint8_t(s.byte);
  uint32_t w[8];
  encode_block<T, FP4_MX_E4M3, 32>(s, [&](int i) { return v.pair(i); }, w);
  *reinterpret_cast<uint4*>(s_codes + at64(r, (run & 1) * 32)) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(s_codes + at64(r, (run & 1) * 32 + 16)) = make_uint4(w[4], w[5], w[6], w[7]);
}
// Blocks along the rows: the thread's run.
template <class T, int FMT>
__device__ __forceinline__ void encode_along(const Run<T>& v, int r, int run, float2 tensor, uint8_t* s_codes, uint8_t* s_scale, bool& bad) {
  encode_run<T, FMT>(r, run, tensor, [&](int i) { return v.pair(i); }, [&](int first, int n) { return v.amax(first, n); }, s_codes, s_scale, bad);
}
// Blocks along the columns: thread t takes columns 2 p and 2 p + 1 (p = t % 64) of rows 32 b .. 32 b + 31 (b = t / 64).  Row `column`
// of the staged codes holds a column's.
template <class T, int FMT>
__device__ __forceinline__ void encode_across(const uint8_t* tile, float2 tensor, uint8_t* s_codes, uint8_t* s_scale, bool& bad) {
  const int p = threadIdx.x & 63, b = threadIdx.x >> 6;
  uint32_t a[32], c[sizeof(T) == 4 ? 32 : 1];              // 16 bits: both columns in a
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint8_t* q = tile + at128(32 * b + i, 2 * p * int(sizeof(T)));
    if constexpr (sizeof(T) == 4) {
      const uint2 w = *reinterpret_cast<const uint2*>(q);
      a[i] = w.x; c[i] = w.y;
    } else {
      a[i] = *reinterpret_cast<const uint32_t*>(q);
    }
  }
  // the largest magnitudes of both columns, of rows [16 h, 16 h + 16)
  uint32_t ma[2], mc[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    ma[h] = a[16 * h];
    if constexpr (sizeof(T) == 4) mc[h] = c[16 * h];
#pragma unroll
    for (int i = 1; i < 16; ++i) {
      ma[h] = TypeOf<T>::most(ma[h], a[16 * h + i]);
      if constexpr (sizeof(T) == 4) mc[h] = TypeOf<T>::most(mc[h], c[16 * h + i]);
    }
    if constexpr (sizeof(T) == 4) { ma[h] &= 0x7FFFFFFFu; mc[h] &= 0x7FFFFFFFu; }
    else { mc[h] = (ma[h] >> 16) & 0x7FFFu; ma[h] &= 0x7FFFu; }
  }
#pragma unroll
  for (int col = 0; col < 2; ++col) {
    const auto value = [&](int i) {
      if constexpr (sizeof(T) == 4) return __uint_as_float(col ? c[i] : a[i]);
      else return col ? TypeOf<T>::hi(a[i]) : TypeOf<T>::lo(a[i]);
    };
    const uint32_t m0 = col ? mc[0] : ma[0], m1 = col ? mc[1] : ma[1];
    encode_run<T, FMT>(2 * p + col, b, tensor, [&](int i) { return pack2(value(2 * i), value(2 * i + 1)); },
                       [&](int first, int n) { return n == 32 ? max(m0, m1) : first ? m1 : m0; }, s_codes, s_scale, bad);
  }
}

// ------------------------------------------------------------------------ global <-> shared ---
// One matrix or one tensor's codes as a kernel sees it.
struct Side {
  CUtensorMap map;             // boxes of 128 rows x 128 bytes (codes in E2M1: 64)
  void* p;
  int64_t ld;                  // elements
  bool wide;                   // the map is there; else the threads copy
};
// A tile's copies in and out.  The first call of the kernel's lives initialises the barrier.
struct Loader {
  uint64_t bar;
  int abort;
};
// Whether the thread asks for the block's tile.  (Called ahead of the wait for the inputs: the switch is a parameter that is not in the constant cache yet.)
__device__ __forceinline__ bool asks_for_tile(int skip_fill) { return threadIdx.x == 0 && !(skip_fill == 0 && blockIdx.x == 0); }
// The tile's copies have come.  (Or did not within the limit: they are given a last millisecond, since a block must not leave ahead of its
// copies, whose place in shared memory would be another block's by then.)
__device__ __forceinline__ bool tile_came(Loader* l, int32_t* status, uint64_t limit_ns) {
  if (mbar_wait(&l->bar, 0, &l->abort, status, limit_ns)) return true;
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(&l->bar, 0))
    if (global_timer_ns() - t0 > 1000000ull) break;
  return false;
}
template <class T>
__device__ __forceinline__ void request_tile(const Side& s, Loader* l, uint8_t* tile, int64_t row0, int64_t col0) {   // one thread
  constexpr int PER = 128 / int(sizeof(T));
#pragma unroll
  for (int i = 0; i < tile_bytes<T>() / BOX_BYTES; ++i) tma_load_2d(tile + i * BOX_BYTES, &s.map, &l->bar, int(col0) + i * PER, int(row0));
}
// Rows off 16-byte boundaries.  A tile that lies whole in the matrix goes without checks, but for its first and last 16 bytes, whose aligned
// pieces may hold bytes that are not the matrix's.  Rows 16 / sizeof(T) apart lie alike within 16 bytes, so a warp takes such
// rows together: how far its pieces are to be shifted is the same in all lanes.
template <class T>
__device__ __forceinline__ bool whole_tile(const Side& s, int64_t row0, int64_t col0, int64_t rows, int64_t cols) {
  return col0 + MX_TILE <= cols && row0 + MX_TILE <= rows;
}
// Words first .. first + 4 of eight, shifted right by `bits`, to `put`.
template <int E, class Put>
__device__ __forceinline__ void shifted(const uint4& lo, const uint4& hi, int mis, Put put) {
  const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const int bits = (mis & 3) * 8;
  const auto from = [&](auto first) {
    constexpr int F = decltype(first)::value;
    uint32_t x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = E == 4 ? w[F + k] : __funnelshift_r(w[F + k], w[F + k + 1], bits);
    put(make_uint4(x[0], x[1], x[2], x[3]));
  };
  switch (mis >> 2) {
    case 0: from(std::integral_constant<int, 0>()); break;
    case 1: from(std::integral_constant<int, 1>()); break;
    case 2: from(std::integral_constant<int, 2>()); break;
    default: from(std::integral_constant<int, 3>()); break;
  }
}
// The warp's rows: step i takes row first_row + i (and, of 16 bits, the row eight further in the upper half of the lanes).
template <class T>
struct WarpRows {
  static constexpr int E = int(sizeof(T)), UNITS = MX_TILE * E / 16, STEPS = MX_TILE / 8 / (32 / UNITS);
  int row, unit;
  __device__ __forceinline__ WarpRows() {
    const int lane = threadIdx.x & 31;
    row = int(threadIdx.x >> 5) * 16 + lane / UNITS * 8;
    unit = lane % UNITS;
  }
};
// Eight 32-bit words of a lane: two aligned pieces, or elements one by one.
struct Words8 {
  uint4 lo, hi;
};
template <class T>
__device__ __forceinline__ Words8 load_elements(const void* p, int n) {       // the first n of 16 / sizeof(T)
  uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16 / int(sizeof(T)); ++i)
    if (i < n) w[i] = sizeof(T) == 4 ? static_cast<const uint32_t*>(p)[i] : static_cast<const unsigned short*>(p)[i];
  return {make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7])};
}
template <class T>
__device__ __forceinline__ uint4 join_elements(const Words8& v) {
  if constexpr (sizeof(T) == 4) return v.lo;
  else return make_uint4(v.lo.x | v.lo.y << 16, v.lo.z | v.lo.w << 16, v.hi.x | v.hi.y << 16, v.hi.z | v.hi.w << 16);
}
template <class T>
__device__ __forceinline__ void copy_whole_tile_in(const Side& s, uint8_t* tile, int64_t row0, int64_t col0, int64_t rows, int64_t cols) {
  constexpr int E = int(sizeof(T)), AT_ONCE = 4;
  const WarpRows<T> at;
  // (only the matrix's first 16 bytes and its last ones can lie in pieces that reach beyond it: rows of a whole tile are long enough)
  const uint8_t *first = static_cast<const uint8_t*>(s.p), *last = first + ((rows - 1) * s.ld + cols) * E;
  const bool at_end = row0 == 0 || row0 + MX_TILE == rows;
  const uint8_t* p = static_cast<const uint8_t*>(s.p) + ((row0 + at.row) * s.ld + col0) * E + at.unit * 16;
  const int64_t pitch = s.ld * E;
#pragma unroll 1
  for (int i0 = 0; i0 < WarpRows<T>::STEPS; i0 += AT_ONCE) {
    Words8 v[AT_ONCE];
    int mis[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      mis[j] = int(reinterpret_cast<uintptr_t>(p) & 15);
      const uint8_t* q = p - mis[j];
      if (at_end && (q < first || q + 32 > last)) {
        v[j] = load_elements<T>(p, 16 / E);
        mis[j] = -1;
      } else {
        v[j] = {reinterpret_cast<const uint4*>(q)[0], reinterpret_cast<const uint4*>(q)[1]};
      }
      p += pitch;
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      uint4* to = reinterpret_cast<uint4*>(tile + at128(at.row + i0 + j, at.unit * 16));
      if (mis[j] < 0) *to = join_elements<T>(v[j]);
      else shifted<E>(v[j].lo, v[j].hi, mis[j], [&](const uint4& x) { *to = x; });
    }
  }
}
template <class T>
__device__ __forceinline__ void copy_whole_tile_out(const Side& s, const uint8_t* tile, int64_t row0, int64_t col0) {
  constexpr int E = int(sizeof(T)), PER = 16 / E, UNITS = WarpRows<T>::UNITS;
  const WarpRows<T> at;
  const int64_t pitch = s.ld * E;
  uint8_t* p = static_cast<uint8_t*>(s.p) + ((row0 + at.row) * s.ld + col0) * E;
#pragma unroll 2
  for (int i = 0; i < WarpRows<T>::STEPS; ++i) {
    // the piece that begins `head` bytes behind its 16 bytes' place in the tile (the last one: what is left at the ends, below)
    const int head = int(-reinterpret_cast<intptr_t>(p) & 15), r = at.row + i;
    if (head == 0 || at.unit < UNITS - 1) {
      const uint4 lo = *reinterpret_cast<const uint4*>(tile + at128(r, at.unit * 16));
      const uint4 hi = *reinterpret_cast<const uint4*>(tile + at128(r, head ? at.unit * 16 + 16 : at.unit * 16));
      shifted<E>(lo, hi, head, [&](const uint4& v) { *reinterpret_cast<uint4*>(p + head + at.unit * 16) = v; });
    }
    p += pitch;
  }
  // PER elements of a row that begins off a boundary: those ahead of its first piece and behind its last
  const int lane = threadIdx.x & 31, e = lane % PER * E, r0 = int(threadIdx.x >> 5) * 16 + lane / PER;
  p = static_cast<uint8_t*>(s.p) + ((row0 + r0) * s.ld + col0) * E;
#pragma unroll 2
  for (int i = 0; i < 16; i += 32 / PER) {
    const int head = int(-reinterpret_cast<intptr_t>(p) & 15), at_byte = e < head ? e : MX_TILE * E - 16 + e;
    if (head) *reinterpret_cast<T*>(p + at_byte) = *reinterpret_cast<const T*>(tile + at128(r0 + i, at_byte));
    p += pitch * (32 / PER);
  }
}
// Any tile, in: a lane takes 16 bytes of the tile's row, from the two aligned pieces that hold them, shifted into
// place; what would touch bytes outside of the matrix, and the row's last piece, goes element by element.
template <class T>
__device__ __forceinline__ void copy_tile_in(const Side& s, uint8_t* tile, int64_t row0, int64_t col0, int64_t rows, int64_t cols) {
  if (whole_tile<T>(s, row0, col0, rows, cols)) return copy_whole_tile_in<T>(s, tile, row0, col0, rows, cols);
  constexpr int E = int(sizeof(T)), PER = 16 / E, UNITS = MX_TILE / PER, STEPS = MX_TILE * UNITS / THREADS, AT_ONCE = 4;
  const uintptr_t first = reinterpret_cast<uintptr_t>(s.p), last = first + uintptr_t(((rows - 1) * s.ld + cols) * E);
  const int unit = threadIdx.x % UNITS;
  const int64_t col = col0 + unit * PER;
#pragma unroll 1
  for (int i0 = 0; i0 < STEPS; i0 += AT_ONCE) {
    Words8 v[AT_ONCE];
    int how[AT_ONCE];                                      // shift in bytes; -1: element by element
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int64_t row = row0 + (i0 + j) * (THREADS / UNITS) + threadIdx.x / UNITS;
      v[j] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
      how[j] = 0;
      if (row < rows && col < cols) {
        const uintptr_t at = first + uintptr_t((row * s.ld + col) * E), piece = at & ~uintptr_t(15);
        how[j] = int(at - piece);
        if (col + PER > cols || piece < first || piece + (how[j] ? 32 : 16) > last) {
          how[j] = -1;
          v[j] = load_elements<T>(reinterpret_cast<const void*>(at), int(cols - col));
        } else {
          v[j].lo = *reinterpret_cast<const uint4*>(piece);
          if (how[j]) v[j].hi = *reinterpret_cast<const uint4*>(piece + 16);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int r = (i0 + j) * (THREADS / UNITS) + threadIdx.x / UNITS;
      uint4* to = reinterpret_cast<uint4*>(tile + at128(r, unit * 16));
      if (how[j] < 0) *to = join_elements<T>(v[j]);
      else shifted<E>(v[j].lo, v[j].hi, how[j], [&](const uint4& x) { *to = x; });
    }
  }
}
// The same, out: whole aligned pieces of 16 bytes from where in the tile's row they lie, then what is left of a row at either end.
template <class T>
__device__ __forceinline__ void copy_tile_out(const Side& s, const uint8_t* tile, int64_t row0, int64_t col0, int64_t rows, int64_t cols) {
  if (whole_tile<T>(s, row0, col0, rows, cols)) return copy_whole_tile_out<T>(s, tile, row0, col0);
  constexpr int E = int(sizeof(T)), PER = 16 / E, UNITS = MX_TILE / PER, STEPS = MX_TILE * UNITS / THREADS;
  const int width = int(cols - col0 < MX_TILE ? cols - col0 : MX_TILE) * E, unit = threadIdx.x % UNITS;
#pragma unroll 2
  for (int i = 0; i < STEPS; ++i) {
    const int r = i * (THREADS / UNITS) + threadIdx.x / UNITS;
    if (row0 + r >= rows) break;
    uint8_t* out = reinterpret_cast<uint8_t*>(static_cast<T*>(s.p) + (row0 + r) * s.ld + col0);
    const int head = int(-reinterpret_cast<intptr_t>(out) & 15), at = head + 16 * unit;      // bytes
    if (at + 16 <= width) {
      uint32_t w[5];
#pragma unroll
      for (int k = 0; k < 5; ++k) w[k] = k < 4 || (at & 3) ? *reinterpret_cast<const uint32_t*>(tile + at128(r, (at & ~3) + 4 * k)) : 0u;
      if (E == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], (at & 3) * 8);
      }
      *reinterpret_cast<uint4*>(out + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  // up to PER - 1 elements at either end: 16 lanes a row
  const int lane = threadIdx.x & 15;
#pragma unroll 2
  for (int r = threadIdx.x / 16; r < MX_TILE; r += THREADS / 16) {
    if (row0 + r >= rows) break;
    uint8_t* out = reinterpret_cast<uint8_t*>(static_cast<T*>(s.p) + (row0 + r) * s.ld + col0);
    int head = int(-reinterpret_cast<intptr_t>(out) & 15);
    if (head > width) head = width;
    const int body = (width - head) & ~15;
    const int at = lane * E < head ? lane * E : lane * E + body;             // elements [0, head) and [head + body, width)
    if (at < width && lane * E < width - body)
      *reinterpret_cast<T*>(out + at) = *reinterpret_cast<const T*>(tile + at128(r, at));
  }
}
template <class T>
__device__ __forceinline__ void send_tile(const Side& s, const uint8_t* tile, int64_t row0, int64_t col0, int64_t cols) {   // one thread
  constexpr int PER = 128 / int(sizeof(T));
#pragma unroll
  for (int i = 0; i < tile_bytes<T>() / BOX_BYTES; ++i)
    if (col0 + i * PER < cols) tma_store_2d(&s.map, tile + i * BOX_BYTES, int(col0) + i * PER, int(row0));
}
__device__ __forceinline__ void copy_scales(uint8_t* dst, const uint8_t* smem, int bytes) {
  for (int i = threadIdx.x; i < bytes / 4; i += THREADS) reinterpret_cast<uint32_t*>(dst)[i] = reinterpret_cast<const uint32_t*>(smem)[i];
}

struct TileAt {
  int64_t row, col;            // tile coordinates
};
__device__ __forceinline__ TileAt tile_at(unsigned t, int64_t col_tiles) {
  const unsigned per_row = unsigned(col_tiles);
  return {int64_t(t / per_row), int64_t(t % per_row)};
}
__device__ __forceinline__ void report(bool bad, int32_t* status) {
  if (__any_sync(0xFFFFFFFFu, bad) && (threadIdx.x & 31) == 0) atomicOr(status, FP4_DEV_NONFINITE);
}

// One direction of an operand as the kernels write it.
struct Codes {
  Side codes;
  uint8_t* scales;
  int64_t tiles;               // 128-element tiles of a row
  bool on;
};

// The largest of the block's values, in every thread.
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* s_max) {
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
  m = s_max[0];
#pragma unroll
  for (int i = 1; i < THREADS / 32; ++i) m = max(m, s_max[i]);
  return m;
}

// ------------------------------------------------------------------ a tensor's amax (NVFP4) ---
// Largest finite magnitude of a matrix as a pattern of fp32, for the block that calls.  (An infinity or a NaN makes its own block's scale a NaN; as the
// tensor's amax it would make every other block's scale, and all codes with it, 0.)  Warps `warp`, `warp + warps`, ... take pieces of a row in
// 16-byte loads, AT_ONCE a lane on their way together; what lies outside of whole aligned pieces goes element by element.  (Maxima of
// integers: their order does not matter.)
struct AmaxArgs {
  const void* x;
  int64_t rows, cols, ld;
  uint32_t* parts;             // one value a block
  uint32_t* amax;              // not null: the block that ends last joins the parts here (`ticket`, 0 between calls, tells it)
  uint32_t* ticket;
};
// The thread's part of it, as a pattern of T; FINITE: of what is finite alone, which costs instructions.
template <class T, bool FINITE>
__device__ __forceinline__ uint32_t thread_amax(const AmaxArgs& a, int64_t warp, int64_t warps) {
  constexpr int E = int(sizeof(T)), AT_ONCE = 8;
  constexpr int64_t PIECE = 32 * AT_ONCE * 16;                               // bytes
  const int lane = threadIdx.x & 31;
  const auto element = [](uintptr_t p) -> uint32_t {
    return E == 4 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const unsigned short*>(p);
  };
  uint32_t m = 0;
  const int64_t pieces = (a.cols * E + PIECE - 1) / PIECE;
#pragma unroll 1
  for (int64_t row = warp / pieces, piece = warp % pieces; row < a.rows;) {
    const uintptr_t begin = reinterpret_cast<uintptr_t>(a.x) + uintptr_t(row * a.ld * E), end = begin + uintptr_t(a.cols * E);
    uintptr_t body = (begin + 15) & ~uintptr_t(15), tail = end & ~uintptr_t(15);
    if (body > end) body = end;
    if (tail < body) tail = body;
    const uintptr_t p = body + uintptr_t(piece * PIECE) + 16 * lane;
    uint4 q[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      q[i] = p + 512 * i < tail ? *reinterpret_cast<const uint4*>(p + 512 * i) : make_uint4(0, 0, 0, 0);
    const auto take = [&](uint32_t w) { m = FINITE ? most_finite<T>(m, w) : TypeOf<T>::most(m, w); };
    if (piece == 0) {                                      // up to 16 / E - 1 elements at either end
      if (begin + lane * E < body) take(element(begin + lane * E));
      if (tail + lane * E < end) take(element(tail + lane * E));
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (FINITE) {
        take(q[i].x); take(q[i].y); take(q[i].z); take(q[i].w);
      } else {
        take(TypeOf<T>::most(TypeOf<T>::most(q[i].x, q[i].y), TypeOf<T>::most(q[i].z, q[i].w)));
      }
    }
    piece += warps;
    if (piece >= pieces) {
      row += piece / pieces;
      piece %= pieces;
    }
  }
  if (FINITE) return m;
  if constexpr (E == 2) return max(m & 0x7FFFu, (m >> 16) & 0x7FFFu);
  else return m & 0x7FFFFFFFu;
}
template <class T>
__device__ __forceinline__ uint32_t amax_of(const AmaxArgs& a, int64_t warp, int64_t warps, uint32_t* s_max) {
  uint32_t m = thread_amax<T, false>(a, warp, warps);
  if (m >= TypeOf<T>::INF) m = thread_amax<T, true>(a, warp, warps);         // (it met something that is not: once more)
  return block_max(__float_as_uint(TypeOf<T>::value(m)), s_max);
}
// One matrix or two in a launch: the first has the first `blocks` blocks.
struct AmaxBatch {
  AmaxArgs a[2];
  int blocks[2];
};
template <class T>
__global__ void __launch_bounds__(THREADS) mx_amax_kernel(const __grid_constant__ AmaxBatch batch) {
  __shared__ uint32_t s_max[THREADS / 32];
  const int second = int(blockIdx.x) >= batch.blocks[0], block = int(blockIdx.x) - (second ? batch.blocks[0] : 0), blocks = batch.blocks[second];
  const AmaxArgs& a = batch.a[second];
  mx_wait_for_inputs();
  mx_let_next_start();
  const uint32_t m = amax_of<T>(a, int64_t(block) * (THREADS / 32) + (threadIdx.x >> 5), int64_t(blocks) * (THREADS / 32), s_max);
  if (threadIdx.x == 0) a.parts[block] = m;
  if (!a.amax) return;
  __shared__ bool last;
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(a.ticket, 1u) == unsigned(blocks) - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  uint32_t all = 0;
  for (int i = threadIdx.x; i < blocks; i += THREADS) all = max(all, *const_cast<volatile uint32_t*>(a.parts + i));
  all = block_max(all, s_max);
  if (threadIdx.x == 0) {
    *a.amax = all;
    *a.ticket = 0;
  }
}

// -------------------------------------------------------------------------- quantisation ---
struct QuantArgs {
  Side x;
  Codes along, across;         // blocks along the rows, along the columns
  int64_t rows, cols;
  // NVFP4: the tensor's amax is there (no parts), is the largest of `parts` values, or (parts < 0) is found by every block for itself, which a
  // tensor that small costs least; the first block notes it then
  uint32_t* amax;
  const uint32_t* part;
  int parts;
  bool backwards;              // the last tile first: what the pass for the amax has left in L2
  int32_t* status;
  uint64_t wait_limit_ns;
  int skip_fill;               // fp4_debug_set
};
// One tensor or two in a launch.
struct QuantBatch {
  QuantArgs a[2];
  unsigned tiles[2];
};
template <class T, int FMT, bool ROWS, bool COLS>
__global__ void __launch_bounds__(THREADS) mx_quantize_kernel(const __grid_constant__ QuantBatch batch) {
  constexpr int CODE_BYTES = MX_TILE * code_row_bytes(FMT);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tile = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* s_along = tile + tile_bytes<T>();
  uint8_t* s_across = s_along + (ROWS ? CODE_BYTES : 0);
  __shared__ __align__(16) uint8_t s_scale[2][1024];
  __shared__ Loader l;
  const int second = blockIdx.x >= batch.tiles[0];
  const QuantArgs& a = batch.a[second];
  const unsigned t = blockIdx.x - (second ? batch.tiles[0] : 0u);
  const TileAt at = tile_at(a.backwards ? batch.tiles[second] - 1 - t : t, mx_tiles(a.cols));
  const int64_t row0 = at.row * MX_TILE, col0 = at.col * MX_TILE;
  if (threadIdx.x == 0) {
    mbar_init(&l.bar, 1);
    l.abort = 0;
    fence_async_smem();
  }
  const bool asks = asks_for_tile(a.skip_fill);
  mx_wait_for_inputs();
  mx_let_next_start();
  if (a.x.wide) {
    if (asks) {
      mbar_arrive_expect_tx(&l.bar, tile_bytes<T>());
      request_tile<T>(a.x, &l, tile, row0, col0);
    }
  } else {
    copy_tile_in<T>(a.x, tile, row0, col0, a.rows, a.cols);
  }
  float2 tensor = make_float2(1.0f, 1.0f);               // 2^k, 2^-k
  if (FMT == FP4_MX_NVFP4) {
    __shared__ uint32_t s_max[THREADS / 32];
    uint32_t m;
    if (a.parts > 0) {
      m = 0;
      for (int i = threadIdx.x; i < a.parts; i += THREADS) m = max(m, a.part[i]);
      m = block_max(m, s_max);
    } else if (a.parts < 0) {
      const AmaxArgs all = {a.x.p, a.rows, a.cols, a.x.ld, nullptr, nullptr, nullptr};
      m = amax_of<T>(all, threadIdx.x >> 5, THREADS / 32, s_max);
    } else {
      m = *a.amax;
    }
    if (a.parts && t == 0 && threadIdx.x == 0) *a.amax = m;
    const int k = mx_tensor_exponent(m);
    tensor = make_float2(pow2_int(k), pow2_int(-k));
  }
  __syncthreads();
  if (a.x.wide && !tile_came(&l, a.status, a.wait_limit_ns)) return;
  bool bad = false;
  if (ROWS) {
    const int r = threadIdx.x & 127, run0 = (threadIdx.x >> 7) * 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) encode_along<T, FMT>(load_run<T>(tile, r, run0 + i), r, run0 + i, tensor, s_along, s_scale[0], bad);
  }
  if (COLS) encode_across<T, FMT>(tile, tensor, s_across, s_scale[1], bad);
  fence_async_smem();
  __syncthreads();
  if (threadIdx.x == 0) {
    if (ROWS) tma_store_2d(&a.along.codes.map, s_along, int(at.col) * code_row_bytes(FMT), int(row0));
    if (COLS) tma_store_2d(&a.across.codes.map, s_across, int(at.row) * code_row_bytes(FMT), int(col0));
  }
  constexpr int BYTES = scale_tile_bytes(FMT);
  if (ROWS) copy_scales(a.along.scales + (at.row * a.along.tiles + at.col) * BYTES, s_scale[0], BYTES);
  if (COLS) copy_scales(a.across.scales + (at.col * a.across.tiles + at.row) * BYTES, s_scale[1], BYTES);
  report(bad, a.status);
  if (threadIdx.x == 0) tma_store_wait_all();
}

// ------------------------------------------------------------------------ dequantisation ---
__device__ __forceinline__ void decode4_e4m3(uint32_t w, float s, float* f) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t t;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(t) : "h"(static_cast<unsigned short>(w >> (16 * i))));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&t));
    f[2 * i] = v.x * s;
    f[2 * i + 1] = v.y * s;
  }
}
__device__ __forceinline__ void decode8_e2m1(uint32_t w, float s, float* f) {
  uint32_t t[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(t[0]), "=r"(t[1]), "=r"(t[2]), "=r"(t[3]) : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&t[i]));
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

struct DequantArgs {
  Side codes, out;
  const uint8_t* scales;
  const uint32_t* amax;
  int64_t rows, cols;
  int32_t* status;
  uint64_t wait_limit_ns;
  int skip_fill;               // fp4_debug_set
};
template <class T, int FMT>
__global__ void __launch_bounds__(THREADS) mx_dequantize_kernel(const __grid_constant__ DequantArgs a) {
  constexpr int BYTES = scale_tile_bytes(FMT), CODE_BYTES = MX_TILE * code_row_bytes(FMT), N = mx_block(FMT);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tile = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* s_codes = tile + tile_bytes<T>();
  __shared__ __align__(16) uint8_t s_scale[BYTES];
  __shared__ Loader l;
  const int64_t col_tiles = mx_tiles(a.cols);
  const TileAt at = tile_at(blockIdx.x, col_tiles);
  const int64_t row0 = at.row * MX_TILE, col0 = at.col * MX_TILE;
  if (threadIdx.x == 0) {
    mbar_init(&l.bar, 1);
    l.abort = 0;
    fence_async_smem();
  }
  const bool asks = asks_for_tile(a.skip_fill);
  mx_wait_for_inputs();
  mx_let_next_start();
  if (asks) {
    mbar_arrive_expect_tx(&l.bar, CODE_BYTES);
    tma_load_2d(s_codes, &a.codes.map, &l.bar, int(at.col) * code_row_bytes(FMT), int(row0));
  }
  copy_scales(s_scale, a.scales + (at.row * col_tiles + at.col) * BYTES, BYTES);
  const float tensor = FMT == FP4_MX_NVFP4 ? pow2_int(mx_tensor_exponent(*a.amax)) : 1.0f;
  __syncthreads();
  if (!tile_came(&l, a.status, a.wait_limit_ns)) return;
  const int r = threadIdx.x & 127, run0 = (threadIdx.x >> 7) * 2;
#pragma unroll
  for (int run = run0; run < run0 + 2; ++run) {
    float f[32];
    if constexpr (FMT == FP4_MX_E4M3) {
      const float s = scale_value<FMT>(s_scale[scale_at(r, run)]);
      const Run8 q = load_run8(s_codes, r, run);
#pragma unroll
      for (int i = 0; i < 8; ++i) decode4_e4m3(q.w[i], s, f + 4 * i);
    } else {
      const uint4 q = *reinterpret_cast<const uint4*>(s_codes + at64(r, run * 16));
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) decode8_e2m1(w[i], scale_value<FMT>(s_scale[scale_at(r, (run * 32 + 8 * i) / N)]), f + 8 * i);
    }
    // (a product of a code, its scale and the tensor's power of two is exact until the last step, which may round or overflow)
    Run<T> v;
#pragma unroll
    for (int i = 0; i < 16; ++i) v.set_pair(i, FMT == FP4_MX_NVFP4 ? f[2 * i] * tensor : f[2 * i], FMT == FP4_MX_NVFP4 ? f[2 * i + 1] * tensor : f[2 * i + 1]);
    store_run(tile, r, run, v);
  }
  fence_async_smem();
  __syncthreads();
  if (!a.out.wide) {
    copy_tile_out<T>(a.out, tile, row0, col0, a.rows, a.cols);
  } else if (threadIdx.x == 0) {
    send_tile<T>(a.out, tile, row0, col0, a.cols);
    tma_store_wait_all();
  }
}

// -------------------------------------------------------------------------------- SwiGLU ---
// h = g sigmoid(g) u in fp32, rounded once.  sigmoid(g) and 1 - sigmoid(g) = sigmoid(-g) from exp(-|g|), which cannot overflow: neither loses its
// digits where it is small.  Two approximate instructions and a square: exp(-|g|) = v^2, v = 2^(-|g| log2(e) / 2) to 2^-22, and the reciprocal to 2^-23;
// the rounded exponent and constant add at most 1.23 |g| 2^-24 to the square.  From g = -87 on the square is below fp32's normal range, where
// what stands beside it may be large enough for an ordinary result (g = -100, u = 3e38: 1.7 % off with the square itself).  So one
// v goes to the small factors and the other comes last; v itself is normal down to g = -174.6, and below that counts as 0.
struct Sigmoid {
  float part, last;            // sigmoid(g) = part last
  float rest;                  // sigmoid(-g)
};
__device__ __forceinline__ Sigmoid sigmoid(float g) {
  float v, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(v) : "f"(fabsf(g) * -0.7213475204444817f));
  const float e = v * v;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  const float last = g < 0.0f ? v : 1.0f;
  return {r * last, last, (g < 0.0f ? 1.0f : e) * r};
}

struct SwigluArgs {
  Side gate, up;               // forward: inputs; backward: d_gate and d_up
  Side dh;                     // backward
  Codes ckpt_gate, ckpt_up;    // forward: written; backward: read
  Side h;
  bool has_h;
  Codes along, across;         // h as an operand
  int64_t rows, cols;
  int32_t* status;
  uint64_t wait_limit_ns;
  int skip_fill;               // fp4_debug_set
};
// h (in `tile`, complete) as an operand and as a matrix.
template <class T>
__device__ __forceinline__ void finish_h(const SwigluArgs& a, const TileAt& at, uint8_t* tile, uint8_t* s_along, uint8_t* s_across,
                                         uint8_t (*s_scale)[512], bool& bad) {
  const int64_t row0 = at.row * MX_TILE, col0 = at.col * MX_TILE;
  if (a.across.on) encode_across<T, FP4_MX_E2M1>(tile, NO_TENSOR_SCALE, s_across, s_scale[1], bad);
  fence_async_smem();
  __syncthreads();
  if (threadIdx.x == 0) {
    if (a.has_h && a.h.wide) send_tile<T>(a.h, tile, row0, col0, a.cols);
    if (a.along.on) tma_store_2d(&a.along.codes.map, s_along, int(at.col) * 64, int(row0));
    if (a.across.on) tma_store_2d(&a.across.codes.map, s_across, int(at.row) * 64, int(col0));
  }
  if (a.has_h && !a.h.wide) copy_tile_out<T>(a.h, tile, row0, col0, a.rows, a.cols);
  if (a.along.on) copy_scales(a.along.scales + (at.row * a.along.tiles + at.col) * 512, s_scale[0], 512);
  if (a.across.on) copy_scales(a.across.scales + (at.col * a.across.tiles + at.row) * 512, s_scale[1], 512);
}
// Shared memory: gate (then h), up (then the checkpoints' codes, in four pieces of 128 rows x 64 bytes: gate and up of either half of the
// columns), and h's codes in either direction as they are wanted.  64 KB of 16-bit inputs: three blocks an SM.  A thread takes its part of up
// into registers before anyone writes codes there.  (Codes beside the inputs, two blocks an SM: 16384 x 13824 358 us; codes from the
// threads to global memory, 16 bytes a row of each: 434.)
template <class T, bool KEEP>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 4 ? 1 : 3) mx_swiglu_fwd_kernel(const __grid_constant__ SwigluArgs a) {
  constexpr int CODES4 = MX_TILE * 64, PIECE = MX_TILE * 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tile = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* t_up = tile + tile_bytes<T>();
  uint8_t* s_along = t_up + tile_bytes<T>();
  uint8_t* s_across = s_along + (a.along.on ? CODES4 : 0);
  __shared__ __align__(16) uint8_t s_scale[4][512];        // along, across, gate, up
  __shared__ Loader l;
  const TileAt at = tile_at(blockIdx.x, mx_tiles(a.cols));
  const int64_t row0 = at.row * MX_TILE, col0 = at.col * MX_TILE;
  if (threadIdx.x == 0) {
    mbar_init(&l.bar, 1);
    l.abort = 0;
    fence_async_smem();
  }
  const bool asks = asks_for_tile(a.skip_fill);
  mx_wait_for_inputs();
  mx_let_next_start();
  if (asks) {
    mbar_arrive_expect_tx(&l.bar, (a.gate.wide ? tile_bytes<T>() : 0) + (a.up.wide ? tile_bytes<T>() : 0));
    if (a.gate.wide) request_tile<T>(a.gate, &l, tile, row0, col0);
    if (a.up.wide) request_tile<T>(a.up, &l, t_up, row0, col0);
  }
  if (!a.gate.wide) copy_tile_in<T>(a.gate, tile, row0, col0, a.rows, a.cols);
  if (!a.up.wide) copy_tile_in<T>(a.up, t_up, row0, col0, a.rows, a.cols);
  __syncthreads();
  if (!tile_came(&l, a.status, a.wait_limit_ns)) return;
  bool bad = false;
  const int r = threadIdx.x & 127, half = threadIdx.x >> 7;
  Run<T> u[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) u[i] = load_run<T>(t_up, r, 2 * half + i);
  if (KEEP) __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int run = 2 * half + i;
    Run<T> g = load_run<T>(tile, r, run);
    if (KEEP) {
      keep_run(g, r, run, t_up + half * PIECE, s_scale[2], bad);
      in_order(g);
      keep_run(u[i], r, run, t_up + (2 + half) * PIECE, s_scale[3], bad);
      in_order(u[i]);
      in_order(g);
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float g0 = g.get(2 * k), g1 = g.get(2 * k + 1);
      const Sigmoid s0 = sigmoid(g0), s1 = sigmoid(g1);
      g.set_pair(k, g0 * s0.part * u[i].get(2 * k) * s0.last, g1 * s1.part * u[i].get(2 * k + 1) * s1.last);
    }
    if (a.has_h || a.across.on) store_run(tile, r, run, g);
    if (a.along.on) encode_along<T, FP4_MX_E2M1>(g, r, run, NO_TENSOR_SCALE, s_along, s_scale[0], bad);
  }
  if (a.across.on) __syncthreads();
  finish_h<T>(a, at, tile, s_along, s_across, s_scale, bad);
  if (KEEP) {
    if (threadIdx.x == 0)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        tma_store_2d(&a.ckpt_gate.codes.map, t_up + i * PIECE, int(at.col) * 128 + 64 * i, int(row0));
        tma_store_2d(&a.ckpt_up.codes.map, t_up + (2 + i) * PIECE, int(at.col) * 128 + 64 * i, int(row0));
      }
    copy_scales(a.ckpt_gate.scales + (at.row * a.ckpt_gate.tiles + at.col) * 512, s_scale[2], 512);
    copy_scales(a.ckpt_up.scales + (at.row * a.ckpt_up.tiles + at.col) * 512, s_scale[3], 512);
  }
  report(bad, a.status);
  if (threadIdx.x == 0) tma_store_wait_all();
}
// Shared memory: dh (then d_gate), the checkpoints' codes (then d_up), and as they are wanted h and its codes.  A thread takes its codes into
// registers before anyone writes d_up there.
template <class T, bool H>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 4 ? 1 : H ? 2 : 3) mx_swiglu_bwd_kernel(const __grid_constant__ SwigluArgs a) {
  constexpr int CODES8 = MX_TILE * 128, CODES4 = MX_TILE * 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tile = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* t_up = tile + tile_bytes<T>();
  uint8_t* t_h = t_up + tile_bytes<T>();
  uint8_t* s_along = t_h + (H ? tile_bytes<T>() : 0);
  uint8_t* s_across = s_along + (H && a.along.on ? CODES4 : 0);
  __shared__ __align__(16) uint8_t s_scale[4][512];        // along, across, gate, up
  __shared__ Loader l;
  const TileAt at = tile_at(blockIdx.x, mx_tiles(a.cols));
  const int64_t row0 = at.row * MX_TILE, col0 = at.col * MX_TILE;
  if (threadIdx.x == 0) {
    mbar_init(&l.bar, 1);
    l.abort = 0;
    fence_async_smem();
  }
  const bool asks = asks_for_tile(a.skip_fill);
  mx_wait_for_inputs();
  mx_let_next_start();
  if (asks) {
    mbar_arrive_expect_tx(&l.bar, 2 * CODES8 + (a.dh.wide ? tile_bytes<T>() : 0));
    tma_load_2d(t_up, &a.ckpt_gate.codes.map, &l.bar, int(at.col) * 128, int(row0));
    tma_load_2d(t_up + CODES8, &a.ckpt_up.codes.map, &l.bar, int(at.col) * 128, int(row0));
    if (a.dh.wide) request_tile<T>(a.dh, &l, tile, row0, col0);
  }
  if (!a.dh.wide) copy_tile_in<T>(a.dh, tile, row0, col0, a.rows, a.cols);
  copy_scales(s_scale[2], a.ckpt_gate.scales + (at.row * a.ckpt_gate.tiles + at.col) * 512, 512);
  copy_scales(s_scale[3], a.ckpt_up.scales + (at.row * a.ckpt_up.tiles + at.col) * 512, 512);
  __syncthreads();
  if (!tile_came(&l, a.status, a.wait_limit_ns)) return;
  bool bad = false;
  const int r = threadIdx.x & 127, half = threadIdx.x >> 7;
  Run8 cg[2], cu[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    cg[i] = load_run8(t_up, r, 2 * half + i);
    cu[i] = load_run8(t_up + CODES8, r, 2 * half + i);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int run = 2 * half + i;
    const float sg = scale_value<FP4_MX_E4M3>(s_scale[2][scale_at(r, run)]), su = scale_value<FP4_MX_E4M3>(s_scale[3][scale_at(r, run)]);
    Run<T> d = load_run<T>(tile, r, run), e, h;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      float g[4], u[4], dg[4], du[4], hv[4];
      decode4_e4m3(cg[i].w[q], sg, g);
      decode4_e4m3(cu[i].w[q], su, u);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const Sigmoid s = sigmoid(g[k]);
        const float gs = g[k] * s.part, dh = d.get(4 * q + k);
        du[k] = dh * gs * s.last;
        dg[k] = dh * u[k] * fmaf(gs, s.rest, s.part) * s.last;      // d/dg g s = s (1 + g (1 - s)) = s + g s (1 - s)
        hv[k] = gs * u[k] * s.last;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        d.set_pair(2 * q + k, dg[2 * k], dg[2 * k + 1]);
        e.set_pair(2 * q + k, du[2 * k], du[2 * k + 1]);
        if (H) h.set_pair(2 * q + k, hv[2 * k], hv[2 * k + 1]);
      }
    }
    store_run(tile, r, run, d);
    store_run(t_up, r, run, e);
    if (H) {
      if (a.has_h || a.across.on) store_run(t_h, r, run, h);
      if (a.along.on) encode_along<T, FP4_MX_E2M1>(h, r, run, NO_TENSOR_SCALE, s_along, s_scale[0], bad);
    }
  }
  fence_async_smem();
  __syncthreads();
  if (threadIdx.x == 0) {
    if (a.up.wide) send_tile<T>(a.up, t_up, row0, col0, a.cols);
    if (a.gate.wide) send_tile<T>(a.gate, tile, row0, col0, a.cols);
  }
  if (!a.up.wide) copy_tile_out<T>(a.up, t_up, row0, col0, a.rows, a.cols);
  if (!a.gate.wide) copy_tile_out<T>(a.gate, tile, row0, col0, a.rows, a.cols);
  if (H) {
    finish_h<T>(a, at, t_h, s_along, s_across, s_scale, bad);
    report(bad, a.status);
  }
  if (threadIdx.x == 0) tma_store_wait_all();
}

// ------------------------------------------------------------------------------ launches ---
int elt_bytes(int dtype) { return dtype == FP4_DTYPE_FP32 ? 4 : 2; }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int make_map(fp4_ctx* ctx, CUtensorMap* map, CUtensorMapDataType type, const void* p, int64_t inner, int64_t outer, int64_t stride_bytes, int box_inner,
             CUtensorMapSwizzle swizzle) {
  const cuuint64_t dims[2] = {cuuint64_t(inner), cuuint64_t(outer)}, strides[1] = {cuuint64_t(stride_bytes)};
  const cuuint32_t box[2] = {cuuint32_t(box_inner), MX_TILE}, elem_strides[2] = {1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(map, type, 2, const_cast<void*>(p), dims, strides, box, elem_strides,
                                                                        CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? FP4_OK : FP4_ERR_CUDA;
}
// A matrix: by TMA where its rows lie on 16-byte boundaries (one that is written: end there too, since a bulk store clips to whole
// 16 bytes).
int matrix_side(fp4_ctx* ctx, Side* s, MxMatrix m, int64_t rows, int64_t cols, int dtype, bool written) {
  const int elt = elt_bytes(dtype);
  s->p = const_cast<void*>(m.p);
  s->ld = m.ld;
  s->wide = (reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && (m.ld * elt) % 16 == 0 && (!written || (cols * elt) % 16 == 0);
  if (!s->wide) return FP4_OK;
  const CUtensorMapDataType type = dtype == FP4_DTYPE_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == FP4_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                             : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return make_map(ctx, &s->map, type, m.p, cols, rows, m.ld * elt, 128 / elt, CU_TENSOR_MAP_SWIZZLE_128B);
}
int codes_side(fp4_ctx* ctx, Side* s, const uint8_t* codes, int64_t rows, int64_t cols, int format, int row = 0) {
  const int64_t pitch = mx_pitch(cols, format);
  if (!row) row = code_row_bytes(format);
  s->wide = true;
  return make_map(ctx, &s->map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, pitch, rows, pitch, row, row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}
int codes_along(fp4_ctx* ctx, Codes* c, const fp4_mx_tensor& q, int64_t rows, int64_t cols, int box_bytes = 0) {
  c->on = q.codes != nullptr;
  c->scales = q.scales;
  c->tiles = mx_tiles(cols);
  return c->on ? codes_side(ctx, &c->codes, q.codes, rows, cols, q.format, box_bytes) : FP4_OK;
}
int codes_across(fp4_ctx* ctx, Codes* c, const fp4_mx_tensor& q, int64_t rows, int64_t cols) {
  c->on = q.codes_t != nullptr;
  c->scales = q.scales_t;
  c->tiles = mx_tiles(rows);
  return c->on ? codes_side(ctx, &c->codes, q.codes_t, cols, rows, q.format) : FP4_OK;
}
template <auto KERNEL, class A>
int launch_tiles(fp4_ctx* ctx, int64_t tiles, int most_smem, int smem, cudaStream_t stream, const A& args) {
  FP4_CUDA_TRY(mx_allow_smem<KERNEL>(ctx->device, 1024 + most_smem));
  return mx_launch<KERNEL>(dim3(unsigned(tiles)), THREADS, 1024 + smem, 1, stream, args);
}

template <class T, int FMT>
int quantize_as(fp4_ctx* ctx, cudaStream_t stream, const QuantBatch& q) {
  constexpr int codes = MX_TILE * code_row_bytes(FMT), one = tile_bytes<T>() + codes;
  const int64_t tiles = int64_t(q.tiles[0]) + q.tiles[1];
  if (q.a[0].along.on && q.a[0].across.on) return launch_tiles<mx_quantize_kernel<T, FMT, true, true>>(ctx, tiles, one + codes, one + codes, stream, q);
  if (q.a[0].across.on) return launch_tiles<mx_quantize_kernel<T, FMT, false, true>>(ctx, tiles, one, one, stream, q);
  return launch_tiles<mx_quantize_kernel<T, FMT, true, false>>(ctx, tiles, one, one, stream, q);
}
// What has to be known of the tensors before they are quantised: for NVFP4 their amax.
template <class T>
int find_amax(fp4_ctx* ctx, cudaStream_t stream, QuantBatch& batch, const fp4_mx_tensor* const* q, int n) {
  constexpr int MOST = MX_SCRATCH_WORDS / 2 - 1;           // parts of a tensor; the scratch ends with two tickets
  AmaxBatch m = {};
  int found = 0;
  for (int i = 0; i < n; ++i) {
    QuantArgs& a = batch.a[i];
    if (q[i]->flags & FP4_MX_AMAX_GIVEN) continue;
    const int64_t bytes = a.rows * a.cols * int64_t(sizeof(T));
    if (bytes <= MX_SMALL_BYTES) {
      a.parts = -1;
      continue;
    }
    const int64_t want = (bytes + 8 * 4096 - 1) / (8 * 4096);
    int blocks = ctx->num_sms * (n > 1 ? 2 : 3);
    if (blocks > MOST) blocks = MOST;
    if (blocks > want) blocks = int(want);
    const bool dense = a.x.ld == a.cols;                   // rows without a gap are one long row
    uint32_t* parts = ctx->mx_scratch + i * MOST;
    m.a[found] = {a.x.p, dense ? 1 : a.rows, dense ? a.rows * a.cols : a.cols, a.x.ld, parts, nullptr, nullptr};
    if (blocks <= MX_FEW_PARTS) {
      a.parts = blocks;
      a.part = parts;
    } else {
      m.a[found].amax = a.amax;
      m.a[found].ticket = ctx->mx_scratch + MX_SCRATCH_WORDS - 1 - i;
    }
    a.backwards = true;
    m.blocks[found++] = blocks;
  }
  if (!found) return FP4_OK;
  KernelScope scope(ctx, stream, KC_ABSMAX, 1);
  return mx_launch<mx_amax_kernel<T>>(dim3(unsigned(m.blocks[0] + m.blocks[1])), THREADS, 0, 1, stream, m);
}
template <class T>
int quantize_from(fp4_ctx* ctx, cudaStream_t stream, QuantBatch& batch, const fp4_mx_tensor* const* q, int n) {
  const int format = q[0]->format;
  if (format == FP4_MX_NVFP4) {
    const int rc = find_amax<T>(ctx, stream, batch, q, n);
    if (rc != FP4_OK) return rc;
  }
  KernelScope scope(ctx, stream, KC_ENCODE, 1);
  if (format == FP4_MX_E2M1) return quantize_as<T, FP4_MX_E2M1>(ctx, stream, batch);
  if (format == FP4_MX_NVFP4) return quantize_as<T, FP4_MX_NVFP4>(ctx, stream, batch);
  return quantize_as<T, FP4_MX_E4M3>(ctx, stream, batch);
}

template <class T, int FMT>
int dequantize_as(fp4_ctx* ctx, cudaStream_t stream, const DequantArgs& a) {
  constexpr int smem = tile_bytes<T>() + MX_TILE * code_row_bytes(FMT);
  return launch_tiles<mx_dequantize_kernel<T, FMT>>(ctx, mx_tiles(a.rows) * mx_tiles(a.cols), smem, smem, stream, a);
}
template <class T>
int dequantize_to(fp4_ctx* ctx, cudaStream_t stream, const DequantArgs& a, int format) {
  if (format == FP4_MX_E2M1) return dequantize_as<T, FP4_MX_E2M1>(ctx, stream, a);
  if (format == FP4_MX_NVFP4) return dequantize_as<T, FP4_MX_NVFP4>(ctx, stream, a);
  return dequantize_as<T, FP4_MX_E4M3>(ctx, stream, a);
}

template <class T>
int swiglu_as(fp4_ctx* ctx, cudaStream_t stream, const SwigluArgs& a, bool bwd) {
  constexpr int codes4 = MX_TILE * 64, tile = tile_bytes<T>();
  const int more = (a.along.on ? codes4 : 0) + (a.across.on ? codes4 : 0);
  if (bwd && (a.has_h || more))
    return launch_tiles<mx_swiglu_bwd_kernel<T, true>>(ctx, mx_tiles(a.rows) * mx_tiles(a.cols), 3 * tile + 2 * codes4, 3 * tile + more, stream, a);
  if (bwd) return launch_tiles<mx_swiglu_bwd_kernel<T, false>>(ctx, mx_tiles(a.rows) * mx_tiles(a.cols), 2 * tile, 2 * tile, stream, a);
  if (a.ckpt_gate.on) return launch_tiles<mx_swiglu_fwd_kernel<T, true>>(ctx, mx_tiles(a.rows) * mx_tiles(a.cols), 2 * tile + 2 * codes4, 2 * tile + more, stream, a);
  return launch_tiles<mx_swiglu_fwd_kernel<T, false>>(ctx, mx_tiles(a.rows) * mx_tiles(a.cols), 2 * tile + 2 * codes4, 2 * tile + more, stream, a);
}
int swiglu(fp4_ctx* ctx, cudaStream_t stream, const SwigluArgs& a, int dtype, bool bwd) {
  KernelScope scope(ctx, stream, KC_ENCODE, 1);
  if (dtype == FP4_DTYPE_BF16) return swiglu_as<__nv_bfloat16>(ctx, stream, a, bwd);
  if (dtype == FP4_DTYPE_FP16) return swiglu_as<__half>(ctx, stream, a, bwd);
  return swiglu_as<float>(ctx, stream, a, bwd);
}

}  // namespace

int launch_mx_quantize(fp4_ctx* ctx, cudaStream_t stream, const MxQuantize* what, int n, int32_t* status) {
  const int dtype = what[0].dtype;
  if (n == 2) {                                            // one launch takes two of a kind
    const fp4_mx_tensor &p = *what[0].q, &q = *what[1].q;
    if (what[1].dtype != dtype || p.format != q.format || !p.codes != !q.codes || !p.codes_t != !q.codes_t ||
        mx_tiles(p.rows) * mx_tiles(p.cols) + mx_tiles(q.rows) * mx_tiles(q.cols) > 0x7FFFFFFF) {
      const int rc = launch_mx_quantize(ctx, stream, what, 1, status);
      return rc != FP4_OK ? rc : launch_mx_quantize(ctx, stream, what + 1, 1, status);
    }
  }
  QuantBatch batch = {};
  const fp4_mx_tensor* q[2] = {};
  for (int i = 0; i < n; ++i) {
    QuantArgs& a = batch.a[i];
    q[i] = what[i].q;
    a.rows = q[i]->rows;
    a.cols = q[i]->cols;
    a.amax = reinterpret_cast<uint32_t*>(q[i]->amax);
    a.status = status;
    a.wait_limit_ns = mx_wait_limit(ctx);
    a.skip_fill = ctx->debug_skip_fill;
    batch.tiles[i] = unsigned(mx_tiles(a.rows) * mx_tiles(a.cols));
    int rc = matrix_side(ctx, &a.x, what[i].x, a.rows, a.cols, dtype, false);
    if (rc == FP4_OK) rc = codes_along(ctx, &a.along, *q[i], a.rows, a.cols);
    if (rc == FP4_OK) rc = codes_across(ctx, &a.across, *q[i], a.rows, a.cols);
    if (rc != FP4_OK) return rc;
  }
  if (dtype == FP4_DTYPE_BF16) return quantize_from<__nv_bfloat16>(ctx, stream, batch, q, n);
  if (dtype == FP4_DTYPE_FP16) return quantize_from<__half>(ctx, stream, batch, q, n);
  return quantize_from<float>(ctx, stream, batch, q, n);
}

int launch_mx_dequantize(fp4_ctx* ctx, cudaStream_t stream, const uint8_t* codes, const uint8_t* scales, const float* amax,
                         int64_t rows, int64_t cols, int format, MxMatrix out, int dtype, int32_t* status) {
  DequantArgs a = {};
  a.scales = scales;
  a.amax = reinterpret_cast<const uint32_t*>(amax);
  a.rows = rows;
  a.cols = cols;
  a.status = status;
  a.wait_limit_ns = mx_wait_limit(ctx);
  a.skip_fill = ctx->debug_skip_fill;
  int rc = codes_side(ctx, &a.codes, codes, rows, cols, format);
  if (rc == FP4_OK) rc = matrix_side(ctx, &a.out, out, rows, cols, dtype, true);
  if (rc != FP4_OK) return rc;
  KernelScope scope(ctx, stream, KC_ENCODE, 1);
  if (dtype == FP4_DTYPE_BF16) return dequantize_to<__nv_bfloat16>(ctx, stream, a, format);
  if (dtype == FP4_DTYPE_FP16) return dequantize_to<__half>(ctx, stream, a, format);
  return dequantize_to<float>(ctx, stream, a, format);
}

int launch_mx_swiglu_fwd(fp4_ctx* ctx, cudaStream_t stream, MxMatrix gate, MxMatrix up, int64_t rows, int64_t cols, int dtype,
                         MxMatrix h, const fp4_mx_tensor* ckpt_gate, const fp4_mx_tensor* ckpt_up, const fp4_mx_tensor* q,
                         int32_t* status) {
  SwigluArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.status = status;
  a.wait_limit_ns = mx_wait_limit(ctx);
  a.skip_fill = ctx->debug_skip_fill;
  a.has_h = h.p != nullptr;
  int rc = matrix_side(ctx, &a.gate, gate, rows, cols, dtype, false);
  if (rc == FP4_OK) rc = matrix_side(ctx, &a.up, up, rows, cols, dtype, false);
  if (rc == FP4_OK && a.has_h) rc = matrix_side(ctx, &a.h, h, rows, cols, dtype, true);
  if (rc == FP4_OK && ckpt_gate) rc = codes_along(ctx, &a.ckpt_gate, *ckpt_gate, rows, cols, 64);
  if (rc == FP4_OK && ckpt_up) rc = codes_along(ctx, &a.ckpt_up, *ckpt_up, rows, cols, 64);
  if (rc == FP4_OK && q) rc = codes_along(ctx, &a.along, *q, rows, cols);
  if (rc == FP4_OK && q) rc = codes_across(ctx, &a.across, *q, rows, cols);
  return rc != FP4_OK ? rc : swiglu(ctx, stream, a, dtype, false);
}

int launch_mx_swiglu_bwd(fp4_ctx* ctx, cudaStream_t stream, MxMatrix dh, const fp4_mx_tensor& gate, const fp4_mx_tensor& up,
                         int64_t rows, int64_t cols, int dtype, MxMatrix dgate, MxMatrix dup, MxMatrix h,
                         const fp4_mx_tensor* q, int32_t* status) {
  SwigluArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.status = status;
  a.wait_limit_ns = mx_wait_limit(ctx);
  a.skip_fill = ctx->debug_skip_fill;
  a.has_h = h.p != nullptr;
  int rc = matrix_side(ctx, &a.dh, dh, rows, cols, dtype, false);
  if (rc == FP4_OK) rc = matrix_side(ctx, &a.gate, dgate, rows, cols, dtype, true);
  if (rc == FP4_OK) rc = matrix_side(ctx, &a.up, dup, rows, cols, dtype, true);
  if (rc == FP4_OK && a.has_h) rc = matrix_side(ctx, &a.h, h, rows, cols, dtype, true);
  if (rc == FP4_OK) rc = codes_along(ctx, &a.ckpt_gate, gate, rows, cols);
  if (rc == FP4_OK) rc = codes_along(ctx, &a.ckpt_up, up, rows, cols);
  if (rc == FP4_OK && q) rc = codes_along(ctx, &a.along, *q, rows, cols);
  if (rc == FP4_OK && q) rc = codes_across(ctx, &a.across, *q, rows, cols);
  return rc != FP4_OK ? rc : swiglu(ctx, stream, a, dtype, true);
}
