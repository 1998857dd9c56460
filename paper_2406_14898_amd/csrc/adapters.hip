// Low-rank adapters of many clients beside a shared projection (C ABI entry
// points), forward and backward over one packed client batch.
//
//   v = x A^T,  y = base + scale v B^T                        (rows' own A, B)
//   dv = scale dy B,  dx = dres + dv A,  dA += dv^T x,  dB += scale dy^T v
//
// With a rank of at most 64 every one of these is bound by the wide operands
// (x, y, dy, dx): each is read or written once, in four kernels.
//
//  * down: v from x.  64-row tiles, the reduction over a workgroup's waves,
//    and over workgroups too when rows are few.
//  * up: y from base and v.  A workgroup covers 64 rows x 256 columns.
//  * bwd_out: one pass over dy gives dv (a part for each block of columns,
//    which dv_sum adds) and dB.
//  * bwd_in: one pass over x and dres gives dx and dA.
//  * join: adds the parts of dA and dB that more than one workgroup left.
//
// Measured on one MI355X, bf16, clients of one slot each (a plain copy of
// 1 GiB moves 5.0 TB/s here, reads alone 6.2):
//   forward, 40583 rows, 4096 -> 12288, rank 16, 32 clients: 2.35 GB in 418 us
//     (down 70 us, 4.9 TB/s of reads; up 350 us, 5.8 TB/s)
//   backward, the same and dres: 2.05 GB in 412 us (out 194, dv_sum 6, in 190,
//     join 13, the gradients' clearing)
//   64 clients of one token, 4096 -> 12288, rank 16: 34 MB in 15.3 us
//   one token, rank 8: 6.1 us
//
// v and dv are fp32.  In bf16 mode a matrix product with them runs on the bf16
// matrix cores in three parts: v = v0 + v1 + v2, all of v's sign, together its 24
// digits.
//
// Rows reach their adapters through a table of segments (runs of rows with
// one slot) in kernel arguments: nothing is uploaded, and a call can be
// captured.  Sums over rows and parts have a fixed order: no atomics.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "../../include/flglm.h"
#include "common.h"
#include "kernels.h"

using namespace flglm;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSegs = 128;     // segments a launch (2 KB of kernel arguments, 3.6 KB with the table of slots)
constexpr int kTile = 64;      // forward: rows of a tile
constexpr int kUpCols = 256;   // forward: columns of a workgroup of `up`
constexpr int kStep = 32;      // backward: rows of a step
constexpr int64_t kMaxStride = 1 << 22;  // elements between rows: 64 of them span at most 2^30 bytes
constexpr int kInCols = 128 * kWaves;  // backward: columns of a workgroup of bwd_in

struct Segs {
  int32_t row0[kSegs], rows[kSegs], slot[kSegs];
  int32_t step0[kSegs + 1];  // first tile / step of each, within the launch
  int count;
};
// Backward: which steps belong to which slot (segments sorted by slot), and how
// they are shared out: worker i takes steps [base + i share, base + (i + 1)
// share), whatever slots these are of, and hands on its sums where the slot
// changes: a slot's first worker to dA / dB itself, the others to parts, part0 +
// (worker - the slot's first) - 1, which join adds.
struct Slots {
  int32_t slot[kSegs], step0[kSegs + 1], part0[kSegs];
  int count, base, share;
  __device__ __host__ int worker(int step) const { return (step - base) / share; }
};

__device__ __forceinline__ int find(const int32_t* first, int count, int v) {
  int lo = 0, hi = count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Rows [row0, row0 + rows) of a matrix as a buffer: what lies past the last row
// reads as zero and is not written, without a branch (which would keep loads
// from being counted, and so every wait would be for all of them).  A lane
// whose column does not exist takes the offset kNowhere.  A NULL matrix, or one
// without rows, reads as zero.
typedef __amdgpu_buffer_rsrc_t Buf;
constexpr uint32_t kNowhere = 1u << 31;
template <typename T>
__device__ __forceinline__ Buf rows_of(const T* p, long row0, long ld, int rows, int width) {
  const int bytes = p && rows > 0 ? (int)(((rows - 1) * ld + width) * (long)sizeof(T)) : 0;
  return __builtin_amdgcn_make_buffer_rsrc((void*)(p + row0 * ld), 0, bytes, 0x00020000);
}
// Byte offset of a lane's column in its row, kNowhere past the width.
template <typename T>
__device__ __forceinline__ uint32_t col_off(int row, long ld, int c, int width) {
  return c < width ? ((uint32_t)row * (uint32_t)ld + c) * (uint32_t)sizeof(T) : kNowhere;
}
constexpr int kOnce = 2;  // cache policy: non-temporal
template <int POLICY = 0>
__device__ __forceinline__ u32x4 buf_ld16(Buf b, uint32_t off) {
  return __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, POLICY);
}
template <int POLICY = 0>
__device__ __forceinline__ void buf_ld8(Vec8<bf16>& v, Buf b, uint32_t off) {
  v.r = buf_ld16<POLICY>(b, off);
}
template <int POLICY = 0>
__device__ __forceinline__ void buf_ld8(Vec8<float>& v, Buf b, uint32_t off) {
  v.r0 = buf_ld16<POLICY>(b, off);
  v.r1 = buf_ld16<POLICY>(b, off + 16);
}
template <int POLICY = 0>
__device__ __forceinline__ void buf_st8(const Vec8<bf16>& v, Buf b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(v.r, b, off, 0, POLICY);
}
template <int POLICY = 0>
__device__ __forceinline__ void buf_st8(const Vec8<float>& v, Buf b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(v.r0, b, off, 0, POLICY);
  __builtin_amdgcn_raw_buffer_store_b128(v.r1, b, off + 16, 0, POLICY);
}
// bf16 between products and memory.  A product leaves lane (m, g) row m at
// columns 8 g (x) and 32 + 8 g (y); an access of whole 128-byte lines is lane
// (m, g) at row m % 8 (x) or 8 + m % 8 (y) and columns 8 (g + 4 (m / 8)).  From
// either to the other: the upper half of each 16 lanes of x is exchanged with
// the lower half of y.  (40583 rows forward, base and y: in halves of lines
// 485 us, in whole ones 457, and past the cache 433.)
__device__ __forceinline__ void turn(u32x4& x, u32x4& y, bool upper) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t give = upper ? x[i] : y[i];
    const uint32_t take = (uint32_t)__builtin_amdgcn_mov_dpp((int)give, 0x128, 0xf, 0xf, true);  // row_ror:8
    if (upper) x[i] = take;
    else y[i] = take;
  }
}
template <typename T> constexpr bool kLines = sizeof(T) == 2;  // an fp32 access of 32 columns is whole lines already
__device__ __forceinline__ void turn(Vec8<bf16>& x, Vec8<bf16>& y, bool upper) { turn(x.r, y.r, upper); }
__device__ __forceinline__ void turn(Vec8<float>&, Vec8<float>&, bool) {}
// This lane's row (of 16) and column (of 64) in access h of two.
template <typename T>
__device__ __forceinline__ int line_row(int h, int m) {
  return kLines<T> ? 8 * h + (m & 7) : m;
}
template <typename T>
__device__ __forceinline__ int line_col(int h, int m, int g) {
  return kLines<T> ? 8 * (g + 4 * (m >> 3)) : 8 * g + 32 * h;
}
__device__ __forceinline__ bf16 buf_ld1(Buf b, uint32_t off, bf16*) {
  return __builtin_bit_cast(bf16, __builtin_amdgcn_raw_buffer_load_b16(b, off, 0, 0));
}
__device__ __forceinline__ float buf_ld1(Buf b, uint32_t off, float*) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0));
}
__device__ __forceinline__ float buf_ldf(Buf b, uint32_t off) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, off, 0, 0));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// How many parts of T hold an fp32 factor.
template <typename T> constexpr int kParts = sizeof(T) == 2 ? 3 : 1;
// Part p of N of x, as T holds it; x becomes the rest.  In bf16 every part but
// the last is cut off towards zero, and a part that would be all of x is half of
// it: no part of a number other than zero is zero or of another sign, and all of
// an infinity's are infinite, so a product with an infinity is the infinity that
// it is in one piece, not a sum of infinities of both signs or of 0 times one.
// (x has 24 digits and a part 8: three parts hold all of it.)
template <int P, int N>
__device__ __forceinline__ float split(float& x, float*) {
  return x;
}
template <int P, int N>
__device__ __forceinline__ bf16 split(float& x, bf16*) {
  if constexpr (P == N - 1) {
    return from_f32<bf16>(x);
  } else {
    constexpr uint32_t kHeld = 0xffff0000u;
    uint32_t bits = __float_as_uint(x) & kHeld;
    if (__uint_as_float(bits) == x) bits = __float_as_uint(0.5f * x) & kHeld;
    x = fabsf(x) < INFINITY ? x - __uint_as_float(bits) : x;
    return __builtin_bit_cast(bf16, (uint16_t)(bits >> 16));
  }
}
// put(p, part p of x) for each of N parts.
template <int N, typename T, int P = 0, typename F>
__device__ __forceinline__ void split_each(float x, F&& put) {
  const T part = split<P, N>(x, (T*)nullptr);
  put(P, part);
  if constexpr (P + 1 < N) split_each<N, T, P + 1>(x, put);
}

// A product over RP ranks with the fp32 factor in parts: its reduction runs over
// parts * RP / 8 chunks of eight slots, part by part.  Step s of 32 slots, lane
// group g: which part and which eight ranks.  Sixteen ranks have four parts, which
// fill two steps.  (Two parts, 16 digits, would do under most results, which are
// rounded to 8, but not where terms cancel.  The third costs short batches 0.2 us
// of 15, rank 64 half a percent, long batches nothing.)
template <typename T, int RP> struct Up {
  static constexpr int parts = sizeof(T) == 2 && RP < 32 ? 4 : kParts<T>;
  static constexpr int steps = (parts * RP + 31) / 32;
  static constexpr int weights = RP < 32 ? 1 : RP / 32;  // different weight fragments of one column
  static constexpr int stride = parts * RP + 8;          // LDS row of one token
  __device__ static __forceinline__ int chunk(int s, int g) { return 4 * s + g; }
  // (of the others both factors are zero: a weight there might be an infinity)
  __device__ static __forceinline__ bool live(int s, int g) { return chunk(s, g) < parts * RP / 8; }
  __device__ static __forceinline__ int rank(int s, int g) { return chunk(s, g) % (RP / 8) * 8; }
};

__device__ __forceinline__ int up_col(int q, int mm) { return 32 * (q >> 1) + 8 * (mm >> 2) + 4 * (q & 1) + (mm & 3); }

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------

// v (or a part of its reduction, part[split][T][r]) of one 64-row tile.
template <typename T, int RT, bool STREAM>
__global__ void __launch_bounds__(kThreads) down_kernel(Segs t, const T* x, long ldx, const T* a, int r, int in,
                                                        float* v, long total_rows) {
  constexpr int RP = 16 * RT;
  constexpr int NI = kTile / 16;
  __shared__ float sh[kWaves][kTile][RP + 1];
  const int seg = find(t.step0, t.count, blockIdx.x);
  const int first = (blockIdx.x - t.step0[seg]) * kTile;
  const int rows = uniform(min(kTile, t.rows[seg] - first)), slot = uniform(t.slot[seg]);
  const long row0 = uniform(t.row0[seg] + first);
  float* out = v + ((long)blockIdx.y * total_rows + row0) * r;
  if (slot < 0) {
    for (int i = threadIdx.x; i < rows * r; i += kThreads) out[i] = 0.f;
    return;
  }
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const Buf xb = rows_of(x, row0, ldx, rows, in), ab = rows_of(a, (long)slot * r, in, r, in);
  f32x4 acc[NI][RT];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // 64-column steps, dealt to the splits and then to the waves in turn: two
  // products over 32 columns each, x loaded in whole lines (40583 rows forward:
  // 424 us instead of 433)
  const int nk = (in + 63) / 64, stride = gridDim.y * kWaves;
  const uint32_t xrow = (uint32_t)ldx * 16 * sizeof(T), arow = (uint32_t)in * 16 * sizeof(T);
  struct Step {
    Vec8<T> av[2][RT], xv[2][NI];
  };
  auto load = [&](Step& s, int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t xo = col_off<T>(line_row<T>(h, m), ldx, 64 * k + line_col<T>(h, m, g), in),
                     ao = col_off<T>(m, in, 64 * k + 8 * g + 32 * h, in);
#pragma unroll
      for (int i = 0; i < NI; ++i) buf_ld8<STREAM ? kOnce : 0>(s.xv[h][i], xb, xo + i * xrow);
#pragma unroll
      for (int j = 0; j < RT; ++j) buf_ld8(s.av[h][j], ab, ao + j * arow);
    }
  };
  auto multiply = [&](Step& s) {
#pragma unroll
    for (int i = 0; i < NI; ++i) turn(s.xv[0][i], s.xv[1][i], m >= 8);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = mma16(s.xv[h][i].frag(), s.av[h][j].frag(), acc[i][j]);
  };
  int k = blockIdx.y * kWaves + w;
  if (rows <= 16) {
    // one token, or a few: more steps in flight, and no loads of rows that do not
    // exist (64 clients of one token, 4096 -> 12288, rank 16: the forward 15.7 us,
    // through the code below 16.7)
    constexpr int U = sizeof(T) == 2 ? (RT == 1 ? 4 : RT == 2 ? 3 : 2) : (RT == 1 ? 2 : 1);
    for (; k < nk; k += U * stride) {
      Vec8<T> av[U][2][RT], xv[U][2];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = 64 * (k + u * stride) + 16 * g + 8 * h;
          const uint32_t ao = col_off<T>(m, in, c, in);
          buf_ld8(xv[u][h], xb, col_off<T>(m, ldx, c, in));
#pragma unroll
          for (int j = 0; j < RT; ++j) buf_ld8(av[u][h][j], ab, ao + j * arow);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < RT; ++j) acc[0][j] = mma16(xv[u][h].frag(), av[u][h][j].frag(), acc[0][j]);
    }
  } else {
    // two steps in flight in turn (past the last they read zero, and so do rows
    // past a tile's last)
    Step s0, s1;
    load(s0, k);
    for (; k < nk; k += 2 * stride) {
      load(s1, k + stride);
      __builtin_amdgcn_sched_barrier(0);  // or the loads sink to their uses
      multiply(s0);
      __builtin_amdgcn_sched_barrier(0);
      load(s0, k + 2 * stride);
      __builtin_amdgcn_sched_barrier(0);
      multiply(s1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sh[w][16 * i + 4 * g + e][16 * j + m] = acc[i][j][e];
  __syncthreads();
  for (int i = threadIdx.x; i < rows * r; i += kThreads) {
    const int row = i / r, c = i - row * r;
    float s = sh[0][row][c];
#pragma unroll
    for (int q = 1; q < kWaves; ++q) s += sh[q][row][c];
    out[i] = s;
  }
}

// y = base + scale v B^T on one 64-row tile and 256 columns; v the sum of
// `parts` partial reductions (parts > 1: also stored to v_out).
// (Five waves a SIMD, of 96 registers, instead of the four of more: 64 clients
// of one token 15.7 us instead of 16.5, 40583 rows 484 instead of 480.)
template <typename T, int RP, bool STREAM>
__global__ void __launch_bounds__(kThreads, (sizeof(T) == 2 && RP <= 32 ? 5 : 1))
    up_kernel(Segs t, const float* v, int parts, long total_rows, float* v_out, const T* b, int r, int out_features,
              float scale, const T* base, long ldb, T* y, long ldy) {
  using U = Up<T, RP>;
  __shared__ __align__(16) T sh[kTile][U::stride];
  const int cols = (out_features + kUpCols - 1) / kUpCols;
  const int tile = blockIdx.x / cols, cb = blockIdx.x - tile * cols;
  const int seg = find(t.step0, t.count, tile);
  const int first = (tile - t.step0[seg]) * kTile;
  const int rows = uniform(min(kTile, t.rows[seg] - first)), slot = uniform(t.slot[seg]);
  const long row0 = uniform(t.row0[seg] + first);
  if (slot < 0) {  // no adapter: v is zero (without parts `down` wrote it), y is base
    if (parts > 1 && cb == 0)
      for (int i = threadIdx.x; i < rows * r; i += kThreads) v_out[row0 * r + i] = 0.f;
    if (base == y) return;
  }
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  // a wave's 64 columns: column tile q, first-operand row mm is column
  // 32 (q / 2) + 8 (mm / 4) + 4 (q % 2) + mm % 4, so that tiles 2h and 2h + 1
  // give a lane eight neighbours, and its row's four lanes 32
  const int c0 = cb * kUpCols + 64 * w;
  const Buf wb = rows_of(slot >= 0 ? b : nullptr, (long)slot * out_features + c0, r, min(64, out_features - c0), r);
  frag_t<T> wf[4][U::weights];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int s = 0; s < U::weights; ++s) {
      Vec8<T> f;
      buf_ld8(f, wb, col_off<T>(up_col(q, m), r, U::live(s, g) ? U::rank(s, g) : r, r));
      wf[q][s] = f.frag();
    }
  if (slot >= 0) {
    // a thread's rank, and one row in kRows; 16 rows at least are staged
    constexpr int kRows = kThreads / RP, kMany = kTile / kRows;
    const int rank = threadIdx.x % RP, row = threadIdx.x / RP;
    auto stage = [&](auto count) {
      constexpr int n = decltype(count)::value;
      float f[n] = {};
      constexpr int nq = n <= 8 ? 4 : 2;  // parts at once
      const uint32_t off = col_off<float>(row, r, rank, r);
      for (int q0 = 0; q0 < parts; q0 += nq) {
        float part[nq][n];
#pragma unroll
        for (int q = 0; q < nq; ++q) {
          const Buf vb = rows_of(v + (q0 + q) * total_rows * r, row0, r, q0 + q < parts ? rows : 0, r);
#pragma unroll
          for (int i = 0; i < n; ++i) part[q][i] = buf_ldf(vb, off + i * (kRows * 4) * (uint32_t)r);
        }
        __builtin_amdgcn_sched_barrier(0);  // all loads before the first sum
#pragma unroll
        for (int q = 0; q < nq; ++q)
#pragma unroll
          for (int i = 0; i < n; ++i) f[i] += part[q][i];
      }
      const Buf ob = rows_of(parts > 1 && cb == 0 ? v_out : nullptr, row0, r, rows, r);
#pragma unroll
      for (int i = 0; i < n; ++i) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(f[i]), ob, col_off<float>(row + i * kRows, r, rank, r), 0,
                                              0);
        split_each<U::parts, T>(f[i], [&](int q, T part) { sh[row + i * kRows][q * RP + rank] = part; });
      }
    };
    if (rows > 16) stage(std::integral_constant<int, kMany>());
    else stage(std::integral_constant<int, 16 / kRows>());
  }
  __syncthreads();
  if (c0 >= out_features) return;
  const Buf bb = rows_of(base, row0, ldb, rows, out_features), yb = rows_of(y, row0, ldy, rows, out_features);
  uint32_t bo[2], yo[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    bo[h] = col_off<T>(line_row<T>(h, m), ldb, c0 + line_col<T>(h, m, g), out_features);
    yo[h] = col_off<T>(line_row<T>(h, m), ldy, c0 + line_col<T>(h, m, g), out_features);
  }
  auto rows16 = [&](int i, Vec8<T> (&bs)[2]) {
    f32x4 acc[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (slot >= 0) {
#pragma unroll
      for (int s = 0; s < U::steps; ++s) {
        Vec8<T> vv;
        if (U::live(s, g)) vv.load(&sh[16 * i + m][8 * U::chunk(s, g)]);
        else vv.zero();
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] = mma16(wf[q][s % U::weights], vv.frag(), acc[q]);
      }
    }
    turn(bs[0], bs[1], m >= 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = bs[h].get(e) + scale * acc[2 * h + (e >> 2)][e & 3];
      bs[h].set(o);
    }
    turn(bs[0], bs[1], m >= 8);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      buf_st8<STREAM ? kOnce : 0>(bs[h], yb, yo[h] + (uint32_t)(16 * i * sizeof(T)) * (uint32_t)ldy);
  };
  auto load16 = [&](int i, Vec8<T> (&bs)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      buf_ld8<STREAM ? kOnce : 0>(bs[h], bb, bo[h] + (uint32_t)(16 * i * sizeof(T)) * (uint32_t)ldb);
  };
  if (rows > kTile - 16) {
    Vec8<T> bs[kTile / 16][2];
#pragma unroll
    for (int i = 0; i < kTile / 16; ++i) load16(i, bs[i]);
#pragma unroll
    for (int i = 0; i < kTile / 16; ++i) rows16(i, bs[i]);
  } else {
    Vec8<T> bs[2], next[2];
    load16(0, bs);
    for (int i = 0; 16 * i < rows; ++i) {
      load16(i + 1, next);  // past the last row: zero
      rows16(i, bs);
      bs[0] = next[0];
      bs[1] = next[1];
    }
  }
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

// Walks the steps [step, end) of one worker and slot.
struct Walk {
  int step, end, seg;
  int row, left;  // the next step's first row, and the rows from there on in its segment
  __device__ __forceinline__ void start(const Segs& t) {
    const int first = (step - t.step0[seg]) * kStep;
    row = uniform(t.row0[seg] + first);
    left = uniform(t.rows[seg] - first);
  }
  // The current step's first row and its rows; moves on.
  __device__ __forceinline__ int next(const Segs& t, int* row0) {
    const int rows = min(kStep, left);
    *row0 = row;
    row += kStep;
    left -= kStep;
    if (++step < end && left <= 0) {
      ++seg;
      row = uniform(t.row0[seg]);
      left = uniform(t.rows[seg]);
    }
    return rows;
  }
};
// Calls run(walk, slot, part) for each slot of a worker's steps; part: where its
// sums go, -1 for the output itself.
template <typename F>
__device__ __forceinline__ void for_slots(const Segs& t, const Slots& sl, int worker, F&& run) {
  int step = sl.base + worker * sl.share;
  const int end = min(sl.step0[sl.count], step + sl.share);
  int k = find(sl.step0, sl.count, step);
  for (; step < end; ++k) {
    Walk wk;
    wk.step = step;
    wk.end = step = min(end, sl.step0[k + 1]);
    wk.seg = find(t.step0, t.count, wk.step);
    wk.start(t);
    const int nth = worker - sl.worker(sl.step0[k]);  // of this slot's workers
    run(wk, uniform(sl.slot[k]), uniform(nth == 0 ? -1 : sl.part0[k] + nth - 1));
  }
}

// LDS rows of a factor [32 tokens][RP] turned to [part][rank][token].
constexpr int kTokStride = kStep + 8;

// One 32-row x 128-column tile of X in a wave's registers: lane (m, g) holds
// rows 8g .. 8g + 7 at columns 8m .. 8m + 7.
// The tile is read once and in whole lines: non-temporal (dy: 484 -> 463 us a
// backward of 40583 rows; of accesses to halves of lines it costs, 487 -> 559 in
// `up` when it had such).
template <typename T>
__device__ __forceinline__ void load_tile(Vec8<T> (&xr)[8], const T* x, long ld, int row0, int rows, int c0, int width,
                                          int m, int g) {
  const Buf b = rows_of(x, row0, ld, rows, width);
  const uint32_t off = col_off<T>(8 * g, ld, c0 + 8 * m, width), row = (uint32_t)ld * sizeof(T);
#pragma unroll
  for (int i = 0; i < 8; ++i) buf_ld8<kOnce>(xr[i], b, off + i * row);
}

// acc[j][q] += X^T W over the tile's 32 rows (xt: the tile turned): columns
// 8 m + j, ranks 16 q + n.  between() runs before each eight products.
template <typename T, int RT, typename F>
__device__ __forceinline__ void outer(f32x4 (&acc)[8][RT], const Vec8<T> (&xt)[8], const T* wt, int m, int g,
                                      F&& between) {
  constexpr int NP = kParts<T>;
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      between();
      Vec8<T> f;
      f.load(wt + ((long)p * 16 * RT + 16 * q + m) * kTokStride + 8 * g);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j][q] = mma16(xt[j].frag(), f.frag(), acc[j][q]);
    }
}

// Waves of a bwd_out workgroup: as many as registers and LDS let run on a CU
// (two a SIMD; one in fp32), because every workgroup along the columns leaves
// a part of dv.
template <typename T> struct OutWaves { static constexpr int n = sizeof(T) == 2 ? 8 : 4; };

// LDS traffic of this wave before the barrier is done, and every wave is here.
// (Global loads and stores stay in flight: __syncthreads would wait for them.)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One step's factor, `ranks` columns of rows `stride` floats apart, on its way
// to LDS: loaded a step ahead.
template <int RP, int NT> struct Factor {
  static_assert(NT % RP == 0, "a thread keeps its rank");
  static constexpr int n = kStep * RP / NT;
  float f[n];
  __device__ static __forceinline__ int rank(int tid) { return tid % RP; }
  __device__ static __forceinline__ int row(int tid, int i) { return tid / RP + i * (NT / RP); }
  __device__ __forceinline__ void load(const float* v, int row0, int rows, int stride, int ranks, int tid) {
    const Buf b = rows_of(v, row0, stride, rows, ranks);
    const uint32_t off = col_off<float>(row(tid, 0), stride, rank(tid), ranks);
#pragma unroll
    for (int i = 0; i < n; ++i) f[i] = buf_ldf(b, off + i * (NT / RP * 4) * (uint32_t)stride);
  }
  // The sum of `parts` such factors, `apart` floats from one another, in order.
  __device__ __forceinline__ void load(const float* v, int row0, int rows, int stride, int ranks, int tid, int parts,
                                       long apart) {
    load(v, row0, rows, stride, ranks, tid);
    for (int q = 1; q < parts; ++q) {
      Factor next;
      next.load(v + q * apart, row0, rows, stride, ranks, tid);
#pragma unroll
      for (int i = 0; i < n; ++i) f[i] += next.f[i];
    }
  }
};

// dv parts (one for each column block) and dB (or a part of it), for the ranks
// [r0, r0 + 16 RT): ranks past 32 are two slices, each with workgroups of its
// own, because the sums of 64 would leave no registers to overlap anything in.
// The slices of a tile run eight workgroups apart, so on one XCD and its L2.
// A step: the tile (loaded two steps before) goes to the wave's own LDS in rows,
// and through registers, turned, into dB; dv reads the rows back and leaves its
// result in their place; one barrier, and the waves' results are added.  Reading
// dy alone in this order takes 150 us for 1.02 GB; with a store of dv's size a
// step beside it 182, whatever its order or place; this kernel 194 (with one
// tile ahead 205).
template <typename T, int RT>
__global__ void __launch_bounds__((64 * OutWaves<T>::n))
    bwd_out_kernel(Segs t, Slots sl, const T* dy, long lddy, const T* b, const float* v, int stride, int out_features,
                   float scale, float* dv_part, long total_rows, float* db, float* db_part, int groups, int slices) {
  constexpr int NW = OutWaves<T>::n, NT = 64 * NW;
  constexpr int RP = 16 * RT, NP = kParts<T>;
  constexpr int kRow = 128 + 16 / (int)sizeof(T);
  constexpr int kDv = RP + 1;
  static_assert(kStep * kDv * 4 <= kStep * kRow * (int)sizeof(T), "dv fits its tile's place");
  __shared__ __align__(16) T wt[2][NP * RP * kTokStride];
  __shared__ __align__(16) T tile[2][NW][kStep * kRow];
  const int group = slices == 1 ? blockIdx.x : (blockIdx.x >> 4) * 8 + (blockIdx.x & 7);
  if (group >= groups) return;
  const int r0 = slices == 1 ? 0 : RP * ((blockIdx.x >> 3) & 1), r = min(RP, stride - r0);
  b += r0;
  v += r0;
  dv_part += r0;
  db += r0;
  db_part += r0;
  const int cols = (out_features + 128 * NW - 1) / (128 * NW);
  const int worker = group / cols, cb = group - worker * cols;
  for_slots(t, sl, worker, [&](Walk& wk, int slot, int part) {
    int tid = threadIdx.x;
    settle(tid);  // addresses are formed anew for each slot: held across slots, they would not fit the registers
    const int lane = tid & 63, w = uniform(tid >> 6), m = lane & 15, g = lane >> 4;
    const int c0 = cb * 128 * NW + 128 * w;
    // this step's rows and the next one's (none: 0)
    int row0, row1 = 0;
    int rows = wk.next(t, &row0), rows1 = 0;
    Vec8<T> xa[8], xb[8], xt[8];
    Factor<RP, NT> va, vb;
    va.load(v, row0, rows, stride, r, tid);
    // B as the second operand of dv = dy B: rank 16 q + m, columns 32 k + 8 g ..
    const Buf bs = rows_of(b, (long)slot * out_features + c0, stride, min(128, out_features - c0), r);
    frag_t<T> bf[4][RT];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        const uint32_t off = col_off<T>(32 * k + 8 * g, stride, 16 * q + m, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) bf[k][q][e] = buf_ld1(bs, off + e * (uint32_t)(stride * sizeof(T)), (T*)nullptr);
      }
    load_tile(xa, dy, lddy, row0, rows, c0, out_features, m, g);
    if (wk.step < wk.end) rows1 = wk.next(t, &row1);
    vb.load(v, row1, rows1, stride, r, tid);
    load_tile(xb, dy, lddy, row1, rows1, c0, out_features, m, g);
    auto stage = [&](T* dst, const Factor<RP, NT>& vn) {
#pragma unroll
      for (int i = 0; i < Factor<RP, NT>::n; ++i) {
        const int row = Factor<RP, NT>::row(tid, i), c = Factor<RP, NT>::rank(tid);
        split_each<NP, T>(vn.f[i], [&](int p, T part) { dst[(p * RP + c) * kTokStride + row] = part; });
      }
    };
    f32x4 acc[8][RT];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int q = 0; q < RT; ++q) acc[j][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    stage(wt[0], va);
    lds_barrier();
    // One step: its tile xr, its factor's registers vc (staged already) and the
    // next step's factor vn.  xr and vc are loaded anew for the step after the
    // next, between the products: eight loads at once would hold the wave up.
    auto step = [&](int buf, Vec8<T> (&xr)[8], Factor<RP, NT>& vc, const Factor<RP, NT>& vn) {
      T* mine = tile[buf][w];
#pragma unroll
      for (int i = 0; i < 8; ++i) xr[i].store(mine + (8 * g + i) * kRow + 8 * m);
      transpose8x8(xr, xt);
      int row2 = 0, rows2 = 0;
      if (wk.step < wk.end) rows2 = wk.next(t, &row2);
      __builtin_amdgcn_sched_barrier(0);
      vc.load(v, row2, rows2, stride, r, tid);
      __builtin_amdgcn_sched_barrier(0);
      const Buf from = rows_of(dy, row2, lddy, rows2, out_features);
      const uint32_t off2 = col_off<T>(8 * g, lddy, c0 + 8 * m, out_features), row_bytes = (uint32_t)lddy * sizeof(T);
      int fetched = 0;
      auto fetch = [&] {
        if (fetched == 8) return;
        buf_ld8<kOnce>(xr[fetched], from, off2 + fetched * row_bytes);
        ++fetched;
        __builtin_amdgcn_sched_barrier(0x387);  // products and global memory stay in order, all else may pass
      };
      __builtin_amdgcn_wave_barrier();
      outer<T, RT>(acc, xt, wt[buf], m, g, fetch);
      f32x4 d[2][RT];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int q = 0; q < RT; ++q) d[h][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          fetch();
          Vec8<T> f;
          f.load(mine + (16 * h + m) * kRow + 32 * k + 8 * g);
#pragma unroll
          for (int q = 0; q < RT; ++q) d[h][q] = mma16(f.frag(), bf[k][q], d[h][q]);
        }
      }
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");  // the rows are read: dv takes their place
      float* dvs = (float*)mine;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < RT; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) dvs[(16 * h + 4 * g + e) * kDv + 16 * q + m] = d[h][q][e];
      stage(wt[buf ^ 1], vn);
      lds_barrier();
      const Buf dst = rows_of(dv_part + cb * total_rows * stride, row0, stride, rows, r);
      const uint32_t off = col_off<float>(Factor<RP, NT>::row(tid, 0), stride, Factor<RP, NT>::rank(tid), r);
#pragma unroll
      for (int i = 0; i < Factor<RP, NT>::n; ++i) {
        const int row = Factor<RP, NT>::row(tid, i), c = Factor<RP, NT>::rank(tid);
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < NW; ++q) s += ((const float*)tile[buf][q])[row * kDv + c];
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(scale * s), dst,
                                              off + i * (NT / RP * 4) * (uint32_t)stride, 0, 0);
      }
      row0 = row1;
      rows = rows1;
      row1 = row2;
      rows1 = rows2;
    };
    // by twos: left in the middle, the loop would wait for all loads at its head
    while (rows1 > 0) {
      step(0, xa, va, vb);
      step(1, xb, vb, va);
    }
    if (rows > 0) step(0, xa, va, vb);
    // all of the old gradient (a part has none: zeros) is read before any is
    // written: one latency
    const bool add = part < 0;
    const long matrix = (long)out_features * stride;
    float* sums = add ? db + slot * matrix : db_part + part * matrix;
    const int cols_left = min(128, out_features - c0);
    const Buf dst = rows_of(sums, c0, stride, cols_left, r), src = rows_of(sums, c0, stride, add ? cols_left : 0, r);
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const uint32_t off = col_off<float>(32 * g, stride, 16 * q + m, r);
      float old[8][4];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) old[j][e] = buf_ldf(src, off + (8 * e + j) * 4 * (uint32_t)stride);
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(old[j][e] + scale * acc[j][q][e]), dst,
                                                off + (8 * e + j) * 4 * (uint32_t)stride, 0, 0);
    }
  });
}

// dv: the column blocks' parts added, into the first of them.
__global__ void __launch_bounds__(kThreads) dv_sum_kernel(float* dv_part, int parts, long n) {
  const long e = ((long)blockIdx.x * kThreads + threadIdx.x) * 4;
  if (e >= n) return;  // n is a multiple of 8
  f32x4 s = *reinterpret_cast<const f32x4*>(dv_part + e);
#pragma unroll 4
  for (int q = 1; q < parts; ++q) s += *reinterpret_cast<const f32x4*>(dv_part + q * n + e);
  *reinterpret_cast<f32x4*>(dv_part + e) = s;
}

// dx and dA (or a part of it); dv is the sum of `parts` parts.  As bwd_out, without a sum over the waves: a
// wave's columns are its own.
template <typename T, int RT, bool STREAM>
__global__ void __launch_bounds__(kThreads, (sizeof(T) == 2 && RT <= 2 ? 2 : 1))
    bwd_in_kernel(Segs t, Slots sl, const T* x, long ldx, const T* a, const float* dv, int parts, long apart, int r,
                  int in, const T* dres, long lddr, T* dx, long lddx, float* da, float* da_part) {
  constexpr int RP = 16 * RT, NP = kParts<T>;
  using U = Up<T, RP>;
  __shared__ __align__(16) T wt[2][NP * RP * kTokStride];
  __shared__ __align__(16) T wr[2][kStep * U::stride];
  constexpr bool kTurned = sizeof(T) == 2;
  constexpr int kTurnedRow = RP + 8;
  __shared__ __align__(16) T aw[kTurned ? kInCols * kTurnedRow : 8];
  const int cols = (in + kInCols - 1) / kInCols;
  const int worker = blockIdx.x / cols, cb = blockIdx.x - worker * cols;
  for_slots(t, sl, worker, [&](Walk& wk, int slot, int part) {
    int tid = threadIdx.x;
    settle(tid);  // as in bwd_out
    const int lane = tid & 63, w = uniform(tid >> 6), m = lane & 15, g = lane >> 4;
    const int c0 = cb * kInCols + 128 * w;
    const bool live = slot >= 0;
    if (!live && (!dx || dx == dres)) return;
    int row0, row1 = 0;
    int rows = wk.next(t, &row0), rows1 = 0;
    Vec8<T> xr[8], xt[8];
    Factor<RP, kThreads> vn;
    auto stage = [&](T* turned, T* in_rows) {
#pragma unroll
      for (int i = 0; i < Factor<RP, kThreads>::n; ++i) {
        const int row = Factor<RP, kThreads>::row(tid, i), c = Factor<RP, kThreads>::rank(tid);
        split_each<NP, T>(vn.f[i], [&](int p, T part) { turned[(p * RP + c) * kTokStride + row] = part; });
        split_each<U::parts, T>(vn.f[i], [&](int p, T part) { in_rows[row * U::stride + p * RP + c] = part; });
      }
    };
    if (live) {
      vn.load(dv, row0, rows, r, r, tid, RT <= 2 ? parts : 1, apart);
      load_tile(xr, x, ldx, row0, rows, c0, in, m, g);
    }
    // A as the first operand of dx = dv A, columns as in `up`: bf16, turned to
    // [column][rank] in LDS (in registers it would cost a second wave a SIMD);
    // fp32, in registers (it would not fit LDS)
    frag_t<T> wf[kTurned ? 1 : 2][4][U::weights];
    if constexpr (!kTurned) {
      const Buf ab = rows_of(live ? a : nullptr, (long)slot * r, in, r, in);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = c0 + 64 * h + up_col(q, m);
#pragma unroll
          for (int s = 0; s < U::weights; ++s) {
            const uint32_t off = U::live(s, g) ? col_off<T>(U::rank(s, g), in, col, in) : kNowhere;
#pragma unroll
            for (int e = 0; e < 8; ++e) wf[h][q][s][e] = buf_ld1(ab, off + e * (uint32_t)(in * sizeof(T)), (T*)nullptr);
          }
        }
    }
    f32x4 acc[8][RT];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int q = 0; q < RT; ++q) acc[j][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    lds_barrier();  // the slot before has read what LDS holds
    if (live) {
      stage(wt[0], wr[0]);
      if constexpr (kTurned) {
        // lanes along the ranks: along the columns their writes would meet in two banks
        const Buf ar = rows_of(a, (long)slot * r, in, r, in);
        constexpr int kAt = kThreads / RP;  // groups of eight columns a pass
#pragma unroll
        for (int i = 0; i < kInCols / 8; i += 4 * kAt) {
          Vec8<T> f[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            buf_ld8(f[u], ar, col_off<T>(tid % RP, in, cb * kInCols + 8 * (i + u * kAt + tid / RP), in));
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const auto e = f[u].frag();
#pragma unroll
            for (int j = 0; j < 8; ++j) aw[(8 * (i + u * kAt + tid / RP) + j) * kTurnedRow + tid % RP] = e[j];
          }
        }
      }
    }
    lds_barrier();
    uint32_t ro[2][2], xo[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        ro[h][u] = col_off<T>(line_row<T>(u, m), lddr, c0 + 64 * h + line_col<T>(u, m, g), in);
        xo[h][u] = col_off<T>(line_row<T>(u, m), lddx, c0 + 64 * h + line_col<T>(u, m, g), in);
      }
    const uint32_t rrow = 16 * sizeof(T) * (uint32_t)lddr, xrow = 16 * sizeof(T) * (uint32_t)lddx;
    for (int buf = 0;; buf ^= 1) {
      const bool more = wk.step < wk.end;
      // what this step adds to, then what the next one takes
      const Buf rb = rows_of(dx ? dres : nullptr, row0, lddr, rows, in), xb = rows_of(dx, row0, lddx, rows, in);
      Vec8<T> bs[2][2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int u = 0; u < 2; ++u) buf_ld8<STREAM ? kOnce : 0>(bs[h][i][u], rb, ro[h][u] + i * rrow);
      if (live) transpose8x8(xr, xt);
      if (more) {
        rows1 = wk.next(t, &row1);
        if (live) {
          vn.load(dv, row1, rows1, r, r, tid, RT <= 2 ? parts : 1, apart);
          load_tile(xr, x, ldx, row1, rows1, c0, in, m, g);
        }
      }
      if (live) outer<T, RT>(acc, xt, wt[buf], m, g, [] {});
      if (dx) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          Vec8<T> f[U::steps];
          if (live) {
#pragma unroll
            for (int s = 0; s < U::steps; ++s) {
              if (U::live(s, g)) f[s].load(wr[buf] + (16 * i + m) * U::stride + 8 * U::chunk(s, g));
              else f[s].zero();
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            f32x4 d[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) d[q] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (live) {
              if constexpr (kTurned) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                  for (int s = 0; s < U::weights; ++s) {
                    Vec8<T> wv;
                    wv.load(aw + (128 * w + 64 * h + up_col(q, m)) * kTurnedRow + U::rank(s, g));
#pragma unroll
                    for (int p = s; p < U::steps; p += U::weights) d[q] = mma16(wv.frag(), f[p].frag(), d[q]);
                  }
              } else {
#pragma unroll
                for (int s = 0; s < U::steps; ++s)
#pragma unroll
                  for (int q = 0; q < 4; ++q) d[q] = mma16(wf[h][q][s % U::weights], f[s].frag(), d[q]);
              }
            }
            turn(bs[h][i][0], bs[h][i][1], m >= 8);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              float o[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] = bs[h][i][u].get(e) + d[2 * u + (e >> 2)][e & 3];
              bs[h][i][u].set(o);
            }
            turn(bs[h][i][0], bs[h][i][1], m >= 8);
#pragma unroll
            for (int u = 0; u < 2; ++u) buf_st8<STREAM ? kOnce : 0>(bs[h][i][u], xb, xo[h][u] + i * xrow);
          }
        }
      }
      if (!more) break;
      if (live) stage(wt[buf ^ 1], wr[buf ^ 1]);
      lds_barrier();
      row0 = row1;
      rows = rows1;
    }
    if (!live) return;
    const bool add = part < 0;
    float* sums = add ? da + (long)slot * r * in : da_part + (long)part * r * in;
    const Buf dst = rows_of(sums, 0, in, r, in), src = rows_of(sums, 0, in, add ? r : 0, in);
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      Vec8<float> o[4];
      uint32_t off[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        off[e] = 16 * q + m < r ? col_off<float>(16 * q + m, in, c0 + 8 * (4 * g + e), in) : kNowhere;
        buf_ld8(o[e], src, off[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = o[e].get(j) + acc[j][q][e];
        o[e].set(s);
        buf_st8(o[e], dst, off[e]);
      }
    }
  });
}

// out[slot] += the parts of its workers, in order; n elements a slot.
// blockIdx.y: the slot's place in the table; .z: which of two.
struct Join {
  Slots sl;
  const float* part;
  float* out;
  long n;
};
__device__ __forceinline__ void join(const Join& j) {
  const int k = blockIdx.y;
  const long e = ((long)blockIdx.x * kThreads + threadIdx.x) * 4;
  if (k >= j.sl.count || j.sl.slot[k] < 0 || e >= j.n) return;
  const int count = j.sl.worker(j.sl.step0[k + 1] - 1) - j.sl.worker(j.sl.step0[k]);
  if (count == 0) return;
  const float* src = j.part + j.sl.part0[k] * j.n + e;
  f32x4* dst = reinterpret_cast<f32x4*>(j.out + j.sl.slot[k] * j.n + e);
  f32x4 s = *dst;
#pragma unroll 4
  for (int i = 0; i < count; ++i) s += *reinterpret_cast<const f32x4*>(src + i * j.n);
  *dst = s;
}
__global__ void __launch_bounds__(kThreads) join_kernel(Join ja, Join jb) {
  if (blockIdx.z) join(jb);
  else join(ja);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || !na || !nb) return false;
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
int launch_status() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FL_OK : set_error(FL_ERR_HIP, hipGetErrorString(e));
}
long cdiv(long a, long b) { return (a + b - 1) / b; }

constexpr long kCus = 256;

struct Run {
  int row0, rows, slot;
};
// Runs of rows with one slot, in row order (adjacent clients of one slot make
// one run); by_slot: sorted by slot, rows in order within it.
int runs_of(const fl_batch_desc* b, const int32_t* client_adapter, bool by_slot, std::vector<Run>* out) {
  try {
    out->reserve(b->num_clients);
    for (int c = 0; c < b->num_clients; ++c) {
      const int r0 = b->cu_seqlens[b->client_seq_ptr[c]], r1 = b->cu_seqlens[b->client_seq_ptr[c + 1]];
      if (!out->empty() && out->back().slot == client_adapter[c]) out->back().rows += r1 - r0;
      else out->push_back({r0, r1 - r0, client_adapter[c]});
    }
    if (by_slot) {
      std::sort(out->begin(), out->end(),
                [](const Run& x, const Run& y) { return x.slot != y.slot ? x.slot < y.slot : x.row0 < y.row0; });
    }
  } catch (const std::bad_alloc&) {
    return set_error(FL_ERR_NOMEM, "out of host memory for the table of clients");
  }
  return FL_OK;
}

// The next launch's segments from runs[i] on.
void fill(const std::vector<Run>& runs, size_t* i, int rows_a_step, Segs* t) {
  t->count = 0;
  int32_t steps = 0;
  for (; *i < runs.size() && t->count < kSegs; ++*i) {
    const Run& q = runs[*i];
    t->row0[t->count] = q.row0;
    t->rows[t->count] = q.rows;
    t->slot[t->count] = q.slot;
    t->step0[t->count++] = steps;
    steps += (int32_t)cdiv(q.rows, rows_a_step);
  }
  t->step0[t->count] = steps;
}

// Forward: workgroups along the reduction of v, for batches whose tiles alone
// do not fill the chip; every wave has a step at least.  `up` adds the parts in
// every block of columns, four loads at a time, which is why they are few and 5
// to 7 cost as much as 8.  (4096 -> 4096, rank 64, 512 rows: 4 parts 18.5 us, 8
// parts 16.6, 16 parts 19.2; 41 tiles: 6 and 4 parts 28.3 and 27.1; 94 tiles: 2
// and 4 parts 42.4 and 49.9; 128 tiles: none and 2 parts 61.8 and 50.3.  4096 ->
// 12288, rank 16, 64 tiles: 3, 4 and 7 parts 44.0, 42.9 and 45.5, of one token
// each 15.9, 15.0 and 16.7.  Where the width allows no more than 5 to 7, they are
// taken: 1280 -> 3840, 23 tiles, 5 and 4 parts 15.4 and 15.7.)  The tiles are those
// launched, of runs of clients with one slot: 256 clients of one token and one
// slot, 4 tiles, 21.8 us a call, without parts 28.0.
int splits_of(const fl_adapter_desc* d, long tiles) {
  long parts = kCus / tiles;
  if (parts > 4 && parts < 8) parts = 4;
  return (int)std::max(1L, std::min<long>({parts, d->in_features / (64 * kWaves), 8}));
}
// Whether operands of this width pass the last-level cache by: from a size on
// that it would not hold for an output's reader, or for the backward; dx in place,
// whose old values may be in the cache, from twice that size on.  (4096 <-> 12288,
// rank 16, the kernels with a scaling of the output behind them: y of 192 MB 234
// us, past the cache 227, of 96 MB 82 and 81, of 48 MB 43 and 48; dx of 128 MB 232
// and 226, of 64 MB 121 and 124; dx of 340 MB, alone, 438 and 412; x of 340 MB, the
// forward alone, 424 and 418.  In place, with a write of the old values before them
// too: y of 96 MB 113 and 112, of 192 MB 220 and 212, of 340 MB 386 and 373; dx of
// 96 MB 204 and 210, of 128 MB 257 and 264, of 192 MB 371 and 373, of 256 MB 492 and
// 491, of 340 MB 642 and 631.)
bool streams(const fl_adapter_desc* d, long rows, int width, bool in_place_dx = false) {
  return d->dtype == FL_BF16 && (size_t)rows * width * 2 >= (in_place_dx ? 2 * kStreamBytes : kStreamBytes);
}
// Backward: columns of a workgroup of bwd_out (OutWaves).
long out_cols(const fl_adapter_desc* d) {
  return cdiv(d->out_features, 128 * (d->dtype == FL_BF16 ? OutWaves<bf16>::n : OutWaves<float>::n));
}
int out_slices(const fl_adapter_desc* d) { return d->rank > 32 ? 2 : 1; }
long in_cols(const fl_adapter_desc* d) { return cdiv(d->in_features, kInCols); }
// Backward: workers that share the steps, for each block of columns; the chip
// holds one workgroup of bwd_out a CU, two of bwd_in (one for ranks past 32 and
// in fp32).
long out_workers(const fl_adapter_desc* d) { return std::max(1L, kCus / (out_cols(d) * out_slices(d))); }
long in_workers(const fl_adapter_desc* d) {
  return std::max(1L, kCus * (d->dtype == FL_BF16 && d->rank <= 32 ? 2 : 1) / in_cols(d));
}
// Shares the steps from the first of a slot >= first_slot on out among
// `workers`; returns their number, and the number of parts.
int share_out(const Segs& t, int first_slot, long workers, Slots* sl, int* parts) {
  sl->count = 0;
  sl->base = -1;
  for (int k = 0; k < t.count; ++k) {
    if (t.slot[k] < first_slot || (sl->count && sl->slot[sl->count - 1] == t.slot[k])) continue;
    if (sl->base < 0) sl->base = t.step0[k];
    sl->slot[sl->count] = t.slot[k];
    sl->step0[sl->count++] = t.step0[k];
  }
  *parts = 0;
  if (!sl->count) return 0;
  const int end = t.step0[t.count], steps = end - sl->base;
  sl->step0[sl->count] = end;
  sl->share = (int)cdiv(steps, workers);
  for (int k = 0; k < sl->count; ++k) {
    sl->part0[k] = *parts;
    if (sl->slot[k] >= 0) *parts += sl->worker(sl->step0[k + 1] - 1) - sl->worker(sl->step0[k]);
  }
  return (int)cdiv(steps, sl->share);
}

struct AdapterWs {
  float* v_part;   // forward: [splits][T][r]
  float* dv_part;  // backward: [column blocks of out][T][r]
  float *da_part, *db_part;
  size_t total;
};
AdapterWs carve(const fl_adapter_desc* d, const fl_batch_desc* b, char* base) {
  AdapterWs w;
  size_t off = 0;
  auto take = [&](size_t n) {
    float* p = base ? (float*)(base + off) : nullptr;
    off = align256(off + n);
    return p;
  };
  const size_t v = (size_t)b->total_tokens * d->rank * 4;
  // (the slots are not known here: as many parts as any table of them gives, all
  // clients' rows being one run of one slot)
  const int splits = splits_of(d, cdiv(b->total_tokens, kTile));
  w.v_part = take(splits > 1 ? splits * v : 0);
  const size_t fwd = off;
  off = 0;
  w.dv_part = take(out_cols(d) * v);
  // at most one part for each boundary between workers
  w.da_part = take((in_workers(d) - 1) * d->rank * d->in_features * 4);
  w.db_part = take((out_workers(d) - 1) * d->rank * d->out_features * 4);
  w.total = std::max(std::max(fwd, off), (size_t)256);
  return w;
}

int check_desc(const fl_adapter_desc* d) {
  if (!d) return set_error(FL_ERR_NULL, "adapter descriptor is NULL");
  if (d->dtype != FL_BF16 && d->dtype != FL_F32) return set_error(FL_ERR_SHAPE, "dtype must be bf16 or fp32");
  if (d->num_adapters < 1 || d->num_adapters > (1 << 16))
    return set_error(FL_ERR_SHAPE, "num_adapters must be in [1, 2^16]");
  if (d->rank < 8 || d->rank > 64 || d->rank % 8)
    return set_error(FL_ERR_SHAPE, "rank must be a multiple of 8 in [8, 64]");
  for (int n : {d->in_features, d->out_features})
    if (n < 8 || n % 8 || n > 65536) return set_error(FL_ERR_SHAPE, "features must be multiples of 8 in [8, 65536]");
  if (!std::isfinite(d->scale)) return set_error(FL_ERR_ARG, "scale is not finite");
  return FL_OK;
}
// One [T, ld] operand of `width` columns.
struct Mat {
  const void* p;
  int64_t ld;
  int width;
  size_t bytes(size_t T, size_t E) const { return p ? ((T - 1) * ld + width) * E : 0; }
};
// Whether two operands share an element: column ranges of one wider buffer
// (equal row strides, no row of one reaching into the other's columns) do not.
bool overlap(const Mat& a, const Mat& b, size_t T, size_t E) {
  if (!overlap(a.p, a.bytes(T, E), b.p, b.bytes(T, E))) return false;
  if (a.ld != b.ld) return true;
  const size_t ld = (size_t)a.ld * E;
  const size_t off = ((uintptr_t)b.p % ld + ld - (uintptr_t)a.p % ld) % ld;  // b's first column behind a's
  return off < a.width * E || off + b.width * E > ld;
}
int check_mat(const Mat& m, bool required) {
  if (!m.p) return required ? set_error(FL_ERR_NULL, "a matrix argument is NULL") : FL_OK;
  if (!al16(m.p)) return set_error(FL_ERR_ALIGN, "a matrix argument is not 16-byte aligned");
  if (m.ld < m.width || m.ld % 8 || m.ld > kMaxStride)
    return set_error(FL_ERR_SHAPE, "a row stride must be a multiple of 8, at least the row's width and at most 2^22");
  return FL_OK;
}

// Calls f.template operator()<T, RT>() for the call's type and rank.
template <typename F>
int dispatch(const fl_adapter_desc* d, F&& f) {
  const int rt = d->rank <= 16 ? 1 : d->rank <= 32 ? 2 : 4;
  if (d->dtype == FL_BF16) {
    if (rt == 1) return f((bf16*)nullptr, std::integral_constant<int, 1>());
    if (rt == 2) return f((bf16*)nullptr, std::integral_constant<int, 2>());
    return f((bf16*)nullptr, std::integral_constant<int, 4>());
  }
  if (rt == 1) return f((float*)nullptr, std::integral_constant<int, 1>());
  if (rt == 2) return f((float*)nullptr, std::integral_constant<int, 2>());
  return f((float*)nullptr, std::integral_constant<int, 4>());
}

}  // namespace

namespace flglm {

int adapter_check(const fl_adapter_desc* d, const fl_batch_desc* b, const int32_t* client_adapter, const void* ws,
                  size_t ws_bytes) {
  if (int rc = check_desc(d)) return rc;
  if (int rc = check_batch(b)) return rc;
  if (!client_adapter || !ws) return set_error(FL_ERR_NULL, "client_adapter / workspace is NULL");
  for (int c = 0; c < b->num_clients; ++c)
    if (client_adapter[c] < -1 || client_adapter[c] >= d->num_adapters)
      return set_error(FL_ERR_ARG, "a client's adapter is outside [-1, num_adapters)");
  if (!al16(ws)) return set_error(FL_ERR_ALIGN, "workspace is not 16-byte aligned");
  if (ws_bytes < carve(d, b, nullptr).total) return set_error(FL_ERR_WORKSPACE, "workspace too small");
  return FL_OK;
}
int adapter_workspace_bytes(const fl_adapter_desc* d, const fl_batch_desc* b, size_t* bytes) {
  if (int rc = check_desc(d)) return rc;
  if (int rc = check_batch(b)) return rc;
  *bytes = carve(d, b, nullptr).total;
  return FL_OK;
}

int adapter_forward(const fl_adapter_desc* d, const fl_batch_desc* batch, const int32_t* client_adapter, const void* x,
                    int64_t ldx, const void* a, const void* b, const void* base, int64_t ld_base, void* y, int64_t ldy,
                    float* v, void* ws, hipStream_t s) {
  std::vector<Run> runs;
  if (int rc = runs_of(batch, client_adapter, false, &runs)) return rc;
  const AdapterWs w = carve(d, batch, (char*)ws);
  long tiles = 0;
  for (const Run& q : runs) tiles += cdiv(q.rows, kTile);
  const int splits = splits_of(d, tiles);
  const long T = batch->total_tokens;
  const long cols = cdiv(d->out_features, kUpCols);
  const bool past_cache = streams(d, T, d->out_features);
  for (size_t i = 0; i < runs.size();) {
    Segs t;
    fill(runs, &i, kTile, &t);
    const int rc = dispatch(d, [&](auto* type, auto rt) {
      using E = std::remove_pointer_t<decltype(type)>;
      constexpr int RT = decltype(rt)::value;
      const auto down = streams(d, T, d->in_features) ? down_kernel<E, RT, kLines<E>> : down_kernel<E, RT, false>;
      hipLaunchKernelGGL(down, dim3(t.step0[t.count], splits), dim3(kThreads), 0, s, t, (const E*)x,
                         ldx, (const E*)a, d->rank, d->in_features, splits > 1 ? w.v_part : v, T);
      if (int e = launch_status()) return e;
      const auto up = past_cache ? up_kernel<E, 16 * RT, kLines<E>> : up_kernel<E, 16 * RT, false>;
      hipLaunchKernelGGL(up, dim3((unsigned)(t.step0[t.count] * cols)), dim3(kThreads), 0, s, t,
                         splits > 1 ? w.v_part : v, splits, T, v, (const E*)b, d->rank, d->out_features, d->scale,
                         (const E*)base, ld_base, (E*)y, ldy);
      return launch_status();
    });
    if (rc) return rc;
  }
  return FL_OK;
}

int adapter_backward(const fl_adapter_desc* d, const fl_batch_desc* batch, const int32_t* client_adapter,
                     const void* dy, int64_t ld_dy, const void* x, int64_t ldx, const void* a, const void* b,
                     const float* v, const void* dres, int64_t ld_dres, void* dx, int64_t ld_dx, float* da, float* db,
                     void* ws, hipStream_t s) {
  std::vector<Run> runs;
  if (int rc = runs_of(batch, client_adapter, true, &runs)) return rc;
  const AdapterWs w = carve(d, batch, (char*)ws);
  const long T = batch->total_tokens;
  const long na = (long)d->rank * d->in_features, nb = (long)d->rank * d->out_features;
  const long cols_in = in_cols(d), cols_out = out_cols(d);
  const bool past_cache = streams(d, T, d->in_features, dx && dx == dres);
  // dv's parts, when few and short, are added where they are read: a launch less
  // (4096 -> 4096, rank 16, 64 rows 20.4 -> 19.2 us, 1024 rows 36.6 -> 35.0; 4096
  // rows 54.8 -> 55.3, and 12 parts of 40583 rows 409 -> 433; past rank 32 the code
  // for it costs the long batches 2 %)
  const bool few = cols_out <= 4 && T <= 1024 && d->rank <= 32;
  const bool one = runs.size() <= kSegs;  // one table holds the batch: dA's and dB's parts are joined in one launch
  auto join = [&](const Join& j, const Join* other) {
    const long n = std::max(j.n, other ? other->n : 0);
    const dim3 grid((unsigned)cdiv(n, 4 * kThreads), std::max(j.sl.count, other ? other->sl.count : 0), other ? 2 : 1);
    hipLaunchKernelGGL(join_kernel, grid, dim3(kThreads), 0, s, j, other ? *other : j);
    return launch_status();
  };
  Slots so, si;
  int parts_out = 0, parts_in = 0;
  bool any = false;
  for (size_t i = 0; i < runs.size();) {
    Segs t;
    fill(runs, &i, kStep, &t);
    const int workers = share_out(t, 0, out_workers(d), &so, &parts_out);
    if (!workers) continue;
    any = true;
    const int rc = dispatch(d, [&](auto* type, auto rt) {
      using E = std::remove_pointer_t<decltype(type)>;
      constexpr int RT = decltype(rt)::value;
      const int groups = (int)(workers * cols_out), slices = out_slices(d);
      hipLaunchKernelGGL((bwd_out_kernel<E, (RT < 2 ? RT : 2)>),
                         dim3((unsigned)(slices == 1 ? groups : cdiv(groups, 8) * 16)),
                         dim3(64 * OutWaves<E>::n), 0, s, t, so, (const E*)dy, ld_dy, (const E*)b, v, d->rank,
                         d->out_features, d->scale, w.dv_part, T, db, w.db_part, groups, slices);
      return launch_status();
    });
    if (rc) return rc;
    if (!one && parts_out) {  // the next launch writes its own parts there
      if (int e = join(Join{so, w.db_part, db, nb}, nullptr)) return e;
    }
  }
  if (any && cols_out > 1 && !few) {  // (of all launches at once: each row's parts are added a single time)
    hipLaunchKernelGGL(dv_sum_kernel, dim3((unsigned)cdiv(T * d->rank, 4 * kThreads)), dim3(kThreads), 0, s, w.dv_part,
                       (int)cols_out, T * d->rank);
    if (int e = launch_status()) return e;
  }
  for (size_t i = 0; i < runs.size();) {
    Segs t;
    fill(runs, &i, kStep, &t);
    const int workers = share_out(t, -1, in_workers(d), &si, &parts_in);
    const int rc = dispatch(d, [&](auto* type, auto rt) {
      using E = std::remove_pointer_t<decltype(type)>;
      constexpr int RT = decltype(rt)::value;
      const auto in = past_cache ? bwd_in_kernel<E, RT, kLines<E>> : bwd_in_kernel<E, RT, false>;
      hipLaunchKernelGGL(in, dim3((unsigned)(workers * cols_in)), dim3(kThreads), 0, s, t, si, (const E*)x, ldx,
                         (const E*)a, w.dv_part, few ? (int)cols_out : 1, T * d->rank, d->rank, d->in_features,
                         (const E*)dres, ld_dres, (E*)dx, ld_dx, da, w.da_part);
      return launch_status();
    });
    if (rc) return rc;
    if (parts_in || (one && parts_out)) {
      const Join jb{so, w.db_part, db, nb};
      if (int e = join(Join{si, w.da_part, da, na}, one ? &jb : nullptr)) return e;
    }
  }
  return FL_OK;
}

}  // namespace flglm

extern "C" {

int fl_adapter_workspace_bytes(const fl_adapter_desc* desc, const fl_batch_desc* batch, size_t* bytes) {
  if (!bytes) return set_error(FL_ERR_NULL, "bytes is NULL");
  return adapter_workspace_bytes(desc, batch, bytes);
}

int fl_adapter_forward(const fl_adapter_desc* desc, const fl_batch_desc* batch, const int32_t* client_adapter,
                       const void* x, int64_t ldx, const void* a, const void* b, const void* base, int64_t ld_base,
                       void* y, int64_t ldy, float* v, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = adapter_check(desc, batch, client_adapter, workspace, workspace_bytes)) return rc;
  const int in = desc->in_features, out = desc->out_features;
  const Mat mx{x, ldx, in}, mb{base, ld_base, out}, my{y, ldy, out};
  if (int rc = check_mat(mx, true)) return rc;
  if (int rc = check_mat(my, true)) return rc;
  if (int rc = check_mat(mb, false)) return rc;
  if (!a || !b || !v) return set_error(FL_ERR_NULL, "a / b / v is NULL");
  if (!al16(a) || !al16(b) || !al16(v)) return set_error(FL_ERR_ALIGN, "a / b / v not 16-byte aligned");
  const size_t T = batch->total_tokens, E = desc->dtype == FL_BF16 ? 2 : 4, n = desc->num_adapters;
  const size_t na = n * desc->rank * in * E, nb = n * desc->rank * out * E, nv = T * desc->rank * 4;
  if (overlap(my, mb, T, E) && !(y == base && ldy == ld_base))
    return set_error(FL_ERR_ALIAS, "y overlaps base without being it");
  if (overlap(my, mx, T, E)) return set_error(FL_ERR_ALIAS, "y overlaps x");
  const void* p[7] = {x, base, y, a, b, v, workspace};
  const size_t len[7] = {mx.bytes(T, E), mb.bytes(T, E), my.bytes(T, E), na, nb, nv, workspace_bytes};
  for (int i = 0; i < 7; ++i)
    for (int j = std::max(i + 1, 3); j < 7; ++j)  // a and b may share memory with x and base, all being read
      if ((j >= 5 || i == 2) && overlap(p[i], len[i], p[j], len[j]))
        return set_error(FL_ERR_ALIAS, "y, v or the workspace overlaps another argument");
  return adapter_forward(desc, batch, client_adapter, x, ldx, a, b, base, ld_base, y, ldy, v, workspace,
                         (hipStream_t)stream);
}

int fl_adapter_backward(const fl_adapter_desc* desc, const fl_batch_desc* batch, const int32_t* client_adapter,
                        const void* dy, int64_t ld_dy, const void* x, int64_t ldx, const void* a, const void* b,
                        const float* v, const void* dres, int64_t ld_dres, void* dx, int64_t ld_dx, float* da,
                        float* db, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = adapter_check(desc, batch, client_adapter, workspace, workspace_bytes)) return rc;
  const int in = desc->in_features, out = desc->out_features;
  const Mat mdy{dy, ld_dy, out}, mx{x, ldx, in}, mr{dres, ld_dres, in}, mdx{dx, ld_dx, in};
  if (int rc = check_mat(mdy, true)) return rc;
  if (int rc = check_mat(mx, true)) return rc;
  if (int rc = check_mat(mr, false)) return rc;
  if (int rc = check_mat(mdx, false)) return rc;
  if (dres && !dx) return set_error(FL_ERR_NULL, "dres without dx");
  if (!a || !b || !v || !da || !db) return set_error(FL_ERR_NULL, "a / b / v / da / db is NULL");
  if (!al16(a) || !al16(b) || !al16(v) || !al16(da) || !al16(db))
    return set_error(FL_ERR_ALIGN, "a / b / v / da / db not 16-byte aligned");
  const size_t T = batch->total_tokens, E = desc->dtype == FL_BF16 ? 2 : 4, n = desc->num_adapters;
  const size_t na = n * desc->rank * in, nb = n * desc->rank * out;
  if (overlap(mdx, mr, T, E) && !(dx == dres && ld_dx == ld_dres))
    return set_error(FL_ERR_ALIAS, "dx overlaps dres without being it");
  if (overlap(mdx, mx, T, E) || overlap(mdx, mdy, T, E)) return set_error(FL_ERR_ALIAS, "dx overlaps x or dy");
  const void* p[10] = {dy, x, dres, dx, a, b, v, da, db, workspace};
  const size_t len[10] = {mdy.bytes(T, E), mx.bytes(T, E), mr.bytes(T, E), mdx.bytes(T, E), na * E, nb * E,
                          T * desc->rank * 4, na * 4, nb * 4, workspace_bytes};
  for (int i = 0; i < 10; ++i)
    for (int j = std::max(i + 1, 4); j < 10; ++j)  // what is only read may share memory
      if ((j >= 7 || i == 3) && overlap(p[i], len[i], p[j], len[j]))
        return set_error(FL_ERR_ALIAS, "dx, da, db or the workspace overlaps another argument");
  return adapter_backward(desc, batch, client_adapter, dy, ld_dy, x, ldx, a, b, v, dres, ld_dres, dx, ld_dx, da, db,
                          workspace, (hipStream_t)stream);
}

}  // extern "C"
