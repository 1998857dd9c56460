// Preference loss over pairs of packed sequences, and its gradient.
//
// Sequence 2p of the batch is the preferred answer of pair p, sequence 2p + 1
// the rejected one.  With x_t the logits of row t, over the labelled rows of
// a sequence s
//   l_s = sum_t x_t[label_t] - logsumexp(x_t),
//   z_p = beta ((l_2p - ref_2p) - (l_2p+1 - ref_2p+1)),
//   L_p = (1 - eps) softplus(-z_p) + eps softplus(z_p),
// and with k_s = beta dL_p/dz_p for the preferred, -k for the rejected one,
//   dlogits_t = grad_scale k_s (onehot(label_t) - softmax(x_t)).
//
// The logits are read once for the loss and once for the gradient: k_s hangs
// on whole sequences, so no row's gradient is known before the last row of
// its pair has been read.  Rows without a label are read in neither.
//
//  * row kernel: the running maximum and sum of exponentials of a row's
//    columns; a row is split over several workgroups when rows are few.
//  * pair kernel: one workgroup a pair joins the parts of its rows, forms the
//    sequence sums, the loss and each row's factors.  The last pair to finish
//    adds the losses in pair order.
//  * gradient kernel: one pass over the logits.
//
// Measured on one MI355X, 8 pairs, 4910 rows of which 3671 carry a label, 130528
// bf16 columns: row 168 us (0.96 GB, 5.7 TB/s; bound by the reads), pair 12 us
// (8 workgroups' latency of a few dependent loads), gradient 395 us (0.96 GB
// read, 1.28 GB written, 5.7 TB/s).
//
// Sums of exponentials are fp32 (values in [0, 1] but for the rounding of the
// maximum, at most 2^24 of them, added in parts); log-probabilities and their
// sums over a sequence are 64 bits, because z is a difference of sums of hundreds
// of rows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/flglm.h"
#include "common.h"
#include "kernels.h"

using namespace flglm;

namespace {

constexpr int kThreads = 256;
constexpr double kLog2e64 = 1.44269504088896340736, kLn2 = 1.0 / kLog2e64;
constexpr float kLog2eLow = (float)(kLog2e64 - (double)kLog2e);  // what the fp32 factor leaves of log2 e
constexpr double kLn2Far = 1.0 / (double)kLog2e;  // of that factor alone, see exp2_far
constexpr int kPairsArg = 128;       // pairs whose bounds travel in one launch's kernel arguments
constexpr int kMaxSplits = 8;        // (one pair, 110 rows of 130528: 8 parts 12.4 us, 16 parts 13.9)
constexpr int kBatch = 2;            // loads of a lane at once
constexpr long kWantGroups = 2048;   // workgroups that fill the chip, four a CU, twice

// Exponentials are powers of two: with M the running maximum of x log2 e, rounded
// up to a whole number and then taken as it is, s = sum of 2^(x log2 e - M), log2 e
// in two parts of fp32, and logsumexp = M ln 2 + ln s.  (Sums of different M are
// joined by powers of two, which are exact: with M between whole numbers, each
// join put the error of an exponential on all that it joined: log-probabilities of
// 130528 columns were off by 1.8e-7, now by 0.8e-7, most of it the rounding of the
// fp32 output.  The fp32 factor
// alone is too small by 1.3e-8 of its size: every logsumexp would be too large by
// that part of the mean distance from the maximum, and a sequence's sum by the sum
// of them.  The second part costs a step of 8 pairs 2 us of 578.)
__device__ __forceinline__ float exp2_less(float x, float M) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2eLow, __builtin_fmaf(x, kLog2e, -M)));
}
// The larger M, the more its rounding moves s: by 2^64 where |M| reaches 2^31,
// and x log2 e overflows for the type's lowest values, with which logits are
// masked.  So in a row whose maximum is past +-kFar, a logit past it counts as
// +-kFar and log2 e is the fp32 factor (a power of two times it: M is exact), and
// a row of nothing but lowest values is uniform.  Below an ordinary maximum such a
// logit gives 2^-infinity = 0 as it is.
__device__ __forceinline__ float exp2_far(float x, float M) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, -M));
}
constexpr float kFar = 0x1p30f;
__device__ __forceinline__ bool far_row(float M) { return fabsf(M) >= kFar * kLog2e; }
__device__ __forceinline__ float saturate(float x) {  // infinities and NaN stay
  return fabsf(x) < INFINITY && fabsf(x) > kFar ? copysignf(kFar, x) : x;
}

// (M, s) pairs; an empty part is (-inf, 0).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  if (m2 == -INFINITY) return;
  if (m == -INFINITY) {
    m = m2;
    s = s2;
    return;
  }
  const float mx = fmaxf(m, m2);
  s = s * __builtin_amdgcn_exp2f(m - mx) + s2 * __builtin_amdgcn_exp2f(m2 - mx);
  m = mx;
}

// Takes 8 N columns into the running (M, s): one new maximum and one rescaling
// for all of them.
template <typename T, int N>
__device__ __forceinline__ void take(float& m, float& s, const Vec8<T> (&v)[N]) {
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int k = 0; k < 8; ++k) top = fmaxf(top, v[u].get(k));
  float mx = fmaxf(m, ceilf(top * kLog2e));
  if (far_row(mx)) {  // nothing but masked columns so far, infinities, or NaN, which a maximum passes over
    mx = fmaxf(m, saturate(top) * kLog2e);
    float sum = 0.f;
    for (int u = 0; u < N; ++u)
      for (int k = 0; k < 8; ++k) {
        const float x = saturate(v[u].get(k));
        if (mx > -INFINITY) sum += exp2_far(x, mx);
        else m = x != x ? x : m;
      }
    if (mx > -INFINITY) {
      s = s * (m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx)) + sum;
      m = mx;
    }
    return;
  }
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k & 3] += exp2_less(v[u].get(k), mx);
  s = s * (m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx)) + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
  m = mx;
}

// Columns [c0, c1) of each labelled row: part[row][split] = (M, s).
// (512 threads a workgroup: one pair 12.4 us, 256 11.7.)
template <typename T>
__global__ void __launch_bounds__(kThreads) pref_row_kernel(const T* logits, long ld, int V, int cols,
                                                            const int32_t* labels, float2* part, uint32_t* done) {
  const long t = blockIdx.x;
  const int sp = blockIdx.y;
  if (t == 0 && sp == 0 && threadIdx.x == 0) *done = 0;  // the pair kernel's count, of the launch behind this one
  const int lab = labels[t];
  if (lab < 0 || lab >= V) return;
  const T* row = logits + t * ld;
  const int c0 = sp * cols, c1 = min(V, c0 + cols);
  float m = -INFINITY, s = 0.f;
  int j0 = c0 + threadIdx.x * 8;
  // whole batches, one loaded while the one before it is taken (8 pairs: 613 us
  // a step, without 622)
  constexpr int kWhole = kBatch * kThreads * 8;
  const int last = c1 - (kBatch - 1) * kThreads * 8;
  if (j0 < last) {
    Vec8<T> va[kBatch], vb[kBatch];  // in turn: moved from one to the other, they would be waited for
    auto load = [&](Vec8<T> (&b)[kBatch]) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) b[u].load(row + j0 + u * kThreads * 8);
      j0 += kWhole;
      __builtin_amdgcn_sched_barrier(0);  // or the loads sink to their uses
    };
    load(va);
    for (;;) {
      if (j0 >= last) {
        take(m, s, va);
        break;
      }
      load(vb);
      take(m, s, va);
      __builtin_amdgcn_sched_barrier(0);
      if (j0 >= last) {
        take(m, s, vb);
        break;
      }
      load(va);
      take(m, s, vb);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  for (; j0 < c1; j0 += kThreads * 8) {
    Vec8<T> v[1];
    v[0].load(row + j0);
    take(m, s, v);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
    join(m, s, m2, s2);
  }
  __shared__ float sm[kThreads / 64], ss[kThreads / 64];
  if ((threadIdx.x & 63) == 0) {
    sm[threadIdx.x >> 6] = m;
    ss[threadIdx.x >> 6] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) join(m, s, sm[w], ss[w]);
    part[t * gridDim.y + sp] = make_float2(m, s);
  }
}

struct PairArgs {
  int32_t cu[2 * kPairsArg + 1];
  int first, count, pairs;  // this launch's pairs [first, first + count) of `pairs`
};

__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) t += sh[w];
  return t;
}

__device__ __forceinline__ double softplus(double u) { return fmax(u, 0.0) + log1p(exp(-fabs(u))); }

// factors[t] = (M, k / s, k, 0): the gradient of row t is k onehot - (k / s)
// 2^(x log2 e - M); k = 0 for a row without a label.
template <typename T>
__global__ void __launch_bounds__(kThreads) pref_pair_kernel(PairArgs a, const T* logits, long ld, int V, int splits,
                                                             const int32_t* labels, const float2* part,
                                                             const float* ref, double beta, double eps, float* logp,
                                                             float* loss, float* loss_sum, f32x4* factors,
                                                             uint32_t* done) {
  __shared__ double sh[kThreads / 64];
  __shared__ bool last;
  const int p = a.first + blockIdx.x;
  const int r0 = a.cu[2 * blockIdx.x], r1 = a.cu[2 * blockIdx.x + 1], r2 = a.cu[2 * blockIdx.x + 2];
  double lp[2] = {0, 0};
  for (int t = r0 + threadIdx.x; t < r2; t += kThreads) {
    const int lab = labels[t];
    f32x4 f = {0.f, 0.f, 0.f, 0.f};
    if (lab >= 0 && lab < V) {
      float x = to_f32(logits[(long)t * ld + lab]), m = -INFINITY, s = 0.f;
#pragma unroll 4
      for (int k = 0; k < splits; ++k) {
        const float2 q = part[(long)t * splits + k];
        join(m, s, q.x, q.y);
      }
      const bool far = far_row(m);
      if (far) x = saturate(x);
      const double l = (double)x - ((double)m * (far ? kLn2Far : kLn2) + log((double)s));
      lp[0] += t < r1 ? l : 0.0;
      lp[1] += t < r1 ? 0.0 : l;
      f[0] = m;
      f[1] = s;
      f[2] = 1.f;
    }
    factors[t] = f;
  }
  lp[0] = block_sum(lp[0], sh);
  lp[1] = block_sum(lp[1], sh);
  double d = lp[0] - lp[1];
  if (ref) d = (lp[0] - (double)ref[2 * p]) - (lp[1] - (double)ref[2 * p + 1]);
  const double z = beta * d;
  // (no 0 times infinity: z is infinite where a label has no probability)
  const double L = (1.0 - eps) * softplus(-z) + (eps > 0.0 ? eps * softplus(z) : 0.0);
  const double k = beta * (eps / (1.0 + exp(-z)) - (1.0 - eps) / (1.0 + exp(z)));
  for (int t = r0 + threadIdx.x; t < r2; t += kThreads) {
    f32x4 f = factors[t];  // this thread's own
    if (f[2] != 0.f) {
      const double kh = t < r1 ? k : -k;
      f[1] = (float)(kh / (double)f[1]);
      f[2] = (float)kh;
      factors[t] = f;
    }
  }
  if (threadIdx.x == 0) {
    logp[2 * p] = (float)lp[0];
    logp[2 * p + 1] = (float)lp[1];
    loss[p] = (float)L;
    last = false;
    if (a.pairs == 1) *loss_sum = (float)L;  // (through the count 1.6 us more)
    else {
      __threadfence();
      last = atomicAdd(done, 1u) == (uint32_t)(a.pairs - 1);
    }
  }
  __syncthreads();
  if (!last) return;
  // every pair's loss is written: added in pair order, whichever came last
  __threadfence();
  double sum = 0;
  for (int i = threadIdx.x; i < a.pairs; i += kThreads)
    sum += (double)__hip_atomic_load(loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sum = block_sum(sum, sh);
  if (threadIdx.x == 0) *loss_sum = (float)sum;
}

__device__ __forceinline__ void store_nt(bf16* p, const Vec8<bf16>& v) {
  __builtin_nontemporal_store(v.r, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store_nt(float* p, const Vec8<float>& v) {
  __builtin_nontemporal_store(v.r0, reinterpret_cast<u32x4*>(p));
  __builtin_nontemporal_store(v.r1, reinterpret_cast<u32x4*>(p + 4));
}

// The first `width` columns of dlogits (past V: 0) of row t; may be the logits
// themselves.  2048 columns a workgroup, so that the chip sweeps through
// memory in order, and from the last row to the first: what the row kernel
// read last is in the last-level cache.  STREAM: the stores are non-temporal.
template <typename T, bool STREAM>
__global__ void __launch_bounds__(kThreads) pref_grad_kernel(const T* logits, long ld, int V, const int32_t* labels,
                                                             const f32x4* factors, float scale, T* dlogits, long ldd,
                                                             int width, int blocks) {
  const uint32_t i = gridDim.x - 1 - blockIdx.x;
  const long t = i / (uint32_t)blocks;
  const int j0 = ((int)(i % (uint32_t)blocks) * kThreads + threadIdx.x) * 8;
  if (j0 >= width) return;
  const int lab = labels[t];
  Vec8<T> v;
  float g[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) g[k] = 0.f;
  if (lab >= 0 && lab < V && j0 < V) {
    v.load(logits + t * ld + j0);
    const f32x4 f = factors[t];
    const float ks = -scale * f[1];
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] = ks * exp2_less(v.get(k), f[0]);
    if (far_row(f[0])) {
      for (int k = 0; k < 8; ++k) g[k] = ks * exp2_far(saturate(v.get(k)), f[0]);
    }
    if ((unsigned)(lab - j0) < 8u) {
#pragma unroll
      for (int k = 0; k < 8; ++k) g[k] += j0 + k == lab ? scale * f[2] : 0.f;
    }
  }
  v.set(g);
  T* out = dlogits + t * ldd + j0;
  if constexpr (STREAM) store_nt(out, v);
  else v.store(out);
}

bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
int launch_status() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FL_OK : set_error(FL_ERR_HIP, hipGetErrorString(e));
}

struct PrefWs {
  f32x4* factors;  // [T]
  float2* part;    // [T][splits]
  uint32_t* done;
  size_t total;
};
// Parts a row is split into: one when the rows alone fill the chip.
int splits_of(long T, long V) {
  const long most = std::max(1L, V / (8 * kThreads));
  return (int)std::min<long>({(kWantGroups + T - 1) / T, most, (long)kMaxSplits});
}
PrefWs carve(long T, long V, char* base) {
  PrefWs w;
  size_t off = 0;
  auto take = [&](size_t n) {
    char* p = base ? base + off : nullptr;
    off = align256(off + n);
    return p;
  };
  w.factors = (f32x4*)take((size_t)T * sizeof(f32x4));
  w.part = (float2*)take((size_t)T * splits_of(T, V) * sizeof(float2));
  w.done = (uint32_t*)take(sizeof(uint32_t));
  w.total = off;
  return w;
}

int check_desc(const fl_preference_desc* d) {
  if (!d) return set_error(FL_ERR_NULL, "preference descriptor is NULL");
  if (d->dtype != FL_BF16 && d->dtype != FL_F32) return set_error(FL_ERR_SHAPE, "dtype must be bf16 or fp32");
  if (d->vocab < 8 || d->vocab % 8 || d->vocab > (1 << 24))
    return set_error(FL_ERR_SHAPE, "vocab must be a multiple of 8 in [8, 2^24]");
  if (!std::isfinite(d->beta) || !(d->beta > 0.f)) return set_error(FL_ERR_ARG, "beta must be finite and > 0");
  if (!(d->label_smoothing >= 0.f && d->label_smoothing <= 0.5f))
    return set_error(FL_ERR_ARG, "label_smoothing must be in [0, 0.5]");
  return FL_OK;
}
int check_pairs(const fl_batch_desc* b) {
  if (int rc = check_batch(b)) return rc;
  for (int c = 0; c < b->num_clients; ++c)
    if ((b->client_seq_ptr[c + 1] - b->client_seq_ptr[c]) % 2)
      return set_error(FL_ERR_CLIENTS, "every client's sequences come in pairs (preferred, rejected)");
  return FL_OK;
}
int check_ws(const fl_preference_desc* d, const fl_batch_desc* b, void* ws, size_t bytes) {
  if (!ws) return set_error(FL_ERR_NULL, "workspace is NULL");
  if (!al16(ws)) return set_error(FL_ERR_ALIGN, "workspace is not 16-byte aligned");
  if (bytes < carve(b->total_tokens, d->vocab, nullptr).total)
    return set_error(FL_ERR_WORKSPACE, "workspace too small");
  return FL_OK;
}
int check_logits(const fl_preference_desc* d, const void* logits, int64_t ld, const int32_t* labels) {
  if (!logits || !labels) return set_error(FL_ERR_NULL, "logits / labels is NULL");
  if (!al16(logits) || ((uintptr_t)labels & 3)) return set_error(FL_ERR_ALIGN, "logits / labels misaligned");
  if (ld < d->vocab || ld % 8 || ld > (int64_t(1) << 32))
    return set_error(FL_ERR_SHAPE, "the logits' row stride must be a multiple of 8, at least vocab and at most 2^32");
  return FL_OK;
}

template <typename T>
int forward(const fl_preference_desc* d, const fl_batch_desc* b, const T* logits, long ld, const int32_t* labels,
            const float* ref, float* logp, float* loss, float* loss_sum, const PrefWs& w, hipStream_t s) {
  const long tokens = b->total_tokens;
  const int V = (int)d->vocab, splits = splits_of(tokens, V);
  const int cols = (int)(((V + splits - 1) / splits + 7) / 8 * 8);
  for (long t0 = 0; t0 < tokens; t0 += kMaxGroups) {
    const unsigned rows = (unsigned)std::min(tokens - t0, kMaxGroups);
    hipLaunchKernelGGL(pref_row_kernel<T>, dim3(rows, splits), dim3(kThreads), 0, s, logits + t0 * ld, ld, V, cols,
                       labels + t0, w.part + t0 * splits, w.done);
    if (int rc = launch_status()) return rc;
  }
  PairArgs a;
  a.pairs = b->num_seqs / 2;
  for (a.first = 0; a.first < a.pairs; a.first += a.count) {
    a.count = std::min(a.pairs - a.first, kPairsArg);
    std::copy(b->cu_seqlens + 2 * a.first, b->cu_seqlens + 2 * (a.first + a.count) + 1, a.cu);
    hipLaunchKernelGGL(pref_pair_kernel<T>, dim3(a.count), dim3(kThreads), 0, s, a, logits, ld, V, splits, labels,
                       w.part, ref, (double)d->beta, (double)d->label_smoothing, logp, loss, loss_sum, w.factors,
                       w.done);
    if (int rc = launch_status()) return rc;
  }
  return FL_OK;
}

template <typename T>
int gradient(const fl_preference_desc* d, long tokens, const T* logits, long ld, const int32_t* labels,
             float grad_scale, T* dlogits, long ldd, int width, const PrefWs& w, hipStream_t s) {
  const int V = (int)d->vocab;
  const long blocks = (width + 8 * kThreads - 1) / (8 * kThreads);
  // A gradient that the last-level cache cannot hold is stored past it (loss and
  // gradient of 4910 rows, 1.28 GB: 568 us instead of 625; with a product that
  // reads the gradient behind them, 612 MB 1131 instead of 1161, 253 MB 844
  // instead of 860, 166 MB 548 instead of 542, 26 MB 319 instead of 317; in place,
  // with a product of 4096 columns, 1.28 GB 8345 instead of 8371, 253 MB 1596
  // instead of 1607, 166 MB and less the same).
  const bool stream = (size_t)tokens * width * sizeof(T) >= kStreamBytes;
  const auto kernel = stream ? pref_grad_kernel<T, true> : pref_grad_kernel<T, false>;
  const long most = kMaxGroups / blocks;  // (a row has 2^14 blocks at most)
  for (long t1 = tokens; t1 > 0;) {
    const long t0 = std::max(0L, t1 - most);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((t1 - t0) * blocks)), dim3(kThreads), 0, s,
                       logits + t0 * ld, ld, V, labels + t0, w.factors + t0, grad_scale, dlogits + t0 * ldd, ldd, width,
                       (int)blocks);
    if (int rc = launch_status()) return rc;
    t1 = t0;
  }
  return FL_OK;
}

}  // namespace

namespace flglm {

int preference_check(const fl_preference_desc* d, const fl_batch_desc* b, const float* ref, float* logp, float* loss,
                     float* loss_sum, void* ws, size_t ws_bytes) {
  if (int rc = check_desc(d)) return rc;
  if (int rc = check_pairs(b)) return rc;
  if (!logp || !loss || !loss_sum) return set_error(FL_ERR_NULL, "logp / loss / loss_sum is NULL");
  if (((uintptr_t)logp & 3) || ((uintptr_t)loss & 3) || ((uintptr_t)loss_sum & 3) || ((uintptr_t)ref & 3))
    return set_error(FL_ERR_ALIGN, "ref_logp / logp / loss / loss_sum misaligned");
  if (int rc = check_ws(d, b, ws, ws_bytes)) return rc;
  const size_t S = b->num_seqs;
  const void* out[3] = {logp, loss, loss_sum};
  const size_t n[3] = {4 * S, 2 * S, 4};
  for (int i = 0; i < 3; ++i) {
    for (int j = i + 1; j < 3; ++j)
      if (overlap(out[i], n[i], out[j], n[j])) return set_error(FL_ERR_ALIAS, "logp / loss / loss_sum overlap");
    if (overlap(out[i], n[i], ws, ws_bytes) || (ref && overlap(out[i], n[i], ref, 4 * S)))
      return set_error(FL_ERR_ALIAS, "logp / loss / loss_sum overlap ref_logp or the workspace");
  }
  return FL_OK;
}

int preference_check_backward(const fl_preference_desc* d, const fl_batch_desc* b, float grad_scale, void* ws,
                              size_t ws_bytes) {
  if (int rc = check_desc(d)) return rc;
  if (int rc = check_pairs(b)) return rc;
  if (!std::isfinite(grad_scale)) return set_error(FL_ERR_ARG, "grad_scale is not finite");
  return check_ws(d, b, ws, ws_bytes);
}

int preference_forward(const fl_preference_desc* d, const fl_batch_desc* b, const void* logits, long ld,
                       const int32_t* labels, const float* ref, float* logp, float* loss, float* loss_sum, void* ws,
                       hipStream_t s) {
  const PrefWs w = carve(b->total_tokens, d->vocab, (char*)ws);
  if (d->dtype == FL_BF16)
    return forward(d, b, (const bf16*)logits, ld, labels, ref, logp, loss, loss_sum, w, s);
  return forward(d, b, (const float*)logits, ld, labels, ref, logp, loss, loss_sum, w, s);
}

int preference_gradient(const fl_preference_desc* d, const fl_batch_desc* b, const void* logits, long ld,
                        const int32_t* labels, float grad_scale, void* dlogits, long ldd, int width, void* ws,
                        hipStream_t s) {
  const PrefWs w = carve(b->total_tokens, d->vocab, (char*)ws);
  if (d->dtype == FL_BF16)
    return gradient(d, b->total_tokens, (const bf16*)logits, ld, labels, grad_scale, (bf16*)dlogits, ldd, width, w,
                    s);
  return gradient(d, b->total_tokens, (const float*)logits, ld, labels, grad_scale, (float*)dlogits, ldd, width, w, s);
}

}  // namespace flglm

extern "C" {

int fl_preference_workspace_bytes(const fl_preference_desc* desc, const fl_batch_desc* batch, size_t* bytes) {
  if (!bytes) return set_error(FL_ERR_NULL, "bytes is NULL");
  if (int rc = check_desc(desc)) return rc;
  if (int rc = check_pairs(batch)) return rc;
  *bytes = carve(batch->total_tokens, desc->vocab, nullptr).total;
  return FL_OK;
}

int fl_preference_forward(const fl_preference_desc* desc, const fl_batch_desc* batch, const void* logits, int64_t ld,
                          const int32_t* labels, const float* ref_logp, float* logp, float* loss, float* loss_sum,
                          void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = preference_check(desc, batch, ref_logp, logp, loss, loss_sum, workspace, workspace_bytes)) return rc;
  if (int rc = check_logits(desc, logits, ld, labels)) return rc;
  const size_t T = batch->total_tokens, S = batch->num_seqs;
  const size_t nl = ((T - 1) * ld + desc->vocab) * (desc->dtype == FL_BF16 ? 2 : 4);
  const void* out[4] = {logp, loss, loss_sum, workspace};
  const size_t n[4] = {4 * S, 2 * S, 4, workspace_bytes};
  for (int i = 0; i < 4; ++i)
    if (overlap(out[i], n[i], logits, nl) || overlap(out[i], n[i], labels, 4 * T))
      return set_error(FL_ERR_ALIAS, "an output or the workspace overlaps the logits or labels");
  if (ref_logp && overlap(workspace, workspace_bytes, ref_logp, 4 * S))
    return set_error(FL_ERR_ALIAS, "the workspace overlaps ref_logp");
  return preference_forward(desc, batch, logits, ld, labels, ref_logp, logp, loss, loss_sum, workspace,
                            (hipStream_t)stream);
}

int fl_preference_backward(const fl_preference_desc* desc, const fl_batch_desc* batch, const void* logits, int64_t ld,
                           const int32_t* labels, float grad_scale, void* dlogits, int64_t ld_d, int64_t width_d,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = preference_check_backward(desc, batch, grad_scale, workspace, workspace_bytes)) return rc;
  if (int rc = check_logits(desc, logits, ld, labels)) return rc;
  if (!dlogits) return set_error(FL_ERR_NULL, "dlogits is NULL");
  if (!al16(dlogits)) return set_error(FL_ERR_ALIGN, "dlogits is not 16-byte aligned");
  if (ld_d < desc->vocab || ld_d % 8 || ld_d > (int64_t(1) << 32))
    return set_error(FL_ERR_SHAPE, "dlogits' row stride must be a multiple of 8, at least vocab and at most 2^32");
  if (width_d < desc->vocab || width_d % 8 || width_d > ld_d || width_d > (1 << 25))
    return set_error(FL_ERR_SHAPE, "dlogits' width must be a multiple of 8 in [vocab, its row stride], at most 2^25");
  const size_t T = batch->total_tokens, E = desc->dtype == FL_BF16 ? 2 : 4;
  const size_t nl = ((T - 1) * ld + desc->vocab) * E, nd = ((T - 1) * ld_d + width_d) * E;
  if (overlap(dlogits, nd, logits, nl) && !(dlogits == logits && ld == ld_d))
    return set_error(FL_ERR_ALIAS, "dlogits overlaps the logits without being them");
  if (overlap(dlogits, nd, labels, 4 * T) || overlap(dlogits, nd, workspace, workspace_bytes) ||
      overlap(workspace, workspace_bytes, logits, nl) || overlap(workspace, workspace_bytes, labels, 4 * T))
    return set_error(FL_ERR_ALIAS, "dlogits or the workspace overlaps another argument");
  return preference_gradient(desc, batch, logits, ld, labels, grad_scale, dlogits, ld_d, (int)width_d, workspace,
                             (hipStream_t)stream);
}

}  // extern "C"
