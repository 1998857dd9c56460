// Global gradient norm over many tensors, and clipping (C ABI entry points).
//
//   n = sqrt(sum over all tensors and elements of g^2),
//   c = min(1, max_norm / (n + 1e-6)),   out = c g  (out may be g itself).
//
// The squares are summed in 64 bits: an fp32 sum of 1e9 squares loses digits,
// and the square of a large fp32 gradient overflows fp32.  The sum is
// deterministic: a workgroup sums one chunk of one tensor into a partial, and
// one workgroup adds the partials in a fixed order.
//
// Tensor tables travel in kernel arguments, kTensors tensors a launch, so a
// call records nothing but kernels (it can be captured) and keeps no state.
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
constexpr int kTensors = 128;                 // tensors a launch (2.6 KB of kernel arguments)
constexpr int kStep = 8 * kThreads;           // elements a workgroup takes at a time
constexpr int64_t kMaxTensors = 1 << 20;
constexpr int64_t kMaxElements = int64_t(1) << 40;
// Bytes from which clipping passes the last-level cache by (1.6 GB into other
// tensors 779 us instead of 834 and 1 GB in place 575 either way, but in place
// 600 MB 366 instead of 360, 300 MB 176 instead of 151).
constexpr size_t kPastCache = size_t(1) << 30;
constexpr double kEps = 1e-6;                 // keeps the quotient finite for a zero norm

struct Table {
  const void* g[kTensors];
  void* out[kTensors];
  int64_t size[kTensors];
  int32_t first[kTensors + 1];  // first block of each tensor within the launch
  int count;
};
struct NormTable {
  const void* g[kTensors];
  int64_t size[kTensors];
  int32_t first[kTensors + 1];
  int count;
};

// The table's entry that block b belongs to (uniform: scalar loads).
template <typename TB>
__device__ __forceinline__ int find(const TB& t, int b) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= b) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int NT>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double sh[NT / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += sh[w];
  return t;
}

// 16 bytes a lane and access, so that an access of a wave is whole lines, and
// 2048 elements a step: fp32 two accesses, bf16 one.  (Eight fp32 elements a lane
// in two halves of lines: norm and clipping of 52 tensors, 6.8 M elements, 19.7
// us instead of 18.5; 0.4 G 817 instead of 779.)
template <typename T>
struct Access {
  using V = std::conditional_t<sizeof(T) == 2, Vec8<T>, Vec4<T>>;
  static constexpr int n = 16 / sizeof(T), step = kStep / (n * kThreads);
  // First element of the thread's access u behind element b.
  __device__ static __forceinline__ int64_t at(int64_t b, int u) { return b + (u * kThreads + (int)threadIdx.x) * n; }
};

// Sums of squares, one partial a workgroup, kBatch steps' loads in flight at once
// (0.4 G fp32: one 305 us, four 262 us, 6.1 TB/s; bound by the reads).
constexpr int kBatch = 4;

template <typename T>
__global__ void __launch_bounds__(kThreads) square_kernel(NormTable t, int chunk, double* part) {
  using A = Access<T>;
  const int k = find(t, blockIdx.x);
  const T* g = (const T*)t.g[k];
  const int64_t n = t.size[k];
  const int64_t b0 = (int64_t)(blockIdx.x - t.first[k]) * chunk;
  const int64_t b1 = min(n, b0 + chunk);
  double acc[4] = {0, 0, 0, 0};
  auto add = [&](const typename A::V& v) {
#pragma unroll
    for (int i = 0; i < A::n; ++i) {
      const double x = v.get(i);
      acc[i & 3] = fma(x, x, acc[i & 3]);
    }
  };
  int64_t b = b0;
  for (; b + kBatch * kStep <= b1; b += kBatch * kStep) {
    typename A::V v[kBatch * A::step];
#pragma unroll
    for (int u = 0; u < kBatch * A::step; ++u) v[u].load(g + A::at(b, u));
#pragma unroll
    for (int u = 0; u < kBatch * A::step; ++u) add(v[u]);
  }
  for (int64_t e = A::at(b, 0); e < b1; e += A::n * kThreads) {
    if (e + A::n <= b1) {
      typename A::V v;
      v.load(g + e);
      add(v);
    } else {
      for (int64_t j = e; j < b1; ++j) {
        const double x = to_f32(g[j]);
        acc[0] = fma(x, x, acc[0]);
      }
    }
  }
  const double s = block_sum<kThreads>((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// One workgroup adds the partials (4096 at most from one tensor of 0.4 G: 4 us,
// of which most is the launch).
constexpr int kFinish = 1024;
__global__ void __launch_bounds__(kFinish) finish_kernel(const double* part, int64_t n, double max_norm, float* out) {
  double a = 0;
  for (int64_t i = threadIdx.x; i < n; i += kFinish) a += part[i];
  const double s = block_sum<kFinish>(a);
  if (threadIdx.x == 0) {
    const double norm = sqrt(s);
    double c = 1.0;
    if (max_norm < INFINITY) {
      c = max_norm / (norm + kEps);
      if (c > 1.0) c = 1.0;  // a NaN stays
    }
    out[0] = (float)norm;
    out[1] = (float)c;
  }
}

// A step a workgroup and done: the chip then sweeps through memory in order,
// which reads and writes faster than as many workgroups each in a stretch of
// its own (0.4 G fp32 in place: 128 K elements a workgroup 640 us, so 540).  From the last
// element to the first: what the norm read last is in the last-level cache (norm
// and clipping of 300 MB in place 151 us, of 400 MB 240; from the first on 180
// and 260; past 1 GB within 1 %).  STREAM: past that cache.
template <typename T, bool STREAM>
__global__ void __launch_bounds__(kThreads) scale_kernel(Table t, const float* norm_coef) {
  using A = Access<T>;
  const float c = norm_coef[1];
  const int block = gridDim.x - 1 - blockIdx.x;
  const int k = find(t, block);
  const T* g = (const T*)t.g[k];
  T* out = (T*)t.out[k];
  if (c == 1.f && g == out) return;
  const int64_t n = t.size[k];
  const int64_t b = (int64_t)(block - t.first[k]) * kStep;
  auto scaled = [&](typename A::V& v) {
    float x[A::n];
#pragma unroll
    for (int i = 0; i < A::n; ++i) x[i] = v.get(i) * c;
    v.set(x);
  };
  if (b + kStep <= n) {
    typename A::V v[A::step];
#pragma unroll
    for (int u = 0; u < A::step; ++u) {
      if constexpr (STREAM) v[u].r = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(g + A::at(b, u)));
      else v[u].load(g + A::at(b, u));
    }
#pragma unroll
    for (int u = 0; u < A::step; ++u) {
      scaled(v[u]);
      if constexpr (STREAM) __builtin_nontemporal_store(v[u].r, reinterpret_cast<u32x4*>(out + A::at(b, u)));
      else v[u].store(out + A::at(b, u));
    }
    return;
  }
  for (int64_t e = A::at(b, 0); e < n; e += A::n * kThreads) {
    if (e + A::n <= n) {
      typename A::V v;
      v.load(g + e);
      scaled(v);
      v.store(out + e);
    } else {
      for (int64_t j = e; j < n; ++j) out[j] = from_f32<T>(to_f32(g[j]) * c);
    }
  }
}

bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na && nb && x < y + nb && y < x + na;
}
int launch_status() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FL_OK : set_error(FL_ERR_HIP, hipGetErrorString(e));
}

// Elements of a chunk: enough chunks to fill the chip, few enough that the
// partials stay small, and a whole batch of loads at least (norm and clipping of
// 52 tensors, 6.8 M fp32 elements: 18.5 us; one step a chunk 20).
int chunk_of(int64_t total) {
  const int64_t want = (total / 4096 + kStep - 1) / kStep * kStep;
  return (int)std::min<int64_t>(std::max<int64_t>(want, kBatch * kStep), 64 * kStep);
}

// The tensors' count and sizes; total elements and chunks.
int check_sizes(int32_t num, const int64_t* sizes, int64_t* total, int64_t* chunks) {
  if (num < 1 || num > kMaxTensors) return set_error(FL_ERR_ARG, "1 <= num_tensors <= 2^20");
  if (!sizes) return set_error(FL_ERR_NULL, "sizes is NULL");
  *total = 0;
  for (int i = 0; i < num; ++i) {
    if (sizes[i] < 0 || sizes[i] > kMaxElements) return set_error(FL_ERR_ARG, "a tensor's size is outside [0, 2^40]");
    *total += sizes[i];
  }
  if (*total > kMaxElements) return set_error(FL_ERR_ARG, "more than 2^40 elements");
  const int64_t chunk = chunk_of(*total);
  *chunks = 0;
  for (int i = 0; i < num; ++i) *chunks += (sizes[i] + chunk - 1) / chunk;
  return FL_OK;
}

// Outputs are written at once by different workgroups: none may overlap
// another, nor a gradient other than the one it replaces.  One sweep over the
// intervals in address order.
int check_outputs(int32_t num, const void* const* grads, void* const* out, const int64_t* sizes, size_t E) {
  struct Range {
    uintptr_t a, b;
    bool written;
  };
  std::vector<Range> r;
  try {
    r.reserve(2 * (size_t)num);
    for (int i = 0; i < num; ++i) {
      if (sizes[i] == 0) continue;
      const size_t n = (size_t)sizes[i] * E;
      r.push_back({(uintptr_t)out[i], (uintptr_t)out[i] + n, true});
      if (out[i] != grads[i]) r.push_back({(uintptr_t)grads[i], (uintptr_t)grads[i] + n, false});
    }
  } catch (const std::bad_alloc&) {
    return set_error(FL_ERR_NOMEM, "out of host memory while checking the outputs");
  }
  std::sort(r.begin(), r.end(), [](const Range& x, const Range& y) { return x.a < y.a; });
  uintptr_t end_read = 0, end_written = 0;
  for (const Range& x : r) {
    if (x.a < end_written || (x.written && x.a < end_read))
      return set_error(FL_ERR_ALIAS, "an output overlaps another output or a gradient that it does not replace");
    uintptr_t& end = x.written ? end_written : end_read;
    end = std::max(end, x.b);
  }
  return FL_OK;
}

}  // namespace

extern "C" {

int fl_grad_norm_workspace_bytes(int32_t num_tensors, const int64_t* sizes, size_t* bytes) {
  if (!bytes) return set_error(FL_ERR_NULL, "bytes is NULL");
  int64_t total, chunks;
  if (int rc = check_sizes(num_tensors, sizes, &total, &chunks)) return rc;
  *bytes = (size_t)std::max<int64_t>(chunks, 1) * sizeof(double);
  return FL_OK;
}

int fl_grad_norm(int32_t dtype, int32_t num_tensors, const void* const* grads, const int64_t* sizes, double max_norm,
                 float* norm_coef, void* workspace, size_t workspace_bytes, void* stream) {
  if (dtype != FL_BF16 && dtype != FL_F32) return set_error(FL_ERR_ARG, "dtype must be bf16 or fp32");
  int64_t total, chunks;
  if (int rc = check_sizes(num_tensors, sizes, &total, &chunks)) return rc;
  if (!grads || !norm_coef || !workspace) return set_error(FL_ERR_NULL, "grads / norm_coef / workspace is NULL");
  if (!(max_norm >= 0.0)) return set_error(FL_ERR_ARG, "max_norm must be >= 0 (infinity: never clip)");
  if (!al16(workspace) || ((uintptr_t)norm_coef & 7))
    return set_error(FL_ERR_ALIGN, "workspace / norm_coef misaligned");
  if (workspace_bytes < (size_t)std::max<int64_t>(chunks, 1) * sizeof(double))
    return set_error(FL_ERR_WORKSPACE, "workspace too small");
  const size_t E = dtype == FL_BF16 ? 2 : 4;
  if (overlap(norm_coef, 8, workspace, workspace_bytes))
    return set_error(FL_ERR_ALIAS, "norm_coef overlaps the workspace");
  for (int i = 0; i < num_tensors; ++i) {
    if (sizes[i] == 0) continue;
    if (!grads[i]) return set_error(FL_ERR_NULL, "a gradient is NULL");
    if (!al16(grads[i])) return set_error(FL_ERR_ALIGN, "gradients must be 16-byte aligned");
    if (overlap(grads[i], sizes[i] * E, workspace, workspace_bytes) || overlap(grads[i], sizes[i] * E, norm_coef, 8))
      return set_error(FL_ERR_ALIAS, "the workspace or norm_coef overlaps a gradient");
  }
  hipStream_t s = (hipStream_t)stream;
  const int chunk = chunk_of(total);
  double* part = (double*)workspace;
  for (int i = 0; i < num_tensors;) {
    NormTable t;
    t.count = 0;
    int64_t blocks = 0;
    for (; i < num_tensors && t.count < kTensors; ++i) {
      const int64_t nb = (sizes[i] + chunk - 1) / chunk;
      if (nb == 0) continue;
      if (t.count && blocks + nb > kMaxGroups) break;  // (one tensor has 2^23 chunks at most)
      t.g[t.count] = grads[i];
      t.size[t.count] = sizes[i];
      t.first[t.count++] = (int32_t)blocks;
      blocks += nb;
    }
    if (!t.count) continue;
    if (dtype == FL_BF16)
      hipLaunchKernelGGL(square_kernel<bf16>, dim3((unsigned)blocks), dim3(kThreads), 0, s, t, chunk, part);
    else
      hipLaunchKernelGGL(square_kernel<float>, dim3((unsigned)blocks), dim3(kThreads), 0, s, t, chunk, part);
    if (int rc = launch_status()) return rc;
    part += blocks;
  }
  hipLaunchKernelGGL(finish_kernel, dim3(1), dim3(kFinish), 0, s, (const double*)workspace, chunks, max_norm,
                     norm_coef);
  return launch_status();
}

int fl_clip_grads(int32_t dtype, int32_t num_tensors, const void* const* grads, void* const* out, const int64_t* sizes,
                  const float* norm_coef, void* stream) {
  if (dtype != FL_BF16 && dtype != FL_F32) return set_error(FL_ERR_ARG, "dtype must be bf16 or fp32");
  int64_t total, chunks;
  if (int rc = check_sizes(num_tensors, sizes, &total, &chunks)) return rc;
  if (!grads || !out || !norm_coef) return set_error(FL_ERR_NULL, "grads / out / norm_coef is NULL");
  if ((uintptr_t)norm_coef & 7) return set_error(FL_ERR_ALIGN, "norm_coef misaligned");
  const size_t E = dtype == FL_BF16 ? 2 : 4;
  for (int i = 0; i < num_tensors; ++i) {
    if (sizes[i] == 0) continue;
    if (!grads[i] || !out[i]) return set_error(FL_ERR_NULL, "a gradient or output is NULL");
    if (!al16(grads[i]) || !al16(out[i]))
      return set_error(FL_ERR_ALIGN, "gradients and outputs must be 16-byte aligned");
    if (overlap(out[i], sizes[i] * E, norm_coef, 8)) return set_error(FL_ERR_ALIAS, "an output overlaps norm_coef");
  }
  if (int rc = check_outputs(num_tensors, grads, out, sizes, E)) return rc;
  hipStream_t s = (hipStream_t)stream;
  const bool past_cache = (size_t)total * E >= kPastCache;
  int64_t done = 0;  // elements of tensor i in the launches before
  for (int i = 0; i < num_tensors;) {
    Table t;
    t.count = 0;
    int64_t blocks = 0;
    while (i < num_tensors && t.count < kTensors && blocks < kMaxGroups) {
      const int64_t n = std::min(sizes[i] - done, (kMaxGroups - blocks) * kStep);  // what still fits this launch
      if (n > 0) {
        t.g[t.count] = (const char*)grads[i] + done * E;
        t.out[t.count] = (char*)out[i] + done * E;
        t.size[t.count] = n;
        t.first[t.count++] = (int32_t)blocks;
        blocks += (n + kStep - 1) / kStep;
        done += n;
      }
      if (done < sizes[i]) break;  // the launch is full
      done = 0;
      ++i;
    }
    if (!t.count) continue;
    const auto bf = past_cache ? scale_kernel<bf16, true> : scale_kernel<bf16, false>;
    const auto f32 = past_cache ? scale_kernel<float, true> : scale_kernel<float, false>;
    hipLaunchKernelGGL(dtype == FL_BF16 ? bf : f32, dim3((unsigned)blocks), dim3(kThreads), 0, s, t, norm_coef);
    if (int rc = launch_status()) return rc;
  }
  return FL_OK;
}

}  // extern "C"
