// Global gradient norm over many tensors and the scaling by it.
//
// Two kernels per list: grad_square_kernel writes one fp64 partial sum of squares per workgroup, grad_scale_kernel adds the
// partials in their order (every workgroup by itself: no kernel in between, no atomics) and scales.  Descriptors travel as
// kernel arguments, kTable tensors a launch: nothing has to be copied to the device, and a captured graph holds them.
// Squares are fp64: no gradient that fits its type overflows them.  Bound: HBM, two reads and one write of every tensor.
#include <algorithm>
#include <cfloat>

#include "common.h"
#include "launch.h"

namespace mote {

namespace {

constexpr int kTable = 120;             // tensors of a launch: 3.8 KB of kernel arguments
constexpr int kThreads = 256;
constexpr int kUnit = 8192;             // elements of a unit of work: 128 (bf16: 64) bytes a thread, all on their way together
constexpr int kPart = kUnit / 2;        // of a unit that is scaled
constexpr int kSquareBlocks = 2048, kScaleBlocks = 2048;   // workgroups of a launch at most
struct Table {
  const void* grad[kTable];
  void* out[kTable];
  int64_t n[kTable];
  int32_t first[kTable + 1];            // first unit of each tensor
  uint32_t bf16[(kTable + 31) / 32];    // a bit per tensor
  int count;
};
static_assert(sizeof(Table) <= 4000, "kernel arguments");

__device__ __forceinline__ int find(const Table& t, int unit) {
  int lo = 0, hi = t.count;             // first[lo] <= unit < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= unit) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* s) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// 16 bytes of a tensor
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const u4& v, int i) { return __uint_as_float(v[i]); }
  static __device__ __forceinline__ u4 scaled(const u4& v, double c) {
    u4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(static_cast<float>(get(v, i) * c));
    return o;
  }
  static __device__ __forceinline__ float one(float v) { return v; }
  static __device__ __forceinline__ float scaled_one(float v, double c) { return static_cast<float>(v * c); }
};
template <> struct Vec<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(const u4& v, int i) { return i & 1 ? bf16_hi(v[i >> 1]) : bf16_lo(v[i >> 1]); }
  static __device__ __forceinline__ u4 scaled(const u4& v, double c) {
    u4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = cvt_pk_bf16(static_cast<float>(bf16_lo(v[i]) * c), static_cast<float>(bf16_hi(v[i]) * c));
    return o;
  }
  static __device__ __forceinline__ float one(uint16_t v) { return bf16_to_f32(v); }
  static __device__ __forceinline__ uint16_t scaled_one(uint16_t v, double c) {
    return static_cast<uint16_t>(cvt_pk_bf16(static_cast<float>(bf16_to_f32(v) * c), 0.0f));
  }
};

template <typename T>
__device__ __forceinline__ double square_unit(const T* g, int n) {
  constexpr int N = Vec<T>::N, V = kUnit / N / kThreads;
  double acc = 0.0;
  if (reinterpret_cast<uintptr_t>(g) % 16 == 0) {
    const u4* const p = reinterpret_cast<const u4*>(g);
    u4 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (i * kThreads + static_cast<int>(threadIdx.x) + 1) * N <= n ? p[i * kThreads + threadIdx.x] : u4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double x = Vec<T>::get(v[i], j);
        acc = fma(x, x, acc);
      }
    const int rest = n / N * N + threadIdx.x;
    if (rest < n) {
      const double x = Vec<T>::one(g[rest]);
      acc = fma(x, x, acc);
    }
  } else {
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const double x = Vec<T>::one(g[i]);
      acc = fma(x, x, acc);
    }
  }
  return acc;
}

__global__ __launch_bounds__(kThreads) void grad_square_kernel(const Table t, double* __restrict__ partial) {
  __shared__ double s[4];
  double acc = 0.0;
  const int units = t.first[t.count];
  int i = find(t, blockIdx.x);
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    while (t.first[i + 1] <= u) ++i;
    const int64_t at = static_cast<int64_t>(u - t.first[i]) * kUnit;
    const int n = static_cast<int>(min(t.n[i] - at, static_cast<int64_t>(kUnit)));
    acc += t.bf16[i >> 5] >> (i & 31) & 1 ? square_unit(static_cast<const uint16_t*>(t.grad[i]) + at, n)
                                          : square_unit(static_cast<const float*>(t.grad[i]) + at, n);
  }
  acc = block_sum(acc, s);
  if (threadIdx.x == 0) partial[blockIdx.x] = acc;
}

// c == 1: a copy, bits as they are
template <typename T>
__device__ __forceinline__ void scale_unit(const T* g, T* o, int n, bool clip, double c) {
  constexpr int N = Vec<T>::N, V = kPart / N / kThreads;
  if ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(o)) % 16 == 0) {
    const u4* const p = reinterpret_cast<const u4*>(g);
    u4* const q = reinterpret_cast<u4*>(o);
    u4 v[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
      if ((i * kThreads + static_cast<int>(threadIdx.x) + 1) * N <= n) v[i] = p[i * kThreads + threadIdx.x];
#pragma unroll
    for (int i = 0; i < V; ++i)
      if ((i * kThreads + static_cast<int>(threadIdx.x) + 1) * N <= n) q[i * kThreads + threadIdx.x] = clip ? Vec<T>::scaled(v[i], c) : v[i];
    const int rest = n / N * N + threadIdx.x;
    if (rest < n) o[rest] = clip ? Vec<T>::scaled_one(g[rest], c) : g[rest];
  } else {
    for (int i = threadIdx.x; i < n; i += kThreads) o[i] = clip ? Vec<T>::scaled_one(g[i], c) : g[i];
  }
}

// Units from the last to the first: what the kernel before read last is still in the memory-side cache.
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(const Table t, const double* __restrict__ partial, int partials, float max_norm,
                                                              float* __restrict__ norm_out) {
  __shared__ double s[4];
  double acc = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < partials; i += kThreads) acc += partial[i];
  const double norm = sqrt(block_sum(acc, s));
  if (blockIdx.x == 0 && threadIdx.x == 0) norm_out[0] = static_cast<float>(norm);
  const double limit = max_norm;
  const bool clip = norm > limit && norm <= DBL_MAX;
  const double c = clip ? limit / norm : 1.0;   // fp64 products: a norm beyond fp32 has a coefficient below its normal range
  const int units = t.first[t.count];
  if (static_cast<int>(blockIdx.x) >= units) return;
  int i = find(t, units - 1 - blockIdx.x);
  for (int u = units - 1 - blockIdx.x; u >= 0; u -= gridDim.x) {
    while (t.first[i] > u) --i;
    if (!clip && t.out[i] == t.grad[i]) continue;
    const int64_t at = static_cast<int64_t>(u - t.first[i]) * kUnit;
    const int n = static_cast<int>(min(t.n[i] - at, static_cast<int64_t>(kUnit)));
    const bool bf16 = t.bf16[i >> 5] >> (i & 31) & 1;
#pragma unroll 1
    for (int h = 0; h < n; h += kPart) {
      const int m = min(n - h, kPart);
      if (bf16) scale_unit(static_cast<const uint16_t*>(t.grad[i]) + at + h, static_cast<uint16_t*>(t.out[i]) + at + h, m, clip, c);
      else scale_unit(static_cast<const float*>(t.grad[i]) + at + h, static_cast<float*>(t.out[i]) + at + h, m, clip, c);
    }
  }
}

// Descriptors [at, at + kTable) of the list in one launch's table.  The caller bounds the elements of all tensors, so that units
// fit an int.
void fill(const GradTensor* g, int at, int n, Table* t) {
  int units = 0, i = 0;
  for (uint32_t& b : t->bf16) b = 0;
  for (; i < kTable && at + i < n; ++i) {
    const GradTensor& s = g[at + i];
    const int64_t u = (s.n + kUnit - 1) / kUnit;
    t->grad[i] = s.grad;
    t->out[i] = s.out;
    t->n[i] = s.n;
    t->first[i] = units;
    if (s.bf16) t->bf16[i >> 5] |= 1u << (i & 31);
    units += static_cast<int>(u);
  }
  t->count = i;
  t->first[i] = units;
}

}  // namespace

size_t grad_clip_workspace_bytes(int n) { return 256 + static_cast<size_t>(n / kTable + 2) * kSquareBlocks * sizeof(double); }

// Results are stored through the caches, where the optimiser finds the last of them.  (Past the caches the scaling takes the same
// time, 118 M elements 154 and 152 us.  A first pass over the gradients of the call before would find more of them, 92 us instead of
// 107; a training step has new ones.)
hipError_t launch_grad_clip(const GradTensor* g, int n, float max_norm, float* norm, void* workspace, hipStream_t stream) {
  double* const partial = static_cast<double*>(workspace);
  int partials = 0;
  Table t{};
  for (int at = 0; at < n; at += kTable) {
    fill(g, at, n, &t);
    const int blocks = std::min(t.first[t.count], kSquareBlocks);
    if (blocks > 0) grad_square_kernel<<<blocks, kThreads, 0, stream>>>(t, partial + partials);
    partials += blocks;
  }
  for (int at = n > 0 ? (n - 1) / kTable * kTable : 0; at >= 0; at -= kTable) {
    fill(g, at, n, &t);
    const int blocks = std::max(std::min(t.first[t.count], kScaleBlocks), 1);
    grad_scale_kernel<<<blocks, kThreads, 0, stream>>>(t, partial, partials, max_norm, norm);
  }
  return hipGetLastError();
}

}  // namespace mote
