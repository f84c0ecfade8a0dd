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
constexpr int kChunk = 16384;           // elements of a unit of work
constexpr int kMaxBlocks = 2048;        // workgroups of a launch
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

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<uint16_t>(uint16_t v) { return bf16_to_f32(v); }

template <typename T>
__device__ __forceinline__ double square_unit(const T* g, int64_t n) {
  double acc = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const double v = to_f32<T>(g[i]);
    acc = fma(v, v, acc);
  }
  return acc;
}

__global__ __launch_bounds__(kThreads) void grad_square_kernel(const Table t, double* __restrict__ partial) {
  __shared__ double s[4];
  double acc = 0.0;
  for (int u = blockIdx.x; u < t.first[t.count]; u += gridDim.x) {
    const int i = find(t, u);
    const int64_t at = static_cast<int64_t>(u - t.first[i]) * kChunk, n = min(t.n[i] - at, static_cast<int64_t>(kChunk));
    acc += t.bf16[i >> 5] >> (i & 31) & 1 ? square_unit(static_cast<const uint16_t*>(t.grad[i]) + at, n)
                                          : square_unit(static_cast<const float*>(t.grad[i]) + at, n);
  }
  acc = block_sum(acc, s);
  if (threadIdx.x == 0) partial[blockIdx.x] = acc;
}

__global__ __launch_bounds__(kThreads) void grad_scale_kernel(const Table t, const double* __restrict__ partial, int partials, float max_norm,
                                                              float* __restrict__ norm_out) {
  __shared__ double s[4];
  double acc = 0.0;
  for (int i = threadIdx.x; i < partials; i += kThreads) acc += partial[i];
  const double norm = sqrt(block_sum(acc, s));
  if (blockIdx.x == 0 && threadIdx.x == 0) norm_out[0] = static_cast<float>(norm);
  const double limit = max_norm;
  const bool clip = norm > limit && norm <= DBL_MAX;
  const double c = clip ? limit / norm : 1.0;   // fp64 products: a norm beyond fp32 has a coefficient below its normal range
  for (int u = blockIdx.x; u < t.first[t.count]; u += gridDim.x) {
    const int i = find(t, u);
    const int64_t at = static_cast<int64_t>(u - t.first[i]) * kChunk, n = min(t.n[i] - at, static_cast<int64_t>(kChunk));
    if (!clip && t.out[i] == t.grad[i]) continue;
    if (t.bf16[i >> 5] >> (i & 31) & 1) {
      const uint16_t* g = static_cast<const uint16_t*>(t.grad[i]) + at;
      uint16_t* o = static_cast<uint16_t*>(t.out[i]) + at;
      for (int64_t j = threadIdx.x; j < n; j += kThreads) o[j] = clip ? static_cast<uint16_t>(cvt_pk_bf16(static_cast<float>(bf16_to_f32(g[j]) * c), 0.0f)) : g[j];
    } else {
      const float* g = static_cast<const float*>(t.grad[i]) + at;
      float* o = static_cast<float*>(t.out[i]) + at;
      for (int64_t j = threadIdx.x; j < n; j += kThreads) o[j] = clip ? static_cast<float>(g[j] * c) : g[j];
    }
  }
}

// Descriptors [at, ...) of the list in one launch's table; returns the number taken.  The caller bounds the elements of all
// tensors, so that units fit an int.
int fill(const GradTensor* g, int at, int n, Table* t) {
  int units = 0, i = 0;
  for (uint32_t& b : t->bf16) b = 0;
  for (; i < kTable && at + i < n; ++i) {
    const GradTensor& s = g[at + i];
    const int64_t u = (s.n + kChunk - 1) / kChunk;
    t->grad[i] = s.grad;
    t->out[i] = s.out;
    t->n[i] = s.n;
    t->first[i] = units;
    if (s.bf16) t->bf16[i >> 5] |= 1u << (i & 31);
    units += static_cast<int>(u);
  }
  t->count = i;
  t->first[i] = units;
  return i;
}

}  // namespace

size_t grad_clip_workspace_bytes(int n) { return 256 + static_cast<size_t>(n / kTable + 2) * kMaxBlocks * sizeof(double); }

hipError_t launch_grad_clip(const GradTensor* g, int n, float max_norm, float* norm, void* workspace, hipStream_t stream) {
  double* const partial = static_cast<double*>(workspace);
  int partials = 0;
  Table t{};
  for (int at = 0; at < n;) {
    const int taken = fill(g, at, n, &t);
    const int blocks = std::min(t.first[t.count], kMaxBlocks);
    if (blocks > 0) grad_square_kernel<<<blocks, kThreads, 0, stream>>>(t, partial + partials);
    partials += blocks;
    at += taken;
  }
  for (int at = 0; at == 0 || at < n;) {
    const int taken = fill(g, at, n, &t);
    const int blocks = std::max(std::min(t.first[t.count], kMaxBlocks), 1);
    grad_scale_kernel<<<blocks, kThreads, 0, stream>>>(t, partial, partials, max_norm, norm);
    at += std::max(taken, 1);
  }
  return hipGetLastError();
}

}  // namespace mote
