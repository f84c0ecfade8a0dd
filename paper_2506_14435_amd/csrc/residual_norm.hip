// The residual stream between two branches of a block: total = a r + b gate * N_post(y), normed = N_pre(total), and its
// gradient.  N is RMSNorm or layer normalisation as in block_extras.hip, here in fp32 throughout.
//
// A row is held in registers between its loads and its stores: NT threads, 8 channels each (NT * 8 >= d), every row
// quantity (mean, variance, the two means of a norm's gradient) is a sum over those threads.  A workgroup keeps the
// parameters of its channels in registers and walks over rows.  Bound: HBM, 8 bytes per bf16 element forward, 12 backward.
#include <algorithm>

#include "common.h"
#include "launch.h"

namespace mote {

namespace {

// 8 values of a row: raw as loaded, and as fp32
template <typename T> struct Row8;
template <> struct Row8<uint16_t> {
  uint4 p;
  __device__ __forceinline__ void load(const uint16_t* s) { p = *reinterpret_cast<const uint4*>(s); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = bf16_lo(p.x); v[1] = bf16_hi(p.x); v[2] = bf16_lo(p.y); v[3] = bf16_hi(p.y);
    v[4] = bf16_lo(p.z); v[5] = bf16_hi(p.z); v[6] = bf16_lo(p.w); v[7] = bf16_hi(p.w);
  }
  static __device__ __forceinline__ void store(uint16_t* d, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(d) = make_uint4(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7]));
  }
};
template <> struct Row8<float> {
  float4 p, q;
  __device__ __forceinline__ void load(const float* s) { p = reinterpret_cast<const float4*>(s)[0]; q = reinterpret_cast<const float4*>(s)[1]; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = p.x; v[1] = p.y; v[2] = p.z; v[3] = p.w; v[4] = q.x; v[5] = q.y; v[6] = q.z; v[7] = q.w;
  }
  static __device__ __forceinline__ void store(float* d, const float (&v)[8]) {
    reinterpret_cast<float4*>(d)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(d)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
};

// Parameters of a thread's 8 channels (absent ones: the neutral value)
__device__ __forceinline__ void load_param(const uint16_t* p, bool in, int c, float neutral, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = neutral;
  if (p != nullptr && in) {
    Row8<uint16_t> r;
    r.load(p + c);
    r.get(v);
  }
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// Sum over the wavefront, the same in every lane: four steps inside rows of 16 lanes, then the four rows
__device__ __forceinline__ float wave_sum_f(float v) {
  v = dpp_add<0xB1>(v);    // lane ^ 1
  v = dpp_add<0x4E>(v);    // lane ^ 2
  v = dpp_add<0x141>(v);   // half-row mirror
  v = dpp_add<0x140>(v);   // row mirror
  const int b = __float_as_int(v);
  return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}

// Sums over the NT threads of a row; buf alternates so that one barrier per sum is enough.
template <int NT>
struct RowSum {
  static constexpr int kWaves = NT / 64;
  float (*buf)[2];   // LDS: [2 * kWaves] of this row
  int turn = 0;
  __device__ __forceinline__ void operator()(float& a, float& b) {
    a = wave_sum_f(a);
    b = wave_sum_f(b);
    if constexpr (NT > 64) {
      float (*const s)[2] = buf + (turn ? kWaves : 0);
      turn ^= 1;
      const int w = (threadIdx.x % NT) >> 6;
      if ((threadIdx.x & 63) == 0) { s[w][0] = a; s[w][1] = b; }
      __syncthreads();
      a = 0.0f;
      b = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) { a += s[i][0]; b += s[i][1]; }
    }
  }
  __device__ __forceinline__ float operator()(float a) {
    float b = 0.0f;
    (*this)(a, b);
    return a;
  }
};

template <int NT> constexpr int rows_of_block() { return NT < 256 ? 256 / NT : 1; }
template <int NT> constexpr int block_threads() { return NT < 256 ? 256 : NT; }

// Normalises v in place to its hat (no gamma, beta); returns 1 / sqrt(var + eps).  Channels beyond d hold zero and stay zero.
template <int NT>
__device__ __forceinline__ float normalise(RowSum<NT>& sum, int kind, float eps, float inv_d, bool in, float (&v)[8]) {
  if (kind == 2) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i];
    const float mean = sum(s) * inv_d;
    if (in)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= mean;
  }
  float q = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) q = fmaf(v[i], v[i], q);
  const float inv = 1.0f / sqrtf(sum(q) * inv_d + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= inv;
  return inv;
}

// total and normed may be r or y
template <int NT, typename T>
__global__ __launch_bounds__(block_threads<NT>()) void residual_norm_kernel(ResidualArgs a, const T* r, const T* y, T* total, T* normed) {
  constexpr int kRows = rows_of_block<NT>();
  __shared__ float s_buf[kRows][2 * (NT / 64)][2];
  const int slot = threadIdx.x / NT, c = (threadIdx.x % NT) * 8;
  const bool in = c < a.d;
  RowSum<NT> sum{s_buf[slot]};
  float g_post[8], b_post[8], gate[8], g_pre[8], b_pre[8];
  load_param(a.post_gamma, in, c, 1.0f, g_post);
  load_param(a.post_beta, in, c, 0.0f, b_post);
  load_param(a.gate, in, c, 1.0f, gate);
  load_param(a.pre_gamma, in, c, 1.0f, g_pre);
  load_param(a.pre_beta, in, c, 0.0f, b_pre);
  const float inv_d = 1.0f / static_cast<float>(a.d);
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kRows; row0 < a.T; row0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const bool live = row0 + slot < a.T;
    const int64_t at = min(row0 + slot, static_cast<int64_t>(a.T) - 1) * a.d + c;
    float rv[8] = {}, v[8] = {};
    if (in) {
      Row8<T> rr, yy;
      yy.load(y + at);
      rr.load(r + at);
      yy.get(v);
      rr.get(rv);
    }
    if (a.post_kind) {
      normalise(sum, a.post_kind, a.post_eps, inv_d, in, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], g_post[i], b_post[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(a.residual_scale, rv[i], a.branch_scale * (gate[i] * v[i]));
    if (in && live) Row8<T>::store(total + at, v);
    if (a.pre_kind) {
      normalise(sum, a.pre_kind, a.pre_eps, inv_d, in, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], g_pre[i], b_pre[i]);
      if (in && live) Row8<T>::store(normed + at, v);
    }
  }
}

// Gradient.  A thread's sums for the parameters of its channels stay in registers over the rows of the workgroup; the row slots of
// a workgroup meet in LDS, and the workgroup leaves one partial row for each parameter gradient that is asked for:
// partial[block][which of `want`][d], summed by residual_params_kernel.  The next row is on its way while one is worked on.
template <int NT, typename T>
__global__ __launch_bounds__(block_threads<NT>()) void residual_norm_backward_kernel(ResidualArgs a, const T* __restrict__ r, const T* __restrict__ y,
                                                                                     const T* __restrict__ d_total, const T* __restrict__ d_normed,
                                                                                     T* __restrict__ dr, T* __restrict__ dy, float* __restrict__ partial, int want) {
  constexpr int kRows = rows_of_block<NT>();
  __shared__ float s_buf[kRows][2 * (NT / 64)][2];
  __shared__ float s_merge[kRows > 1 ? block_threads<NT>() * 8 : 1];
  const int slot = threadIdx.x / NT, c = (threadIdx.x % NT) * 8;
  const bool in = c < a.d;
  RowSum<NT> sum{s_buf[slot]};
  float g_post[8], b_post[8], gate[8], g_pre[8];
  load_param(a.post_gamma, in, c, 1.0f, g_post);
  load_param(a.post_beta, in, c, 0.0f, b_post);
  load_param(a.gate, in, c, 1.0f, gate);
  load_param(a.pre_gamma, in, c, 1.0f, g_pre);
#pragma unroll
  for (int i = 0; i < 8; ++i) gate[i] *= a.branch_scale;
  float p[5][8] = {};   // gate (without the branch scale), post gamma, post beta, pre gamma, pre beta
  const float inv_d = 1.0f / static_cast<float>(a.d);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  struct Raw {
    Row8<T> y, r, n, t;
  };
  auto load = [&](int64_t row) __attribute__((always_inline)) {
    Raw q;
    if (in) {
      const int64_t at = min(row, static_cast<int64_t>(a.T) - 1) * a.d + c;
      q.y.load(y + at);
      q.r.load(r + at);
      if (d_normed != nullptr) q.n.load(d_normed + at);
      if (d_total != nullptr) q.t.load(d_total + at);
    }
    return q;
  };
  constexpr bool kAhead = NT < 1024;   // 128 registers a thread have no room for a second row
  int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + slot;
  Raw next = load(row);
  for (; row - slot < a.T; row += step) {
    const Raw raw = next;
    if constexpr (kAhead) {
      next = load(row + step);
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool store = in && row < a.T;
    const int64_t at = row * a.d + c;
    float hat_y[8] = {}, z[8], up[8] = {}, hat[8] = {}, dn[8] = {}, inv_y = 1.0f;
    if (in) {
      raw.y.get(hat_y);
      raw.r.get(hat);
    }
    if (store) {   // behind the last row it is that row once more, with zero gradients: nothing of it reaches a sum
      if (d_normed != nullptr) raw.n.get(dn);
      if (d_total != nullptr) raw.t.get(up);
    }
    if (a.post_kind) {
      inv_y = normalise(sum, a.post_kind, a.post_eps, inv_d, in, hat_y);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = fmaf(hat_y[i], g_post[i], b_post[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = hat_y[i];
    }
    if (d_normed != nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i) hat[i] = fmaf(gate[i], z[i], a.residual_scale * hat[i]);
      const float inv = normalise(sum, a.pre_kind, a.pre_eps, inv_d, in, hat);
      float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[3][i] = fmaf(dn[i], hat[i], p[3][i]);
        p[4][i] += dn[i];
        dn[i] *= g_pre[i];
        m1 += dn[i];
        m2 = fmaf(dn[i], hat[i], m2);
      }
      sum(m1, m2);
      m1 = a.pre_kind == 2 ? m1 * inv_d * inv : 0.0f;
      m2 *= inv_d * inv;
#pragma unroll
      for (int i = 0; i < 8; ++i) up[i] = fmaf(inv, dn[i], up[i] - fmaf(hat[i], m2, m1));
    }
    if (store) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = a.residual_scale * up[i];
      Row8<T>::store(dr + at, o);
    }
    if (!in)
#pragma unroll
      for (int i = 0; i < 8; ++i) up[i] = 0.0f;   // the mean of a layer norm's gradient reaches channels beyond d
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[0][i] = fmaf(up[i], z[i], p[0][i]);
      up[i] *= gate[i];
    }
    if (a.post_kind) {
      float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[1][i] = fmaf(up[i], hat_y[i], p[1][i]);
        p[2][i] += up[i];
        up[i] *= g_post[i];
        m1 += up[i];
        m2 = fmaf(up[i], hat_y[i], m2);
      }
      sum(m1, m2);
      m1 = a.post_kind == 2 ? m1 * inv_d * inv_y : 0.0f;
      m2 *= inv_d * inv_y;
#pragma unroll
      for (int i = 0; i < 8; ++i) up[i] = fmaf(inv_y, up[i], -fmaf(hat_y[i], m2, m1));
    }
    if (store) Row8<T>::store(dy + at, up);
    if constexpr (!kAhead) next = load(row + step);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) p[0][i] *= a.branch_scale;
  float* out = partial + static_cast<int64_t>(blockIdx.x) * __builtin_popcount(want) * a.d + c;
#pragma unroll
  for (int w = 0; w < 5; ++w) {
    if (!(want >> w & 1)) continue;
    if constexpr (kRows > 1) {
      __syncthreads();
      if (slot > 0) Row8<float>::store(s_merge + threadIdx.x * 8, p[w]);
      __syncthreads();
      if (slot == 0)
#pragma unroll
        for (int k = 1; k < kRows; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) p[w][i] += s_merge[(threadIdx.x + k * NT) * 8 + i];
    }
    if (slot == 0 && in) Row8<float>::store(out, p[w]);
    out += a.d;
  }
}

// Sums of the partial rows in their order: 64 columns of a parameter gradient per workgroup, 16 slices of the rows.
__global__ __launch_bounds__(1024) void residual_params_kernel(const float* __restrict__ partial, int rows, int d, int want, ResidualGrads out) {
  __shared__ float s_p[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), part = threadIdx.x >> 6, n = gridDim.y;
  float* const all[5] = {out.gate, out.post_gamma, out.post_beta, out.pre_gamma, out.pre_beta};
  float* dst = nullptr;
  int k = blockIdx.y;
#pragma unroll
  for (int w = 0; w < 5; ++w)
    if (want >> w & 1) {
      if (k == 0) dst = all[w];
      --k;
    }
  float s = 0.0f;
  if (c < d) {
    const float* const p = partial + static_cast<int64_t>(blockIdx.y) * d + c;
#pragma unroll 16
    for (int i = part; i < rows; i += 16) s += p[static_cast<int64_t>(i) * n * d];
  }
  s_p[part][threadIdx.x & 63] = s;
  __syncthreads();
  if (part == 0 && c < d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += s_p[i][threadIdx.x];
    dst[c] = s;
  }
}

template <int NT, typename T>
void forward(const ResidualArgs& a, const void* r, const void* y, void* total, void* normed, hipStream_t stream) {
  constexpr int kRows = rows_of_block<NT>();
  const int blocks = static_cast<int>(std::min<int64_t>((static_cast<int64_t>(a.T) + kRows - 1) / kRows, 2048));
  residual_norm_kernel<NT, T><<<blocks, block_threads<NT>(), 0, stream>>>(a, static_cast<const T*>(r), static_cast<const T*>(y), static_cast<T*>(total),
                                                                          static_cast<T*>(normed));
}

int threads_of_row(int d) {
  int nt = 64;
  while (nt * 8 < d) nt *= 2;
  return nt;
}
// As many workgroups as the registers let reside (158 of them a thread for bf16, 186 for fp32: three and two workgroups of
// 256 threads per CU), at least two rows for each slot: every workgroup leaves a partial row.  (8191 x 2048 bf16, the rows'
// kernel and the sums behind it: two 57.3 + 4.8 us, three 49.0 + 6.2.)
int backward_blocks(int T, int d, bool f32) {
  const int nt = threads_of_row(d), rows = std::max(256 / nt, 1);
  const int most = std::max((f32 ? 512 : 768) * 256 / std::max(nt, 256), 256);
  return static_cast<int>(std::max<int64_t>(std::min<int64_t>((static_cast<int64_t>(T) + 2 * rows - 1) / (2 * rows), most), 1));
}

template <int NT, typename T>
void backward(const ResidualArgs& a, const void* r, const void* y, const void* d_total, const void* d_normed, void* dr, void* dy, float* partial,
              int want, hipStream_t stream) {
  residual_norm_backward_kernel<NT, T><<<backward_blocks(a.T, a.d, sizeof(T) == 4), block_threads<NT>(), 0, stream>>>(
      a, static_cast<const T*>(r), static_cast<const T*>(y), static_cast<const T*>(d_total), static_cast<const T*>(d_normed), static_cast<T*>(dr),
      static_cast<T*>(dy), partial, want);
}

}  // namespace

#define MOTE_ROW_DISPATCH(CALL)                 \
  switch (threads_of_row(a.d)) {                \
    case 64: CALL(64); break;                   \
    case 128: CALL(128); break;                 \
    case 256: CALL(256); break;                 \
    case 512: CALL(512); break;                 \
    default: CALL(1024); break;                 \
  }

hipError_t launch_residual_norm(const ResidualArgs& a, bool f32, const void* r, const void* y, void* total, void* normed, hipStream_t stream) {
#define MOTE_CALL(NT) f32 ? forward<NT, float>(a, r, y, total, normed, stream) : forward<NT, uint16_t>(a, r, y, total, normed, stream)
  MOTE_ROW_DISPATCH(MOTE_CALL)
#undef MOTE_CALL
  return hipGetLastError();
}

size_t residual_norm_workspace_bytes(int T, int d) {
  return 256 + static_cast<size_t>(backward_blocks(std::max(T, 1), d, false)) * 5 * d * sizeof(float);
}

hipError_t launch_residual_norm_backward(const ResidualArgs& a, bool f32, const void* r, const void* y, const void* d_total, const void* d_normed, void* dr,
                                         void* dy, const ResidualGrads& grads, void* workspace, hipStream_t stream) {
  const int want = (grads.gate ? 1 : 0) | (grads.post_gamma ? 2 : 0) | (grads.post_beta ? 4 : 0) | (grads.pre_gamma ? 8 : 0) | (grads.pre_beta ? 16 : 0);
  float* const partial = static_cast<float*>(workspace);
  int rows = 0;
  if (a.T > 0) {
    rows = backward_blocks(a.T, a.d, f32);
#define MOTE_CALL(NT)                                                                                      \
  f32 ? backward<NT, float>(a, r, y, d_total, d_normed, dr, dy, partial, want, stream)                      \
      : backward<NT, uint16_t>(a, r, y, d_total, d_normed, dr, dy, partial, want, stream)
    MOTE_ROW_DISPATCH(MOTE_CALL)
#undef MOTE_CALL
  }
  if (want) residual_params_kernel<<<dim3((a.d + 63) / 64, __builtin_popcount(want)), 1024, 0, stream>>>(partial, rows, a.d, want, grads);
  return hipGetLastError();
}

}  // namespace mote
