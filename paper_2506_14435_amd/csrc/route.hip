// Scored routing (softmax or sigmoid scores, selection bias, groups, top-k, renormalised weights) and its gradient.
#include <algorithm>
#include <cfloat>

#include "common.h"
#include "launch.h"

namespace mote {

constexpr int kRtTokens = 4;      // tokens of a workgroup
constexpr int kRtThreads = 256;
constexpr int kRtRow = 66;        // doubles of an LDS row of 64 keys: rows of the four tokens of a wavefront start in different banks

__device__ __forceinline__ double shfl16(double v, int off) { return __shfl_xor(v, off, 16); }

// LDS written and read by lanes of one wavefront
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// One token by 16 lanes: lane s owns the experts s + 16 v.  l_row: its finished logits in LDS; key_row, grp_row: LDS scratch
// of 64 doubles (groups only).  Returns the scores of the lane's experts in sc.
__device__ __forceinline__ void route_token(const RouteArgs& a, const double* l_row, double* key_row, double* grp_row, int tok, bool live,
                                            bool masked, double (&sc)[4], int* s_cnt) {
  const int s = threadIdx.x & 15, E = a.E;
  double l[4], key[4];
  double mx = -INFINITY;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    l[v] = s + 16 * v < E ? l_row[s + 16 * v] : -INFINITY;
    mx = fmax(mx, l[v]);
  }
  double lse_sum = 1.0;
  if (a.sigmoid) {
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] = s + 16 * v < E ? 1.0 / (1.0 + exp(-l[v])) : 0.0;
  } else {
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) mx = fmax(mx, shfl16(mx, off));
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      sc[v] = s + 16 * v < E ? exp(l[v] - mx) : 0.0;
      sum += sc[v];
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) sum += shfl16(sum, off);
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] = sc[v] / sum;
    lse_sum = sum;
  }
  const bool by_logit = a.bias == nullptr && !(a.n_groups > 1 && a.group_top == 2);
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int e = s + 16 * v;
    key[v] = -INFINITY;
    if (e < E) {
      key[v] = by_logit ? l[v] : sc[v] + (a.bias ? static_cast<double>(a.bias[e]) : 0.0);
      if (key[v] != key[v]) key[v] = -DBL_MAX;
    }
  }
  if (a.n_groups > 1) {
    const int G = a.n_groups, n = E / G;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (s + 16 * v < E) key_row[s + 16 * v] = key[v];
    wave_lds_fence();
    double gs[4];
    for (int i = 0; i < 4; ++i) {
      const int g = s + 16 * i;
      gs[i] = -INFINITY;
      if (g < G) {
        double t1 = -INFINITY, t2 = -INFINITY;
        for (int j = 0; j < n; ++j) {
          const double kv = key_row[g * n + j];
          if (kv > t1) { t2 = t1; t1 = kv; }
          else if (kv > t2) t2 = kv;
        }
        gs[i] = a.group_top == 2 ? t1 + t2 : t1;
        grp_row[g] = gs[i];
      }
    }
    wave_lds_fence();
    uint64_t open = 0;
    for (int i = 0; i < 4; ++i) {
      const int g = s + 16 * i;
      int rank = 0;
      for (int j = 0; j < G; ++j) {
        const double o = grp_row[j];
        rank += (o > gs[i] || (o == gs[i] && j < g)) ? 1 : 0;
      }
      const uint64_t m = __ballot(g < G && rank < a.top_groups);
      open |= ((m >> (threadIdx.x & 48)) & 0xFFFFull) << (16 * i);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int e = s + 16 * v;
      if (e < E && !((open >> (e / n)) & 1)) key[v] = -INFINITY;
    }
  }
  int my_e = -1;
  for (int j = 0; j < a.k; ++j) {
    double b = -INFINITY;
    int be = 1 << 20;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (key[v] > b) { b = key[v]; be = s + 16 * v; }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) {
      const double ob = shfl16(b, off);
      const int oe = __shfl_xor(be, off, 16);
      const bool take = ob > b || (ob == b && oe < be);
      b = take ? ob : b;
      be = take ? oe : be;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (be == s + 16 * v) key[v] = -INFINITY;
    if (s == j && be < E) my_e = be;
  }
  if (masked) my_e = -1;
  // weights: lane j < k has slot j
  const bool have = my_e >= 0;
  const double ls = have ? l_row[my_e] : 0.0;
  double w = 0.0;
  if (a.renormalise) {
    // log of the score (softmax: up to a constant of the row)
    double al = -INFINITY;
    if (have) al = a.sigmoid ? fmin(ls, 0.0) - log1p(exp(-fabs(ls))) : ls;
    double m = al;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) m = fmax(m, shfl16(m, off));
    const double ex = have ? exp(al - m) : 0.0;
    double sum = ex;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) sum += shfl16(sum, off);
    w = have ? ex / sum : 0.0;
  } else if (have) {
    w = a.sigmoid ? 1.0 / (1.0 + exp(-ls)) : exp(ls - mx) / lse_sum;
  }
  if (live && s < a.k) {
    a.topk_idx[static_cast<int64_t>(tok) * a.k + s] = my_e;
    a.topk_w[static_cast<int64_t>(tok) * a.k + s] = have ? static_cast<float>(w * static_cast<double>(a.scale)) : 0.0f;
    if (have && s_cnt != nullptr) atomicAdd(&s_cnt[my_e], 1);
  }
  if (live && a.logits != nullptr) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (s + 16 * v < E) a.logits[static_cast<int64_t>(tok) * E + s + 16 * v] = static_cast<float>(l[v]);
  }
  if (masked || !live) {
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] = 0.0;
  }
}

// Four tokens per workgroup; wavefront w sums a quarter of the channels, lane e has expert e.
__global__ __launch_bounds__(kRtThreads) void route_kernel(RouteArgs a) {
  __shared__ double s_l[4][kRtTokens][kRtRow];
  __shared__ double s_key[kRtTokens][kRtRow], s_grp[kRtTokens][kRtRow];
  __shared__ int s_cnt[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t0 = blockIdx.x * kRtTokens;
  if (threadIdx.x < 64) s_cnt[threadIdx.x] = 0;
  double acc[kRtTokens] = {0.0, 0.0, 0.0, 0.0};
  const int e = min(lane, a.E - 1);
  for (int c = wave; c < a.d; c += 4) {
    const double w = bf16_to_f32(a.w_router[static_cast<int64_t>(c) * a.E + e]);
#pragma unroll
    for (int t = 0; t < kRtTokens; ++t)
      acc[t] = fma(static_cast<double>(bf16_to_f32(a.x[static_cast<int64_t>(min(t0 + t, a.T - 1)) * a.d + c])), w, acc[t]);
  }
#pragma unroll
  for (int t = 0; t < kRtTokens; ++t) s_l[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < kRtTokens; t += 4) {
    s_l[0][t][lane] = ((s_l[0][t][lane] + s_l[1][t][lane]) + s_l[2][t][lane]) + s_l[3][t][lane];
  }
  __syncthreads();
  if (wave == 0) {
    const int t = lane >> 4, tok = t0 + t;
    const bool live = tok < a.T;
    const bool masked = live && a.mask != nullptr && a.mask[tok] == 0;
    double sc[4];
    route_token(a, s_l[0][t], s_key[t], s_grp[t], tok, live, masked, sc, a.part_cnt ? s_cnt : nullptr);
    if (a.part_sum != nullptr) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        sc[v] += __shfl_xor(sc[v], 16, 64);
        sc[v] += __shfl_xor(sc[v], 32, 64);
        if (lane < 16) a.part_sum[static_cast<int64_t>(blockIdx.x) * 64 + lane + 16 * v] = sc[v];
      }
    }
  }
  __syncthreads();
  if (a.part_cnt != nullptr && threadIdx.x < 64) a.part_cnt[static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x] = s_cnt[threadIdx.x];
}

// Counts and score sums of all workgroups, in their order.
__global__ __launch_bounds__(1024) void route_stats_kernel(const double* __restrict__ part_sum, const int32_t* __restrict__ part_cnt, int blocks,
                                                           int E, int32_t* __restrict__ counts, float* __restrict__ score_sum) {
  __shared__ double s_sum[16][64];
  __shared__ int s_cnt[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double a = 0.0;
  int c = 0;
  for (int b = wave; b < blocks; b += 16) {
    if (score_sum != nullptr) a += part_sum[static_cast<int64_t>(b) * 64 + lane];
    if (counts != nullptr) c += part_cnt[static_cast<int64_t>(b) * 64 + lane];
  }
  s_sum[wave][lane] = a;
  s_cnt[wave][lane] = c;
  __syncthreads();
  if (wave == 0 && lane < E) {
    for (int w = 1; w < 16; ++w) { a += s_sum[w][lane]; c += s_cnt[w][lane]; }
    if (score_sum != nullptr) score_sum[lane] = static_cast<float>(a);
    if (counts != nullptr) counts[lane] = c;
  }
}

static int route_blocks(int T) { return (T + kRtTokens - 1) / kRtTokens; }

size_t route_workspace_bytes(int T) { return 256 + static_cast<size_t>(route_blocks(T)) * 64 * (sizeof(double) + sizeof(int32_t)); }

hipError_t launch_route(RouteArgs a, int32_t* counts, float* score_sum, void* workspace, hipStream_t stream) {
  const int blocks = route_blocks(a.T);
  const bool stats = counts != nullptr || score_sum != nullptr;
  if (stats) {
    a.part_sum = static_cast<double*>(workspace);
    a.part_cnt = reinterpret_cast<int32_t*>(a.part_sum + static_cast<int64_t>(blocks) * 64);
  }
  if (a.T > 0) route_kernel<<<blocks, kRtThreads, 0, stream>>>(a);
  if (stats) route_stats_kernel<<<1, 1024, 0, stream>>>(a.part_sum, a.part_cnt, blocks, a.E, counts, score_sum);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void route_import_kernel(const int32_t* __restrict__ idx, const float* __restrict__ w, int n, int E,
                                                           int32_t* __restrict__ topk_idx, float* __restrict__ topk_p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int e = idx[i];
  const bool ok = e >= 0 && e < E;
  topk_idx[i] = ok ? e : 0;
  topk_p[i] = ok ? w[i] : 0.0f;
}

hipError_t launch_route_import(const int32_t* idx, const float* w, int n, int E, int32_t* topk_idx, float* topk_p, hipStream_t stream) {
  if (n > 0) route_import_kernel<<<(n + 255) / 256, 256, 0, stream>>>(idx, w, n, E, topk_idx, topk_p);
  return hipGetLastError();
}

// -------------------------------------------------------------------------------------------------------- gradient

// dL/dlogits of one token by 16 lanes (lane s: experts s + 16 v), fp32.
__device__ __forceinline__ void route_grad_token(const RouteBackwardArgs& a, int tok, bool live, float (&g)[4]) {
  const int s = threadIdx.x & 15, E = a.E;
  float l[4], sc[4], om[4], up[4], sel[4], q[4];
  const int64_t row = static_cast<int64_t>(tok) * E;
  float mx = -INFINITY;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int e = s + 16 * v;
    l[v] = e < E ? a.logits[row + e] : -INFINITY;
    q[v] = e < E && a.d_score_sum != nullptr ? a.d_score_sum[e] : 0.0f;
    up[v] = 0.0f;
    sel[v] = 0.0f;
    mx = fmaxf(mx, l[v]);
  }
  auto sum16 = [](float v) {
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) v += __shfl_xor(v, off, 16);
    return v;
  };
  for (int j = 0; j < a.k; ++j) {
    const int e = a.topk_idx[static_cast<int64_t>(tok) * a.k + j];
    const float d = a.d_topk_w[static_cast<int64_t>(tok) * a.k + j];
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (e == s + 16 * v && e < E) { up[v] += d; sel[v] += 1.0f; }
  }
  if (a.sigmoid) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float t = expf(-fabsf(l[v])), r = 1.0f / (1.0f + t);
      sc[v] = l[v] >= 0.0f ? r : t * r;
      om[v] = l[v] >= 0.0f ? t * r : r;   // 1 - s
    }
  } else {
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 16));
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      sc[v] = s + 16 * v < E ? expf(l[v] - mx) : 0.0f;
      om[v] = 1.0f;
      sum += sc[v];
    }
    sum = sum16(sum);
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] /= sum;
  }
  if (a.renormalise) {
    // softmax over log s of the selected
    float al[4], m = -INFINITY;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      al[v] = a.sigmoid ? fminf(l[v], 0.0f) - log1pf(expf(-fabsf(l[v]))) : l[v];
      if (sel[v] > 0.0f) m = fmaxf(m, al[v]);
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 16));
    float p[4], sum = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      p[v] = sel[v] > 0.0f ? expf(al[v] - m) : 0.0f;
      sum += p[v] * sel[v];
    }
    sum = sum16(sum);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    float dot = 0.0f, dq = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      p[v] *= inv;
      dot += p[v] * up[v];
      dq += sc[v] * q[v];
    }
    dot = sum16(dot);
    dq = sum16(dq);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      g[v] = a.scale * p[v] * (up[v] - sel[v] * dot) * om[v];
      g[v] += a.sigmoid ? sc[v] * om[v] * q[v] : sc[v] * (q[v] - dq);
    }
  } else {
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      up[v] = a.scale * up[v] + q[v];
      dot += sc[v] * up[v];
    }
    dot = sum16(dot);
#pragma unroll
    for (int v = 0; v < 4; ++v) g[v] = a.sigmoid ? sc[v] * om[v] * up[v] : sc[v] * (up[v] - dot);
  }
  const bool masked = a.mask != nullptr && a.mask[tok] == 0;
#pragma unroll
  for (int v = 0; v < 4; ++v)
    if (!live || masked || s + 16 * v >= E) g[v] = 0.0f;
}

__global__ __launch_bounds__(256) void route_dlogits_kernel(RouteBackwardArgs a) {
  const int tok = blockIdx.x * 16 + (threadIdx.x >> 4), s = threadIdx.x & 15;
  float g[4];
  route_grad_token(a, min(tok, a.T - 1), tok < a.T, g);
  if (tok < a.T)
#pragma unroll
    for (int v = 0; v < 4; ++v) a.g[static_cast<int64_t>(tok) * 64 + s + 16 * v] = g[v];
}

__global__ __launch_bounds__(256) void route_dx_kernel(RouteBackwardArgs a) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(a.T) * a.d) return;
  const int64_t t = i / a.d;
  const int c = static_cast<int>(i - t * a.d);
  float s = 0.0f;
  for (int e = 0; e < a.E; ++e) s = fmaf(a.g[t * 64 + e], bf16_to_f32(a.w_router[static_cast<int64_t>(c) * a.E + e]), s);
  a.dx[i] = s;
}

__global__ __launch_bounds__(256) void route_dw_kernel(RouteBackwardArgs a) {
  const int c = blockIdx.x, e = threadIdx.x & 63, part = threadIdx.x >> 6;
  __shared__ float s_p[4][64];
  float s = 0.0f;
  for (int t = part; t < a.T; t += 4) s = fmaf(bf16_to_f32(a.x[static_cast<int64_t>(t) * a.d + c]), a.g[static_cast<int64_t>(t) * 64 + e], s);
  s_p[part][e] = s;
  __syncthreads();
  if (threadIdx.x < a.E) a.dw[static_cast<int64_t>(c) * a.E + e] = ((s_p[0][e] + s_p[1][e]) + s_p[2][e]) + s_p[3][e];
}

size_t route_backward_workspace_bytes(int T, int d, int E) {
  (void)d; (void)E;
  return 256 + static_cast<size_t>(T) * 64 * sizeof(float);
}

hipError_t launch_route_backward(RouteBackwardArgs a, void* workspace, hipStream_t stream) {
  a.g = static_cast<float*>(workspace);
  if (a.T > 0) route_dlogits_kernel<<<(a.T + 15) / 16, 256, 0, stream>>>(a);
  if (a.T > 0 && a.dx) route_dx_kernel<<<static_cast<unsigned>((static_cast<int64_t>(a.T) * a.d + 255) / 256), 256, 0, stream>>>(a);
  if (a.dw) route_dw_kernel<<<a.d, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace mote
