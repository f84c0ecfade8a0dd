// Scored routing (softmax or sigmoid scores, selection bias, groups, top-k, renormalised weights) and its gradient.
#include <algorithm>
#include <cfloat>

#include "common.h"
#include "launch.h"

namespace mote {

// ------------------------------------------------------------------------------------------------------- forward
//
// A workgroup of eight wavefronts owns 32 tokens.  Logits: bf16 MFMA (32 tokens x 32 experts x 16 channels, twice: the
// router's rows [d, E] are read as pairs of experts, so one operand has the even and one the odd experts), the wavefronts
// split the channels in units of 64.  The fp32 accumulators of a unit are added to fp64 sums: what is left is the rounding
// inside a unit, which has a bound, and an index may depend on it only where two keys are closer than that bound.  There the
// logits in question are summed again in fp64, so that the indices are those of fp64 logits.  (fp64 MFMA on every logit would
// be bound by its issue: 8192 x 2048 x 64 27 us at its peak rate, against 7 us for the hidden states from HBM.)
constexpr int kRtTokens = 32;     // tokens of a workgroup
constexpr int kRtWaves = 8;
constexpr int kRtThreads = 64 * kRtWaves;
constexpr int kRtUnit = 64;       // channels of a unit
constexpr int kRtRow = 65;        // elements of an LDS row of 64 logits or keys: the rows of a wavefront's four tokens start in different banks
// Bound of a unit's rounding, in units of 2^-24 |x| |w| (Euclidean norms, which bound sum |x w|): four chained instructions, each
// of which aligns 16 products and the addend to the largest of them; measured at most 6.1 units of sum |x w| per instruction
// over normal, one-signed, wide-range and one-large inputs, taken as 16.  Plus the rounding of a logit to fp32.
constexpr float kRtBound = (4 * 16 + 2) * 0x1p-24f * 1.02f;

// LDS written and read by lanes of one wavefront
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Reductions over the 16 lanes of a DPP row, the same result in all of them
template <int CTRL> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return __int_as_float(dpp<CTRL>(__float_as_int(v))); }
template <int CTRL> __device__ __forceinline__ double dpp(double v) {
  return __hiloint2double(dpp<CTRL>(__double2hiint(v)), dpp<CTRL>(__double2loint(v)));
}
template <typename T, typename F> __device__ __forceinline__ T row_reduce(T v, F f) {
  v = f(v, dpp<0xB1>(v));    // lane ^ 1
  v = f(v, dpp<0x4E>(v));    // lane ^ 2
  v = f(v, dpp<0x141>(v));   // half-row mirror
  return f(v, dpp<0x140>(v));
}
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double max_of(double a, double b) { return fmax(a, b); }
template <typename T> __device__ __forceinline__ T row_max(T v) { return row_reduce(v, [](T a, T b) { return max_of(a, b); }); }
template <typename T> __device__ __forceinline__ T row_min(T v) { return -row_max(-v); }
template <typename T> __device__ __forceinline__ T row_sum(T v) { return row_reduce(v, [](T a, T b) { return a + b; }); }
__device__ __forceinline__ int row_or(int v) { return row_reduce(v, [](int a, int b) { return a | b; }); }
__device__ __forceinline__ int row_min_int(int v) { return row_reduce(v, [](int a, int b) { return min(a, b); }); }
__device__ __forceinline__ float exp_of(float v) { return expf(v); }
__device__ __forceinline__ double exp_of(double v) { return exp(v); }
__device__ __forceinline__ float abs_of(float v) { return fabsf(v); }
__device__ __forceinline__ double abs_of(double v) { return fabs(v); }
template <typename R> constexpr R lowest_of() { return sizeof(R) == 8 ? static_cast<R>(-DBL_MAX) : static_cast<R>(-FLT_MAX); }

// Selection for one token by the 16 lanes of a DPP row; lane s has the experts s + 16 v.
//   R = float : all keys in fp32 from logits that are off by at most `tol`; returns in every lane of the row whether two keys
//               are too close for that
//   R = double: the same on fp64 keys; bit v of `exact`: the logit of the lane's expert is settled.  `again` gets the experts
//               (bit v) whose logits have to be settled, 0 in every lane of the row: the selection is final
// The selected experts go to sel[0 .. k) (the caller has filled it with -1), lowest index first among equal keys.
// sc: scores of the lane's experts, shift and total: softmax is exp(l - shift) / total.
template <typename R>
__device__ __forceinline__ bool route_select(const RouteArgs& a, const double* l_row, R* key_row, R* grp_row, volatile int* sel, float tol, int exact, int* again,
                                             float (&sc)[4], float& shift, float& total) {
  constexpr bool kExact = sizeof(R) == 8;
  const int s = threadIdx.x & 15, E = a.E;
  const R kNone = -INFINITY;
  double l[4];
  R key[4], score[4];
  float mx = -INFINITY;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    l[v] = s + 16 * v < E ? l_row[s + 16 * v] : static_cast<double>(-INFINITY);
    mx = fmaxf(mx, static_cast<float>(l[v]));
  }
  const bool by_logit = a.bias == nullptr && !(a.n_groups > 1 && a.group_top == 2);
  total = 1.0f;
  if (a.sigmoid) {
    shift = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      score[v] = s + 16 * v < E ? R(1) / (R(1) + exp_of(static_cast<R>(-l[v]))) : R(0);
      sc[v] = static_cast<float>(score[v]);
    }
  } else {
    mx = row_max(mx);
    shift = mx;
    R sum = 0;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      score[v] = s + 16 * v < E ? exp_of(static_cast<R>(l[v] - static_cast<double>(mx))) : R(0);
      sum += score[v];
    }
    sum = row_sum(sum);
    total = static_cast<float>(sum);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      score[v] /= sum;
      sc[v] = static_cast<float>(score[v]);
    }
  }
  // how far a key may be off: the logits' bound through the score's slope (a quarter for the sigmoid, at most 2 P for the softmax)
  // and, in fp32, the rounding of the score
  float delta = tol;
  if (!by_logit) {
    delta = a.sigmoid ? 0.25f * tol : 2.2f * tol;
    if (!kExact) delta += (a.sigmoid ? 8.0f : 16.0f + 4.0f * fabsf(mx)) * 0x1p-24f;
    if (!(tol < 0.05f)) delta = INFINITY;
  }
  const R slack = kExact ? R(0x1p-50) : R(4 * 0x1p-24);
  auto near = [&](R x, R y, float width) { return !(abs_of(x - y) > static_cast<R>(width) + slack * (abs_of(x) + abs_of(y))); };
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int e = s + 16 * v;
    key[v] = kNone;
    if (e < E) {
      key[v] = by_logit ? static_cast<R>(l[v]) : score[v] + (a.bias ? static_cast<R>(a.bias[e]) : R(0));
      if (key[v] != key[v]) key[v] = lowest_of<R>();
    }
  }
  bool close = false;
  int more = 0;
  if (a.n_groups > 1) {
    const int G = a.n_groups, n = E / G;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (s + 16 * v < E) key_row[s + 16 * v] = key[v];
    wave_lds_fence();
    R gs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = s + 16 * i;
      gs[i] = kNone;
      if (g < G) {
        R t1 = kNone, t2 = kNone;
        for (int j = 0; j < n; ++j) {
          const R kv = key_row[g * n + j];
          t2 = max_of(t2, kv > t1 ? t1 : kv);
          t1 = max_of(t1, kv);
        }
        gs[i] = a.group_top == 2 ? t1 + t2 : t1;
        grp_row[g] = gs[i];
      }
    }
    wave_lds_fence();
    uint64_t open = 0;
    R worst_in = INFINITY, best_out = kNone;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (16 * i >= G) break;
      const int g = s + 16 * i;
      int rank = 0;
      for (int j = 0; j < G; ++j) {
        const R o = grp_row[j];
        rank += (o > gs[i] || (o == gs[i] && j < g)) ? 1 : 0;
      }
      const bool in = g < G && rank < a.top_groups;
      if (g < G) {
        if (in) worst_in = -max_of(-worst_in, -gs[i]);
        else best_out = max_of(best_out, gs[i]);
      }
      open |= ((__ballot(in) >> (threadIdx.x & 48)) & 0xFFFFull) << (16 * i);
    }
    worst_in = row_min(worst_in);
    best_out = row_max(best_out);
    const float width = 2.0f * static_cast<float>(a.group_top) * delta;
    if (best_out > kNone && near(worst_in, best_out, width)) {
      if constexpr (kExact) {   // every unsettled expert of the groups around the border
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int e = s + 16 * v;
          if (e < E && !(exact >> v & 1)) {
            const R g = grp_row[e / n];
            if (near(g, worst_in, width) || near(g, best_out, width)) more |= 1 << v;
          }
        }
      } else {
        close = true;
      }
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int e = s + 16 * v;
      if (e < E && !((open >> (e / n)) & 1)) key[v] = kNone;
    }
  }
  R first[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) first[v] = key[v];
  R last = INFINITY;
  int surplus = 0;   // keys taken less rounds: equal keys are close
  for (int j = 0; j <= a.k; ++j) {
    const R m = row_max(max_of(max_of(key[0], key[1]), max_of(key[2], key[3])));
    if constexpr (kExact) {
      if (j == a.k) break;
      int e_min = 64;
#pragma unroll
      for (int v = 3; v >= 0; --v)
        if (key[v] == m && m > kNone) e_min = s + 16 * v;
      e_min = row_min_int(e_min);
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (e_min == s + 16 * v) {
          sel[j] = e_min;
          key[v] = kNone;
        }
      if (m > kNone) {   // unsettled experts whose key may be on the other side of this one
        int count = 0, open = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (first[v] > kNone && near(first[v], m, 2.0f * delta)) {
            ++count;
            if (!(exact >> v & 1)) open |= 1 << v;
          }
        if (row_sum(count) > 1) more |= open;
      }
    } else {
      if (j > 0 && m > kNone && near(last, m, 2.0f * delta)) close = true;
      last = m;
      surplus -= m > kNone && s == 0 ? 1 : 0;
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (key[v] == m && m > kNone) {   // equal keys go together
          if (j < a.k) sel[j] = s + 16 * v;
          key[v] = kNone;
          ++surplus;
        }
    }
  }
  if constexpr (!kExact) close |= row_sum(surplus) > 0;
  if constexpr (kExact) *again = more;
  return close;
}

// fp64 logits of the experts e0, e1 of a token by one wavefront.
__device__ __forceinline__ void exact_logits(const RouteArgs& a, int tok, int e0, int e1, double* l_row) {
  const int lane = threadIdx.x & 63;
  const uint16_t* const xr = a.x + static_cast<int64_t>(tok) * a.d;
  double s0 = 0.0, s1 = 0.0;
#pragma unroll 8
  for (int c = lane; c < a.d; c += 64) {
    const double xv = bf16_to_f32(xr[c]);
    s0 = fma(xv, static_cast<double>(bf16_to_f32(a.w_router[c * a.E + e0])), s0);
    s1 = fma(xv, static_cast<double>(bf16_to_f32(a.w_router[c * a.E + e1])), s1);
  }
  s0 = wave_sum(s0);
  s1 = wave_sum(s1);
  if (lane == 0) {
    l_row[e0] = s0;
    l_row[e1] = s1;
  }
}

struct RouteLds {
  union {
    double red[4][32 * 64];                    // partial sums of four wavefronts: one lane's 32 logits in stride
    struct {
      double key[kRtTokens][kRtRow], grp[kRtTokens][kRtRow];
    } pick;
  };
  double l[kRtTokens][kRtRow];                 // finished logits
  float nx[kRtWaves][64], nw[kRtWaves][2][64]; // shares of |x|^2 of the tokens and of |w|^2 of the experts
  uint32_t orx[kRtWaves][64], orw[kRtWaves];   // bits of the values: all zero or not
  int sel[kRtTokens][8];
  double sum[kRtWaves][64];
  int cnt[64];
};

// 64 channels of the 32 tokens and of all experts
struct RouteUnit {
  u4 x[4];
  uint32_t w[32];
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float dot2(uint32_t v, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v), __builtin_bit_cast(bf16x2, v), c, false);
}

// PAIRS: E is even, two experts of a row are one aligned word.
template <bool PAIRS>
__global__ __launch_bounds__(kRtThreads) void route_kernel(RouteArgs a) {
  __shared__ RouteLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 31, g = lane >> 5;
  const int t0 = blockIdx.x * kRtTokens;
  const int units = a.d / kRtUnit;
  if (tid < 64) lds.cnt[tid] = 0;
  if (tid < kRtTokens * 8) lds.sel[tid >> 3][tid & 7] = -1;

  const uint16_t* const xr = a.x + static_cast<int64_t>(min(t0 + r, a.T - 1)) * a.d + 8 * g;
  const unsigned row_bytes = 2u * a.E;
  const int e_lo = PAIRS ? 2 * min(r, a.E / 2 - 1) : min(2 * r, a.E - 1), e_hi = min(2 * r + 1, a.E - 1);
  auto load = [&](int u) __attribute__((always_inline)) {
    RouteUnit q;
    u = min(u, units - 1);
#pragma unroll
    for (int s = 0; s < 4; ++s) q.x[s] = *reinterpret_cast<const u4*>(xr + u * kRtUnit + 16 * s);
    const char* const wb = reinterpret_cast<const char*>(a.w_router) + static_cast<size_t>(u) * kRtUnit * row_bytes;   // uniform
    const unsigned lo = 8u * g * row_bytes + 2u * e_lo, hi = 8u * g * row_bytes + 2u * e_hi;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const char* const p = wb + (16 * s + i) * row_bytes;
        if constexpr (PAIRS) q.w[8 * s + i] = *reinterpret_cast<const uint32_t*>(p + lo);
        else q.w[8 * s + i] = *reinterpret_cast<const uint16_t*>(p + lo) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p + hi)) << 16;
      }
    return q;
  };
  double even[16], odd[16];
#pragma unroll
  for (int v = 0; v < 16; ++v) even[v] = odd[v] = 0.0;
  float nx = 0.0f, nw0 = 0.0f, nw1 = 0.0f;
  uint32_t orx = 0, orw = 0;
  auto compute = [&](const RouteUnit& q) __attribute__((always_inline)) {
    v16f c0, c1;
#pragma unroll
    for (int v = 0; v < 16; ++v) c0[v] = c1[v] = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u4 b0, b1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        b0[i] = __builtin_amdgcn_perm(q.w[8 * s + 2 * i + 1], q.w[8 * s + 2 * i], 0x05040100u);
        b1[i] = __builtin_amdgcn_perm(q.w[8 * s + 2 * i + 1], q.w[8 * s + 2 * i], 0x07060302u);
        nx = dot2(q.x[s][i], nx);
        nw0 = dot2(b0[i], nw0);
        nw1 = dot2(b1[i], nw1);
        orx |= q.x[s][i];
        orw |= b0[i] | b1[i];
      }
      c0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q.x[s]), __builtin_bit_cast(bf16x8, b0), c0, 0, 0, 0);
      c1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q.x[s]), __builtin_bit_cast(bf16x8, b1), c1, 0, 0, 0);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      even[v] += static_cast<double>(c0[v]);
      odd[v] += static_cast<double>(c1[v]);
    }
  };
  if (wave < units) {
    RouteUnit p = load(wave), q;
    for (int u = wave; u < units; u += 2 * kRtWaves) {
      q = load(u + kRtWaves);
      compute(p);
      if (u + kRtWaves >= units) break;
      p = load(u + 2 * kRtWaves);
      compute(q);
    }
  }
  // Sums over the wavefronts in a fixed order: 4 .. 7 onto 0 .. 3, then all four.  Element v of a lane is token
  // (v & 3) + 8 (v >> 2) + 4 g, experts 2 r (even) and 2 r + 1 (odd).
  lds.nx[wave][lane] = nx;
  lds.nw[wave][0][lane] = nw0;
  lds.nw[wave][1][lane] = nw1;
  lds.orx[wave][lane] = orx & 0x7FFF7FFFu;
  const bool any_w = __ballot((orw & 0x7FFF7FFFu) != 0) != 0;
  if (lane == 0) lds.orw[wave] = any_w;
  double* const mine = lds.red[wave & 3] + lane;
  if (wave >= 4) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      mine[64 * v] = even[v];
      mine[64 * (16 + v)] = odd[v];
    }
  }
  __syncthreads();
  if (wave < 4) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      mine[64 * v] += even[v];
      mine[64 * (16 + v)] += odd[v];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = tid + i * kRtThreads;
    const double sum = ((lds.red[0][at] + lds.red[1][at]) + lds.red[2][at]) + lds.red[3][at];
    const int v = at >> 6, ln = at & 63;
    lds.l[(v & 3) + 8 * ((v >> 2) & 3) + 4 * (ln >> 5)][2 * (ln & 31) + (v >> 4)] = sum;
  }
  __syncthreads();

  // Selection: 16 lanes per token, all 32 at once.
  const int t = tid >> 4, s = tid & 15, tok = t0 + t;
  const bool live = tok < a.T;
  const bool masked = live && a.mask != nullptr && a.mask[tok] == 0;
  float x2 = lds.nx[s & 7][t + 32 * (s >> 3)];
  int bits = static_cast<int>(lds.orx[s & 7][t + 32 * (s >> 3)]);
  x2 = row_sum(x2);
  bits = row_or(bits);
  float w2 = 0.0f;
  int w_nan = 0;
  uint32_t wbits = 0;
#pragma unroll
  for (int v = 0; v < 4; ++v) {   // lane s: experts s + 16 v
    float n = 0.0f;
#pragma unroll
    for (int i = 0; i < kRtWaves; ++i) n += lds.nw[i][s & 1][(s >> 1) + 8 * v] + lds.nw[i][s & 1][(s >> 1) + 8 * v + 32];
    const bool in = s + 16 * v < a.E;
    w2 = fmaxf(w2, in ? n : 0.0f);
    w_nan |= in && n != n;
  }
#pragma unroll
  for (int i = 0; i < kRtWaves; ++i) wbits |= lds.orw[i];
  w_nan = row_or(w_nan);
  w2 = row_max(w2);
  // squares that underflow say nothing; products below the smallest normal value are off by an absolute amount
  const bool zero = bits == 0 || wbits == 0;
  float tol = kRtBound * sqrtf(x2) * sqrtf(w2) + 0x1p-120f;
  if (w_nan || !(x2 > 0x1p-80f && w2 > 0x1p-80f)) tol = INFINITY;
  if (zero) tol = 0.0f;
  float sc[4], shift, total;
  float* const fkey = reinterpret_cast<float*>(lds.pick.key[t]);
  float* const fgrp = reinterpret_cast<float*>(lds.pick.grp[t]);
  const bool vague = !(tol < INFINITY);   // the bound says nothing: every logit of the token is settled
  const bool close = (route_select<float>(a, lds.l[t], fkey, fgrp, lds.sel[t], tol, 0, nullptr, sc, shift, total) || vague) && live && !masked;
  if (__ballot(close)) {   // rare: settle what is too close
    int exact = zero ? 15 : 0, again = 0, all = 0;
#pragma unroll
    for (int v = 0; v < 4; ++v) all |= s + 16 * v < a.E ? 1 << v : 0;
    for (;;) {
      if (s < 8) lds.sel[t][s] = -1;
      wave_lds_fence();
      route_select<double>(a, lds.l[t], lds.pick.key[t], lds.pick.grp[t], lds.sel[t], tol, exact, &again, sc, shift, total);
      again = close ? (vague ? all : again) & ~exact : 0;
      uint64_t b[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) b[v] = __ballot(again >> v & 1);
      if (!(b[0] | b[1] | b[2] | b[3])) break;
      for (int q = 0; q < 4; ++q) {
        uint64_t m = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) m |= ((b[v] >> (16 * q)) & 0xFFFFull) << (16 * v);
        while (m) {
          const int e0 = __builtin_ctzll(m);
          m &= m - 1;
          const int e1 = m ? __builtin_ctzll(m) : e0;
          if (m) m &= m - 1;
          exact_logits(a, t0 + (wave << 2) + q, e0, e1, lds.l[(wave << 2) + q]);
        }
      }
      exact |= again;
      wave_lds_fence();
    }
  }
  wave_lds_fence();
  // weights: lane j < k has slot j
  const int e = s < a.k && !masked ? static_cast<volatile int*>(lds.sel[t])[s] : -1;
  const bool have = e >= 0;
  const double l = have ? lds.l[t][e] : 0.0;
  float w = 0.0f;
  if (a.renormalise) {
    // a softmax over log s of the selected (softmax scores: log s is the logit up to a constant of the row)
    const float ref = row_max(have ? static_cast<float>(l) : -INFINITY);
    float al = static_cast<float>(l - static_cast<double>(ref));
    if (a.sigmoid) {
      const float lf = static_cast<float>(l);
      al = fminf(lf, 0.0f) - log1pf(expf(-fabsf(lf)));
      const float top = row_max(have ? al : -INFINITY);
      al -= top;
    }
    const float ex = have ? expf(al) : 0.0f;
    w = ex / row_sum(ex);
  } else {
    w = a.sigmoid ? 1.0f / (1.0f + expf(-static_cast<float>(l))) : expf(static_cast<float>(l - static_cast<double>(shift))) / total;
  }
  if (live && s < a.k) {
    a.topk_idx[static_cast<int64_t>(tok) * a.k + s] = e;
    a.topk_w[static_cast<int64_t>(tok) * a.k + s] = have ? w * a.scale : 0.0f;
    if (have && a.part_cnt != nullptr) atomicAdd(&lds.cnt[e], 1);
  }
  if (live && a.logits != nullptr) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (s + 16 * v < a.E) a.logits[static_cast<int64_t>(tok) * a.E + s + 16 * v] = static_cast<float>(lds.l[t][s + 16 * v]);
  }
  if (a.part_sum == nullptr) return;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    double d = live && !masked ? static_cast<double>(sc[v]) : 0.0;
    d += __shfl_xor(d, 16, 64);
    d += __shfl_xor(d, 32, 64);
    if (lane < 16) lds.sum[wave][lane + 16 * v] = d;
  }
  __syncthreads();
  if (tid < 64) {
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kRtWaves; ++i) d += lds.sum[i][tid];
    a.part_sum[static_cast<int64_t>(blockIdx.x) * 64 + tid] = d;
    a.part_cnt[static_cast<int64_t>(blockIdx.x) * 64 + tid] = lds.cnt[tid];
  }
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
  if (a.T > 0) {
    if (a.E % 2 == 0 && (reinterpret_cast<uintptr_t>(a.w_router) & 3) == 0) route_kernel<true><<<blocks, kRtThreads, 0, stream>>>(a);
    else route_kernel<false><<<blocks, kRtThreads, 0, stream>>>(a);
  }
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
