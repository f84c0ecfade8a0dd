// Scored routing (softmax or sigmoid scores, selection bias, groups, top-k, renormalised weights) and its gradient.
#include <algorithm>
#include <cfloat>
#include <climits>

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
// How far a logit may be off.  An instruction adds its 16 channels in two steps of eight; a step cuts the products (and a smaller
// addend) at 2^-24 of the largest product's exponent, adds them and rounds to fp32 (read off the instruction with products that cancel).
// In units of 2^-24, with Euclidean norms: step j = 0 .. 7 of a unit is off by at most 8 |x_j| q_j, q the largest power of two not above
// any |w| of its eight channels, and by the sum so far, at most that of |x_i| |w_i| over the steps i <= j.  For all units that is
//   8 |x| sqrt(sum q^2) + sqrt(sum ((8 - j) |x_j|)^2) |w|     (of normal values 3.9 + 5.1 |x| |w|)
// however the values lie; without the q's, where they would have to be found in the loop, sqrt(sum ((16 - j) |x_j|)^2) |w|, 12.8.
// (Measured: one unit of products that take each other's bits is off by 11.1 |x| |w|, 0.93 of the bound.)
constexpr float kLogitBound = 0x1p-24f * 1.05f;

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
__device__ __forceinline__ int row_max(int v) { return row_reduce(v, [](int a, int b) { return max(a, b); }); }
__device__ __forceinline__ float row_max(float v) { return row_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ double row_max(double v) { return row_reduce(v, [](double a, double b) { return fmax(a, b); }); }
template <typename T> __device__ __forceinline__ T row_sum(T v) { return row_reduce(v, [](T a, T b) { return a + b; }); }
__device__ __forceinline__ double wave_max(double v) {
  v = row_max(v);
  v = fmax(v, __shfl_xor(v, 16, kWave));
  return fmax(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ double wave_add(double v) {
  v = row_sum(v);
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}
__device__ __forceinline__ double wave_min(double v) { return -wave_max(-v); }

// Hardware exp2: a unit of 2^-24, and |v| units for the rounding of its argument.  From fp64 the fraction of the exponent alone is
// rounded: for the weights; the scores of all experts, of which keys and sums are made, are four times as many (8192 x 2048 x 64 27.4 us with
// fp64 for them too, 1 x 2048 x 16 10.8 instead of 10.5).
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }
__device__ __forceinline__ float exp_of(double v) {
  double t = v * 1.4426950408889634;
  t = t < -200.0 ? -200.0 : t > 200.0 ? 200.0 : t;   // 0 and inf in fp32
  const double n = __builtin_rint(t);
  return __builtin_ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(t - n)), static_cast<int>(n));
}
// fp32 values as integers of the same order, and back; kNoKey is below all of them
constexpr int kNoKey = INT_MIN;
__device__ __forceinline__ int order_of(float v) {
  const int b = __float_as_int(v);
  return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float value_of(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7FFFFFFF)); }

__device__ __forceinline__ bool keys_are_logits(const RouteArgs& a) { return a.bias == nullptr && !(a.n_groups > 1 && a.group_top == 2); }

// How far a key may be off where the logits are off by tol: the score's slope is at most a quarter (sigmoid) or twice the score
// (softmax), of which none is above `most`.  Not for large tol, where a slope says nothing.
__device__ __forceinline__ float key_tolerance(const RouteArgs& a, float tol, float most) {
  if (keys_are_logits(a)) return tol;
  return tol < 0.05f ? (a.sigmoid ? 0.25f : 2.2f * most) * tol : INFINITY;
}
template <typename R>
__device__ __forceinline__ bool near_keys(R x, R y, float width, R slack) {
  return !(fabs(x - y) > static_cast<R>(width) + slack * (fabs(x) + fabs(y)));
}

// Scores of one token by the 16 lanes of a DPP row, lane s: experts s + 16 v.  Softmax is exp(l - shift) / total.
__device__ __forceinline__ void route_scores(const RouteArgs& a, const double* l_row, float (&sc)[4], double& shift, float& total) {
  const int s = threadIdx.x & 15;
  double l[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) l[v] = s + 16 * v < a.E ? l_row[s + 16 * v] : static_cast<double>(-INFINITY);
  shift = 0.0;
  total = 1.0f;
  if (a.sigmoid) {
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] = __builtin_amdgcn_rcpf(1.0f + exp_of(static_cast<float>(-l[v])));
  } else {
    shift = row_max(fmax(fmax(l[0], l[1]), fmax(l[2], l[3])));
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] = exp_of(static_cast<float>(l[v] - shift));
    total = row_sum((sc[0] + sc[1]) + (sc[2] + sc[3]));
    const float inv = __builtin_amdgcn_rcpf(total);
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] *= inv;
  }
#pragma unroll
  for (int v = 0; v < 4; ++v)
    if (s + 16 * v >= a.E) sc[v] = 0.0f;
}

// Selection for one token by the 16 lanes of a DPP row, on fp32 keys; the selected experts go to sel[0 .. k), which the caller
// has filled with -1, and the first one that is not to sel[k].  Returns in every lane of the row: 0, the selection is final; j in
// 1 .. k, only the experts sel[j - 1] and sel[j] are too close to be told apart; -1, more hangs on logits that are off by
// `tol` and scores by the rounding of exp_of and rcp.
// key_row, grp_row: 64 and 128 integers of LDS (groups only).
__device__ __forceinline__ int route_select(const RouteArgs& a, const double* l_row, const float (&sc)[4], double shift, float total, int* key_row, int* grp_row,
                                            int* sel, float tol) {
  const int s = threadIdx.x & 15, E = a.E;
  const bool by_logit = keys_are_logits(a);
  const float most = a.sigmoid ? 1.0f : 1.001f / total;   // the largest score
  float delta = key_tolerance(a, tol, most);
  if (!by_logit) delta += (a.sigmoid ? 8.0f : most * (16.0f + 4.0f * fabsf(static_cast<float>(shift)))) * 0x1p-24f;
  const float slack = 4 * 0x1p-24f;
  int key[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int e = s + 16 * v;
    float f = -INFINITY;
    if (e < E) f = by_logit ? static_cast<float>(l_row[e]) : sc[v] + (a.bias ? a.bias[e] : 0.0f);
    if (f != f) f = -FLT_MAX;
    key[v] = f > -INFINITY ? order_of(f) : kNoKey;
  }
  bool many = false;
  if (a.n_groups > 1) {
    const int G = a.n_groups, n = E / G;
#pragma unroll
    for (int v = 0; v < 4; ++v) key_row[s + 16 * v] = key[v];
    wave_lds_fence();
    float worst_in = INFINITY, best_out = -INFINITY;   // the least that a group inside, the most that one outside may have
    uint64_t open = 0;
#pragma unroll 1
    for (int i = 0; 16 * i < G; ++i) {
      const int g = s + 16 * i;
      int t1 = kNoKey, t2 = kNoKey;
#pragma unroll 1
      for (int j = 0; j < n; j += 8) {
        int kv[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) kv[q] = key_row[min(g * n + min(j + q, n - 1), 63)];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int c = j + q < n ? kv[q] : kNoKey;
          t2 = max(t2, min(c, t1));
          t1 = max(t1, c);
        }
      }
      int gs = t1;
      float lost = slack * fabsf(value_of(t1));   // by rounding the keys and their sum: of the size of the keys, which may cancel
      if (a.group_top == 2) {
        gs = t2 == kNoKey ? kNoKey : order_of(value_of(t1) + value_of(t2));
        lost += slack * fabsf(value_of(t2));
      }
      if (g < G) {
        grp_row[g] = gs;
        grp_row[64 + g] = __float_as_int(lost);
      }
    }
    wave_lds_fence();
#pragma unroll 1
    for (int i = 0; 16 * i < G; ++i) {
      const int g = s + 16 * i, gs = grp_row[min(g, G - 1)];
      int rank = 0;
#pragma unroll 1
      for (int j = 0; j < G; j += 8) {
        int o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = grp_row[min(j + q, G - 1)];
#pragma unroll
        for (int q = 0; q < 8; ++q) rank += j + q < G && (o[q] > gs || (o[q] == gs && j + q < g)) ? 1 : 0;
      }
      const bool in = g < G && rank < a.top_groups;
      if (g < G && gs != kNoKey) {
        const float lost = __int_as_float(grp_row[64 + g]), score = value_of(gs);   // +inf inside: a NaN, which fminf passes over
        if (in) worst_in = fminf(worst_in, score - lost);
        else best_out = fmaxf(best_out, score + lost);
      }
      open |= ((__ballot(in) >> (threadIdx.x & 48)) & 0xFFFFull) << (16 * i);
    }
    worst_in = -row_max(-worst_in);
    best_out = row_max(best_out);
    const float width = 2.0f * static_cast<float>(a.group_top) * delta;
    const unsigned inv_n = 65536u / static_cast<unsigned>(n) + 1u;   // e / n for e < 64
    many = !(worst_in - best_out > width);   // also where both are below the range of fp32
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (!((open >> (((s + 16 * v) * inv_n) >> 16)) & 1)) key[v] = kNoKey;
  }
  // a lane's keys in descending order, their experts in the bytes of ex
  int ex = s | (s + 16) << 8 | (s + 32) << 16 | (s + 48) << 24;
  auto order = [&](int i, int j) __attribute__((always_inline)) {
    const bool swap = key[j] > key[i];
    const int ki = swap ? key[j] : key[i], kj = swap ? key[i] : key[j];
    const int bi = (ex >> (8 * i)) & 0xFF, bj = (ex >> (8 * j)) & 0xFF, x = swap ? bi ^ bj : 0;
    key[i] = ki;
    key[j] = kj;
    ex ^= x << (8 * i) | x << (8 * j);
  };
  order(0, 1); order(2, 3); order(0, 2); order(1, 3); order(1, 2);
  float last = INFINITY, before = INFINITY;
  int surplus = 0, pair = 0;   // keys taken less rounds: equal keys of several lanes go together
#pragma unroll 1
  for (int j = 0; j <= a.k + 1; ++j) {
    const int m = row_max(key[0]);
    const float mv = value_of(m);
    const bool some = m != kNoKey, hit = some && key[0] == m;
    if (j <= a.k) {
      const bool close = some && j > 0 && near_keys(last, mv, 2.0f * delta, slack);
      many |= close && pair != 0;
      pair = close ? j : pair;
      surplus += (hit ? 1 : 0) - (some && s == 0 ? 1 : 0);
      if (hit) sel[j] = ex & 0xFF;
    } else {
      many |= some && pair == a.k && near_keys(before, mv, 2.0f * delta, slack);   // a third one at the end of the selection
    }
    before = last;
    last = mv;
    key[0] = hit ? key[1] : key[0];
    key[1] = hit ? key[2] : key[1];
    key[2] = hit ? key[3] : key[2];
    key[3] = hit ? kNoKey : key[3];
    ex = hit ? ex >> 8 : ex;
  }
  return many || row_sum(surplus) > 0 ? -1 : pair;
}

// The same for one token by a whole wavefront (lane e: expert e), on fp64 keys: the rare case, compact rather than fast.
// exact: bit e, the logit of expert e is settled; the others are off by tol.  Returns the experts whose logits have to be
// settled for the selection to be that of fp64 logits (0: it is final, sel is written).
// The keys of settled experts are as good as fp64, but for softmax scores with something added: the denominator has the logits of
// all experts in it.  An error of tol in those that are not settled moves it by a factor 1 + r, |r| <= (exp(tol) - 1) times the sum of
// their scores, and with it the difference of two keys by r times that of their scores.  Where that could change their order, the
// experts with the larger ones of those scores are settled too, round by round, until it cannot.
__device__ __forceinline__ uint64_t route_select_exact(const RouteArgs& a, const double* l_row, double* key_row, double* grp_row, int* sel, float tol,
                                                       uint64_t exact) {
  const int e = threadIdx.x & 63, E = a.E;
  const double kNone = -INFINITY, slack = 0x1p-50;
  const bool shared = !a.sigmoid && !keys_are_logits(a);
  const double l = e < E ? l_row[e] : kNone;
  double key = l, score = 0.0;
  if (!keys_are_logits(a)) {
    if (a.sigmoid) {
      key = 1.0 / (1.0 + exp(-l));
    } else {
      key = exp(l - wave_max(l));
      if (e >= E) key = 0.0;
      key /= wave_add(key);
      score = key;
    }
    if (a.bias && e < E) key += static_cast<double>(a.bias[e]);
  }
  if (key != key) key = -DBL_MAX;
  if (e >= E) key = kNone;
  const float width = 2.0f * key_tolerance(a, tol, shared ? static_cast<float>(wave_max(score)) * 1.001f : 1.0f);
  uint64_t more = 0, heavy = 0;   // heavy: of the scores that are not settled those around their mean and above, one at least
  double moved = 0.0;             // bounds |r|
  if (shared) {
    const bool open = e < E && !((exact >> e) & 1);
    const double mass = wave_add(open ? score : 0.0), mean = mass / static_cast<double>(max(E - __builtin_popcountll(exact), 1));
    moved = mass * (tol < 0.05f ? 1.1f * tol : INFINITY);
    heavy = __ballot(open && !(score < 0.99 * mean));
  }
  if (a.n_groups > 1) {
    const int G = a.n_groups, n = E / G;
    key_row[e] = key;
    grp_row[e] = score;
    wave_lds_fence();
    double t1 = kNone, t2 = kNone, mass = 0.0;   // mass: all scores of the group, at least those in its key
    if (e < G)
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const double kv = key_row[e * n + j];
        t2 = fmax(t2, fmin(kv, t1));
        t1 = fmax(t1, kv);
        mass += grp_row[e * n + j];
      }
    const double gs = a.group_top == 2 ? t1 + t2 : t1;
    wave_lds_fence();
    grp_row[e] = gs;
    wave_lds_fence();
    key_row[e] = a.group_top == 2 ? t2 : t1;   // the smallest key of the group's score
    wave_lds_fence();
    int rank = 0;
#pragma unroll 1
    for (int j = 0; j < G; ++j) {
      const double o = grp_row[j];
      rank += (o > gs || (o == gs && j < e)) ? 1 : 0;
    }
    const uint64_t open = __ballot(e < G && rank < a.top_groups);
    const double worst_in = wave_min(e < G && rank < a.top_groups ? gs : INFINITY), best_out = wave_max(e < G && rank >= a.top_groups ? gs : kNone);
    const double mine = grp_row[min(e / n, G - 1)];
    const float w = width * static_cast<float>(a.group_top);
    const double least = key_row[min(e / n, G - 1)];
    if (best_out > kNone && near_keys(worst_in, best_out, w, slack)) {   // what makes the scores of the groups around the border
      more |= __ballot(key > kNone && (key > least || near_keys(key, least, width, slack)) &&
                       (near_keys(mine, worst_in, w, slack) || near_keys(mine, best_out, w, slack)));
      if (shared && (more & ~exact) == 0) {
        const double most = wave_max(e < G && (near_keys(gs, worst_in, w, slack) || near_keys(gs, best_out, w, slack)) ? mass : 0.0);
        if (!(worst_in - best_out > most * moved)) more |= heavy;
      }
    }
    if (e < E && !((open >> (e / n)) & 1)) key = kNone;
  }
  const double first = key;
  int got = -1;
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {
    const double m = wave_max(key);
    if (!(m > kNone)) break;
    const int win = __builtin_ctzll(__ballot(key == m));   // lowest index among equal keys
    if (e == j) got = win;
    if (e == win) key = kNone;
    // experts whose key may lie on the other side of this one, itself included
    const double won = __shfl(score, win, kWave);
    const bool close = first > kNone && near_keys(first, m, shared ? key_tolerance(a, tol, static_cast<float>(score + won)) * 1.001f : width, slack);
    const uint64_t at = __ballot(close);
    if (__builtin_popcountll(at) > 1) {
      more |= at;
      if (shared && (at & ~exact) == 0 && __ballot(close && !(fabs(first - m) >= fabs(score - won) * moved))) more |= heavy;
    }
  }
  if (e < 8) sel[e] = got;
  return more & ~exact;
}

struct RouteLds {
  union {
    struct {
      unsigned char w[kRtWaves][kRtUnit * 128 + 128];  // a unit of router rows of each wavefront (columns beyond E of the last row are read, never used)
      unsigned char x[kRtWaves][kRtTokens * 128];      // and of the tokens
    } stage;
    double red[kRtWaves][32 * 64];                     // partial sums: the 32 (16) of a lane in stride
    struct {
      double key[kRtTokens][kRtRow], grp[kRtTokens][kRtRow];
      double sum[kRtWaves][64];
    } pick;
  };
  double l[kRtTokens][kRtRow];                 // finished logits
  float nx[kRtWaves][kRtTokens], px[kRtWaves][kRtTokens];   // shares of the tokens' sums
  float nw[kRtWaves][128];                     // shares of |w|^2 of the experts (two each), or of |w|^2 and the sum of q^2
  uint32_t orx[kRtWaves][kRtTokens], orw[kRtWaves]; // bits of the values: all zero or not
  float x2[kRtTokens], p2[kRtTokens], w2, q2;  // sums of the tokens, the largest ones of the experts; x2, w2 0: nothing but zeros
  int sel[kRtTokens][9];
  int cnt[64];
};
static_assert(sizeof(RouteLds) <= 160 * 1024, "LDS of a CU");

// The router's weights as the operands of route_kernel: for a unit of 64 channels, operand f of step s is 64 lanes of 16
// bytes, lane 32 g + r: channels 16 s + 8 g .. + 7 of expert r (NF = 1, E <= 32) or 2 r + f (NF = 2).  And as columns [E, d],
// for logits that are settled (reading them out of the operands, a line of memory for 16 bytes, took 13000 cycles for two).
// One unit per workgroup, which also leaves every expert's shares of |w|^2 and of the sum of q^2 and the bits of its values.
constexpr int kLayThreads = 1024;   // four elements and one or two pieces a thread: the kernel is a chain of latencies
template <int NF>
__global__ __launch_bounds__(kLayThreads) void route_layout_kernel(const uint16_t* __restrict__ w, int d, int E, u4* __restrict__ ops, u4* __restrict__ cols,
                                                                   float* __restrict__ w2, float* __restrict__ q2, uint32_t* __restrict__ bits) {
  __shared__ uint16_t s_w[kRtUnit][64 + 2];
  __shared__ float s_n[16][64], s_q[16][64];
  __shared__ uint32_t s_any[16][64];
  const int u = blockIdx.x, tid = threadIdx.x, e = tid & 63, part = tid >> 6;
  const uint16_t* const src = w + static_cast<int64_t>(u) * kRtUnit * E;
  uint16_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = e < E ? src[(4 * part + i) * E + e] : 0;
  float n = 0.0f;
  uint32_t any = 0, q = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s_w[4 * part + i][e] = v[i];
    n = fmaf(bf16_to_f32(v[i]), bf16_to_f32(v[i]), n);
    any |= v[i] & 0x7FFFu;
    q = max(q, v[i] & 0x7F80u);
  }
  s_n[part][e] = n;
  s_q[part][e] = __uint_as_float(q << 16);
  s_any[part][e] = any;
  __syncthreads();
  // the lower threads write the operands, the upper ones the columns: eight channels of an expert each
  const bool op = tid < 512;
  const int i = tid & 511, lane = i & 63, f = (i >> 6) % NF, s = (i >> 6) / NF;
  const int c = op ? 16 * s + 8 * (lane >> 5) : 8 * (i & 7), col = op ? (NF == 2 ? 2 * (lane & 31) + f : lane & 31) : i >> 3;
  if (op ? i < 4 * NF * 64 : col < E) {
    u4 o;
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = s_w[c + 2 * q][col] | static_cast<uint32_t>(s_w[c + 2 * q + 1][col]) << 16;
    if (op) ops[static_cast<int64_t>(u) * 4 * NF * 64 + i] = o;
    else cols[static_cast<int64_t>(col) * (d >> 3) + u * 8 + (i & 7)] = o;
  }
  if (part == 0) {
    n = 0.0f;
    any = 0;
    float sum_q = 0.0f;
#pragma unroll
    for (int j = 0; j < 16; j += 2) {   // eight channels
      n += s_n[j][e] + s_n[j + 1][e];
      any |= s_any[j][e] | s_any[j + 1][e];
      const float most = fmaxf(s_q[j][e], s_q[j + 1][e]);
      sum_q = fmaf(most, most, sum_q);
    }
    w2[u * 64 + e] = n;
    q2[u * 64 + e] = sum_q;
    bits[u * 64 + e] = any;
  }
}

// fp64 logits of two experts of a token by one wavefront, eight channels of both a lane and round (half a wavefront for each expert,
// twice the rounds: 16301 x 3584 x 60 72.5 us instead of 69.7).  Code that a workgroup in fifty reaches is fetched from memory when
// it does (some 1000 cycles for 64 bytes of it, under the stream of the hidden states): here and below it is short rather than unrolled.
template <bool COLS>
__device__ __forceinline__ void settle_two(const RouteArgs& a, int tok, int e0, int e1, double* l_row) {
  const int lane = threadIdx.x & 63;
  const uint16_t* const xr = a.x + static_cast<int64_t>(tok) * a.d;
  double s0 = 0.0, s1 = 0.0;
#pragma unroll 2
  for (int c = 8 * lane; c < a.d; c += 8 * 64) {
    const u4 x = *reinterpret_cast<const u4*>(xr + c);
    u4 w[2];
    if constexpr (COLS) {
      w[0] = a.cols[(static_cast<int64_t>(e0) * a.d + c) >> 3];
      w[1] = a.cols[(static_cast<int64_t>(e1) * a.d + c) >> 3];
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint16_t* const p = a.w_router + static_cast<size_t>(c) * a.E + (h ? e1 : e0);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[h][q] = p[2 * q * a.E] | static_cast<uint32_t>(p[(2 * q + 1) * a.E]) << 16;
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {   // fp64 products: of large values, beyond fp32, they are finite
      const double lo = bf16_lo(x[q]), hi = bf16_hi(x[q]);
      s0 = fma(lo, static_cast<double>(bf16_lo(w[0][q])), s0);
      s0 = fma(hi, static_cast<double>(bf16_hi(w[0][q])), s0);
      s1 = fma(lo, static_cast<double>(bf16_lo(w[1][q])), s1);
      s1 = fma(hi, static_cast<double>(bf16_hi(w[1][q])), s1);
    }
  }
  s0 = wave_add(s0);
  s1 = wave_add(s1);
  if (lane == 0) {
    l_row[e0] = s0;
    l_row[e1] = s1;
  }
  wave_lds_fence();
}

// Puts the experts sel[j - 1] and sel[j], whose logits are settled, into their order; lanes 0 and 1 of the wavefront have one each.
// A softmax score is exp(l - shift) / total with an fp32 total, off by `part` of it at most (the other logits' tol, 16 roundings of
// the exponentials weighted by their shares, 6 of their sum): that moves the difference of two keys by `part` of the scores' difference.
// False where this could change the order.
__device__ __forceinline__ bool order_two(const RouteArgs& a, const double* l_row, int* sel, int j, int e0, int e1, double shift, float total, float tol) {
  const int lane = threadIdx.x & 63, e = lane == 0 ? e0 : e1;
  double key = l_row[e], score = 0.0;
  if (!keys_are_logits(a)) {
    score = exp(a.sigmoid ? -key : key - shift);
    score = a.sigmoid ? 1.0 / (1.0 + score) : score / static_cast<double>(total);
    key = score;
    if (a.bias) key += static_cast<double>(a.bias[e]);
    if (key != key) key = -DBL_MAX;
  }
  const double other = __shfl(key, 1, kWave), apart = fabs(score - __shfl(score, 1, kWave));
  const float part = a.sigmoid || keys_are_logits(a) ? 0.0f : (tol < 0.05f ? 1.1f * tol + 32 * 0x1p-24f : INFINITY);
  if (__builtin_amdgcn_readfirstlane(static_cast<int>(fabs(key - other) < apart * part))) return false;
  if (lane == 0 && !(key > other || (key == other && e0 < e1))) {
    sel[j - 1] = e1;
    sel[j] = e0;
  }
  return true;
}

// 64 channels of the 32 tokens and the router's rows of these channels: operands (LAID) or the rows as they lie in memory
template <int NL>
struct RouteUnit {
  u4 x[4];
  u4 w[NL];
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float dot2(uint32_t v, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v), __builtin_bit_cast(bf16x2, v), c, false);
}

// LAID: the router's weights come as operands, from route_layout_kernel.  Otherwise (up to kRouteUnlaidTokens: one launch) the rows of a
// unit come as they lie in memory, NL loads of 16 bytes a lane (8 NL >= E), and are turned into the operands of NF = 2 through
// LDS.  PAIRS: E is even, two experts of a row are one aligned word.  (Loading those words from memory takes the
// address unit as long for four bytes as for 16: 580 cycles a unit, of 36 loads instead of 12.)
// The logits' sums of units [u_lo, u_hi), one set per wavefront, in lds.red (a barrier is still to come), the norms' shares in
// lds.nx, nw, orx and orw.
template <int NF, bool LAID, int NL, bool PAIRS>
__device__ __forceinline__ void route_logits(const RouteArgs& a, RouteLds& lds, int t0, int u_lo, int u_hi) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 31, g = lane >> 5;
  // neighbouring units go to one wavefront: at any time the eight read places of a row that lie far apart (rows are often a
  // multiple of 4096 bytes, and so are the places of one memory channel)
  const int units = a.d / kRtUnit, u_begin = u_lo + wave * (u_hi - u_lo) / kRtWaves, u_end = u_lo + (wave + 1) * (u_hi - u_lo) / kRtWaves;

  // 16-byte pieces of the tokens' units: eight lanes read the 128 bytes of a token, piece p of token t goes to place p ^ (t & 7) of
  // its 128 bytes of LDS, which spreads the operand reads (32 tokens, one piece) over the banks.  (Operands straight from memory
  // touch the 32 rows four times each: 8192 x 2048 50000 cycles instead of 23000 up to the logits.)  The whole offset is the lane's: a
  // scalar offset has no part in the range check, and tokens behind the last one must not be read.
  const uint32_t x_bytes = 2u * a.d;
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.x) + static_cast<int64_t>(t0) * a.d, 0,
                                                                      static_cast<int>(min(a.T - t0, kRtTokens) * x_bytes), 0x00020000);   // zeros behind the last token
  const int x_lane = static_cast<int>((lane >> 3) * x_bytes) + 16 * (lane & 7);
  const uint32_t row_bytes = 2u * a.E;
  const __amdgpu_buffer_rsrc_t rw = LAID ? __builtin_amdgcn_make_buffer_rsrc(const_cast<u4*>(a.ops), 0, units * 4 * NF * 1024, 0x00020000)
                                         : __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.w_router), 0, static_cast<int>(a.d * row_bytes), 0x00020000);
  auto load = [&](int u) __attribute__((always_inline)) {
    RouteUnit<NL> q;
    u = min(u, u_end - 1);
    const uint32_t base = static_cast<uint32_t>(u) * (LAID ? 4u * NF * 1024u : kRtUnit * row_bytes);
#pragma unroll
    for (int i = 0; i < NL; ++i) q.w[i] = __builtin_amdgcn_raw_buffer_load_b128(rw, 16 * lane + base + 1024 * i, 0, 0);   // zeros behind the last row
#pragma unroll
    for (int i = 0; i < 4; ++i) q.x[i] = __builtin_amdgcn_raw_buffer_load_b128(rx, x_lane + (static_cast<uint32_t>(8 * i) * x_bytes + 2u * kRtUnit * u), 0, 0);
    __builtin_amdgcn_sched_barrier(0);   // the loads of a unit leave before the work on the one in front of it
    return q;
  };
  unsigned char* const stage = lds.stage.w[wave];
  const unsigned char* const col = stage + 8 * g * row_bytes + 4 * r;   // experts 2 r, 2 r + 1 of row 8 g; beyond E what lies there
  double acc[NF][16];
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[f][v] = 0.0;
  float nx[4] = {}, nw[NF] = {};   // nx, orx: tokens 8 i + lane / 8, step lane % 8 of the units
  uint32_t orx[4] = {}, orw = 0;
  unsigned char* const x_stage = lds.stage.x[wave];
  const unsigned char* const x_row = x_stage + r * 128;
  auto compute = [&](const RouteUnit<NL>& q) __attribute__((always_inline)) {
    if constexpr (!LAID) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        *reinterpret_cast<u4*>(stage + 1024 * i + 16 * lane) = q.w[i];
        orw |= q.w[i].x | q.w[i].y | q.w[i].z | q.w[i].w;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      *reinterpret_cast<u4*>(x_stage + (8 * i + (lane >> 3)) * 128 + 16 * ((lane & 7) ^ (lane >> 3))) = q.x[i];
      nx[i] = dot2(q.x[i].x, dot2(q.x[i].y, dot2(q.x[i].z, dot2(q.x[i].w, nx[i]))));
      orx[i] |= q.x[i].x | q.x[i].y | q.x[i].z | q.x[i].w;
    }
    wave_lds_fence();
    v16f c[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) c[f][v] = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u4 x = *reinterpret_cast<const u4*>(x_row + 16 * ((2 * s + g) ^ (r & 7)));
      u4 b[NF];
      if constexpr (LAID) {
#pragma unroll
        for (int f = 0; f < NF; ++f) b[f] = q.w[NF * s + f];
      } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const unsigned char* const p = col + (16 * s + i) * row_bytes;
          if constexpr (PAIRS) w[i] = *reinterpret_cast<const uint32_t*>(p);
          else w[i] = *reinterpret_cast<const uint16_t*>(p) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p + 2)) << 16;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          b[0][i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
          b[1][i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
          nw[0] = dot2(b[0][i], nw[0]);
          nw[1] = dot2(b[1][i], nw[1]);
        }
      }
#pragma unroll
      for (int f = 0; f < NF; ++f) c[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, b[f]), c[f], 0, 0, 0);
    }
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[f][v] += static_cast<double>(c[f][v]);
    wave_lds_fence();
  };
  float op_n = 0.0f, op_q = 0.0f;   // LAID: this wavefront's shares of the units' |w|^2 and sum of q^2 of expert `lane`
  uint32_t op_any = 0;
  if constexpr (LAID)
    for (int u = wave; u < units; u += kRtWaves) {
      op_n += a.op_w2[u * 64 + lane];
      op_q += a.op_q2[u * 64 + lane];
      op_any |= a.op_bits[u * 64 + lane];
    }
  if (u_begin < u_end) {
    RouteUnit<NL> p = load(u_begin), q;
#pragma unroll 1
    for (int u = u_begin; u < u_end; u += 2) {
      q = load(u + 1);
      compute(p);
      if (u + 1 >= u_end) break;
      p = load(u + 2);
      compute(q);
    }
  }
  // Sums over the wavefronts in their order.  Element v of a lane is token (v & 3) + 8 (v >> 2) + 4 g of the lane's expert.
#pragma unroll
  for (int i = 0; i < 4; ++i) {   // over the eight lanes of a token
    const float share = static_cast<float>((LAID ? 8 : 16) - (lane & 7));
    float n = nx[i] * (share * share), p = nx[i];
    int o = static_cast<int>(orx[i] & 0x7FFF7FFFu);
    n += dpp<0xB1>(n); n += dpp<0x4E>(n); n += dpp<0x141>(n);
    if constexpr (LAID) {
      p += dpp<0xB1>(p); p += dpp<0x4E>(p); p += dpp<0x141>(p);
    }
    o |= dpp<0xB1>(o); o |= dpp<0x4E>(o); o |= dpp<0x141>(o);
    if ((lane & 7) == 0) {
      lds.nx[wave][8 * i + (lane >> 3)] = n;
      if constexpr (LAID) lds.px[wave][8 * i + (lane >> 3)] = p;
      lds.orx[wave][8 * i + (lane >> 3)] = o;
    }
  }
  if constexpr (!LAID) {
    lds.nw[wave][2 * r + 64 * g] = nw[0];
    lds.nw[wave][2 * r + 64 * g + 1] = nw[1];
    const bool any_w = __ballot((orw & 0x7FFF7FFFu) != 0) != 0;
    if (lane == 0) lds.orw[wave] = any_w;
  } else {
    lds.nw[wave][lane] = op_n;
    lds.nw[wave][64 + lane] = op_q;
    op_any = __ballot(op_any != 0) != 0;
    if (lane == 0) lds.orw[wave] = op_any;
  }
  __syncthreads();   // the sums take the place of the rows
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int v = 0; v < 16; ++v) lds.red[wave][64 * (16 * f + v) + lane] = acc[f][v];
}

// Sums over the wavefronts in their order: |w|^2 (and the sum of q^2) of expert `lane`, those of token
// `lane`, and element `at` of lds.red, which is the logit of token_of(at) and expert_of(at).
struct Norms {
  float n, p;
  uint32_t any;
};
template <bool LAID>
__device__ __forceinline__ Norms expert_norm(const RouteLds& lds) {
  const int lane = threadIdx.x & 63;
  Norms r{};
#pragma unroll
  for (int i = 0; i < kRtWaves; ++i) {
    r.n += LAID ? lds.nw[i][lane] : lds.nw[i][lane] + lds.nw[i][lane + 64];
    if constexpr (LAID) r.p += lds.nw[i][lane + 64];
    r.any |= lds.orw[i];
  }
  return r;
}
template <bool LAID>
__device__ __forceinline__ Norms token_norm(const RouteLds& lds) {
  const int lane = threadIdx.x & 31;
  Norms r{};
#pragma unroll
  for (int i = 0; i < kRtWaves; ++i) {
    r.n += lds.nx[i][lane];
    if constexpr (LAID) r.p += lds.px[i][lane];
    r.any |= lds.orx[i][lane];
  }
  return r;
}
__device__ __forceinline__ double element_sum(const RouteLds& lds, int at) {
  double sum = lds.red[0][at];
#pragma unroll
  for (int w = 1; w < kRtWaves; ++w) sum += lds.red[w][at];
  return sum;
}
__device__ __forceinline__ int token_of(int at) { return ((at >> 6) & 3) + 8 * ((at >> 8) & 3) + 4 * ((at >> 5) & 1); }
template <int NF> __device__ __forceinline__ int expert_of(int at) { return NF == 2 ? 2 * (at & 31) + (at >> 10) : at & 31; }

// The experts' largest and the tokens' own sums for the bound: one that is not a number must not get lost in the maximum, and zero
// stands for zeros only.
__device__ __forceinline__ float expert_max(const RouteArgs& a, float n) {
  n = static_cast<int>(threadIdx.x & 63) < a.E ? (n == n ? n : INFINITY) : 0.0f;
  n = row_max(n);
  n = fmaxf(n, __shfl_xor(n, 16, 64));
  return fmaxf(n, __shfl_xor(n, 32, 64));
}
template <bool LAID>
__device__ __forceinline__ void put_w2(const RouteArgs& a, RouteLds& lds, const Norms& r) {
  const float n = expert_max(a, r.n);
  if ((threadIdx.x & 63) == 0) lds.w2 = r.any ? fmaxf(n, 0x1p-149f) : 0.0f;
  if constexpr (LAID) {
    const float q = expert_max(a, r.p);
    if ((threadIdx.x & 63) == 0) lds.q2 = q;
  }
}
__device__ __forceinline__ void put_x2(RouteLds& lds, const Norms& r) {
  lds.x2[threadIdx.x & 31] = r.any ? fmaxf(r.n == r.n ? r.n : INFINITY, 0x1p-149f) : 0.0f;
  lds.p2[threadIdx.x & 31] = r.p;
}
__device__ __forceinline__ void route_start(RouteLds& lds) {
  if (threadIdx.x < 64) lds.cnt[threadIdx.x] = 0;
  if (threadIdx.x < kRtTokens * 9) (&lds.sel[0][0])[threadIdx.x] = -1;
}

// From the logits (lds.l) to the outputs
// LAID: the bound knows the q's; COLS: there are columns of the router's weights
template <bool LAID, bool COLS>
__device__ __forceinline__ void route_finish(const RouteArgs& a, RouteLds& lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t0 = blockIdx.x * kRtTokens;
  // Selection: 16 lanes per token, all 32 at once.
  const int t = tid >> 4, s = tid & 15, tok = t0 + t;
  const bool live = tok < a.T;
  const bool masked = live && a.mask != nullptr && a.mask[tok] == 0;
  // squares that underflow say nothing; products below the smallest normal value are off by an absolute amount
  const float x2 = lds.x2[t], w2 = lds.w2;
  bool zero = x2 == 0.0f || w2 == 0.0f;   // all logits are exactly zero
  float tol = sqrtf(x2) * sqrtf(w2);
  if constexpr (LAID) tol += 8.0f * sqrtf(lds.p2[t]) * sqrtf(lds.q2);
  tol = kLogitBound * tol + 0x1p-120f;
  if (!(x2 > 0x1p-80f && w2 > 0x1p-80f)) tol = INFINITY;
  if (zero) tol = 0.0f;
  const bool vague = !(tol < INFINITY);   // the bound says nothing: every logit of the token is settled
  float sc[4], total;
  double shift;
  route_scores(a, lds.l[t], sc, shift, total);
  int state = route_select(a, lds.l[t], sc, shift, total, reinterpret_cast<int*>(lds.pick.key[t]), reinterpret_cast<int*>(lds.pick.grp[t]), lds.sel[t], tol);
  if (vague || (state > 0 && zero)) state = -1;
  if (!live || masked) state = 0;
  // Rare: the logits that a selection hangs on are settled by the token's wavefront.  Two experts are put in order; otherwise the
  // selection is made again in fp64 until it hangs on no logit that is not settled.
  if (__ballot(state != 0)) {
    wave_lds_fence();
    const uint64_t all = ~0ull >> (64 - a.E);
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
      const int st = __builtin_amdgcn_readlane(state, 0);
      const bool z = __builtin_amdgcn_readlane(zero, 0);
      const float tol_q = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(tol), 0));
      // the next row of lanes takes the place of the first
      state = __shfl(state, lane + 16, kWave);
      tol = __shfl(tol, lane + 16, kWave);
      zero = __shfl(static_cast<int>(zero), lane + 16, kWave) != 0;
      if (st == 0) continue;
      const int tq = 4 * wave + q;
      double* const l_row = lds.l[tq];
      int* const sel = lds.sel[tq];
      if (st > 0) {
        const int e0 = __builtin_amdgcn_readfirstlane(sel[st - 1]), e1 = __builtin_amdgcn_readfirstlane(sel[st]);
        settle_two<COLS>(a, t0 + tq, e0, e1, l_row);
        if (order_two(a, l_row, sel, st, e0, e1, __shfl(shift, 16 * q, kWave), __shfl(total, 16 * q, kWave), tol_q)) continue;
      }
      uint64_t exact = z ? all : 0, next = tol_q < INFINITY ? 0 : all;
      for (;;) {
        exact |= next;
#pragma unroll 1
        while (next) {
          const int e0 = __builtin_ctzll(next);
          next &= next - 1;
          const int e1 = next ? __builtin_ctzll(next) : e0;
          if (next) next &= next - 1;
          settle_two<COLS>(a, t0 + tq, e0, e1, l_row);
        }
        next = route_select_exact(a, l_row, lds.pick.key[tq], lds.pick.grp[tq], sel, tol_q, exact);
        if (next == 0) break;
      }
    }
    wave_lds_fence();
    route_scores(a, lds.l[t], sc, shift, total);
  }
  wave_lds_fence();
  // weights: lane j < k has slot j
  const int e = s < a.k && !masked ? lds.sel[t][s] : -1;
  const bool have = e >= 0;
  const double l = have ? lds.l[t][e] : 0.0;
  float w = 0.0f;
  if (a.renormalise) {
    // a softmax over log s of the selected (softmax scores: log s is the logit up to a constant of the row); fp64, because the
    // logits of a row may be large beside their differences
    double al = l;
    if (a.sigmoid) al = fmin(l, 0.0) - static_cast<double>(0.69314718f * __builtin_amdgcn_logf(1.0f + exp_of(-fabs(l))));
    al -= row_max(have ? al : static_cast<double>(-INFINITY));
    const float ex = have ? exp_of(al) : 0.0f;
    w = ex / row_sum(ex);
  } else {
    w = a.sigmoid ? 1.0f / (1.0f + exp_of(-l)) : exp_of(l - shift) / total;
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
    if (lane < 16) lds.pick.sum[wave][lane + 16 * v] = d;
  }
  __syncthreads();
  if (tid < 64) {
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kRtWaves; ++i) d += lds.pick.sum[i][tid];
    a.part_sum[static_cast<int64_t>(blockIdx.x) * 64 + tid] = d;
    a.part_cnt[static_cast<int64_t>(blockIdx.x) * 64 + tid] = lds.cnt[tid];
  }
}

template <int NF, bool LAID, int NL, bool PAIRS>
__global__ __launch_bounds__(kRtThreads) void route_kernel(RouteArgs a) {
  __shared__ __attribute__((aligned(16))) RouteLds lds;
  const int tid = threadIdx.x, wave = tid >> 6;
  route_start(lds);
  route_logits<NF, LAID, NL, PAIRS>(a, lds, blockIdx.x * kRtTokens, 0, a.d / kRtUnit);
  if (wave == 0) put_w2<LAID>(a, lds, expert_norm<LAID>(lds));
  else if (wave == 1 && (tid & 63) < kRtTokens) put_x2(lds, token_norm<LAID>(lds));
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2 * NF; ++i) {
    const int at = tid + i * kRtThreads;
    lds.l[token_of(at)][expert_of<NF>(at)] = element_sum(lds, at);
  }
  __syncthreads();
  route_finish<LAID, LAID>(a, lds);
}

// Few tokens and many channels: the bytes of the router's rows and of the tokens, at the 30 a cycle that a CU takes in, are
// what a workgroup's time is made of.  Shares of the channels go to workgroups of their own, which leave their sums
// and norms in memory, and a second kernel adds them in order and goes on.  Workgroups behind those write the weights as columns, from
// which it settles logits (out of the rows a pair is a line of memory for each channel, at those 30 bytes a cycle: 64 x 3584 x 64 in
// groups, with a pair to settle 24.5 us, out of columns 19.8; with a border between groups 39 and 30; with nothing to settle 16.2).
struct RoutePart {
  double l[kRtTokens * 64];        // in the order of lds.red
  float nx[kRtTokens], nw[64];
  uint32_t orx[kRtTokens], orw, unused[31];
};
template <int NL, bool PAIRS>
__global__ __launch_bounds__(kRtThreads) void route_part_kernel(RouteArgs a, RoutePart* __restrict__ parts, u4* __restrict__ cols, int blocks, int shares) {
  __shared__ __attribute__((aligned(16))) RouteLds lds;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, units = a.d / kRtUnit;
  const int block = blockIdx.x / shares, share = blockIdx.x - block * shares;
  if (block >= blocks) {   // eight channels of an expert a thread
    const int first = static_cast<int>(blockIdx.x) - blocks * shares, step = static_cast<int>(gridDim.x) - blocks * shares;
    if (lane < a.E)
      for (int u = first; u < units; u += step) {
        const int c = u * kRtUnit + 8 * wave;
        const uint16_t* const p = a.w_router + static_cast<size_t>(c) * a.E + lane;
        u4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = p[2 * q * a.E] | static_cast<uint32_t>(p[(2 * q + 1) * a.E]) << 16;
        cols[(static_cast<int64_t>(lane) * a.d + c) >> 3] = o;
      }
    return;
  }
  RoutePart& out = parts[blockIdx.x];
  route_logits<2, false, NL, PAIRS>(a, lds, block * kRtTokens, share * units / shares, (share + 1) * units / shares);
  if (wave == 0) {
    const Norms r = expert_norm<false>(lds);
    out.nw[lane] = r.n;
    if (lane == 0) out.orw = r.any;
  } else if (wave == 1 && lane < kRtTokens) {
    const Norms r = token_norm<false>(lds);
    out.nx[lane] = r.n;
    out.orx[lane] = r.any;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) out.l[tid + i * kRtThreads] = element_sum(lds, tid + i * kRtThreads);
}
__global__ __launch_bounds__(kRtThreads) void route_join_kernel(RouteArgs a, const RoutePart* __restrict__ parts, int shares) {
  __shared__ __attribute__((aligned(16))) RouteLds lds;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const RoutePart* const in = parts + static_cast<int64_t>(blockIdx.x) * shares;
  route_start(lds);
  double sum[4] = {};
  Norms r{};
#pragma unroll 4
  for (int s = 0; s < shares; ++s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += in[s].l[tid + i * kRtThreads];
    if (wave == 0) {
      r.n += in[s].nw[lane];
      r.any |= in[s].orw;
    } else if (wave == 1 && lane < kRtTokens) {
      r.n += in[s].nx[lane];
      r.any |= in[s].orx[lane];
    }
  }
  if (wave == 0) put_w2<false>(a, lds, r);
  else if (wave == 1 && lane < kRtTokens) put_x2(lds, r);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = tid + i * kRtThreads;
    lds.l[token_of(at)][expert_of<2>(at)] = sum[i];
  }
  __syncthreads();
  route_finish<false, true>(a, lds);
}

// Counts and score sums of all workgroups in a fixed order: 16 experts per workgroup, 64 slices of the partial sums.
__global__ __launch_bounds__(1024) void route_stats_kernel(const double* __restrict__ part_sum, const int32_t* __restrict__ part_cnt, int blocks,
                                                           int E, int32_t* __restrict__ counts, float* __restrict__ score_sum) {
  __shared__ double s_sum[64][17];
  __shared__ int s_cnt[64][17];
  const int col = threadIdx.x & 15, slice = threadIdx.x >> 4, e = blockIdx.x * 16 + col;
  double a = 0.0;
  int c = 0;
#pragma unroll 8
  for (int b = slice; b < blocks; b += 64) {
    a += part_sum[static_cast<int64_t>(b) * 64 + e];
    c += part_cnt[static_cast<int64_t>(b) * 64 + e];
  }
  s_sum[slice][col] = a;
  s_cnt[slice][col] = c;
  __syncthreads();
  if (threadIdx.x < 256) {   // 16 lanes per expert, four slices each
    const int i = threadIdx.x >> 4, q = threadIdx.x & 15;
    a = (s_sum[q][i] + s_sum[q + 16][i]) + (s_sum[q + 32][i] + s_sum[q + 48][i]);
    c = (s_cnt[q][i] + s_cnt[q + 16][i]) + (s_cnt[q + 32][i] + s_cnt[q + 48][i]);
    a = row_sum(a);
    c = row_sum(c);
    const int expert = blockIdx.x * 16 + i;
    if (q == 0 && expert < E) {
      if (score_sum != nullptr) score_sum[expert] = static_cast<float>(a);
      if (counts != nullptr) counts[expert] = c;
    }
  }
}

static int route_blocks(int T) { return (T + kRtTokens - 1) / kRtTokens; }
static size_t align256(size_t v) { return (v + 255) & ~size_t{255}; }
static int route_operands(int E) { return E <= 32 ? 1 : 2; }

// Up to this many tokens the workgroups are too few for the chip, and weights that are laid out first come too late: their kernel
// takes longer than it saves.  One kernel, or split, and laid out first, in us, 128 tokens: 896 x 8 8.9, 10.7; 2048 x 16 11.5, 12.9;
// 2048 x 64 13.5, 16.4; 3584 x 64 17.1, 21.8; 1024 tokens: 9.7, 11.1; 12.0, 14.1; 17.6, 19.5; 21.6, 24.6; 2048 tokens: 2048 x 64 19.9,
// 19.4, 3584 x 64 25.2, 24.8 (but 1500 x 896 x 8 9.8, 11.9).
constexpr int kRouteUnlaidTokens = 1024;
// Shares of the channels: a unit for each wavefront, 16 at most (d = 16384, E = 64: 16 shares 18.7 us, 32 of them 24.4), a workgroup
// per CU at most, from 256 KB of operands for a workgroup of 32 tokens on (below, the second launch takes what it saves).  One
// workgroup, and split, in us: d = 1280, E = 64 12.1, 12.9; 2048 x 64 14.5, 13.0; 3584 x 64 19.9, 14.8; 7168 x 64 32.7, 19.1;
// 2048 x 32 13.0, 12.0; 4096 x 16 16.0, 13.3; 1024 x 8 8.8, 10.3.
static int route_shares(int T, int d, int E) {
  if (T == 0 || T > kRouteUnlaidTokens || d * (kRtTokens + E) < 1 << 17) return 1;
  return std::min({d / (kRtUnit * kRtWaves), 16, 256 / route_blocks(T)});
}
size_t route_split_bytes(int T, int d, int E) {
  const int shares = route_shares(T, d, E);
  return shares > 1 ? align256(static_cast<size_t>(route_blocks(T)) * shares * sizeof(RoutePart)) + align256(static_cast<size_t>(E) * d * 2) : 0;
}

size_t route_stats_bytes(int T) { return align256(static_cast<size_t>(route_blocks(T)) * 64 * (sizeof(double) + sizeof(int32_t)) + 1); }
size_t route_layout_bytes(int T, int d, int E) {
  return T > kRouteFewTokens ? align256(static_cast<size_t>(d / kRtUnit) * (4 * route_operands(E) * 1024 + 64 * 12) + static_cast<size_t>(E) * d * 2) : 0;
}
// A split has fewer shares as the workgroups become more, and there is none above kRouteUnlaidTokens: the largest one of all
// numbers of tokens up to T.
size_t route_workspace_bytes(int T, int d, int E, bool stats) {
  size_t n = route_layout_bytes(T, d, E);
  for (int t = kRtTokens; t - kRtTokens < std::min(T, kRouteUnlaidTokens); t += kRtTokens) n = std::max(n, route_split_bytes(t, d, E));
  return (stats ? route_stats_bytes(T) : 0) + n;
}

hipError_t launch_route(RouteArgs a, int32_t* counts, float* score_sum, void* workspace, bool split, hipStream_t stream) {
  const int blocks = route_blocks(a.T), units = a.d / kRtUnit;
  const bool stats = counts != nullptr || score_sum != nullptr;
  char* ws = static_cast<char*>(workspace);
  if (stats) {
    a.part_sum = reinterpret_cast<double*>(ws);
    a.part_cnt = reinterpret_cast<int32_t*>(a.part_sum + static_cast<int64_t>(blocks) * 64);
    ws += route_stats_bytes(a.T);
  }
  // odd E: two experts of a row are two words (64 x 3584 x 63 in one workgroup for 32 tokens 42 us, 128 tokens laid out 22)
  const bool lay = a.T > kRouteUnlaidTokens || (a.T > kRouteFewTokens && !split && (route_shares(a.T, a.d, a.E) > 1 || (a.E > 16 && a.E % 2 != 0)));
  if (lay) {
    const int nf = route_operands(a.E);
    u4* const ops = reinterpret_cast<u4*>(ws);
    u4* const cols = ops + static_cast<int64_t>(units) * 4 * nf * 64;
    float* const w2 = reinterpret_cast<float*>(cols + static_cast<int64_t>(a.E) * a.d / 8);
    float* const q2 = w2 + units * 64;
    uint32_t* const bits = reinterpret_cast<uint32_t*>(q2 + units * 64);
    a.ops = ops;
    a.cols = cols;
    a.op_w2 = w2;
    a.op_q2 = q2;
    a.op_bits = bits;
    if (nf == 1) {
      route_layout_kernel<1><<<units, kLayThreads, 0, stream>>>(a.w_router, a.d, a.E, ops, cols, w2, q2, bits);
      route_kernel<1, true, 4, true><<<blocks, kRtThreads, 0, stream>>>(a);
    } else {
      route_layout_kernel<2><<<units, kLayThreads, 0, stream>>>(a.w_router, a.d, a.E, ops, cols, w2, q2, bits);
      route_kernel<2, true, 8, true><<<blocks, kRtThreads, 0, stream>>>(a);
    }
  } else if (split) {
    const int shares = route_shares(a.T, a.d, a.E);
    RoutePart* const parts = reinterpret_cast<RoutePart*>(ws);
    u4* const cols = reinterpret_cast<u4*>(ws + align256(static_cast<size_t>(blocks) * shares * sizeof(RoutePart)));
    a.cols = cols;
    const int grid = blocks * shares + std::min(units, std::max(256 - blocks * shares, 16));   // columns on the CUs that are left
    if (a.E <= 16 && a.E % 2 == 0) route_part_kernel<2, true><<<grid, kRtThreads, 0, stream>>>(a, parts, cols, blocks, shares);
    else if (a.E <= 16) route_part_kernel<2, false><<<grid, kRtThreads, 0, stream>>>(a, parts, cols, blocks, shares);
    else if (a.E % 2 == 0) route_part_kernel<8, true><<<grid, kRtThreads, 0, stream>>>(a, parts, cols, blocks, shares);
    else route_part_kernel<8, false><<<grid, kRtThreads, 0, stream>>>(a, parts, cols, blocks, shares);
    route_join_kernel<<<blocks, kRtThreads, 0, stream>>>(a, parts, shares);
  } else if (a.T > 0) {
    if (a.E <= 16 && a.E % 2 == 0) route_kernel<2, false, 2, true><<<blocks, kRtThreads, 0, stream>>>(a);
    else if (a.E <= 16) route_kernel<2, false, 2, false><<<blocks, kRtThreads, 0, stream>>>(a);
    else if (a.E % 2 == 0) route_kernel<2, false, 8, true><<<blocks, kRtThreads, 0, stream>>>(a);
    else route_kernel<2, false, 8, false><<<blocks, kRtThreads, 0, stream>>>(a);
  }
  if (stats) route_stats_kernel<<<(a.E + 15) / 16, 1024, 0, stream>>>(a.part_sum, a.part_cnt, blocks, a.E, counts, score_sum);
  return hipGetLastError();
}

// A caller's routing for the dispatch plan: what is no expert becomes -1, which the plan and the combine pass over.
__global__ __launch_bounds__(256) void route_import_kernel(const int32_t* __restrict__ idx, const float* __restrict__ w, int n, int E,
                                                           int32_t* __restrict__ topk_idx, float* __restrict__ topk_p, int32_t* __restrict__ row_of) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int e = idx[i];
  const bool ok = e >= 0 && e < E;
  topk_idx[i] = ok ? e : -1;
  topk_p[i] = ok ? w[i] : 0.0f;
  if (!ok) row_of[i] = -1;
}

hipError_t launch_route_import(const int32_t* idx, const float* w, int n, int E, int32_t* topk_idx, float* topk_p, int32_t* row_of, hipStream_t stream) {
  if (n > 0) route_import_kernel<<<(n + 255) / 256, 256, 0, stream>>>(idx, w, n, E, topk_idx, topk_p, row_of);
  return hipGetLastError();
}

// -------------------------------------------------------------------------------------------------------- gradient

// dL/dlogits of one token by 16 lanes (lane s: experts s + 16 v), fp32.  slot_e, slot_d: LDS of the token's eight slots.
__device__ __forceinline__ void route_grad_token(const RouteBackwardArgs& a, int tok, bool live, int* slot_e, float* slot_d, float (&g)[4]) {
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
  // every lane sees all slots: one load each, then LDS
  if (s < 8) {
    slot_e[s] = s < a.k ? a.topk_idx[static_cast<int64_t>(tok) * a.k + s] : -1;
    slot_d[s] = s < a.k ? a.d_topk_w[static_cast<int64_t>(tok) * a.k + s] : 0.0f;
  }
  wave_lds_fence();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int e = slot_e[j];
    const float d = slot_d[j];
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (e == s + 16 * v && e < E) { up[v] += d; sel[v] += 1.0f; }
  }
  if (a.sigmoid) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float t = exp_of(-fabsf(l[v])), r = __builtin_amdgcn_rcpf(1.0f + t);
      sc[v] = l[v] >= 0.0f ? r : t * r;
      om[v] = l[v] >= 0.0f ? t * r : r;   // 1 - s
    }
  } else {
    mx = row_max(mx);
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      sc[v] = s + 16 * v < E ? exp_of(l[v] - mx) : 0.0f;
      om[v] = 1.0f;
      sum += sc[v];
    }
    sum = row_sum(sum);
#pragma unroll
    for (int v = 0; v < 4; ++v) sc[v] /= sum;
  }
  if (a.renormalise) {
    // softmax over log s of the selected
    float al[4], m = -INFINITY;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      al[v] = a.sigmoid ? fminf(l[v], 0.0f) - 0.69314718f * __builtin_amdgcn_logf(1.0f + exp_of(-fabsf(l[v]))) : l[v];
      if (sel[v] > 0.0f) m = fmaxf(m, al[v]);
    }
    m = row_max(m);
    float p[4], sum = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      p[v] = sel[v] > 0.0f ? exp_of(al[v] - m) : 0.0f;
      sum += p[v] * sel[v];
    }
    sum = row_sum(sum);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    float dot = 0.0f, dq = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      p[v] *= inv;
      dot += p[v] * up[v];
      dq += sc[v] * q[v];
    }
    dot = row_sum(dot);
    dq = row_sum(dq);
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
    dot = row_sum(dot);
#pragma unroll
    for (int v = 0; v < 4; ++v) g[v] = a.sigmoid ? sc[v] * om[v] * up[v] : sc[v] * (up[v] - dot);
  }
  const bool masked = a.mask != nullptr && a.mask[tok] == 0;
#pragma unroll
  for (int v = 0; v < 4; ++v)
    if (!live || masked || s + 16 * v >= E) g[v] = 0.0f;
}

// The two products of the gradient run on the bf16 MFMA with exact operands: x and w_router are bf16, an fp32 dlogits is the sum of
// three bf16 terms (8 bits of its 24 each, cut and not rounded, so that the rest is exact).  route_dlogits_kernel writes the
// terms as operands of both:
//   ga [tile of 32 tokens][term][step of 16 experts][lane]: lane 32 g + r, experts 16 s + 8 g .. + 7 of token r        (dx)
//   gb [step of 16 tokens][term][32 experts][lane]: lane 32 g + r, tokens 8 g .. + 7 of the step, expert 32 n + r      (dw)
// and the router's weights for dx, wa [32 channels][step of 16 experts][lane]: experts 16 s + 8 g .. + 7 of channel r.
// Bound of the whole: HBM, x read once and dx (fp32) written once; the terms are 12 bytes per token and expert and stay in the caches.
__device__ __forceinline__ void three_terms(float g, uint32_t (&t)[3]) {
  const uint32_t b = __float_as_uint(g);
  if ((b & 0x7F800000u) == 0x7F800000u) {   // infinity and NaN: one term
    t[0] = (b >> 16) | ((b & 0x7FFFFFu) ? 0x40u : 0u);
    t[1] = t[2] = 0u;
    return;
  }
  const float r1 = g - __uint_as_float(b & 0xFFFF0000u);
  const uint32_t b1 = __float_as_uint(r1);
  const float r2 = r1 - __uint_as_float(b1 & 0xFFFF0000u);
  t[0] = b >> 16;
  t[1] = b1 >> 16;
  t[2] = __float_as_uint(r2) >> 16;
}

// 32 tokens per workgroup, 16 lanes each; the workgroups behind those lay out the weights, 32 channels each.
// NS: steps of 16 experts, NT: tiles of 32.
template <int NS, int NT>
__global__ __launch_bounds__(512) void route_dlogits_kernel(RouteBackwardArgs a) {
  __shared__ float s_g[32][65];
  __shared__ int s_e[32][8], s_keep[32];
  __shared__ float s_d[32][8];
  const int tid = threadIdx.x, tiles = (a.T + 31) / 32;
  if (static_cast<int>(blockIdx.x) >= tiles) {
    const int ct = blockIdx.x - tiles;
    for (int i = tid; i < NS * 64; i += 512) {
      const int lane = i & 63, s = i >> 6, e = 16 * s + 8 * (lane >> 5);
      const uint16_t* const row = a.w_router + static_cast<int64_t>(32 * ct + (lane & 31)) * a.E;
      u4 o;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t lo = e + 2 * q < a.E ? row[e + 2 * q] : 0, hi = e + 2 * q + 1 < a.E ? row[e + 2 * q + 1] : 0;
        o[q] = lo | hi << 16;
      }
      a.wa[static_cast<int64_t>(ct) * NS * 64 + i] = o;
    }
    return;
  }
  const int t = tid >> 4, s = tid & 15, tok = blockIdx.x * 32 + t;
  float g[4];
  route_grad_token(a, min(tok, a.T - 1), tok < a.T, s_e[t], s_d[t], g);
#pragma unroll
  for (int v = 0; v < 4; ++v) s_g[t][s + 16 * v] = g[v];
  if (s == 0) s_keep[t] = tok < a.T && (a.mask == nullptr || a.mask[tok] != 0);
  __syncthreads();
  if (tid < 64) {   // a bit for every token that takes part, 16 in a word
    const uint32_t b = static_cast<uint32_t>(__ballot(tid < 32 && s_keep[tid & 31] != 0));
    if (tid < 2) a.keep[blockIdx.x * 2 + tid] = (b >> (16 * tid)) & 0xFFFFu;
  }
#pragma unroll 1
  for (int i = tid; i < (NS + 2 * NT) * 64; i += 512) {
    const bool first = i < NS * 64;
    const int j = first ? i : i - NS * 64, lane = j & 63, q = j >> 6;      // q: step of experts, or 2 * tile of experts + step of tokens
    const int at_t = first ? lane & 31 : 16 * (q & 1) + 8 * (lane >> 5), at_e = first ? 16 * q + 8 * (lane >> 5) : 32 * (q >> 1) + (lane & 31);
    u4 o[3];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      uint32_t lo[3], hi[3];
      three_terms(first ? s_g[at_t][at_e + 2 * h] : s_g[at_t + 2 * h][at_e], lo);
      three_terms(first ? s_g[at_t][at_e + 2 * h + 1] : s_g[at_t + 2 * h + 1][at_e], hi);
#pragma unroll
      for (int p = 0; p < 3; ++p) o[p][h] = lo[p] | hi[p] << 16;
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      if (first) a.ga[((static_cast<int64_t>(blockIdx.x) * 3 + p) * NS + q) * 64 + lane] = o[p];
      else a.gb[((static_cast<int64_t>(blockIdx.x) * 2 + (q & 1)) * 3 + p) * (NT * 64) + (q >> 1) * 64 + lane] = o[p];
    }
  }
}

__device__ __forceinline__ v16f mfma_bf16(u4 a, u4 b, v16f c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// dx: a wavefront has 64 tokens, whose terms stay in registers, and a slice of the channels, whose weights come 32 channels at
// a time.  Slices of 256 channels (the terms are read once for 64 KB of dx), fewer while that leaves SIMDs without a wavefront.
template <int NS>
__global__ __launch_bounds__(256) void route_dx_kernel(RouteBackwardArgs a, int slice) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, g = lane >> 5;
  const int c_begin = (blockIdx.y * 4 + wave) * slice, c_end = min(c_begin + slice, a.d);
  if (c_begin >= a.d) return;
  const int tile = blockIdx.x * 2, tiles = (a.T + 31) / 32;
  u4 ga[2][3][NS];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int s = 0; s < NS; ++s) ga[m][p][s] = a.ga[((static_cast<int64_t>(min(tile + m, tiles - 1)) * 3 + p) * NS + s) * 64 + lane];
  u4 w[NS];
  auto load = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < NS; ++s) w[s] = a.wa[(static_cast<int64_t>(min(c, a.d - 32) >> 5) * NS + s) * 64 + lane];
  };
  load(c_begin);
#pragma unroll 1
  for (int c = c_begin; c < c_end; c += 32) {
    v16f acc[2];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[m][v] = 0.0f;
    u4 b[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) b[s] = w[s];
    load(c + 32);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 2; p >= 0; --p)   // smallest terms first
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) acc[m] = mfma_bf16(ga[m][p][s], b[s], acc[m]);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int t = (tile + m) * 32 + (v & 3) + 8 * (v >> 2) + 4 * g;
        if (t < a.T) a.dx[static_cast<int64_t>(t) * a.d + c + r] = acc[m][v];
      }
  }
}

// dw: a workgroup has 128 channels and a share of the tokens, which its eight wavefronts split; their sums meet in LDS.  A
// step is 16 tokens: 4 KB of x as it lies in memory, turned into operands through LDS (a word of two channels of eight
// tokens each: even and odd channels are two operands), against the terms of the step.  With several shares
// (blockIdx.y) the sums go to dw_part, which route_dw_sum_kernel adds in order.
constexpr int kDwWaves = 8, kDwChannels = 128;
template <int NT>
__global__ __launch_bounds__(64 * kDwWaves) void route_dw_kernel(RouteBackwardArgs a, int steps_per_wave) {
  __shared__ __attribute__((aligned(16))) union {
    unsigned char x[kDwWaves][16 * 2 * kDwChannels];
    float sum[kDwWaves / 2][4 * NT * 16][64];
  } lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, g = lane >> 5;
  const int c0 = blockIdx.x * kDwChannels, steps = (a.T + 15) / 16;
  const int first = (blockIdx.y * kDwWaves + wave) * steps_per_wave, last = min(first + steps_per_wave, steps);
  v16f acc[2][2][NT];   // half of the channels, even / odd, tile of experts
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[j][o][n][v] = 0.0f;
  struct Step {
    u4 x[4], g[3][NT];
    uint32_t keep;   // a padding token has no part, whatever its row holds
  };
  auto load = [&](int s) __attribute__((always_inline)) {
    Step q;
    s = min(s, last - 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * s + 4 * i + (lane >> 4);
      const uint16_t* const row = a.x + static_cast<int64_t>(min(t, a.T - 1)) * a.d + c0 + 8 * (lane & 15);
      q.x[i] = *reinterpret_cast<const u4*>(row);
    }
    q.keep = load_uniform(a.keep + s);
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int n = 0; n < NT; ++n) q.g[p][n] = a.gb[(static_cast<int64_t>(s) * 3 + p) * (NT * 64) + n * 64 + lane];
    __builtin_amdgcn_sched_barrier(0);
    return q;
  };
  unsigned char* const stage = lds.x[wave];
  auto compute = [&](const Step& q) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = (q.keep >> (4 * i + (lane >> 4))) & 1;
      *reinterpret_cast<u4*>(stage + 1024 * i + 16 * lane) = in ? q.x[i] : u4{0u, 0u, 0u, 0u};
    }
    wave_lds_fence();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint32_t*>(stage + (8 * g + i) * 256 + 128 * j + 4 * r);
      u4 even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        even[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
        odd[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
      }
#pragma unroll
      for (int p = 2; p >= 0; --p)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[j][0][n] = mfma_bf16(even, q.g[p][n], acc[j][0][n]);
          acc[j][1][n] = mfma_bf16(odd, q.g[p][n], acc[j][1][n]);
        }
    }
    wave_lds_fence();
  };
  if (first < last) {
    Step p = load(first), q;
#pragma unroll 1
    for (int s = first; s < last; s += 2) {
      q = load(s + 1);
      compute(p);
      if (s + 1 >= last) break;
      p = load(s + 2);
      compute(q);
    }
  }
  // sums of the wavefronts, a tree in a fixed order
#pragma unroll 1
  for (int half = kDwWaves / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int v = 0; v < 16; ++v) lds.sum[wave - half][((j * 2 + o) * NT + n) * 16 + v][lane] = acc[j][o][n][v];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[j][o][n][v] += lds.sum[wave][((j * 2 + o) * NT + n) * 16 + v][lane];
    }
  }
  if (wave != 0) return;
  const bool whole = gridDim.y == 1;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int c = c0 + 64 * j + 2 * ((v & 3) + 8 * (v >> 2) + 4 * g) + o, e = 32 * n + r;
          if (!whole) a.dw_part[(static_cast<int64_t>(blockIdx.y) * a.d + c) * (32 * NT) + e] = acc[j][o][n][v];
          else if (e < a.E) a.dw[static_cast<int64_t>(c) * a.E + e] = acc[j][o][n][v];
        }
}

template <int NT>
__global__ __launch_bounds__(256) void route_dw_sum_kernel(const float* __restrict__ part, int parts, int d, int E, float* __restrict__ dw) {
  const int i = blockIdx.x * 256 + threadIdx.x, c = i / (32 * NT), e = i % (32 * NT);
  if (c >= d) return;
  const int64_t stride = static_cast<int64_t>(d) * 32 * NT;
  float s = 0.0f;
#pragma unroll 8
  for (int p = 0; p < parts; ++p) s += part[p * stride + i];
  if (e < E) dw[static_cast<int64_t>(c) * E + e] = s;
}

__global__ __launch_bounds__(256) void zero_kernel(float* __restrict__ p, int64_t n) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) p[i] = 0.0f;
}

namespace {
int steps_of(int E) { return E <= 16 ? 1 : E <= 32 ? 2 : 4; }
// Shares of the tokens: one workgroup per CU, at least four steps of 16 tokens for each wavefront.  (d = 896, E = 8, T = 2048 with at
// least eight: 12.8 us instead of 9.7; d = 2048, E = 64, T = 16000 with two workgroups per CU: 44.8 instead of 33.5.)
int dw_shares(int T, int d) {
  const int want = std::max(256 / (d / kDwChannels), 1), most = (T + 16 * kDwWaves * 4 - 1) / (16 * kDwWaves * 4);
  return std::max(std::min(want, most), 1);
}
struct BackwardLayout {
  size_t ga, gb, wa, keep, part, bytes;
};
BackwardLayout backward_layout(int T, int d, int E) {
  const size_t tiles = (static_cast<size_t>(T) + 31) / 32, ns = steps_of(E), nt = E <= 32 ? 1 : 2;
  BackwardLayout l;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t p = at; at += align256(n); return p; };
  l.ga = take(tiles * 3 * ns * 1024);
  l.gb = take(tiles * 2 * 3 * nt * 1024);
  l.wa = take(static_cast<size_t>(d / 32) * ns * 1024);
  l.keep = take(tiles * 2 * sizeof(uint32_t));
  l.part = take(dw_shares(T, d) > 1 ? static_cast<size_t>(dw_shares(T, d)) * d * 32 * nt * sizeof(float) : 0);
  l.bytes = std::max<size_t>(at, 256);
  return l;
}
}  // namespace

size_t route_backward_workspace_bytes(int T, int d, int E) { return backward_layout(T, d, E).bytes; }

hipError_t launch_route_backward(RouteBackwardArgs a, void* workspace, hipStream_t stream) {
  if (a.T == 0) {
    const int64_t n = static_cast<int64_t>(a.d) * a.E;
    if (a.dw) zero_kernel<<<static_cast<unsigned>((n + 255) / 256), 256, 0, stream>>>(a.dw, n);
    return hipGetLastError();
  }
  const BackwardLayout l = backward_layout(a.T, a.d, a.E);
  char* const ws = static_cast<char*>(workspace);
  a.ga = reinterpret_cast<u4*>(ws + l.ga);
  a.gb = reinterpret_cast<u4*>(ws + l.gb);
  a.wa = reinterpret_cast<u4*>(ws + l.wa);
  a.keep = reinterpret_cast<uint32_t*>(ws + l.keep);
  a.dw_part = reinterpret_cast<float*>(ws + l.part);
  const unsigned lay = static_cast<unsigned>((a.T + 31) / 32 + a.d / 32);
  int slice = 256;
  while (slice > 32 && static_cast<int64_t>((a.T + 63) / 64) * ((a.d + slice - 1) / slice) < 1024) slice /= 2;
  const dim3 dx_grid((a.T + 63) / 64, (a.d + 4 * slice - 1) / (4 * slice));
  const int shares = dw_shares(a.T, a.d), steps = (a.T + 15) / 16, per_wave = (steps + shares * kDwWaves - 1) / (shares * kDwWaves);
  const dim3 dw_grid(a.d / kDwChannels, shares);
  const unsigned sum_grid = static_cast<unsigned>((static_cast<int64_t>(a.d) * (a.E <= 32 ? 32 : 64) + 255) / 256);
#define MOTE_BACKWARD(NS_, NT_)                                                                                              \
  route_dlogits_kernel<NS_, NT_><<<lay, 512, 0, stream>>>(a);                                                                \
  if (a.dx) route_dx_kernel<NS_><<<dx_grid, 256, 0, stream>>>(a, slice);                                                      \
  if (a.dw) route_dw_kernel<NT_><<<dw_grid, 64 * kDwWaves, 0, stream>>>(a, per_wave);                                        \
  if (a.dw && shares > 1) route_dw_sum_kernel<NT_><<<sum_grid, 256, 0, stream>>>(a.dw_part, shares, a.d, a.E, a.dw)
  switch (steps_of(a.E)) {
    case 1: MOTE_BACKWARD(1, 1); break;
    case 2: MOTE_BACKWARD(2, 1); break;
    default: MOTE_BACKWARD(4, 2); break;
  }
#undef MOTE_BACKWARD
  return hipGetLastError();
}

}  // namespace mote
