// The router's gate by scores and its gradient.  One wavefront per token; a lane holds VPL consecutive experts, so that a group of experts is a run of
// lanes.  Bound: reading the logits (and writing their gradient), then the rounds of the selection.
//
// The choice is that of 64-bit scores: with a bias or sums of two, ranks of different experts come within 32-bit rounding of one another once in some
// thousand tokens, and which one is taken would then hang on how the exponential was rounded.  Where the order of the scores is that of the
// logits (no bias, groups that count by their best), the logits themselves are compared.
#include "block.h"
#include <limits.h>
#include <type_traits>

namespace {

// ---- the order of ranks as whole numbers: removed experts lie below every rank, -inf included
template <typename R> struct Key;
template <> struct Key<float> {
  typedef int type;
  static constexpr int NONE = INT_MIN;
  static __device__ __forceinline__ int of(float v) {
    const int b = __float_as_int(v + 0.0f);       // -0 ties with +0
    return b ^ ((b >> 31) & 0x7fffffff);
  }
};
template <> struct Key<double> {
  typedef long long type;
  static constexpr long long NONE = LLONG_MIN;
  static __device__ __forceinline__ long long of(double v) {
    const long long b = __double_as_longlong(v + 0.0);
    return b ^ ((b >> 63) & 0x7fffffffffffffffLL);
  }
};
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_max(int v) {
  return max(v, __builtin_amdgcn_update_dpp(INT_MIN, v, CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ long long dpp_max(long long v) {
  const int hi = __builtin_amdgcn_update_dpp(INT_MIN, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  const unsigned int lo = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)(unsigned int)v, CTRL, ROWS, 0xf, false);
  return max(v, (long long)hi << 32 | lo);
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ long long lane_value(long long v, int lane) {
  return (long long)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned int)__builtin_amdgcn_readlane((int)(unsigned int)v, lane);
}
// over the wavefront: rows of 16 lanes, then row 0 -> 1, 2 -> 3 and the low half -> the high half
template <typename T> __device__ __forceinline__ T wave_top(T v) {
  v = dpp_max<0x111, 0xf>(v);
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  return lane_value(v, 63);
}
template <typename T> __device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  return v;
}
// exp(x - top) where top is the largest of the row's; infinities included
__device__ __forceinline__ float exp_under(float x, float top) { return x == top ? 1.0f : expf(x - top); }
__device__ __forceinline__ double exp_under(double x, double top) { return x == top ? 1.0 : exp(x - top); }

// a lane's VPL logits; experts past E and masked ones are -inf
template <int VPL> __device__ __forceinline__ void load_row(const float *row, int E, int lane, float (&x)[VPL]) {
  if (VPL % 4 == 0 && E % 4 == 0) {
#pragma unroll
    for (int i = 0; i < VPL; i += 4) {
      const int e = lane * VPL + i;
      float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (e < E) v = *reinterpret_cast<const float4 *>(row + e);
      x[i] = v.x; x[(i + 1) % VPL] = v.y; x[(i + 2) % VPL] = v.z; x[(i + 3) % VPL] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = lane * VPL + i < E ? row[lane * VPL + i] : -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) x[i] = x[i] != x[i] ? -INFINITY : x[i];
}

// The two largest of a group's ranks, -inf where it has fewer that count.
template <typename R> struct Best {
  R first, second;
  __device__ __forceinline__ void add(R v) {
    const R low = v < first ? v : first;
    first = v > first ? v : first;
    second = low > second ? low : second;
  }
  __device__ __forceinline__ void join(R f, R s) {
    add(f);
    second = s > second ? s : second;
  }
  __device__ __forceinline__ R worth(int best) const { return best == 2 && second > (R)-INFINITY ? first + second : first; }
};

// Which groups stay: bit g.  Lane g holds what group g is worth (lanes past the groups: nothing).
template <typename R> __device__ __forceinline__ unsigned long long kept_groups(R worth, int groups, int kept, int lane) {
  int before = 0;
  const auto mine = Key<R>::of(worth);
  for (int j = 0; j < groups; ++j) {
    const auto other = lane_value(mine, j);
    before += other > mine || (other == mine && j < lane);
  }
  return __ballot(lane < groups && before < kept);
}

// ---- forward.  WIDE: ranks are 64-bit scores (and bias); else the logits.
template <int VPL, bool WIDE>
__global__ void __launch_bounds__(256) score_gate_kernel(const float *__restrict__ logits, const float *__restrict__ bias, int T, int E, int k,
                                                         smoe_gate_rule rule, int32_t *__restrict__ idx, float *__restrict__ gates) {
  typedef typename std::conditional<WIDE, double, float>::type R;
  typedef typename Key<R>::type K;
  __shared__ R s_rank[4][VPL * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * 4 + wave;
  if (t >= T) return;                       // wavefronts share nothing
  float x[VPL];
  load_row<VPL>(logits + (size_t)t * E, E, lane, x);
  const bool softmax = rule.score == SMOE_SCORE_SOFTMAX;
  float top = -INFINITY;
  if (softmax && (WIDE || !rule.renormalise)) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) top = fmaxf(top, x[i]);
    top = wave_max(top);
  }
  R rank[VPL];
  if constexpr (WIDE) {
    double s[VPL], sum = 0.0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      s[i] = softmax ? exp_under((double)x[i], (double)top) : 1.0 / (1.0 + exp(-(double)x[i]));
      sum += lane * VPL + i < E ? s[i] : 0.0;
    }
    if (softmax) sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int e = lane * VPL + i;
      double r = softmax ? s[i] / sum : s[i];
      if (bias && e < E) r += (double)bias[e];
      rank[i] = x[i] == -INFINITY || r != r ? -INFINITY : r;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) rank[i] = x[i];
  }
  K key[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i) key[i] = lane * VPL + i < E ? Key<R>::of(rank[i]) : Key<R>::NONE;

  if (rule.kept_groups < rule.groups) {
    const int per = E / rule.groups, run = per / VPL;      // experts and lanes of a group
    unsigned long long kept;
    Best<R> best{(R)-INFINITY, (R)-INFINITY};
    if (run * VPL == per && (run & (run - 1)) == 0) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) best.add(rank[i]);
      for (int d = 1; d < run; d <<= 1) {
        const R f = __shfl_xor(best.first, d, 64), s = __shfl_xor(best.second, d, 64);
        best.join(f, s);
      }
      kept = kept_groups(__shfl(best.worth(rule.group_best), min(lane * run, 63), 64), rule.groups, rule.kept_groups, lane);
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i) s_rank[wave][lane * VPL + i] = rank[i];
      if (lane < rule.groups)
        for (int i = 0; i < per; ++i) best.add(s_rank[wave][lane * per + i]);
      kept = kept_groups(best.worth(rule.group_best), rule.groups, rule.kept_groups, lane);
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (!((kept >> min((lane * VPL + i) / per, 63)) & 1)) key[i] = Key<R>::NONE;
  }

  // k rounds of the wavefront's largest key; equal ones go to the lower expert, which lies in the lower lane or before it in the same
  int my_e = 0;
  float my_x = -INFINITY;
  for (int j = 0; j < k; ++j) {
    K most = key[0];
#pragma unroll
    for (int i = 1; i < VPL; ++i) most = max(most, key[i]);
    const K found = wave_top(most);
    const int from = __ffsll((long long)__ballot(most == found)) - 1;
    int at = VPL - 1;
    float value = x[VPL - 1];
#pragma unroll
    for (int i = VPL - 2; i >= 0; --i)
      if (key[i] == found) { at = i; value = x[i]; }
    at = __builtin_amdgcn_readlane(at, from);
    value = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(value), from));
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (lane == from && i == at) key[i] = Key<R>::NONE;
    if (lane == j) { my_e = from * VPL + at; my_x = value; }
  }

  // lane j < k: the weight of slot j
  float w;
  if (rule.renormalise) {
    // sigmoid's scores are taken times exp(-m), m the largest kept logit where that is negative: their ratios stay where they all underflow
    const float most = wave_max(my_x);
    const float m = softmax ? most : fminf(most, 0.f);
    if (most == -INFINITY) w = 1.0f;
    else if (softmax) w = exp_under(my_x, m);
    else w = my_x <= 0.f ? expf(my_x - m) / (1.0f + expf(my_x)) : 1.0f / (1.0f + expf(-my_x));
    w = lane < k ? w : 0.f;
    w /= wave_sum(w);
  } else if (softmax) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) sum += lane * VPL + i < E ? exp_under(x[i], top) : 0.f;
    w = exp_under(my_x, top) / wave_sum(sum);
  } else {
    w = 1.0f / (1.0f + expf(-my_x));
  }
  if (lane < k) {
    idx[(size_t)t * k + lane] = my_e;
    gates[(size_t)t * k + lane] = rule.scale * w;
  }
}

// ---- gradient.  ROW: softmax scores that are not renormalised, whose gradient reaches every logit of the row.
template <int VPL, bool ROW>
__global__ void __launch_bounds__(256) score_gate_bwd_kernel(const float *__restrict__ logits, const int32_t *__restrict__ idx,
                                                             const float *__restrict__ dgates, int T, int E, int k, smoe_gate_rule rule,
                                                             float *__restrict__ dlogits) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= T) return;
  int e = -1;
  float dw = 0.f, x_e = -INFINITY;
  if (lane < k) {
    e = idx[(size_t)t * k + lane];
    dw = rule.scale * dgates[(size_t)t * k + lane];
    if ((unsigned)e < (unsigned)E) x_e = logits[(size_t)t * E + e];
    else e = -1;
    if (x_e != x_e) x_e = -INFINITY;
  }
  const bool live = e >= 0 && x_e != -INFINITY;
  float p[VPL], d_e, total = 0.f;
  if constexpr (ROW) {
    float x[VPL], top = -INFINITY, sum = 0.f;
    load_row<VPL>(logits + (size_t)t * E, E, lane, x);
#pragma unroll
    for (int i = 0; i < VPL; ++i) top = fmaxf(top, x[i]);
    top = wave_max(top);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      p[i] = x[i] == -INFINITY ? 0.f : exp_under(x[i], top);
      sum += p[i];
    }
    sum = wave_sum(sum);
    const float inv = sum > 0.f ? 1.0f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) p[i] *= inv;
    d_e = live ? dw * exp_under(x_e, top) * inv : 0.f;
    total = wave_sum(d_e);
  } else if (rule.renormalise) {
    const bool softmax = rule.score == SMOE_SCORE_SOFTMAX;
    const float most = wave_max(live ? x_e : -INFINITY);
    const float m = softmax ? most : fminf(most, 0.f);
    float q = 0.f;
    if (live) q = softmax ? exp_under(x_e, m) : x_e <= 0.f ? expf(x_e - m) / (1.0f + expf(x_e)) : 1.0f / (1.0f + expf(-x_e));
    const float sum = wave_sum(q);
    q = sum > 0.f ? q / sum : 0.f;
    const float mean = wave_sum(q * dw);
    d_e = live ? q * (dw - mean) : 0.f;
    if (!softmax) d_e *= 1.0f / (1.0f + expf(x_e));       // 1 - sigmoid
  } else {
    d_e = live ? dw / ((1.0f + expf(-x_e)) * (1.0f + expf(x_e))) : 0.f;
  }
  float out[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i) out[i] = ROW ? -total * p[i] : 0.f;
  for (int j = 0; j < k; ++j) {
    const int at = __builtin_amdgcn_readlane(e, j);
    const float d = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(d_e), j));
#pragma unroll
    for (int i = 0; i < VPL; ++i) out[i] += lane * VPL + i == at ? d : 0.f;
  }
  float *row = dlogits + (size_t)t * E;
  if (VPL % 4 == 0 && E % 4 == 0) {
#pragma unroll
    for (int i = 0; i < VPL; i += 4)
      if (lane * VPL + i < E)
        *reinterpret_cast<float4 *>(row + lane * VPL + i) = make_float4(out[i], out[(i + 1) % VPL], out[(i + 2) % VPL], out[(i + 3) % VPL]);
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (lane * VPL + i < E) row[lane * VPL + i] = out[i];
  }
}

template <bool WIDE, typename F> void by_width(int E, F f) {
  if (E <= 64) f(std::integral_constant<int, 1>{});
  else if (E <= 128) f(std::integral_constant<int, 2>{});
  else if (E <= 256) f(std::integral_constant<int, 4>{});
  else if (E <= 512) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
}

}  // namespace

int launch_score_gate(hipStream_t s, const float *logits, const float *bias, int T, int E, int k, const smoe_gate_rule &rule, int32_t *idx, float *gates) {
  const dim3 grid(ceil_div(T, 4)), block(256);
  const bool wide = bias || (rule.kept_groups < rule.groups && rule.group_best > 1);
  by_width<false>(E, [&](auto v) {
    constexpr int VPL = decltype(v)::value;
    if (wide) hipLaunchKernelGGL((score_gate_kernel<VPL, true>), grid, block, 0, s, logits, bias, T, E, k, rule, idx, gates);
    else hipLaunchKernelGGL((score_gate_kernel<VPL, false>), grid, block, 0, s, logits, bias, T, E, k, rule, idx, gates);
  });
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

int launch_score_gate_bwd(hipStream_t s, const float *logits, const int32_t *idx, const float *dgates, int T, int E, int k, const smoe_gate_rule &rule,
                          float *dlogits) {
  const dim3 grid(ceil_div(T, 4)), block(256);
  const bool row = rule.score == SMOE_SCORE_SOFTMAX && !rule.renormalise;
  by_width<false>(E, [&](auto v) {
    constexpr int VPL = decltype(v)::value;
    if (row) hipLaunchKernelGGL((score_gate_bwd_kernel<VPL, true>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
    else hipLaunchKernelGGL((score_gate_bwd_kernel<VPL, false>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
  });
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
