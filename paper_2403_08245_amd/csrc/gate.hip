// The router's gate by scores and its gradient.  A lane holds VPL consecutive experts, so that a group of experts is a run of lanes; a token is 16 lanes (or
// a wavefront: many experts, large k, and every token whose choice fp32 cannot tell).  Bound: the rounds of the selection, then reading the logits and writing
// their gradient (32768 tokens of 256 experts in groups, k = 8: 22.3 us forward, where its logits take 6.7; 9.8 backward, 34 MB written, 3.6 TB/s).
//
// The choice is that of 64-bit ranks: with a bias or sums of two, ranks of different experts come within 32-bit rounding of one another once in some
// thousand tokens, and which one is taken would then hang on how the exponential was rounded.  Where ranks are scores alone (no bias, and groups that count by
// their best or all stay) the logits themselves are compared, which is the order of the exact scores.
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

// a lane's VPL entries of a row; those past E are -inf, and so are NaN
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
  for (int i = 0; i < VPL; ++i) x[i] = fmaxf(x[i], -INFINITY);      // the larger of a number and NaN is the number
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

// ---- forward, one token of the wavefront.  WIDE: ranks are 64-bit scores (and bias); else the logits.  s_rank: VPL * 64 of the wavefront's own.
template <int VPL, bool WIDE>
__device__ __forceinline__ void gate_token(const float *__restrict__ logits, const float *__restrict__ bias, int t, int E, int k, const smoe_gate_rule &rule,
                                           int32_t *__restrict__ idx, float *__restrict__ gates, void *ranks) {
  typedef typename std::conditional<WIDE, double, float>::type R;
  typedef typename Key<R>::type K;
  R *const s_rank = (R *)ranks;
  const int lane = threadIdx.x & 63;
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
      for (int i = 0; i < VPL; ++i) s_rank[lane * VPL + i] = rank[i];
      if (lane < rule.groups)
        for (int i = 0; i < per; ++i) best.add(s_rank[lane * per + i]);
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

template <int VPL, bool WIDE>
__global__ void __launch_bounds__(256) score_gate_kernel(const float *__restrict__ logits, const float *__restrict__ bias, int T, int E, int k,
                                                         smoe_gate_rule rule, int32_t *__restrict__ idx, float *__restrict__ gates) {
  __shared__ double s_rank[4][VPL * 64];
  const int wave = threadIdx.x >> 6, t = blockIdx.x * 4 + wave;
  if (t < T) gate_token<VPL, WIDE>(logits, bias, t, E, k, rule, idx, gates, s_rank[wave]);      // wavefronts share nothing
}

// ---- forward, four tokens of a wavefront at once, 16 lanes each.
// Ranks are fp32 here, and every step says whether rounding could have decided it: then the wavefront takes that token again by gate_token.  A rank
// becomes a whole number between 0 and 2^23 over the row's range (good to 2.5: three roundings to 2^-24 of it, and the cut), with the expert's number below it, so that the largest of them names
// its expert, ties included, and one that was taken is found by comparing.  Two picks (or groups) are told apart where they differ by more
// than what the exponential, the sums and this rounding can be off by.
__device__ __forceinline__ unsigned int row16_max(unsigned int v) {      // over rows of 16 lanes, in all of them
  v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
  v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
  v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
  return max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));
}
template <int CTRL> __device__ __forceinline__ float turned16(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, turned16<0x121>(v));
  v = fmaxf(v, turned16<0x122>(v));
  v = fmaxf(v, turned16<0x124>(v));
  return fmaxf(v, turned16<0x128>(v));
}
__device__ __forceinline__ float row16_sum(float v) {
  v += turned16<0x121>(v);
  v += turned16<0x122>(v);
  v += turned16<0x124>(v);
  return v + turned16<0x128>(v);
}

template <int VPL, bool WIDE, bool SOFTMAX>
__global__ void __launch_bounds__(256, VPL <= 16 ? 8 : 4) score_gate_rows_kernel(const float *__restrict__ logits, const float *__restrict__ bias, int T, int E, int k,
                                                              smoe_gate_rule rule, int32_t *__restrict__ idx, float *__restrict__ gates) {
  constexpr int INDEX = VPL <= 4 ? 6 : VPL <= 8 ? 7 : VPL <= 16 ? 8 : 9, BITS = VPL <= 16 ? 23 : 22, MASK = (1 << INDEX) - 1;
  constexpr int EXACT = VPL <= 4 ? 1 : VPL / 4;             // VPL of gate_token
  __shared__ double s_rank[4][EXACT * 64];
  const int lane = threadIdx.x & 15, wave = threadIdx.x >> 6;
  const int t0 = (blockIdx.x * 4 + wave) * 4;
  if (t0 >= T) return;
  const int t = min(t0 + (((int)threadIdx.x & 63) >> 4), T - 1);      // rows past the last repeat it
  float x[VPL];
  load_row<VPL>(logits + (size_t)t * E, E, lane, x);        // the padding is -inf like a masked expert
  float rank[VPL];
  float top = -INFINITY, sum = 0.f;
  float off = 0.f;                                          // what a rank may be off by
  if (SOFTMAX && (WIDE || !rule.renormalise)) {
    float low = INFINITY;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      top = fmaxf(top, x[i]);
      low = fminf(low, x[i] == -INFINITY ? INFINITY : x[i]);
    }
    top = row16_max(top);
    low = -row16_max(-low);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      rank[i] = exp_under(x[i], top);
      sum += rank[i];
    }
    sum = row16_sum(sum);
    off = (top - low + 40.f) * 0x1p-24f / sum;              // the largest is 1 / sum
  }
  float hi = -INFINITY, lo = INFINITY;                      // the row's range
  if constexpr (WIDE) {
    float b[VPL];
    if (bias) {
      load_row<VPL>(bias, E, lane, b);
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i) b[i] = 0.f;
    }
    const float inv = SOFTMAX ? 1.0f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      // sigmoid: the exponent's rounding moves it by at most 0.224 2^-23, exponential, sum and reciprocal by 1.75 2^-23
      const float r = b[i] + (SOFTMAX ? rank[i] * inv : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x[i])));
      const bool masked = x[i] == -INFINITY;
      rank[i] = masked ? -INFINITY : r;
      hi = fmaxf(hi, rank[i]);
      lo = fminf(lo, masked ? INFINITY : r);                // a bias of -inf makes the range infinite, and the token unsure
    }
    if (!SOFTMAX) off = 8 * 0x1p-24f;
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      rank[i] = x[i];
      hi = fmaxf(hi, x[i]);
      lo = fminf(lo, x[i] == -INFINITY ? INFINITY : x[i]);
    }
    off = 0.f;
  }
  hi = row16_max(hi);
  lo = -row16_max(-lo);
  const float range = hi - lo;
  if (WIDE) off += 0x1p-23f * fmaxf(fabsf(hi), fabsf(lo));
  bool unsure = !(range > 0x1p-100f && range < 0x1p100f);
  const float unit = ((float)(1 << BITS) - 8.f) / range;
  const float wide_gap = 6.f + 2.f * off * unit;                // two cut ranks, each off by 2.5 and `off`
  unsure |= !(wide_gap < (float)(1 << BITS));
  const int gap = unsure ? 0 : (int)wide_gap;

  bool kept = lane * VPL < E;                               // the lane's group, and lanes past the experts are in none
  if (rule.kept_groups < rule.groups) {
    const int run = E / rule.groups / VPL;                  // lanes of a group (the launcher says that it is a whole number)
    const bool even = (run & (run - 1)) == 0;
    const int group = even ? 0 : lane / run, at = lane - group * run;
    float first = -INFINITY, second = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      second = __builtin_amdgcn_fmed3f(first, second, rank[i]);
      first = fmaxf(first, rank[i]);
    }
    if (even) {
      for (int d = 1; d < run; d <<= 1) {
        const float f = __shfl_xor(first, d, 16), s = __shfl_xor(second, d, 16);
        second = fmaxf(__builtin_amdgcn_fmed3f(first, second, f), s);
        first = fmaxf(first, f);
      }
    } else {
      const float own_first = first, own_second = second;
      for (int d = 1; d < run; ++d) {
        const int from = (lane + d - (at + d >= run ? run : 0)) & 15;
        const float f = __shfl(own_first, from, 16), s = __shfl(own_second, from, 16);
        second = fmaxf(__builtin_amdgcn_fmed3f(first, second, f), s);
        first = fmaxf(first, f);
      }
    }
    float worth = rule.group_best == 2 && second > -INFINITY ? first + second : first;
    worth = kept ? worth : NAN;
    const float error = 4.f * off + 0x1p-22f * fabsf(worth);
    const float above = worth == -INFINITY ? worth : worth + error, under = worth == -INFINITY ? worth : worth - error;
    int at_least = 0, surely = 0;                           // groups that may come before this one, and that do
    auto meet = [&](float other) {
      at_least += other >= under;
      surely += other > above;
    };
    if (even) {
      for (int d = run; d < 16; d += run) meet(__shfl_xor(worth, d, 16));
    } else {
      for (int g = 0; g < rule.groups; ++g) {
        const float other = __shfl(worth, g * run, 16);
        meet(g == group ? NAN : other);
      }
    }
    unsure |= kept && at_least >= rule.kept_groups && surely < rule.kept_groups;
    kept &= at_least < rule.kept_groups;
  }
  // Masked experts and those of other groups have 0 here, as the row's least has: where one of them comes near a pick, the token is unsure.
  unsigned int key[VPL];
  const float from = kept ? lo : INFINITY;
  const unsigned int name = (unsigned int)(MASK - lane * VPL) + 1u;
#pragma unroll
  for (int i = 0; i < VPL; ++i) key[i] = ((unsigned int)fmaxf((rank[i] - from) * unit, 0.f) << INDEX) + name - (unsigned int)i;
  // k rounds, and the largest of what is left.  Keys are under 2^31, so of their distances to the last pick, without sign, those of smaller keys are
  // the larger ones, and the largest is the next pick's.
  int my_e = 0;
  unsigned int last = 0x80000000u;
  for (int j = 0; j <= k; ++j) {
    unsigned int found = key[0] - last;
#pragma unroll
    for (int i = 1; i < VPL; ++i) found = max(found, key[i] - last);
    found = row16_max(found) + last;
    unsure |= j > 0 && (int)((last - 1u) >> INDEX) - (int)((found - 1u) >> INDEX) < gap;
    last = found;
    if (lane == j) my_e = MASK - (int)((found - 1u) & MASK);
  }
  unsure |= hi == INFINITY;
  const bool mine = lane < k;
  const float my_x0 = mine && my_e < E ? logits[(size_t)t * E + my_e] : -INFINITY;
  const float my_x = my_x0 != my_x0 ? -INFINITY : my_x0;
  float w;
  if (rule.renormalise) {
    const float most = row16_max(my_x);
    const float m = SOFTMAX ? most : fminf(most, 0.f);
    if (SOFTMAX) w = exp_under(my_x, m);
    else w = my_x <= 0.f ? expf(my_x - m) / (1.0f + expf(my_x)) : 1.0f / (1.0f + expf(-my_x));
    w = mine ? w : 0.f;
    w /= row16_sum(w);
  } else {
    w = SOFTMAX ? exp_under(my_x, top) / sum : 1.0f / (1.0f + expf(-my_x));
  }
  const unsigned long long again = __ballot(unsure);
  if (mine && !((again >> ((int)threadIdx.x & 48)) & 0xffffull) && t0 + (((int)threadIdx.x & 63) >> 4) < T) {
    idx[(size_t)t * k + lane] = my_e;
    gates[(size_t)t * k + lane] = rule.scale * w;
  }
  if (again == 0) return;
  for (int q = 0; q < 4; ++q)
    if (t0 + q < T && ((again >> (16 * q)) & 0xffffull)) gate_token<EXACT, WIDE>(logits, bias, t0 + q, E, k, rule, idx, gates, s_rank[wave]);
}

// ---- gradient.  ROW: softmax scores that are not renormalised, whose gradient reaches every logit of the row.
template <int VPL, bool ROW>
__global__ void __launch_bounds__(256) score_gate_bwd_kernel(const float *logits, const int32_t *idx, const float *dgates, int T, int E, int k, smoe_gate_rule rule,
                                                             float *dlogits) {
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

// Four tokens of a wavefront, 16 lanes each (k <= 16).  Where the gradient reaches the kept logits only, the wavefront clears its tokens' rows, which lie
// behind one another, and puts the k values into them behind that: the lines are in L2.
template <int VPL, bool ROW>
__global__ void __launch_bounds__(256) score_gate_bwd_rows_kernel(const float *logits, const int32_t *idx, const float *dgates, int T, int E, int k, smoe_gate_rule rule,
                                                                  float *dlogits) {
  const int lane = threadIdx.x & 15;
  const int t0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 4;
  if (t0 >= T) return;
  const int t = min(t0 + (((int)threadIdx.x & 63) >> 4), T - 1);      // rows past the last repeat it
  int e = -1;
  float dw = 0.f, x_e = -INFINITY;
  if (lane < k) {
    e = idx[(size_t)t * k + lane];
    dw = rule.scale * dgates[(size_t)t * k + lane];
    if ((unsigned)e < (unsigned)E) x_e = fmaxf(logits[(size_t)t * E + e], -INFINITY);
    else e = -1;
  }
  const bool live = e >= 0 && x_e != -INFINITY;
  float d_e;
  if constexpr (ROW) {
    float p[VPL], top = -INFINITY, sum = 0.f;
    load_row<VPL>(logits + (size_t)t * E, E, lane, p);
#pragma unroll
    for (int i = 0; i < VPL; ++i) top = fmaxf(top, p[i]);
    top = row16_max(top);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      p[i] = p[i] == -INFINITY ? 0.f : exp_under(p[i], top);
      sum += p[i];
    }
    sum = row16_sum(sum);
    const float inv = sum > 0.f ? 1.0f / sum : 0.f;
    d_e = live ? dw * exp_under(x_e, top) * inv : 0.f;
    const float total = row16_sum(d_e) * inv;
#pragma unroll
    for (int i = 0; i < VPL; ++i) p[i] *= -total;
    for (int j = 0; j < k; ++j) {
      const int at = __shfl(e, j, 16) - lane * VPL;
      const float d = __shfl(d_e, j, 16);
#pragma unroll
      for (int i = 0; i < VPL; ++i) p[i] += at == i ? d : 0.f;
    }
    float *row = dlogits + (size_t)t * E;
    if (t0 + (((int)threadIdx.x & 63) >> 4) >= T) return;
    if (VPL % 4 == 0 && E % 4 == 0) {
#pragma unroll
      for (int i = 0; i < VPL; i += 4)
        if (lane * VPL + i < E) *reinterpret_cast<float4 *>(row + lane * VPL + i) = make_float4(p[i], p[(i + 1) % VPL], p[(i + 2) % VPL], p[(i + 3) % VPL]);
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (lane * VPL + i < E) row[lane * VPL + i] = p[i];
    }
  } else {
    const bool softmax = rule.score == SMOE_SCORE_SOFTMAX;
    if (rule.renormalise) {
      const float most = row16_max(live ? x_e : -INFINITY);
      const float m = softmax ? most : fminf(most, 0.f);
      float q = 0.f;
      if (live) q = softmax ? exp_under(x_e, m) : x_e <= 0.f ? expf(x_e - m) / (1.0f + expf(x_e)) : 1.0f / (1.0f + expf(-x_e));
      const float sum = row16_sum(q);
      q = sum > 0.f ? q / sum : 0.f;
      const float mean = row16_sum(q * dw);
      d_e = live ? q * (dw - mean) : 0.f;
      if (!softmax) d_e *= 1.0f / (1.0f + expf(x_e));       // 1 - sigmoid
    } else {
      d_e = live ? dw / ((1.0f + expf(-x_e)) * (1.0f + expf(x_e))) : 0.f;
    }
    float value = 0.f;                                      // of every slot that names the lane's expert
    for (int j = 0; j < k; ++j) {
      const int other = __shfl(e, j, 16);
      const float d = __shfl(d_e, j, 16);
      value += other == e ? d : 0.f;
    }
    // dlogits may be the logits: what was read has arrived (it is in `value`) before the rows are cleared
    __asm__ volatile("s_waitcnt vmcnt(0)" : "+v"(value)::"memory");
    float *rows = dlogits + (size_t)t0 * E;
    const int n = min(4, T - t0) * E, at = (int)threadIdx.x & 63;
    if (E % 4 == 0) {
      for (int i = at * 4; i < n; i += 256) *reinterpret_cast<float4 *>(rows + i) = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
      for (int i = at; i < n; i += 64) rows[i] = 0.f;
    }
    __asm__ volatile("s_waitcnt vmcnt(0)" : "+v"(value)::"memory");
    if (live && t0 + (((int)threadIdx.x & 63) >> 4) < T) dlogits[(size_t)t * E + e] = value;
  }
}

template <typename F> void by_width(int E, F f) {
  if (E <= 64) f(std::integral_constant<int, 1>{});
  else if (E <= 128) f(std::integral_constant<int, 2>{});
  else if (E <= 256) f(std::integral_constant<int, 4>{});
  else if (E <= 512) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
}

}  // namespace

int launch_score_gate(hipStream_t s, const float *logits, const float *bias, int T, int E, int k, const smoe_gate_rule &rule, int32_t *idx, float *gates) {
  const dim3 block(256);
  const bool grouped = rule.kept_groups < rule.groups;
  const bool wide = bias || (grouped && rule.group_best > 1);
  // Four tokens a wavefront: where 16 lanes hold a row, and a group is a run of lanes.  Four / one, us: 4 tokens of 256 experts 4.4 / 6.6, 16384 of 64 5.3 / 9.3, of
  // 160 14.7 / 33.8, of 512 25.4 / 54.1, 32768 of 128 9.8 / 17, of 256 22.3 / 66.5; logits that are all equal, so that every token is taken
  // again, 86 / 64.
  const int vpl = E <= 64 ? 4 : E <= 128 ? 8 : E <= 256 ? 16 : 32;
  if (E <= 512 && k <= 16 && (!grouped || E / rule.groups % vpl == 0)) {
    const dim3 grid(ceil_div(T, 16));
    auto go = [&](auto v) {
      constexpr int VPL = decltype(v)::value;
      auto as = [&](auto w, auto softmax) {
        hipLaunchKernelGGL((score_gate_rows_kernel<VPL, decltype(w)::value, decltype(softmax)::value>), grid, block, 0, s, logits, bias, T, E, k, rule, idx, gates);
      };
      if (rule.score == SMOE_SCORE_SOFTMAX) wide ? as(std::true_type{}, std::true_type{}) : as(std::false_type{}, std::true_type{});
      else wide ? as(std::true_type{}, std::false_type{}) : as(std::false_type{}, std::false_type{});
    };
    if (vpl == 4) go(std::integral_constant<int, 4>{});
    else if (vpl == 8) go(std::integral_constant<int, 8>{});
    else if (vpl == 16) go(std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, 32>{});
    SMOE_LAUNCH_CHECK();
    return SMOE_OK;
  }
  const dim3 grid(ceil_div(T, 4));
  by_width(E, [&](auto v) {
    constexpr int VPL = decltype(v)::value;
    if (wide) hipLaunchKernelGGL((score_gate_kernel<VPL, true>), grid, block, 0, s, logits, bias, T, E, k, rule, idx, gates);
    else hipLaunchKernelGGL((score_gate_kernel<VPL, false>), grid, block, 0, s, logits, bias, T, E, k, rule, idx, gates);
  });
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

int launch_score_gate_bwd(hipStream_t s, const float *logits, const int32_t *idx, const float *dgates, int T, int E, int k, const smoe_gate_rule &rule,
                          float *dlogits) {
  const dim3 block(256);
  const bool row = rule.score == SMOE_SCORE_SOFTMAX && !rule.renormalise;
  // four tokens / one token a wavefront, us: 4 tokens of 256 experts 2.8 / 3.1, 16384 of 64 (softmax) 4.6 / 7.6, of 512 (sigmoid) 9 / 13.5, 32768 of 256 9.8 / 17.3
  if (k <= 16 && (!row || E <= 256)) {
    const dim3 grid(ceil_div(T, 16));
    if (!row) hipLaunchKernelGGL((score_gate_bwd_rows_kernel<1, false>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
    else if (E <= 64) hipLaunchKernelGGL((score_gate_bwd_rows_kernel<4, true>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
    else if (E <= 128) hipLaunchKernelGGL((score_gate_bwd_rows_kernel<8, true>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
    else hipLaunchKernelGGL((score_gate_bwd_rows_kernel<16, true>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
    SMOE_LAUNCH_CHECK();
    return SMOE_OK;
  }
  const dim3 grid(ceil_div(T, 4));
  by_width(E, [&](auto v) {
    constexpr int VPL = decltype(v)::value;
    if (row) hipLaunchKernelGGL((score_gate_bwd_kernel<VPL, true>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
    else hipLaunchKernelGGL((score_gate_bwd_kernel<VPL, false>), grid, block, 0, s, logits, idx, dgates, T, E, k, rule, dlogits);
  });
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
