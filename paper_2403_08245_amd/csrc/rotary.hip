// Rotary positions of query and key rows, and the two ways between rows and the paged cache: writing them (turned and rounded to 8 bits
// where asked) and reading them back.  All are bound by memory: a row is read once and written once.
//
// A wavefront takes one token's rows, or some of them, d_head / 8 lanes a row and 8 elements a lane.  The angles belong to the token:
// each lane works out the sine and cosine of one pair (two for rows over 128), and the wavefront shares them through LDS, so they cost
// a token one evaluation a lane, however many heads it has.
//
// An angle is p f modulo one turn, of the 64-bit fraction of a turn that a position adds: one integer product that wraps, whose upper 32
// bits are the angle as a signed number of 2^-32 turns.
#include "cache.h"

namespace {

constexpr int WAVES = 4;
constexpr int MAX_PAIRS = 256;      // rows of at most 512 elements
constexpr int BATCH = 4;            // rows a lane has in flight

template <typename T> struct Eight;   // 8 elements of a row as they are loaded and stored
template <> struct Eight<bf16_t> {
  typedef bf16_t vec __attribute__((ext_vector_type(8)));
  vec v;
  __device__ __forceinline__ void load(const bf16_t *p) { v = *reinterpret_cast<const vec *>(p); }
  __device__ __forceinline__ void store(bf16_t *p) const { *reinterpret_cast<vec *>(p) = v; }
  __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
  __device__ __forceinline__ void set(int i, float x) { v[i] = (bf16_t)x; }
};
template <> struct Eight<float> {
  typedef float vec __attribute__((ext_vector_type(4)));
  vec v[2];
  __device__ __forceinline__ void load(const float *p) { v[0] = reinterpret_cast<const vec *>(p)[0]; v[1] = reinterpret_cast<const vec *>(p)[1]; }
  __device__ __forceinline__ void store(float *p) const { reinterpret_cast<vec *>(p)[0] = v[0]; reinterpret_cast<vec *>(p)[1] = v[1]; }
  __device__ __forceinline__ float get(int i) const { return v[i >> 2][i & 3]; }
  __device__ __forceinline__ void set(int i, float x) { v[i >> 2][i & 3] = x; }
};

// the sum of 8 elements' shares, in their order
__device__ __forceinline__ void sum_parts(const float *src, size_t stride, int shares, int e0, Eight<float> &y) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  f32x4 lo = f32x4{0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll 4
  for (int k = 0; k < shares; ++k) {
    const f32x4 *p = reinterpret_cast<const f32x4 *>(src + k * stride + e0);
    lo += p[0];
    hi += p[1];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y.set(i, lo[i]);
    y.set(4 + i, hi[i]);
  }
}

struct Work {          // how the rows of a launch are dealt to wavefronts
  int groups;          // wavefronts a token
  int per;             // rows of each
  int lanes_log2;      // lanes a row
};

// Rounds a row to e4m3 with a power of two of its own (the lanes of a row hold it, 8 elements each).  e is the smallest whole number with
// amax 2^-e <= 448 = 1.75 * 2^8: the exponent of amax less 8, one more where its fraction is past 1.75.  Multiplying by 2^-e is exact but
// for values that are far below the smallest of e4m3 anyway, so the only rounding is the one to 3 mantissa bits.
__device__ __forceinline__ uint2 to_e4m3(float (&y)[8], int lanes, unsigned int &byte) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(y[i]);
    if (a < INFINITY) amax = fmaxf(amax, a);
    else y[i] = NAN;     // infinite or NaN: NaN as stored
  }
  for (int x = lanes >> 1; x > 0; x >>= 1) amax = fmaxf(amax, __shfl_xor(amax, x, 64));
  const unsigned int bits = __float_as_uint(amax);
  byte = (unsigned int)max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
  const float inv = __uint_as_float((254u - byte) << 23);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= inv;
  uint2 q;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  q.x = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  q.y = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  return q;
}

// CACHE: -1 none (Q and K go to Qr and Kr), else the cache's format, and the rows of K and V go there.  PARTS: those rows come as fp32 shares.
template <typename T, int CACHE, bool PARTS>
__global__ void __launch_bounds__(64 * WAVES) turn_rows_kernel(TurnArgs a, smoe_cache c, smoe_places places, Work w, int N, int page_shift) {
  __shared__ float2 angle[WAVES][MAX_PAIRS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const unsigned int item = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + wave);
  const int row = (int)(item / (unsigned int)w.groups), group = (int)(item - (unsigned int)row * (unsigned int)w.groups);
  const bool live = row < a.rows;
  const int rot = a.rotary.turns ? a.rotary.rot : 0;

  int pos = 0, id = -1;
  if (live) {
    if constexpr (CACHE < 0) {
      pos = a.positions ? a.positions[row] : row % a.T;
    } else {
      int seq;
      find_place(places, N, row, seq, pos);
      id = find_page(places, c.pages, page_shift, seq, pos);
    }
    for (int i = lane; i < rot >> 1; i += 64) {
      const uint32_t part = (uint32_t)((a.rotary.turns[i] * (uint64_t)(int64_t)pos) >> 32);
      float s, k;
      sincospif((float)(int32_t)part * 0x1p-31f, &s, &k);
      angle[wave][i] = make_float2(k * a.rotary.amplitude, (a.back ? -s : s) * a.rotary.amplitude);
    }
  }
  __syncthreads();
  if (!live) return;

  const int lanes = 1 << w.lanes_log2, rows_at_once = 64 >> w.lanes_log2;
  const int e0 = (lane & (lanes - 1)) * 8, sub = lane >> w.lanes_log2;
  const bool active = e0 < a.d;
  const int half = rot >> 1;
  const bool whole = half % 8 == 0;               // both elements of 8 pairs lie in two whole chunks
  // y = x * co + partner * si of each element; the elements from `rot` on keep theirs
  float co[8], si[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = e0 + i;
    co[i] = 1.f;
    si[i] = 0.f;
    if (e < rot) {
      const bool first = a.rotary.interleaved ? !(e & 1) : e < half;
      const float2 t = angle[wave][a.rotary.interleaved ? e >> 1 : first ? e : e - half];
      co[i] = t.x;
      si[i] = first ? -t.y : t.y;
    }
  }
  const int total = a.hq + a.hk + (CACHE >= 0 ? a.hk : 0), last = min((group + 1) * w.per, total);
  for (int j0 = group * w.per; j0 < last; j0 += rows_at_once * BATCH) {
    Eight<T> x[BATCH], p[BATCH];
    Eight<float> xf[PARTS ? BATCH : 1], pf[PARTS ? BATCH : 1];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int j = j0 + u * rows_at_once + sub;
      if (PARTS && j >= a.hq) {
        if (j < last) {
          const bool value = j >= a.hq + a.hk;
          const size_t width = (size_t)a.hk * a.d, slab = width * a.rows;
          const float *src = a.parts + (value ? slab : 0) + (size_t)row * width + (size_t)(j - a.hq - (value ? a.hk : 0)) * a.d;
          sum_parts(src, 2 * slab, a.shares, e0, xf[PARTS ? u : 0]);
          if (!value && !a.rotary.interleaved && e0 < rot) {
            if (whole) {
              sum_parts(src, 2 * slab, a.shares, e0 < half ? e0 + half : e0 - half, pf[PARTS ? u : 0]);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int e = e0 + i;
                float sum = 0.f;
                if (e < rot)
                  for (int k = 0; k < a.shares; ++k) sum += src[k * 2 * slab + (e < half ? e + half : e - half)];
                pf[PARTS ? u : 0].set(i, sum);
              }
            }
          }
        }
      } else if (j < last && active) {
        const T *src = j < a.hq ? (const T *)a.Q + ((size_t)row * a.hq + j) * a.d
                       : j < a.hq + a.hk ? (const T *)a.K + ((size_t)row * a.hk + (j - a.hq)) * a.d
                                         : (const T *)a.V + ((size_t)row * a.hk + (j - a.hq - a.hk)) * a.d;
        x[u].load(src + e0);
        if (!a.rotary.interleaved && e0 < rot) {
          if (whole) {
            p[u].load(src + (e0 < half ? e0 + half : e0 - half));
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int e = e0 + i;
              p[u].set(i, e < rot ? to_f32<T>(src[e < half ? e + half : e - half]) : 0.f);
            }
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int j = j0 + u * rows_at_once + sub;
      const bool mine = j < last && active;
      const bool turned = j < a.hq + a.hk;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool part = PARTS && j >= a.hq;
        const float v = part ? xf[PARTS ? u : 0].get(i) : x[u].get(i);
        const float other = a.rotary.interleaved ? (part ? xf[PARTS ? u : 0].get(i ^ 1) : x[u].get(i ^ 1)) : (part ? pf[PARTS ? u : 0].get(i) : p[u].get(i));
        y[i] = turned && e0 + i < rot ? fmaf(other, si[i], v * co[i]) : v;
      }
      if (CACHE < 0 || j < a.hq) {
        if (mine) {
          T *dst = j < a.hq ? (T *)a.Qr + ((size_t)row * a.hq + j) * a.d : (T *)a.Kr + ((size_t)row * a.hk + (j - a.hq)) * a.d;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u].set(i, y[i]);
          x[u].store(dst + e0);
        }
      }
      if constexpr (CACHE >= 0) {
        const bool store = mine && j >= a.hq && id >= 0;
        const bool value = !turned;
        const size_t at = ((size_t)id * c.h + (j - a.hq - (value ? a.hk : 0))) * c.page + (pos & (c.page - 1));
        if constexpr (CACHE == SMOE_CACHE_BF16) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u].set(i, y[i]);
          if (store) x[u].store((T *)(value ? c.V : c.K) + at * a.d + e0);
        } else {
          unsigned int byte;
          const uint2 q = to_e4m3(y, lanes, byte);
          if (store) {
            *reinterpret_cast<uint2 *>((uint8_t *)(value ? c.V : c.K) + at * a.d + e0) = q;
            if (e0 == 0) (value ? c.V_exp : c.K_exp)[at] = (uint8_t)byte;
          }
        }
      }
    }
  }
}

// Rows back from the cache, as bf16: both formats' values are exact there.
template <int FORMAT>
__global__ void __launch_bounds__(64 * WAVES) cache_read_kernel(smoe_cache c, smoe_places places, Work w, int rows, int N, int page_shift, bf16_t *K, bf16_t *V) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const unsigned int item = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + wave);
  const int row = (int)(item / (unsigned int)w.groups), group = (int)(item - (unsigned int)row * (unsigned int)w.groups);
  if (row >= rows) return;
  int seq, pos;
  find_place(places, N, row, seq, pos);
  const int id = find_page(places, c.pages, page_shift, seq, pos);
  const int lanes = 1 << w.lanes_log2, rows_at_once = 64 >> w.lanes_log2;
  const int e0 = (lane & (lanes - 1)) * 8, sub = lane >> w.lanes_log2;
  const int last = min((group + 1) * w.per, 2 * c.h);
  for (int j0 = group * w.per; j0 < last; j0 += rows_at_once * BATCH) {
    Eight<bf16_t> x[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int j = j0 + u * rows_at_once + sub;
      const bool value = j >= c.h;
      x[u].v = 0;
      if (j < last && id >= 0) {
        const size_t at = ((size_t)id * c.h + (j - (value ? c.h : 0))) * c.page + (pos & (c.page - 1));
        if constexpr (FORMAT == SMOE_CACHE_BF16) {
          x[u].load((const bf16_t *)(value ? c.V : c.K) + at * c.d_head + e0);
        } else {
          typedef float f32x2 __attribute__((ext_vector_type(2)));
          const uint2 q = *reinterpret_cast<const uint2 *>((const uint8_t *)(value ? c.V : c.K) + at * c.d_head + e0);
          const float scale = e4m3_scale((value ? c.V_exp : c.K_exp)[at]);
          const f32x2 y0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, false), y1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, true);
          const f32x2 y2 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, false), y3 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, true);
          const float y[8] = {y0[0], y0[1], y1[0], y1[1], y2[0], y2[1], y3[0], y3[1]};
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u].set(i, y[i] * scale);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int j = j0 + u * rows_at_once + sub;
      const bool value = j >= c.h;
      if (j < last) x[u].store((value ? V : K) + ((size_t)row * c.h + (j - (value ? c.h : 0))) * c.d_head + e0);
    }
  }
}

Work deal(int rows, int per_token, int d) {
  Work w;
  w.lanes_log2 = 0;
  while ((8 << w.lanes_log2) < d) ++w.lanes_log2;
  const int at_once = 64 >> w.lanes_log2;
  w.per = at_once * BATCH;
  w.groups = ceil_div(per_token, w.per);
  (void)rows;
  return w;
}
bool grid_of(const Work &w, int rows, unsigned int &blocks) {
  const unsigned long long n = ((unsigned long long)rows * w.groups + WAVES - 1) / WAVES;
  blocks = (unsigned int)n;
  return n <= 0xffffffffull / (64 * WAVES);   // fewer than 2^32 threads a launch
}
int log2_of(int n) { return __builtin_ctz((unsigned int)n); }

}  // namespace

int launch_turn(hipStream_t s, smoe_dtype dt, const TurnArgs &a) {
  const Work w = deal(a.rows, a.hq + a.hk, a.d);
  unsigned int blocks;
  if (!grid_of(w, a.rows, blocks)) return SMOE_ERR_UNSUPPORTED;
  if (dt == SMOE_BF16) turn_rows_kernel<bf16_t, -1, false><<<blocks, 64 * WAVES, 0, s>>>(a, smoe_cache{}, smoe_places{}, w, 1, 0);
  else turn_rows_kernel<float, -1, false><<<blocks, 64 * WAVES, 0, s>>>(a, smoe_cache{}, smoe_places{}, w, 1, 0);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

int launch_cache_append(hipStream_t s, const TurnArgs &a, const smoe_cache &c, const smoe_places &p) {
  const Work w = deal(a.rows, a.hq + 2 * a.hk, a.d);
  unsigned int blocks;
  if (!grid_of(w, a.rows, blocks)) return SMOE_ERR_UNSUPPORTED;
  const int N = p.lens ? a.rows / p.sequences : 1, shift = log2_of(c.page);
  auto go = [&](auto kernel) { kernel<<<blocks, 64 * WAVES, 0, s>>>(a, c, p, w, N, shift); };
  if (c.format == SMOE_CACHE_BF16) a.parts ? go(turn_rows_kernel<bf16_t, SMOE_CACHE_BF16, true>) : go(turn_rows_kernel<bf16_t, SMOE_CACHE_BF16, false>);
  else a.parts ? go(turn_rows_kernel<bf16_t, SMOE_CACHE_E4M3, true>) : go(turn_rows_kernel<bf16_t, SMOE_CACHE_E4M3, false>);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

int launch_cache_read(hipStream_t s, const smoe_cache &c, const smoe_places &p, int rows, void *K, void *V) {
  const Work w = deal(rows, 2 * c.h, c.d_head);
  unsigned int blocks;
  if (!grid_of(w, rows, blocks)) return SMOE_ERR_UNSUPPORTED;
  const int N = p.lens ? rows / p.sequences : 1, shift = log2_of(c.page);
  if (c.format == SMOE_CACHE_BF16) cache_read_kernel<SMOE_CACHE_BF16><<<blocks, 64 * WAVES, 0, s>>>(c, p, w, rows, N, shift, (bf16_t *)K, (bf16_t *)V);
  else cache_read_kernel<SMOE_CACHE_E4M3><<<blocks, 64 * WAVES, 0, s>>>(c, p, w, rows, N, shift, (bf16_t *)K, (bf16_t *)V);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
