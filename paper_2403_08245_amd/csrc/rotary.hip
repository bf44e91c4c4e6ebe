// Rotary positions of query and key rows, and the two ways between rows and the paged cache: writing them (turned and rounded to 8 bits
// where asked) and reading them back.  All are bound by memory: a row is read once and written once.
//
// A wavefront takes one token's rows, or some of them, d_head / 8 lanes a row and 8 elements a lane.  The angles belong to the token:
// each lane works out the sine and cosine of one pair (more for rows over 128), and the wavefront shares them through LDS, so they cost
// a token one evaluation a lane, however many heads it has.  Its first rows are on their way meanwhile.
// Measured: queries and keys of 8192 tokens, 16 + 4 heads of 128, bf16, 84 MB: 19.6 us (4.3 TB/s; 15.8 where the caches hold them); of 32768
// tokens, 32 + 4 heads, 604 MB: 104 us (5.8 TB/s).  A large copy runs at 5.1.
//
// An angle is p f modulo one turn, of the 64-bit fraction of a turn that a position adds: one integer product that wraps, whose upper 32
// bits are the angle as a signed number of 2^-32 turns.
#include "cache.h"
#include <type_traits>

namespace {

constexpr int WAVES = 4;
constexpr int MAX_PAIRS = 256;      // rows of at most 512 elements
// Rows a lane has in flight.  2: a decoding step's four tokens 3.0 us, the queries and keys of 8192 tokens (16 + 4 heads of 128) 19.4; 4: 3.5
// and 21.2; 1: 2.9 and 18.5, but rows of 64 half turned 26.4 instead of 22.2.  (One launch behind another, from a captured graph; by
// itself, under a trace, the first is 3.5.)
constexpr int BATCH = 2;
constexpr int TOKENS = 16;          // of a wavefront, where rows are copied between the cache and plain tensors
constexpr int MOST = 8;             // rounds of rows a wavefront takes (32768 tokens of 36 heads: 4 108.6, 8 107.9, 16 116 us)
// Rounds of rows that fill the chip as a wavefront each; with more, a wavefront takes several (8192 tokens of 20 heads in bf16: 19.4 us, with
// 16384 here 20.7; in fp32 37.4 and 35.4).
constexpr int MANY_ITEMS = 8192;

template <typename T> struct Eight;   // 8 elements of a row as they are loaded and stored
template <> struct Eight<bf16_t> {
  typedef bf16_t vec __attribute__((ext_vector_type(8)));
  vec v;
  __device__ __forceinline__ void load(const bf16_t *p) { v = *reinterpret_cast<const vec *>(p); }
  __device__ __forceinline__ void store(bf16_t *p) const { *reinterpret_cast<vec *>(p) = v; }
  __device__ __forceinline__ void load_once(const bf16_t *p) { v = __builtin_nontemporal_load(reinterpret_cast<const vec *>(p)); }   // kept by no cache
  template <bool ONCE> __device__ __forceinline__ void store_as(bf16_t *p) const {
    if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<vec *>(p));
    else store(p);
  }
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

// the sum of 8 elements' shares, in their order, eight of them requested together
__device__ __forceinline__ void sum_parts(const float *src, size_t stride, int shares, int e0, Eight<float> &y) {
  constexpr int AHEAD = 8;
  Eight<float> part[AHEAD];
#pragma unroll
  for (int i = 0; i < 8; ++i) y.set(i, 0.f);
#pragma unroll 1
  for (int k0 = 0; k0 < shares; k0 += AHEAD) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (k0 + k < shares) part[k].load(src + (k0 + k) * stride + e0);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (k0 + k < shares) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y.set(i, y.get(i) + part[k].get(i));
      }
  }
}

// How the rows of a launch are dealt to wavefronts: d / 8 lanes a row, as many rows at once as 64 lanes hold.
struct Work {
  int groups;          // wavefronts a token
  int per;             // rows of each
  int lanes;           // lanes a row, d / 8
  int at_once;         // rows at once, 64 / lanes
};
// The wavefront's share of it: a token and some of its rows.
struct Item {
  int row, group;
};
__device__ __forceinline__ Item item_of(const Work &w) {
  const unsigned int item = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + (threadIdx.x >> 6));
  const unsigned int row = item / (unsigned int)w.groups;
  return Item{(int)row, (int)(item - row * (unsigned int)w.groups)};
}

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
  if (byte == 247u) {      // e = 120, of values past 1.75 * 2^127: the code above 240 would stand for 2^128, which neither bf16 nor fp32 holds
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fabsf(y[i]) > 240.f ? copysignf(240.f, y[i]) : y[i];
  }
  uint2 q;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  q.x = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  q.y = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  return q;
}

// CACHE: -1 none (Q and K go to Qr and Kr), else the cache's format, and the rows of K and V go there.  PARTS: those rows come as fp32 shares, and those of
// Q, with WIDE, as fp32.
template <typename T, int CACHE, bool PARTS, bool WIDE = false>
__global__ void __launch_bounds__(64 * WAVES) turn_rows_kernel(TurnArgs a, smoe_cache c, smoe_places places, Work w, int N, int page_shift) {
  __shared__ float2 s_angle[WAVES][MAX_PAIRS];
  constexpr int AHEAD = PARTS ? 1 : BATCH;        // a decoding pass has few rows for many wavefronts
  float2 *const angle = s_angle[threadIdx.x >> 6];
  const int lane = threadIdx.x & 63;
  const Item item = item_of(w);
  const int row = item.row;
  if (row >= a.rows) return;                      // a wavefront shares nothing with its block's others
  const int rot = a.rotary.turns ? a.rotary.rot : 0, half = rot >> 1;
  const bool whole = half % 8 == 0;               // both elements of 8 pairs lie in two whole chunks
  const int sub = lane / w.lanes, e0 = (lane - sub * w.lanes) * 8;
  const int total = a.hq + a.hk + (CACHE >= 0 ? a.hk : 0), end = min((item.group + 1) * w.per, total);

  Eight<T> x[AHEAD], p[AHEAD];                    // elements, and their partners where those are another chunk's
  Eight<float> xf, pf;                            // the same in fp32: sums of shares, wide queries
  auto mine = [&](int j) { return j < end && sub < w.at_once; };
  auto load = [&](int u, int j) {
    if (!mine(j)) return;
    if (PARTS && j >= a.hq) {
      const bool value = j >= a.hq + a.hk;
      const size_t width = (size_t)a.hk * a.d, slab = width * a.rows;
      const float *src = a.parts + (value ? slab : 0) + (size_t)row * width + (size_t)(j - a.hq - (value ? a.hk : 0)) * a.d;
      sum_parts(src, 2 * slab, a.shares, e0, xf);
      if (value || a.rotary.interleaved || e0 >= rot) return;
      if (whole) {
        sum_parts(src, 2 * slab, a.shares, e0 < half ? e0 + half : e0 - half, pf);
        return;
      }
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const int e = e0 + i;
        float sum = 0.f;
        if (e < rot)
          for (int k = 0; k < a.shares; ++k) sum += src[k * 2 * slab + (e < half ? e + half : e - half)];
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (t == i) pf.set(t, sum);
      }
      return;
    }
    if (WIDE) {
      const float *src = (const float *)a.Q + ((size_t)row * a.hq + j) * a.d;
      xf.load(src + e0);
      if (a.rotary.interleaved || e0 >= rot) return;
      if (whole) {
        pf.load(src + (e0 < half ? e0 + half : e0 - half));
        return;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = e0 + i;
        pf.set(i, e < rot ? src[e < half ? e + half : e - half] : 0.f);
      }
      return;
    }
    const T *src = j < a.hq ? (const T *)a.Q + ((size_t)row * a.hq + j) * a.d
                   : j < a.hq + a.hk ? (const T *)a.K + ((size_t)row * a.hk + (j - a.hq)) * a.d
                                     : (const T *)a.V + ((size_t)row * a.hk + (j - a.hq - a.hk)) * a.d;
    x[u].load(src + e0);
    if (a.rotary.interleaved || e0 >= rot) return;
    if (whole) {
      p[u].load(src + (e0 < half ? e0 + half : e0 - half));
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + i;
      p[u].set(i, e < rot ? to_f32<T>(src[e < half ? e + half : e - half]) : 0.f);
    }
  };
  int j0 = item.group * w.per + sub;
  // the first rows are on their way while the angles are worked out
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) load(u, j0 + u * w.at_once);

  int pos = 0, id = -1;
  if constexpr (CACHE < 0) {
    pos = a.positions ? a.positions[row] : row % a.T;
  } else {
    int seq;
    find_place(places, N, row, seq, pos);
    id = find_page(places, c.pages, page_shift, seq, pos);
  }
  for (int i = lane; i < half; i += 64) {
    const uint32_t part = (uint32_t)((a.rotary.turns[i] * (uint64_t)(int64_t)pos) >> 32);
    float s, k;
    // to 24 bits of half a turn, 9.4e-8 radians at most: fp32 rows come out 2.8e-8 off in the root mean square, 2.2e-8 with the angle in 64 bits
    sincospif((float)(int32_t)part * 0x1p-31f, &s, &k);
    angle[i] = make_float2(k * a.rotary.amplitude, (a.back ? -s : s) * a.rotary.amplitude);
  }
  // LDS operations of one wavefront execute in order; the compiler keeps to it, too
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // y = x * co + partner * si of each element; the elements from `rot` on keep theirs
  float co[8], si[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = e0 + i;
    co[i] = 1.f;
    si[i] = 0.f;
    if (e < rot) {
      const bool first = a.rotary.interleaved ? !(e & 1) : e < half;
      const float2 t = angle[a.rotary.interleaved ? e >> 1 : first ? e : e - half];
      co[i] = t.x;
      si[i] = first ? -t.y : t.y;
    }
  }
  while (true) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int j = j0 + u * w.at_once;
      const bool turned = j < a.hq + a.hk, part = PARTS && (WIDE || j >= a.hq);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = part ? xf.get(i) : x[u].get(i);
        const float other = a.rotary.interleaved ? (part ? xf.get(i ^ 1) : x[u].get(i ^ 1)) : (part ? pf.get(i) : p[u].get(i));
        y[i] = turned && e0 + i < rot ? fmaf(other, si[i], v * co[i]) : v;
      }
      if (CACHE < 0 || j < a.hq) {
        if (WIDE && mine(j)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) xf.set(i, y[i]);
          xf.store((float *)a.Qr + ((size_t)row * a.hq + j) * a.d + e0);
        } else if (mine(j)) {
          T *dst = j < a.hq ? (T *)a.Qr + ((size_t)row * a.hq + j) * a.d : (T *)a.Kr + ((size_t)row * a.hk + (j - a.hq)) * a.d;
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u].set(i, y[i]);
          x[u].store(dst + e0);
        }
      }
      if constexpr (CACHE >= 0) {
        const bool store = mine(j) && j >= a.hq && id >= 0, value = !turned;
        const size_t at = ((size_t)id * c.h + (j - a.hq - (value ? a.hk : 0))) * c.page + (pos & (c.page - 1));
        if constexpr (CACHE == SMOE_CACHE_BF16) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u].set(i, y[i]);
          if (store) x[u].store((T *)(value ? c.V : c.K) + at * a.d + e0);
        } else {
          unsigned int byte;
          const uint2 q = to_e4m3(y, w.lanes, byte);
          if (store) {
            *reinterpret_cast<uint2 *>((uint8_t *)(value ? c.V : c.K) + at * a.d + e0) = q;
            if (e0 == 0) (value ? c.V_exp : c.K_exp)[at] = (uint8_t)byte;
          }
        }
      }
    }
    j0 += w.at_once * AHEAD;
    if (j0 - sub >= end) break;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(u, j0 + u * w.at_once);
  }
}

// Rows to the cache without a turn (WRITE), or back from it as bf16, where both formats' values are exact.  A wavefront takes 16 tokens' rows
// of one head, keys or values: positions that follow one another lie side by side on a page, so that what it writes there (or
// reads) is 2 or 4 KB in a row, and the 16 exponents one piece.  Rows on their way into the cache are dead afterwards and kept by no cache;
// ONCE: nor is what is written, where it is more than the caches could hold until it is used.
// Quantising 34.7 thousand tokens of 8 heads, 213 MB, us: 49.5 so (46.8 with the pages past the caches, too, which costs 12 if they are read
// back next; 53.6 all through the caches; 51 with a token a wavefront); of 4 heads of 64 16.6 (18.1; 35.5 with a token a wavefront).  Reading the
// former back, 213 MB again: 33.1 past the caches, 47.9 through them.
template <int FORMAT, bool WRITE, int D, bool ONCE>
__global__ void __launch_bounds__(64 * WAVES) cache_rows_kernel(smoe_cache c, smoe_places places, bf16_t *K, bf16_t *V, int tokens, int N, int page_shift, unsigned int items) {
  constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, ROUNDS = TOKENS / AT_ONCE;
  const int lane = threadIdx.x & 63, sub = lane / LANES, e0 = (lane % LANES) * 8;
  const unsigned int item = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + (threadIdx.x >> 6));
  if (item >= items) return;
  const unsigned int per_tile = 2u * c.h, tile = item / per_tile, j = item - tile * per_tile;
  const bool value = j >= (unsigned int)c.h;
  const int head = (int)(j - (value ? c.h : 0));
  bf16_t *const outside = (value ? V : K) + (size_t)head * D + e0;
  uint8_t *const pages = (uint8_t *)(value ? c.V : c.K), *const exps = value ? c.V_exp : c.K_exp;
  Eight<bf16_t> x[ROUNDS];
  size_t at[ROUNDS];          // the row in the cache
  bool mine[ROUNDS], there[ROUNDS];
#pragma unroll
  for (int u = 0; u < ROUNDS; ++u) {
    const long long t = (long long)tile * TOKENS + u * AT_ONCE + sub;
    mine[u] = t < tokens;
    const int token = mine[u] ? (int)t : 0;
    if (WRITE && mine[u]) x[u].load_once(outside + (size_t)token * c.h * D);
    int seq, pos;
    find_place(places, N, token, seq, pos);
    const int id = find_page(places, c.pages, page_shift, seq, pos);
    there[u] = mine[u] && id >= 0;
    at[u] = ((size_t)max(id, 0) * c.h + head) * c.page + (pos & (c.page - 1));
  }
  if constexpr (!WRITE) {
    uint2 q[ROUNDS];
    unsigned int byte[ROUNDS];
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) {
      x[u].v = 0;
      if constexpr (FORMAT == SMOE_CACHE_BF16) {
        if (there[u]) x[u].load((const bf16_t *)pages + at[u] * D + e0);
      } else {
        q[u] = uint2{0, 0};
        byte[u] = 1;
        if (there[u]) {
          q[u] = *reinterpret_cast<const uint2 *>(pages + at[u] * D + e0);
          byte[u] = exps[at[u]];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) {
      if constexpr (FORMAT == SMOE_CACHE_E4M3) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const float scale = e4m3_scale(byte[u]);
        const f32x2 y0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u].x, false), y1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u].x, true);
        const f32x2 y2 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u].y, false), y3 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u].y, true);
        const float y[8] = {y0[0], y0[1], y1[0], y1[1], y2[0], y2[1], y3[0], y3[1]};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u].set(i, y[i] * scale);
      }
      if (mine[u]) x[u].template store_as<ONCE>(outside + (size_t)(tile * TOKENS + u * AT_ONCE + sub) * c.h * D);
    }
  } else {
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) {
      if constexpr (FORMAT == SMOE_CACHE_BF16) {
        if (there[u]) x[u].template store_as<ONCE>((bf16_t *)pages + at[u] * D + e0);
      } else {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[u].get(i);
        unsigned int byte;
        const uint2 q = to_e4m3(y, LANES, byte);
        if (there[u]) {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          const u32x2 codes = {q.x, q.y};
          u32x2 *const dst = reinterpret_cast<u32x2 *>(pages + at[u] * D + e0);
          if constexpr (ONCE) __builtin_nontemporal_store(codes, dst);
          else *dst = codes;
          if (e0 == 0) exps[at[u]] = (uint8_t)byte;
        }
      }
    }
  }
}

// Small launches spread a token's rows over wavefronts, one round of rows each; large ones keep a token's rows together, up to `most` rounds of
// them, which share its angles and its place.
Work deal(int rows, int per_token, int d, int most) {
  Work w;
  w.lanes = d / 8;
  w.at_once = 64 / w.lanes;
  const int rounds = ceil_div(per_token, w.at_once);
  const long long each = std::min<long long>(std::max<long long>((long long)rows * rounds / MANY_ITEMS, 1), std::min(most, rounds));
  w.groups = ceil_div(rounds, (int)each);
  w.per = ceil_div(rounds, w.groups) * w.at_once;
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
  const Work w = deal(a.rows, a.hq + a.hk, a.d, MOST);
  unsigned int blocks;
  if (!grid_of(w, a.rows, blocks)) return SMOE_ERR_UNSUPPORTED;
  if (dt == SMOE_BF16) turn_rows_kernel<bf16_t, -1, false><<<blocks, 64 * WAVES, 0, s>>>(a, smoe_cache{}, smoe_places{}, w, 1, 0);
  else turn_rows_kernel<float, -1, false><<<blocks, 64 * WAVES, 0, s>>>(a, smoe_cache{}, smoe_places{}, w, 1, 0);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

namespace {
template <bool WRITE> int launch_rows(hipStream_t s, const smoe_cache &c, const smoe_places &p, int tokens, void *K, void *V) {
  const unsigned long long items = 2ull * c.h * ceil_div(tokens, TOKENS), blocks = (items + WAVES - 1) / WAVES;
  if (blocks > 0xffffffffull / (64 * WAVES)) return SMOE_ERR_UNSUPPORTED;   // fewer than 2^32 threads a launch
  auto go = [&](auto kernel) {
    kernel<<<(unsigned int)blocks, 64 * WAVES, 0, s>>>(c, p, (bf16_t *)K, (bf16_t *)V, tokens, p.lens ? tokens / p.sequences : 1, log2_of(c.page), (unsigned int)items);
  };
  auto by_once = [&](auto d_c, auto once_c) {
    constexpr int D = decltype(d_c)::value;
    constexpr bool ONCE = decltype(once_c)::value;
    c.format == SMOE_CACHE_BF16 ? go(cache_rows_kernel<SMOE_CACHE_BF16, WRITE, D, ONCE>) : go(cache_rows_kernel<SMOE_CACHE_E4M3, WRITE, D, ONCE>);
  };
  // pages are read again from half the last-level cache down, rows by the launch that comes next, with as much of its own
  const size_t written = (size_t)tokens * c.h * c.d_head * (WRITE && c.format == SMOE_CACHE_E4M3 ? 2 : 4);
  const bool once = written > LAST_LEVEL_CACHE / (WRITE ? 2 : 4);
  auto by_d = [&](auto d_c) { once ? by_once(d_c, std::true_type{}) : by_once(d_c, std::false_type{}); };
  c.d_head == 128 ? by_d(std::integral_constant<int, 128>{}) : by_d(std::integral_constant<int, 64>{});
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
}  // namespace

bool cache_append_fits(int rows, int hq, int hk, int d) {
  unsigned int blocks;
  return grid_of(deal(rows, hq + 2 * hk, d, 1), rows, blocks);   // a round of rows each: the most wavefronts
}

int launch_cache_append(hipStream_t s, const TurnArgs &a, const smoe_cache &c, const smoe_places &p) {
  if (!a.rotary.turns && !a.parts) return launch_rows<true>(s, c, p, a.rows, (void *)a.K, (void *)a.V);
  const Work w = deal(a.rows, a.hq + 2 * a.hk, a.d, a.parts ? 1 : MOST);
  unsigned int blocks;
  if (!grid_of(w, a.rows, blocks)) return SMOE_ERR_UNSUPPORTED;
  const int N = p.lens ? a.rows / p.sequences : 1, shift = log2_of(c.page);
  auto go = [&](auto kernel) { kernel<<<blocks, 64 * WAVES, 0, s>>>(a, c, p, w, N, shift); };
  auto by_format = [&](auto f_c) {
    constexpr int F = decltype(f_c)::value;
    if (!a.parts) go(turn_rows_kernel<bf16_t, F, false>);
    else if (a.wide) go(turn_rows_kernel<bf16_t, F, true, true>);
    else go(turn_rows_kernel<bf16_t, F, true>);
  };
  if (c.format == SMOE_CACHE_BF16) by_format(std::integral_constant<int, SMOE_CACHE_BF16>{});
  else by_format(std::integral_constant<int, SMOE_CACHE_E4M3>{});
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

int launch_cache_read(hipStream_t s, const smoe_cache &c, const smoe_places &p, int rows, void *K, void *V) { return launch_rows<false>(s, c, p, rows, K, V); }
