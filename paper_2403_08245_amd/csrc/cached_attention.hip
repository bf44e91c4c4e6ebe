// Attention of the last N positions of every sequence over the paged cache: the decoding form of attention.hip.
//
// Bound by memory: every key and value is read once for the N * G query rows of its head, and 32 rows at most share a read, so a byte of
// the cache meets 16 to 32 multiplications a row where the matrix cores could do 300.  What counts is that all compute units read from the
// first microsecond to the last, whatever the lengths are: a sequence's keys are cut into pieces of about the same length over the
// whole batch, one block a piece, and a second kernel joins the pieces of a sequence from their maxima and sums.
//
// Inside a block four wavefronts take steps of 32 keys in turn, from memory straight to registers.  Scores are worked out transposed,
// S^T[key][query] = K Q^T on 16 x 16 x 32 matrix instructions, so a lane owns one query column: its running maximum and sum are scalars of
// the lane, and its eight weights of a step already lie as the second product's operand, O^T[column][query] = V^T P^T, whose contraction
// runs over the keys in the order the lanes hold them.  A lane reads its eight keys' values for D / 16 columns and turns them
// into the operands of D / 16 instructions by byte permutations.  No LDS traffic of theirs (two tiles of queries, and fp32 ones,
// wait in LDS) and no barrier until a piece ends.
// Values in e4m3 are widened to bf16, scaled, as they are used: exactly, and at half the bytes.
//
// Measured (reads alone reach 6.5 TB/s here, a copy 5.1): 256 sequences of 500, 8 heads, 524 MB 81 us (6.5 TB/s); 64 of 100 to 8192, 4 heads,
// 240 MB 50 us; 64 of 3 to 8192, 142 MB 31 us (4.6); 90001 and 131072 in e4m3, 8 heads of 24 rows, 456 MB 85.5 us (5.3); one of 301
// 6.8 us.  What bounds the short ones is a chain of dependent reads (lengths, page numbers, keys) and, where sequences are cut, the second
// launch of 4 us; the counters show 1.02 times the bytes of the cache fetched.
#include "cache.h"
#include <algorithm>
#include <type_traits>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int STEP = 32;         // keys of a step
constexpr int WAVES = 4;
constexpr int MAX_TARGET = 768;  // pieces that the whole batch is cut into, about (Dims::target), at most
// As many pieces as blocks are resident, three a compute unit (one new token) or two: a few more would run by themselves at the end (64
// sequences of up to 8192 positions: 768 pieces 31.1 us, 1024 33.0; two long ones of three tokens: 512 82.8, 1024 94.4).
constexpr int T_ONE = 768, T_MULTI = 512, T_TWO = 512;
// Sequences of no more steps are not cut, and where the table holds no longer ones there is no second kernel (one of 301 positions 6.5 us, with a line
// at 8 steps 9.4; a thousand of up to 300 21.3 and 170).
constexpr int WHOLE_STEPS = 16;
// Steps of a piece, at least: one sequence of 4096, 4 heads, 16 12.5 us, 8 10.7, 4 10.0; four of 900 to 4096 12.8, 11.1, 12.5
// (taken before the reads went past the caches).
constexpr int MIN_STEPS = 8;
constexpr int MOST_PIECES = 256; // of a unit (one of 131072, one head: 21.4 us; 512 23.5)

struct Dims {
  int N, G, R;                   // R = N * G query rows of a (sequence, head)
  int tiles;                     // row tiles of each
  int units;                     // tiles * h: what a sequence is worked on as
  int shift;                     // page = 1 << shift
  int cap;                       // positions the table can hold
  int rows;                      // rows a piece leaves in the workspace
  int target;                    // pieces that the whole batch is cut into, about
  bool whole;                    // the table holds too few positions for a sequence to be cut
};

// ------------------------------------------------------------------------------------------------ the cut
// Steps of a sequence; one without keys has one, whose block writes its zeros.
__device__ __forceinline__ int length_of(const int32_t *lens, int b, int cap) { return min(max(lens[b], 0), cap); }
__device__ __forceinline__ int steps_of(int len) { return max((len + STEP - 1) / STEP, 1); }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <int CTRL, int ROWS> __device__ __forceinline__ int shifted(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
// inclusive sums over the lanes
__device__ __forceinline__ int scan_add(int v) {
  v += shifted<0x111, 0xf>(v);
  v += shifted<0x112, 0xf>(v);
  v += shifted<0x114, 0xf>(v);
  v += shifted<0x118, 0xf>(v);
  v += shifted<0x142, 0xa>(v);
  v += shifted<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ float scan_add(float v) {
  auto f = [](int x) { return __int_as_float(x); };
  v += f(shifted<0x111, 0xf>(__float_as_int(v)));
  v += f(shifted<0x112, 0xf>(__float_as_int(v)));
  v += f(shifted<0x114, 0xf>(__float_as_int(v)));
  v += f(shifted<0x118, 0xf>(__float_as_int(v)));
  v += f(shifted<0x142, 0xa>(__float_as_int(v)));
  v += f(shifted<0x143, 0xc>(__float_as_int(v)));
  return v;
}
__device__ __forceinline__ int at_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

struct Place {
  int b, len, n;       // sequence, its length, the pieces each of its units is cut into
  int local;           // number within what is counted of this sequence
  int slot;            // pieces of cut sequences before this sequence's
};
// Which sequence does number `index` belong to, counting the pieces of all units (JOIN false), or the units that are cut (JOIN true), in the
// order of the sequences?  Every wavefront finds its own: a lane takes ceil(B / 64) sequences in a row.  The length of a piece follows from
// the batch's steps; their sum is a floating number (a few roundings longer or shorter pieces), the same in every wavefront of both kernels.
// With the hundredth that it is longer there are fewer than `target` cut units, and fewer than twice as many pieces of cut units.
constexpr int HELD = 4;   // lengths a lane keeps in registers, requested together
template <bool JOIN> __device__ __forceinline__ bool find_piece(const int32_t *lens, int B, const Dims &d, int index, int lane, Place &p) {
  const int each = (B + 63) >> 6, first = lane * each, end = min(first + each, B);
  int held[HELD];
  float sum = 0.f;
  auto batch = [&](int from) {
    if (each == 1) {
      held[0] = from < end ? lens[from] : -1;
      held[0] = from < end ? min(max(held[0], 0), d.cap) : -1;
#pragma unroll
      for (int i = 1; i < HELD; ++i) held[i] = -1;
      return;
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = from + i < end ? lens[from + i] : -1;
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = from + i < end ? min(max(held[i], 0), d.cap) : -1;
  };
#pragma unroll 1
  for (int c = 0; c < each; c += HELD) {
    batch(first + c);
#pragma unroll
    for (int i = 0; i < HELD; ++i) sum += held[i] >= 0 ? (float)steps_of(held[i]) : 0.f;
  }
  const float total = __int_as_float(at_lane(__float_as_int(scan_add(sum)), 63)) * (float)d.units;
  const int per = max((int)fminf(total * (1.01f / (float)d.target), 1e9f) + 1, MIN_STEPS);
  // ceil(steps / per) by a reciprocal: steps and per are whole numbers under 2^26, so the quotient is off by less than one
  const float inv = 1.0f / (float)per;
  auto pieces_of = [&](int len) {
    const int steps = steps_of(len);
    if (steps <= WHOLE_STEPS) return 1;
    int n = (int)((float)steps * inv);
    n += n * per < steps ? 1 : 0;
    n += n * per < steps ? 1 : 0;
    n -= (n - 1) * per >= steps ? 1 : 0;
    return min(n, MOST_PIECES);
  };
  int pieces = 0, cut_pieces = 0, cut_units = 0;
#pragma unroll 1
  for (int c = 0; c < each; c += HELD) {
    if (each > HELD) batch(first + c);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int n = held[i] >= 0 ? pieces_of(held[i]) : 0;
      pieces += n;
      cut_pieces += n > 1 ? n : 0;
      cut_units += n > 1 ? 1 : 0;
    }
  }
  const int counted = (JOIN ? cut_units : pieces) * d.units;
  cut_pieces *= d.units;
  const int upto = scan_add(counted), slots_upto = scan_add(cut_pieces);
  const unsigned long long past = __ballot(upto > index);
  if (!past) return false;
  const int owner = __ffsll((long long)past) - 1;
  int before = at_lane(upto - counted, owner), slot = at_lane(slots_upto - cut_pieces, owner);
  if (each == 1) {                            // that lane's only one
    p.b = owner;
    p.len = at_lane(held[0], owner);
    p.n = at_lane(pieces, owner);
    p.local = index - before;
    p.slot = slot;
    return true;
  }
#pragma unroll 1
  for (int c = 0; c < each; c += 64) {        // that lane's sequences, one a lane
    const int b = owner * each + c + lane;
    const bool have = c + lane < each && b < B;
    const int len = have ? length_of(lens, b, d.cap) : 0, n = have ? pieces_of(len) : 0;
    const int all = n * d.units, cut = n > 1 ? all : 0, here = JOIN ? (n > 1 ? d.units : 0) : all;
    const int to = scan_add(here), slots_to = scan_add(cut);
    const unsigned long long found = __ballot(before + to > index);
    if (found) {
      const int l = __ffsll((long long)found) - 1;
      p.b = owner * each + c + l;
      p.len = at_lane(len, l);
      p.n = at_lane(n, l);
      p.local = index - before - at_lane(to - here, l);
      p.slot = slot + at_lane(slots_to - cut, l);
      return true;
    }
    before += at_lane(to, 63);
    slot += at_lane(slots_to, 63);
  }
  return false;
}

// What a piece leaves: its rows' sums of weighted values [rows][D], then their maxima and sums of weights [rows] each.
__host__ __device__ inline size_t slot_floats(int rows, int D) { return ((size_t)rows * (D + 2) + 3) & ~(size_t)3; }

// ------------------------------------------------------------------------------------------------ a step's operands
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const void *p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000); }
// ONCE: bytes that nothing will read again are kept by no cache.
template <bool ONCE> __device__ __forceinline__ u32x4 load4(__amdgpu_buffer_rsrc_t w, int at) { return __builtin_amdgcn_raw_buffer_load_b128(w, at, 0, ONCE ? 2 : 0); }
template <bool ONCE> __device__ __forceinline__ u32x2 load2(__amdgpu_buffer_rsrc_t w, int at) { return __builtin_amdgcn_raw_buffer_load_b64(w, at, 0, ONCE ? 2 : 0); }
template <bool ONCE> __device__ __forceinline__ uint32_t load1(__amdgpu_buffer_rsrc_t w, int at) { return __builtin_amdgcn_raw_buffer_load_b32(w, at, 0, ONCE ? 2 : 0); }

// two bf16 of the lower or upper two of four e4m3 codes, scaled
template <bool UPPER> __device__ __forceinline__ uint32_t widen(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, UPPER));
}

// The upper of the two bf16 numbers that stand for x: cut towards zero, from the next number below it, so that what is left for the lower is
// never zero and both have x's sign.  Infinity times x is then infinity times either, and their sum, not a NaN; rounded to the nearest, the
// lower would be zero or of the other sign for half of all x.  The two are within 2^-16 of x (2^-17 with the nearest).
__device__ __forceinline__ float upper_part(float x) { return __uint_as_float(__float_as_uint(x * (1.f - 0x1p-23f)) & 0xffff0000u); }

// The same offset, but what is added to it stays an immediate of the loads: hoisted out of the loop, every sum would take a register.
__device__ __forceinline__ int here(int at) {
  __asm__ volatile("" : "+v"(at));
  return at;
}
// the largest over the lanes of a query (lane % 16)
__device__ __forceinline__ float max_of_query(float x) {
  unsigned int b = __float_as_uint(x);
  u32x2 r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  unsigned int r0 = r[0], r1 = r[1];
  x = fmaxf(__uint_as_float(r0), __uint_as_float(r1));
  b = __float_as_uint(x);
  r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  r0 = r[0], r1 = r[1];
  return fmaxf(__uint_as_float(r0), __uint_as_float(r1));
}

// A group of 16 keys, which lies on one page: windows over its rows and exponents (wave-uniform).  Rows past the length and pages that do not
// exist lie outside and read as zeros: no product of a weight of zero with whatever the cache holds there.
struct Group {
  const char *K, *V;
  const uint8_t *K_exp, *V_exp;
  int left;              // rows within the length
  bool exists;
};

// Keys: lane -> key (lane % 16) of each of the two groups, D / 4 elements of its row.  Which elements go with which instruction is
// free as long as the queries' fragments follow (query_offset).
template <int D, int FORMAT> struct Keys {
  static constexpr int BYTES = FORMAT == SMOE_CACHE_BF16 ? D * 2 : D, LOADS = BYTES / 64;
  u32x4 v[2][LOADS];
  uint32_t e[2];
  static __device__ __forceinline__ int lane_offset(int lane) { return (lane & 15) * BYTES + (lane >> 4) * 16; }
  template <bool ONCE> __device__ __forceinline__ void load(int t, const Group &p, int at, int lane) {
    const __amdgpu_buffer_rsrc_t rows = window(p.K, p.left * BYTES);
    at = here(at);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) v[t][i] = load4<ONCE>(rows, at + i * 64);
    if constexpr (FORMAT == SMOE_CACHE_E4M3) e[t] = __builtin_amdgcn_raw_buffer_load_b8(window(p.K_exp, p.left), lane & 15, 0, 0);
  }
  // first element of the lane's eight of instruction ks
  static __device__ __forceinline__ int query_offset(int ks, int lane) {
    return FORMAT == SMOE_CACHE_BF16 ? ks * 32 + (lane >> 4) * 8 : (ks >> 1) * 64 + (lane >> 4) * 16 + (ks & 1) * 8;
  }
  __device__ __forceinline__ bf16x8 frag(int t, int ks) const {
    if constexpr (FORMAT == SMOE_CACHE_BF16) {
      return __builtin_bit_cast(bf16x8, v[t][ks]);
    } else {
      const uint32_t a = v[t][ks >> 1][(ks & 1) * 2], b = v[t][ks >> 1][(ks & 1) * 2 + 1];
      const float scale = e4m3_scale(e[t]);
      return __builtin_bit_cast(bf16x8, u32x4{widen<false>(a, scale), widen<true>(a, scale), widen<false>(b, scale), widen<true>(b, scale)});
    }
  }
};

// Values: lane -> keys 4 (lane / 16) + 0..3 of both groups, columns D / 16 * (lane % 16) and on.
template <int D, int FORMAT> struct Values {
  static constexpr int COLS = D / 16, WORDS = COLS / 2;    // columns of a lane, 32-bit words of them as bf16
  static constexpr int KEPT = FORMAT == SMOE_CACHE_BF16 ? WORDS : WORDS / 2;
  static constexpr int BYTES = FORMAT == SMOE_CACHE_BF16 ? D * 2 : D;
  uint32_t v[8][KEPT];
  uint32_t e[2];
  static __device__ __forceinline__ int lane_offset(int lane) { return (lane >> 4) * 4 * BYTES + (lane & 15) * KEPT * 4; }
  template <bool ONCE> __device__ __forceinline__ void load(int t, const Group &p, int at, int lane) {
    const __amdgpu_buffer_rsrc_t rows = window(p.V, p.left * BYTES);
    at = here(at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (KEPT == 4) {
        const u32x4 x = load4<ONCE>(rows, at + i * BYTES);
#pragma unroll
        for (int w = 0; w < 4; ++w) v[4 * t + i][w] = x[w];
      } else if constexpr (KEPT == 2) {
        const u32x2 x = load2<ONCE>(rows, at + i * BYTES);
        v[4 * t + i][0] = x[0];
        v[4 * t + i][1] = x[1];
      } else {
        v[4 * t + i][0] = load1<ONCE>(rows, at + i * BYTES);
      }
    }
    if constexpr (FORMAT == SMOE_CACHE_E4M3) e[t] = load1<false>(window(p.V_exp, p.left ? 16 : 0), (lane >> 4) * 4);
  }
};
// The same as bf16.
template <int D> struct Columns {
  static constexpr int WORDS = D / 32;
  uint32_t v[8][WORDS];
  template <int FORMAT> __device__ __forceinline__ Columns(const Values<D, FORMAT> &x, const int (&left)[2], int g) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (FORMAT == SMOE_CACHE_BF16) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) v[k][w] = x.v[k][w];
      } else {
        // the exponents behind the length are masked: a scale of what lies there could make a NaN of zero
        const float scale = 4 * g + (k & 3) < left[k >> 2] ? e4m3_scale((x.e[k >> 2] >> (8 * (k & 3))) & 255u) : 0.f;
#pragma unroll
        for (int w = 0; w < WORDS / 2; ++w) {
          v[k][2 * w] = widen<false>(x.v[k][w], scale);
          v[k][2 * w + 1] = widen<true>(x.v[k][w], scale);
        }
      }
    }
  }
  // column j of the lane's, its eight keys
  __device__ __forceinline__ bf16x8 frag(int j) const {
    u32x4 r;
#pragma unroll
    for (int m = 0; m < 4; ++m) r[m] = __builtin_amdgcn_perm(v[2 * m + 1][j / 2], v[2 * m][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, r);
  }
  // The same with zeros for the keys whose bit is not set.  (`pick` is the permutation of even columns: an opaque value, so that a loop
  // around this does not hold every column's operand in registers.)
  __device__ __forceinline__ bf16x8 frag(int j, unsigned int keys, unsigned int pick) const {
    u32x4 r;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      r[m] = __builtin_amdgcn_perm(v[2 * m + 1][j / 2], v[2 * m][j / 2], j % 2 ? pick + 0x02020202u : pick);
      r[m] &= (keys >> (2 * m) & 1 ? 0xffffu : 0u) | (keys >> (2 * m + 1) & 1 ? 0xffff0000u : 0u);
    }
    return __builtin_bit_cast(bf16x8, r);
  }
  // is any of them infinite or NaN?
  __device__ __forceinline__ bool odd() const {
    bool found = false;
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int w = 0; w < WORDS; ++w) found |= (v[k][w] & 0x7f80u) == 0x7f80u || (v[k][w] & 0x7f800000u) == 0x7f800000u;
    return found;
  }
};

// ------------------------------------------------------------------------------------------------ one piece
// ONE: a single new token a sequence, so that every position within the length is seen by every query.
// WIDE: the queries are fp32, and meet the keys as two bf16 numbers.
template <int D, int FORMAT, int RT, bool ONE, bool ONCE, bool WIDE>
__global__ void __launch_bounds__(64 * WAVES, RT == 1 && ONE ? 3 : 2)
    cached_attention_kernel(const void *Q, smoe_cache c, smoe_places p, Dims d, bf16_t *O, float *LSE, float *ws) {
  constexpr int KS = D / 32, COLS = D / 16, ROW = D + 4;     // padded: a wavefront's 16 rows start in 16 different banks
  // The queries' fragments: in registers, or, two tiles of them or two numbers each, in LDS, until the piece ends (held in registers they
  // spilled, and a reload in the loop waits for every request under way: two sequences of 90001 and 131072 positions in e4m3 133 us).
  // Two tiles of heads of 128 still take all 256 registers and spill some, 15 in bf16 and 4 in e4m3 (7 with fp32 queries): stored before, and
  // reloaded in and behind, the loop of the last steps, where not every query sees every key; the loop of the others has no access to scratch.
  constexpr bool SHARED = RT > 1 || WIDE;
  constexpr int FRAGS = RT * KS * (WIDE ? 2 : 1);
  union Shared {
    float acc[WAVES][RT * 16][ROW];
    bf16x8 q[SHARED ? FRAGS : 1][64];
  };
  __shared__ __attribute__((aligned(16))) char s_mem[sizeof(Shared)];
  Shared &shared = *reinterpret_cast<Shared *>(s_mem);
  auto &s_acc = shared.acc;
  auto &s_q = shared.q;
  __shared__ float s_m[WAVES][RT * 16], s_l[WAVES][RT * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  Place at;
  if (d.whole) {              // no sequence can be long enough to be cut: a block for each unit
    at.b = (int)blockIdx.x / d.units;
    at.len = length_of(p.lens, at.b, d.cap);
    at.n = 1;
    at.local = (int)blockIdx.x - at.b * d.units;
    at.slot = 0;
  } else if (!find_piece<false>(p.lens, p.sequences, d, (int)blockIdx.x, lane, at)) {
    return;                   // the grid is an upper bound
  }
  // everything of the piece is wave-uniform, and is told so: the windows below live in scalar registers
  const int pieces = uniform(at.n), len = uniform(at.len), b = uniform(at.b);
  const int unit = uniform(at.local / pieces), piece = uniform(at.local) - unit * pieces;
  const int tile = uniform(unit / c.h), hh = unit - tile * c.h;
  const int all_steps = steps_of(len), long_ = uniform((all_steps + pieces - 1) / pieces);
  const int step0 = piece * long_, step1 = min(step0 + long_, all_steps);

  // the lane's query of each 16, and the first position it does not see
  const int row0 = tile * RT * 16, rows = min(RT * 16, d.R - row0);
  int seen[RT], token[RT];
  bf16x8 q[RT][KS], q_low[WIDE ? RT : 1][KS];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row0 + min(t * 16 + col, rows - 1);
    token[t] = r / d.G;
    seen[t] = len - d.N + token[t] + 1;
    const size_t src = (((size_t)b * d.R + r) * c.h + hh) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (SHARED && (t * KS + ks) % WAVES != wave) continue;       // a wavefront's share of them
      const size_t e = src + Keys<D, FORMAT>::query_offset(ks, lane);
      if constexpr (WIDE) {
        const f32x4 *x = reinterpret_cast<const f32x4 *>((const float *)Q + e);
        const f32x4 lo = x[0], hi = x[1];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = i < 4 ? lo[i] : hi[i - 4];
          const float up = upper_part(y);
          q[t][ks][i] = (bf16_t)up;
          q_low[t][ks][i] = (bf16_t)(y - up);
        }
      } else {
        q[t][ks] = *reinterpret_cast<const bf16x8 *>((const bf16_t *)Q + e);
      }
    }
  }
  const int token0 = row0 / d.G, token1 = (row0 + rows - 1) / d.G;
  const int all_see = len - d.N + token0 + 1;               // every query of the tile sees the keys before this one

  constexpr float LOG2E = 1.4426950408889634f;
  const float scale = LOG2E / sqrtf((float)D);
  f32x4 acc[RT][COLS];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int j = 0; j < COLS; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  constexpr int BYTES = FORMAT == SMOE_CACHE_BF16 ? D * 2 : D;
  const int32_t *table = p.block_table + (size_t)b * p.width;
  // The wavefront's next 64 page numbers, one a lane: two for each of its steps from the `from`-th on.
  int ids = -1;
  auto fetch_pages = [&](int from) {
    const int key = (step0 + wave + (from + (lane >> 1)) * WAVES) * STEP + 16 * (lane & 1);
    ids = (unsigned)key < (unsigned)d.cap ? table[key >> d.shift] : -1;    // whatever the length: it may still be on its way
    ids = here(ids);      // waited for at this place, not where a number is used in the loop
  };
  auto group_of = [&](int step, int t, int id) {
    const int key = step * STEP + 16 * t;
    Group x;
    x.exists = (unsigned)id < (unsigned)c.pages && step < step1 && key < len;
    const size_t row = ((size_t)(x.exists ? id : 0) * c.h + hh) * c.page + (key & (c.page - 1));
    x.left = x.exists ? min(len - key, 16) : 0;
    x.K = (const char *)c.K + row * BYTES;
    x.V = (const char *)c.V + row * BYTES;
    x.K_exp = c.K_exp + row;
    x.V_exp = c.V_exp + row;
    return x;
  };
  // The keys of the next step are requested when this one's have met the queries, its values when this one's have met the weights: a
  // wavefront always has requests of 8 to 16 KB under way in bf16 and heads of 128, half of it in e4m3, and half of either in heads of 64.
  Keys<D, FORMAT> k;
  Values<D, FORMAT> v;
  const int k_at = Keys<D, FORMAT>::lane_offset(lane), v_at = Values<D, FORMAT>::lane_offset(lane);
  int s = step0 + wave;
  fetch_pages(0);
  Group now[2] = {group_of(s, 0, at_lane(ids, 0)), group_of(s, 1, at_lane(ids, 1))};
#pragma unroll
  for (int t = 0; t < 2; ++t) k.template load<ONCE>(t, now[t], k_at, lane);
#pragma unroll
  for (int t = 0; t < 2; ++t) v.template load<ONCE>(t, now[t], v_at, lane);
  if (SHARED) {
#pragma unroll
    for (int f = 0; f < RT * KS; ++f)
      if (f % WAVES == wave) {
        s_q[f][lane] = q[f / KS][f % KS];
        if constexpr (WIDE) s_q[RT * KS + f][lane] = q_low[f / KS][f % KS];
      }
    __syncthreads();
  }
  int i = 1;                // which of the wavefront's steps is next
  // TAIL: not every query sees every key of the step.
  auto take_step = [&](auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    const int key0 = s * STEP, q_at = here(lane);
    if ((i & 31) == 0) fetch_pages(i);
    const Group next[2] = {group_of(s + WAVES, 0, at_lane(ids, 2 * (i & 31))), group_of(s + WAVES, 1, at_lane(ids, 2 * (i & 31) + 1))};
    ++i;
    f32x4 sc[RT][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int t = 0; t < RT; ++t) sc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 f = k.frag(i, ks);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          sc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, SHARED ? s_q[t * KS + ks][q_at] : q[t][ks], sc[t][i], 0, 0, 0);
          if constexpr (WIDE) sc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, s_q[RT * KS + t * KS + ks][q_at], sc[t][i], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) k.template load<ONCE>(t, next[t], k_at, lane);
    // The weights as two bf16 numbers, the second what the first's rounding left: the products then carry 16 bits of them, and the output's own
    // rounding is the only one (error against 64 bits 2.1e-3 -> 1.7e-3).  The matrix cores have the time: only where 32 rows share a read does it
    // show (two sequences of 90001 and 131072 positions in e4m3, 24 rows: 82.3 -> 85.5 us; 64 ragged ones of 4 rows 31.1 both).
    bf16x8 pb[RT], pl[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x4 (&x)[2] = sc[t];
      if (TAIL || !now[0].exists || !now[1].exists) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((TAIL && key0 + 16 * i + 4 * g + e >= seen[t]) || !now[i].exists) x[i][e] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
      mx = max_of_query(mx);
      const float m_new = fmaxf(m[t], mx), base = m_new == -INFINITY ? 0.f : m_new;   // no inf - inf while nothing was seen
      const float alpha = __builtin_amdgcn_exp2f((m[t] - base) * scale);
      m[t] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = __builtin_amdgcn_exp2f((x[i][e] - base) * scale);   // the difference first: huge scores cancel exactly
          sum += w;
          const float up = upper_part(w);
          pb[t][4 * i + e] = (bf16_t)up;
          pl[t][4 * i + e] = (bf16_t)(w - up);
        }
      l[t] = l[t] * alpha + sum;
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int j = 0; j < COLS; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][j][e] *= alpha;
      }
    }
    const int left[2] = {now[0].left, now[1].left};
    const Columns<D> y(v, left, g);
    if (!ONE && TAIL && __any(y.odd())) {
      // Infinite or NaN values at positions that some queries see and others do not: a weight of zero would not keep them out, so each
      // token's queries take their own product, over the values that the token sees.
#pragma unroll 1
      for (int n = token0; n <= token1; ++n) {
        const int sees = len - d.N + n + 1;
        unsigned int keys = 0;
        const unsigned int pick = (unsigned int)here(0x05040100);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) keys |= key0 + 16 * (kk >> 2) + 4 * g + (kk & 3) < sees ? 1u << kk : 0u;
#pragma unroll
        for (int j = 0; j < COLS; ++j)
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const bf16x8 f = y.frag(j, keys, pick);
            f32x4 with = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pb[t], acc[t][j], 0, 0, 0);
            with = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pl[t], with, 0, 0, 0);
            if (token[t] == n) acc[t][j] = with;
          }
      }
    } else {
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const bf16x8 f = y.frag(j);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pb[t], acc[t][j], 0, 0, 0);
          acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pl[t], acc[t][j], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      v.template load<ONCE>(t, next[t], v_at, lane);
      now[t] = next[t];
    }
    s += WAVES;
  };
#pragma unroll 1
  while (s < step1 && (s + 1) * STEP <= all_see) take_step(std::false_type{});
#pragma unroll 1
  while (s < step1) take_step(std::true_type{});

  if (SHARED) __syncthreads();                // the queries are done with
  // The wavefronts' parts meet in LDS.  A lane holds columns 4 COLS g + COLS e + j of its query, j and e running.
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float sum = l[t];
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (t * 16 + col < rows) {
      float *dst = s_acc[wave][t * 16 + col] + 4 * COLS * g;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < COLS; j += 4) *reinterpret_cast<f32x4 *>(dst + e * COLS + j) = f32x4{acc[t][j][e], acc[t][j + 1][e], acc[t][j + 2][e], acc[t][j + 3][e]};
      if (g == 0) {
        s_m[wave][t * 16 + col] = m[t];
        s_l[wave][t * 16 + col] = sum;
      }
    }
  }
  __syncthreads();
  float *out = ws + (size_t)uniform(at.slot + at.local) * slot_floats(d.rows, D);
  for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * WAVES) {
    const int r = i / (D / 4), x = (i - r * (D / 4)) * 4;
    float top = s_m[0][r];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w][r]);
    const float base = top == -INFINITY ? 0.f : top;
    f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f((s_m[w][r] - base) * scale);
      total = fmaf(s_l[w][r], f, total);
      const f32x4 y = *reinterpret_cast<const f32x4 *>(&s_acc[w][r][x]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(y[e], f, sum[e]);
    }
    if (pieces == 1) {
      // nothing attended: zeros, also where weights of zero met infinite values and the sums are NaN
      const float inv = 1.f / total;
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(total == 0.f ? 0.f : sum[e] * inv);
      const size_t row = ((size_t)b * d.R + row0 + r) * c.h + hh;
      *reinterpret_cast<bf16x4 *>(O + row * D + x) = o;
      if (x == 0) LSE[row] = total == 0.f ? -INFINITY : fmaf(top, scale, __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
    } else {
      *reinterpret_cast<f32x4 *>(out + (size_t)r * D + x) = sum;
      if (x == 0) {
        out[(size_t)d.rows * D + r] = top;
        out[(size_t)d.rows * (D + 1) + r] = total;
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ the join
// A block takes some rows of a cut unit, D / 4 lanes a row, or several such groups, which take its pieces in turn and meet in LDS in a
// fixed order: one row a block where few units are cut, into many pieces, and more of them where the units fill the chip.
// A thousand lanes a block only where there are hardly any blocks: one sequence of 131072 positions, one head, 8 rows 21.0 us (22.5 with 256);
// one of 4096 with 4 heads of 4 rows 12.5 (11.6).
constexpr int JOIN_AHEAD = 8, JOIN_FEW = 8;
template <int D, int JOIN_THREADS> __global__ void __launch_bounds__(JOIN_THREADS)
    cached_attention_join_kernel(smoe_places p, Dims d, int h, int rows_log2, const float *ws, bf16_t *O, float *LSE) {
  constexpr int LANES = D / 4, GROUPS = JOIN_THREADS / LANES;
  __shared__ __attribute__((aligned(16))) float s_acc[GROUPS][D + 4];
  __shared__ float s_m[GROUPS], s_l[GROUPS];
  const int lane = threadIdx.x & 63;
  Place at;
  if (!find_piece<true>(p.lens, p.sequences, d, (int)blockIdx.x, lane, at)) return;
  const int unit = at.local, tile = unit / h, hh = unit - tile * h;
  const int each = GROUPS >> rows_log2;                     // groups of a row
  const int group = threadIdx.x / LANES, x = (threadIdx.x % LANES) * 4;
  const int r = ((int)blockIdx.y << rows_log2) + group / each, sub = group & (each - 1);
  const bool mine = r < d.rows && tile * d.rows + r < d.R;
  const float scale = 1.4426950408889634f / sqrtf((float)D);
  const size_t stride = slot_floats(d.rows, D);
  const float *base = ws + (size_t)(at.slot + unit * at.n) * stride;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if (mine) {
#pragma unroll 1
    for (int i0 = sub; i0 < at.n; i0 += each * JOIN_AHEAD) {
      float pm[JOIN_AHEAD], pl[JOIN_AHEAD];
      f32x4 y[JOIN_AHEAD];
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; ++u) {
        const int i = i0 + u * each;
        if (i < at.n) {
          const float *src = base + (size_t)i * stride;
          pm[u] = src[(size_t)d.rows * D + r];
          pl[u] = src[(size_t)d.rows * (D + 1) + r];
          y[u] = *reinterpret_cast<const f32x4 *>(src + (size_t)r * D + x);
        }
      }
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; ++u) {
        if (i0 + u * each >= at.n) break;
        const float top = fmaxf(m, pm[u]), safe = top == -INFINITY ? 0.f : top;
        const float old = __builtin_amdgcn_exp2f((m - safe) * scale), now = __builtin_amdgcn_exp2f((pm[u] - safe) * scale);
        m = top;
        l = fmaf(l, old, pl[u] * now);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(acc[e], old, y[u][e] * now);
      }
    }
  }
  *reinterpret_cast<f32x4 *>(&s_acc[group][x]) = acc;
  if (x == 0) {
    s_m[group] = m;
    s_l[group] = l;
  }
  __syncthreads();
  if (!mine || sub != 0) return;
  float top = m;
  for (int w = 1; w < each; ++w) top = fmaxf(top, s_m[group + w]);
  const float safe = top == -INFINITY ? 0.f : top;
  f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
  for (int w = 0; w < each; ++w) {
    const float f = __builtin_amdgcn_exp2f((s_m[group + w] - safe) * scale);
    total = fmaf(s_l[group + w], f, total);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(s_acc[group + w][x + e], f, sum[e]);
  }
  const float inv = 1.f / total;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(total == 0.f ? 0.f : sum[e] * inv);      // nothing attended: zeros, also where the sums are NaN
  const size_t row = ((size_t)at.b * d.R + tile * d.rows + r) * h + hh;
  *reinterpret_cast<bf16x4 *>(O + row * D + x) = o;
  if (x == 0) LSE[row] = total == 0.f ? -INFINITY : fmaf(top, scale, __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// Query rows that share a read of the cache: 16, or 32 where there are more.
int row_tiles(int R) { return R > 16 ? 2 : 1; }

}  // namespace

constexpr size_t MAX_SLOTS = 2 * MAX_TARGET;
bool cached_attention_fits(int B, int N, int G, int h) {
  // query rows within 31 bits, and one-dimensional grids of fewer than 2^32 threads
  const long long R = (long long)N * G;
  if (R > 0x7fffffffLL || B * (double)R * h > 0x7fffffff) return false;
  const long long rows = 16 * row_tiles((int)R);
  return (R + rows - 1) / rows * h * B <= 0x7fffffffLL / 256 - 2 * MAX_TARGET;
}

size_t cached_attention_workspace_bytes(int N, int G, int d_head, int positions) {
  if (positions <= WHOLE_STEPS * STEP) return 0;           // nothing is cut
  const int R = N * G;
  return align256(MAX_SLOTS * slot_floats(std::min(R, 16 * row_tiles(R)), d_head) * sizeof(float));
}

int launch_cached_attention(hipStream_t s, const void *Q, bool wide, int N, int G, const smoe_cache &c, const smoe_places &p, void *O, float *LSE, void *ws) {
  Dims d;
  d.N = N;
  d.G = G;
  d.R = N * G;
  const int rt = row_tiles(d.R);
  d.tiles = ceil_div(d.R, 16 * rt);
  d.rows = std::min(d.R, 16 * rt);
  d.shift = __builtin_ctz((unsigned int)c.page);
  d.cap = p.width * c.page;
  const long long units = (long long)d.tiles * c.h, all = units * p.sequences;
  d.units = (int)units;
  d.target = rt == 1 && N == 1 ? T_ONE : rt == 1 ? T_MULTI : T_TWO;
  d.whole = d.cap <= WHOLE_STEPS * STEP;
  // pieces at most: a sequence's are ceil(steps / per) <= 1 + steps / per, and at most its share of the table's positions; without cuts a
  // block numbers its unit directly, so the grid is exact
  const long long most = d.whole ? all : std::min<long long>(all + d.target, all * ceil_div(ceil_div(d.cap, STEP), MIN_STEPS));
  auto go = [&](auto kernel, auto join, auto join_few) {
    kernel<<<(unsigned int)most, 64 * WAVES, 0, s>>>(Q, c, p, d, (bf16_t *)O, LSE, (float *)ws);
    if (hipGetLastError() != hipSuccess) return SMOE_ERR_HIP;
    if (d.whole) return SMOE_OK;
    const long long cut = std::min<long long>(all, d.target);                  // units, at most
    const bool few = cut * d.rows <= JOIN_FEW;
    int rows_log2 = 0;
    while ((2 << rows_log2) <= 256 * 4 / c.d_head && (1 << rows_log2) < d.rows && cut * ceil_div(d.rows, 2 << rows_log2) >= 512) ++rows_log2;
    const dim3 grid((unsigned int)cut, ceil_div(d.rows, 1 << rows_log2));
    if (few) join_few<<<grid, 1024, 0, s>>>(p, d, c.h, rows_log2, (const float *)ws, (bf16_t *)O, LSE);
    else join<<<grid, 256, 0, s>>>(p, d, c.h, rows_log2, (const float *)ws, (bf16_t *)O, LSE);
    return hipGetLastError() == hipSuccess ? SMOE_OK : SMOE_ERR_HIP;
  };
  auto by_rows = [&](auto d_c, auto f_c, auto once_c, auto wide_c) {
    constexpr int D = decltype(d_c)::value, F = decltype(f_c)::value;
    constexpr bool ONCE = decltype(once_c)::value, WIDE = decltype(wide_c)::value;
    auto join = cached_attention_join_kernel<D, 256>, join_few = cached_attention_join_kernel<D, 1024>;
    return rt > 1   ? go(cached_attention_kernel<D, F, 2, false, ONCE, WIDE>, join, join_few)
           : N > 1 ? go(cached_attention_kernel<D, F, 1, false, ONCE, WIDE>, join, join_few)
                   : go(cached_attention_kernel<D, F, 1, true, ONCE, WIDE>, join, join_few);
  };
  auto by_wide = [&](auto d_c, auto f_c, auto once_c) { return wide ? by_rows(d_c, f_c, once_c, std::true_type{}) : by_rows(d_c, f_c, once_c, std::false_type{}); };
  // Where one tile holds all rows a key is read by one block, and the next call reads another layer's: past the caches, then, unless the
  // cache is so small that several layers' stay in the last-level cache (256 MB) from one token to the next.  64 sequences of up to 8192
  // positions, 135 MB, read in turn with four more such caches: 33.0 us past the caches, 36.4 through them; 64 of 100 to 8192, 240 MB, 51.2 /
  // 55.9; one of 4096, 17 MB, 11.6 / 11.8 in turn with 35 more, but 15.0 / 13.3 where all stay; one of 301 7.3 / 6.5.
  const size_t held = (size_t)std::min<long long>(c.pages, (long long)p.sequences * p.width) * c.page * c.h * c.d_head * (c.format == SMOE_CACHE_BF16 ? 4 : 2);
  const bool once = d.tiles == 1 && held > LAST_LEVEL_CACHE / 4;
  auto by_once = [&](auto d_c, auto f_c) { return once ? by_wide(d_c, f_c, std::true_type{}) : by_wide(d_c, f_c, std::false_type{}); };
  auto by_format = [&](auto d_c) {
    return c.format == SMOE_CACHE_BF16 ? by_once(d_c, std::integral_constant<int, SMOE_CACHE_BF16>{}) : by_once(d_c, std::integral_constant<int, SMOE_CACHE_E4M3>{});
  };
  return c.d_head == 128 ? by_format(std::integral_constant<int, 128>{}) : by_format(std::integral_constant<int, 64>{});
}
