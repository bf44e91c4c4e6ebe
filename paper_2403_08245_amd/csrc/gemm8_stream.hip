// The products in 8 bits for many rows: persistent blocks, one per compute unit, four wavefronts 2 x 2 over a 256 x 256 (or 128 x 256) tile,
// v_mfma_scale_f32_32x32x64_f8f6f4 with the weights as the first operand, so that a lane holds four consecutive columns of a row.
// Bound: the matrix cores at twice the rate of bf16; an instruction reads as many bytes of operands in as many cycles, so the loop is the
// one of the bf16 kernels (gemm_stream.hip) with stages of 128 elements instead of 64: the same 128 bytes a row.
// 8192 x 8192 x 8192: 485 us, 2.27 PFLOP/s, 0.93 of the library's product of the same box; the matrix cores are busy for 0.77 of the cycles.  Of the rest 4 % are the
// rows' powers of two (gathered, four bytes a row and stage), 6 % misses of L2, by timing copies of the loop without the one or with rows that
// stay there; with no loads in the loop at all it takes 413 us.
//
// A stage is 128 elements of the contraction.  Rows come as whole 128-byte lines, 16-byte chunks permuted by the row; weights lie in memory as
// they are read from LDS (smoe_weights8), 2 KB for 16 columns; both go to LDS directly, and so do the powers of two: four bytes for a row or column and
// stage.  Two slots.  The first half of a stage multiplies what is in registers and reads the second half's operands; then the slot is
// free, and the second half issues the loads of the stage after next, waits for the next stage and reads its first half.
// The loader walks the block's list of tiles ahead of the multiplying side, so a tile's first stages land while the one before it is written out.
//
// Operands of an instruction: lane (r, h) = (lane % 32, lane / 32) holds elements 16 h .. 16 h + 15 and 32 + 16 h .. of row or column r, and the power
// of two of its elements 32 h .. 32 h + 31.
#include "block.h"
#include "gemm_epilogue.h"
#include <type_traits>

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int B8_BYTES = TB * ROW8;                     // weights of a stage, 256 columns
constexpr int MAX_E8 = 256;

template <int FM_, bool ONCE_ = false> struct Shape8 {
  static constexpr int FM = FM_;                        // 32-row fragments per wavefront
  static constexpr bool ONCE = ONCE_;                   // weights that no further tile reads pass the caches
  static constexpr int TM = FM * 64;                    // tile rows; columns are TB = 256
  static constexpr int A_BYTES = TM * ROW8;
  static constexpr int NLA = A_BYTES / 4096, NLB = B8_BYTES / 4096;   // load instructions per wavefront and stage
  static constexpr int NL = NLA + NLB + 2;              // and the powers of two of the rows and the columns
  // LDS: rows of two slots, weights of two, then powers of two of rows and columns, then each wavefront's patch
  static constexpr int OFF_B = 2 * A_BYTES, OFF_EA = OFF_B + 2 * B8_BYTES, OFF_EB = OFF_EA + 2 * TM * 4, OFF_PATCH = OFF_EB + 2 * TB * 4;
  static constexpr int LDS_BYTES = OFF_PATCH + 4 * EPI_WAVE_BYTES;
};
using Big8 = Shape8<4>;
using Half8 = Shape8<2>;
using Half8Once = Shape8<2, true>;

enum { OUT_BF16, OUT_F16, OUT_SWIGLU, OUT_GELU, OUT_BF16_REST };
// store instructions that a wavefront issues per tile
template <int FM, int OUT> constexpr int Stores8 = FM * (OUT == OUT_BF16 ? 8 : OUT == OUT_BF16_REST ? 10 : OUT == OUT_F16 ? 9 : OUT == OUT_SWIGLU ? 3 : 5);

// first[e] = M-tiles of the experts before e, by every wavefront for itself (all write the same); returns first[E]
template <int TM> __device__ __forceinline__ int number_tiles8(const int32_t *offsets, int E, int *first, int lane) {
  int base = 0;
  if (lane == 0) first[0] = 0;
  for (int c0 = 0; c0 < E; c0 += 64) {
    const int x = c0 + lane;
    int n = x < E ? (offsets[x + 1] - offsets[x] + TM - 1) / TM : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(n, d, 64);
      if (lane >= d) n += up;
    }
    if (x < E) first[x + 1] = base + n;
    base += __builtin_amdgcn_readlane(n, 63);
  }
  return base;
}
template <int TM>
__device__ __forceinline__ void find_tile8(const int32_t *offsets, const int *first, int E, int tile, int lane, int &e, int &row0, int &row_end) {
  e = E - 1;
  for (int c0 = 0; c0 < E; c0 += 64) {
    const unsigned long long owns = __ballot(first[min(c0 + lane, E - 1) + 1] > tile);
    if (!owns) continue;
    e = c0 + __ffsll((long long)owns) - 1;
    break;
  }
  row0 = __builtin_amdgcn_readfirstlane(offsets[e]) + (tile - __builtin_amdgcn_readfirstlane(first[e])) * TM;
  row_end = __builtin_amdgcn_readfirstlane(offsets[e + 1]);
}

// Sources of the loader's current tile: range-checked windows and per-lane byte offsets at step 0.
template <typename S> struct Loader8 {
  int32x4 win_a, win_ea, win_b, win_eb;
  uint32_t oa[S::NLA], oea, ob, oeb;
  uint32_t group_bytes;              // of a group of 16 columns: steps * 2048
  uint32_t row_step, group_step, row_exps_step, group_exps_step;      // bytes a source moves per stage
  int step, uwave;
  int again;                         // S::ONCE: above 0 where the expert has further tiles
  __device__ __forceinline__ void load(int I, uint32_t lds0, int slot) const {
    if (I < S::NLA) {
      load16_to_lds_checked(win_a, oa[I] + (uint32_t)step * row_step, lds0 + slot * S::A_BYTES + uwave * (S::NLA * 1024), I * 1024);
    } else if (I < S::NLA + S::NLB) {
      const int J = I - S::NLA;
      const uint32_t off = ob + ((uint32_t)(J >> 1) * group_bytes + (uint32_t)step * group_step + (uint32_t)(J & 1) * 1024u);
      const uint32_t lds = lds0 + S::OFF_B + slot * B8_BYTES + uwave * (S::NLB * 1024);
      if (S::ONCE) load16_to_lds_checked_or_once(win_b, off, lds + J * 1024, again);
      else load16_to_lds_checked(win_b, off, lds, J * 1024);
    } else if (I == S::NLA + S::NLB) {
      load4_to_lds_checked(win_ea, oea + (uint32_t)step * row_exps_step, lds0 + S::OFF_EA + slot * (S::TM * 4) + (uwave & (S::TM / 64 - 1)) * 256);
    } else {
      load4_to_lds_checked(win_eb, oeb + (uint32_t)step * group_exps_step, lds0 + S::OFF_EB + slot * (TB * 4) + uwave * 256);
    }
  }
};

// a wavefront's operands of 64 elements
template <int FM> struct Frags8 {
  i32x8 a[FM], b[FR];
};
template <int FM> struct Exps8 {
  int a[FM], b[FR];
};
// Where the lane reads in a slot.
struct Reader8 {
  uint32_t fa[4], fb;                // chunk kk of the rows' fragments; of the columns': further chunks lie 512 bytes on
  uint32_t ea, eb;
  int shift;                         // of the power of two in its four bytes
  // part `i` of half s: fragment b0 a0 b1 b2 b3 a1 .., 16 bytes of each, twice
  template <typename S> __device__ __forceinline__ void read(Frags8<S::FM> &f, int i, const char *smem, int slot, int s) const {
    const int frag = i >> 1, t = i & 1, kk = 2 * s + t;
    const char *a = smem + slot * S::A_BYTES, *b = smem + S::OFF_B + slot * B8_BYTES;
    const bool rows = frag == 1 || frag > FR;
    const int n = frag == 0 ? 0 : frag == 1 ? 0 : frag <= FR ? frag - 1 : frag - FR;
    const i32x4 v = rows ? *reinterpret_cast<const i32x4 *>(a + fa[kk] + n * 4096) : *reinterpret_cast<const i32x4 *>(b + fb + kk * 512 + n * 4096);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (rows) f.a[n][4 * t + q] = v[q];
      else f.b[n][4 * t + q] = v[q];
    }
  }
  template <typename S> __device__ __forceinline__ void read_exps(Exps8<S::FM> &x, const char *smem, int slot) const {
#pragma unroll
    for (int n = 0; n < S::FM; ++n) x.a[n] = *reinterpret_cast<const int *>(smem + S::OFF_EA + slot * (S::TM * 4) + ea + n * 128);
#pragma unroll
    for (int n = 0; n < FR; ++n) x.b[n] = *reinterpret_cast<const int *>(smem + S::OFF_EB + slot * (TB * 4) + eb + n * 128);
  }
  template <int FM> __device__ __forceinline__ void shift_exps(Exps8<FM> &x) const {
#pragma unroll
    for (int n = 0; n < FM; ++n) x.a[n] = (int)((unsigned)x.a[n] >> shift);
#pragma unroll
    for (int n = 0; n < FR; ++n) x.b[n] = (int)((unsigned)x.b[n] >> shift);
  }
};

// The products of one half of a stage; behind(i) issues what goes behind product i.  LDS reads and loads are spread one or two behind a product: in
// bursts they queue up in front of the next product.
template <bool FIRST, int HALF_, int FM, typename Behind>
__device__ __forceinline__ void multiply8(const Frags8<FM> &f, const Exps8<FM> &x, f32x16 (&acc)[FM][FR], Behind behind) {
  f32x16 zero;
#pragma unroll
  for (int q = 0; q < 16; ++q) zero[q] = 0.f;
  sched_fence();
#pragma unroll
  for (int m = 0; m < FM; ++m) {
#pragma unroll
    for (int n = 0; n < FR; ++n) {
      acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.b[n], f.a[m], FIRST ? zero : acc[m][n], 0, 0, 2 * HALF_, x.b[n], 2 * HALF_, x.a[m]);
      sched_fence();
      behind(m * FR + n);
      sched_fence();
    }
  }
}
// part `i` of n things spread over the products from .. to: does it go behind product p?
__device__ constexpr bool goes_behind(int i, int n, int p, int from, int to) {
  const int at = from + i * (to - from) / n;
  return at == p;
}

// One stage in slot `cur`, the next in `nxt`.  f[0] holds the columns and the first rows of its first half, x its powers of two on entry, and the next
// stage's on exit.
// STORES: at least that many stores were issued after the next stage's loads.
template <bool FIRST, int STORES, typename S, typename Slot, typename Next>
__device__ __forceinline__ void stage8(const Loader8<S> &ld, const Reader8 &rd, Frags8<S::FM> (&f)[2], Exps8<S::FM> &x, f32x16 (&acc)[S::FM][FR], const char *smem,
                                       uint32_t lds0, Slot cur, Next nxt) {
  constexpr int FM = S::FM, P = FM * FR, PARTS = 2 * (FM + FR), HEAD = 2 * (FR + 1);
  // Products 0 .. P - 1 are the first half's, P .. 2 P - 1 the second's.  The first half's further rows are read by TAIL (they are needed from product 4 on),
  // the second half by FREE, behind which the slot is free; loads go behind the products to LOADED; the next stage is waited for behind
  // LANDED.  8192 x 8192 x 8192, us, by FREE, LOADED, LANDED (of 16 + 16): 12, 29, 24 485; 11, 32, 26 488; 13, 28, 28 490; 15, 30, 22 496; 16, 28, 26 500 to 508.
  constexpr int TAIL = P == 16 ? 3 : 2, FREE = P * 3 / 4, LOADED = P + P * 13 / 16, LANDED = P + P / 2;
  auto load_at = [](int i) { return FREE + i * (LOADED - FREE) / S::NL; };
  constexpr int EARLY = [] { int n = 0; for (int i = 0; i < S::NL; ++i) n += FREE + i * (LOADED - FREE) / S::NL <= LANDED; return n; }();
  auto loads = [&](int p) {
#pragma unroll
    for (int i = 0; i < S::NL; ++i)
      if (load_at(i) == p) ld.load(i, lds0, (int)cur);
  };
  multiply8<FIRST, 0>(f[0], x, acc, [&](int p) {
#pragma unroll
    for (int i = HEAD; i < PARTS; ++i)
      if (goes_behind(i - HEAD, PARTS - HEAD, p, 0, TAIL)) rd.template read<S>(f[0], i, smem, (int)cur, 0);
#pragma unroll
    for (int i = 0; i < PARTS; ++i)
      if (goes_behind(i, PARTS, p, TAIL, FREE)) rd.template read<S>(f[1], i, smem, (int)cur, 1);
    if (p == FREE) __syncthreads();      // every wavefront holds the stage: its slot is free
    loads(p);
  });
  Exps8<FM> y;
  multiply8<false, 1>(f[1], x, acc, [&](int p) {
    loads(P + p);
    if (P + p == LANDED) {
      wait_loads<(EARLY + STORES < 63 ? EARLY + STORES : 63)>();
      __syncthreads();
      rd.template read_exps<S>(y, smem, (int)nxt);
    }
#pragma unroll
    for (int i = 0; i < HEAD; ++i)
      if (goes_behind(i, HEAD, P + p, LANDED, 2 * P)) rd.template read<S>(f[0], i, smem, (int)nxt, 0);
  });
  rd.shift_exps(y);
  x = y;
}

// The rows of a weighted sum: fp16 with a power of two for the wavefront's 128 columns of a row, as many bytes as bf16 and three bits more, so that the
// sum carries little but its own rounding (16384 tokens, 8 experts, 4096 -> 2 x 14336: error against 64 bits 2.7e-3 with bf16 rows,
// 2.1e-3 so; the plain form's 1.7e-3).  Where the largest values of all 32 rows lie in [2^-6, 2^15) (or are 0) they are stored as they are, good
// to 2^-11 of a value and 2^-19 of the largest; else times the power of two that brings the largest into [2^14, 2^15).
// exps: 141 for values as they are, else the largest's exponent, biased by 127 (15 .. 254; infinite and NaN rows take the largest finite value's).
template <int FM, typename DestFn, typename ExpFn>
__device__ __forceinline__ void store_wave_tile_f16(const f32x16 (&acc)[FM][FR], char *patch, DestFn dest, ExpFn put_exp, int lane) {
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  acc_settle();
  RowStore<decltype(dest(0, 0))> pend;
#pragma unroll
  for (int fm = 0; fm < FM; ++fm) {
    sched_fence();
    float v[FR][16], most = 0.f;
#pragma unroll
    for (int fn = 0; fn < FR; ++fn)
#pragma unroll
      for (int i = 0; i < 16; ++i) v[fn][i] = acc_read(acc[fm][fn][i]);
#pragma unroll
    for (int fn = 0; fn < FR; ++fn)
#pragma unroll
      for (int i = 0; i < 16; i += 2) most = fmaxf(most, fmaxf(fabsf(v[fn][i]), fabsf(v[fn][i + 1])));
    most = fmaxf(most, __shfl_xor(most, 32, 64));
    unsigned int e = 141u;
    if (__any(most != 0.f && !(most >= 0x1p-6f && most < 0x1p15f))) {
      if (__any(most == INFINITY)) {
        most = 0.f;
#pragma unroll
        for (int fn = 0; fn < FR; ++fn)
#pragma unroll
          for (int i = 0; i < 16; ++i) most = fmaxf(most, finite_abs(v[fn][i]));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
      }
      e = max(__float_as_uint(most) >> 23, 15u);
      const float scale = __uint_as_float((268u - e) << 23);
#pragma unroll
      for (int fn = 0; fn < FR; ++fn)
#pragma unroll
        for (int i = 0; i < 16; ++i) v[fn][i] *= scale;
    }
    put_exp(fm, e);
#pragma unroll
    for (int half = 0; half < 2; ++half)
      pipe_block(pend, patch, lane, [&] {
#pragma unroll
        for (int f2 = 0; f2 < 2; ++f2)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float *x = &v[half * 2 + f2][g * 4];
            const f16x4 o = __builtin_convertvector(f32x4_t{x[0], x[1], x[2], x[3]}, f16x4);
            patch_put(patch, lane, f2, g, __builtin_bit_cast(bf16x4, o));
          }
      }, dest(fm, half));
  }
  sched_fence();
  issue_row_store(pend);
}

// The rows in bf16 of a weighted sum, and what rounding took from them (S2S8Args::rest): of 64 columns a lane has every other four, and with its neighbour's in
// the other half of the wavefront the 16 bytes of its row.
template <int FM, typename DestFn, typename RestFn>
__device__ __forceinline__ void store_wave_tile_rest(const f32x16 (&acc)[FM][FR], char *patch, DestFn dest, RestFn put_rest, int lane) {
  acc_settle();
  RowStore<decltype(dest(0, 0))> pend;
#pragma unroll
  for (int fm = 0; fm < FM; ++fm)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      unsigned int word[2];
      pipe_block(pend, patch, lane, [&] {
#pragma unroll
        for (int f2 = 0; f2 < 2; ++f2) {
          unsigned int bits = 0;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 v;
            unsigned int t[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float x = acc_read(acc[fm][half * 2 + f2][g * 4 + q]);
              v[q] = (bf16_t)x;
              t[q] = bf16_rest_at_14(x);
            }
            // bits 14 and 15 of each, four to a word, in front of those of the g before
            const unsigned int lo = __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0501u), hi = __builtin_amdgcn_perm(t[3], t[2], 0x05010c0cu);
            bits = ((lo | hi) & 0xc0c0c0c0u) | ((bits >> 2) & 0x3f3f3f3fu);
            patch_put(patch, lane, f2, g, v);
          }
          word[f2] = bits;
        }
      }, dest(fm, half));
      const unsigned int other[2] = {(unsigned int)__shfl_xor((int)word[0], 32, 64), (unsigned int)__shfl_xor((int)word[1], 32, 64)};
      put_rest(fm, half, i32x4{(int)word[0], (int)other[0], (int)word[1], (int)other[1]});
    }
  sched_fence();
  issue_row_store(pend);
}

// Sixteen values of a row's block of 32 (its other lane has the rest): their codes, four to a word, and the block's byte.
__device__ __forceinline__ unsigned int pack_block(float (&h)[16], unsigned int (&code)[4]) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(h[i]));       // NaN is passed over, and comes out of the conversion as NaN
  amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
  unsigned int byte = e4m3_byte(amax);
  if (__any(byte > 246u)) {                                            // infinities, and values next to fp32's end: as e4m3_scaled has them
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = fmaxf(amax, finite_abs(h[i]));
    amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
    byte = e4m3_byte(amax);
#pragma unroll
    for (int g = 0; g < 4; ++g) code[g] = e4m3_four(h[4 * g], h[4 * g + 1], h[4 * g + 2], h[4 * g + 3], byte);
    return byte;
  }
  const float inv = __uint_as_float((254u - byte) << 23);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(h[4 * g] * inv, h[4 * g + 1] * inv, 0, false);
    code[g] = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(h[4 * g + 2] * inv, h[4 * g + 3] * inv, lo, true);
  }
  return byte;
}

// EVEN: an even number of stages, so that every tile starts in slot 0 and slots are constants.
template <typename S, int OUT, bool SCATTER, bool EVEN>
__global__ void __launch_bounds__(NTHREADS, 1) s2s8_stream_kernel(S2S8Args a, int tiles_n, int group_m, uint32_t magic_a, uint32_t magic_sum) {
  constexpr bool HIDDEN = OUT == OUT_SWIGLU || OUT == OUT_GELU;
  constexpr int STORES = Stores8<S::FM, OUT>;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ int s_off[MAX_E8 + 1], s_first[MAX_E8 + 1];
  // order indices of the rows of up to four open tiles, and the tiles: the loader has opened tile n + 2 and requested the rows of n + 3 while
  // tile n is written out (a tile has two stages at least).
  __shared__ int s_idx[4][S::TM];
  __shared__ __attribute__((aligned(16))) int s_tile[4][4];

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int uwave = __builtin_amdgcn_readfirstlane(wave);
  const int uwm = uwave >> 1, uwn = uwave & 1;
  const int G = gridDim.x;
  const int pos = ((int)blockIdx.x & 7) * (G >> 3) + ((int)blockIdx.x >> 3);   // blocks b, b + 8, ... share an XCD and get consecutive tiles
  const int steps = (a.W.d_in + ROW8 - 1) / ROW8;
  const int ns = max(steps, 2);                         // a contraction of one stage has a second one of zeros
  for (int i = threadIdx.x; i <= a.W.E; i += NTHREADS) s_off[i] = a.offsets[i];
  __syncthreads();
  const int m_tiles = number_tiles8<S::TM>(s_off, a.W.E, s_first, lane);
  const long long total = (long long)m_tiles * tiles_n;
  const int tiles = (int)((total - pos + G - 1) / G);   // of this block: pos, pos + G, ..
  auto args = [&]() {                                   // read again where they are used, once a tile
    auto p = (const __attribute__((address_space(4))) S2S8Args *)__builtin_amdgcn_kernarg_segment_ptr();
    __asm__ volatile("" : "+s"(p));
    return p;
  };
  struct Tile {
    int seq;                        // position in this block's list (-1 before the first)
    int e, row0, row_end, n0;       // n0: first column, or hidden unit
  };
  auto next_tile = [&](Tile &t) -> bool {
    const int seq = t.seq + 1;
    if (seq >= tiles) return false;
    int mt, nt;
    tile_coords(seq * G + pos, m_tiles, tiles_n, group_m, mt, nt);
    t.seq = seq;
    find_tile8<S::TM>(s_off, s_first, args()->W.E, mt, lane, t.e, t.row0, t.row_end);
    t.n0 = nt * (OUT == OUT_SWIGLU ? TB / 2 : TB);
    *reinterpret_cast<int4 *>(s_tile[seq & 3]) = make_int4(t.e, t.row0, t.row_end, t.n0);
    return true;
  };
  auto follow = [&](Tile &t) -> bool {
    if (t.seq + 1 >= tiles) return false;
    ++t.seq;
    const int4 v = *reinterpret_cast<const int4 *>(s_tile[t.seq & 3]);
    t.e = __builtin_amdgcn_readfirstlane(v.x);
    t.row0 = __builtin_amdgcn_readfirstlane(v.y);
    t.row_end = __builtin_amdgcn_readfirstlane(v.z);
    t.n0 = __builtin_amdgcn_readfirstlane(v.w);
    return true;
  };
  // order indices of a tile's rows (rows past the segment repeat its last one's)
  auto fetch_rows = [&](const Tile &t) {
    const auto p = args();
    const int32_t *o = p->a_map.o ? p->a_map.o : p->c_map.o;
    if (!o) return;
    const int part = wave & (S::TM / 64 - 1);
    const int i = min(t.row0 + part * 64 + lane, t.row_end - 1);
    load4_to_lds(o + i, __builtin_amdgcn_readfirstlane(lds_address((const char *)&s_idx[t.seq & 3][0])) + (uwave & (S::TM / 64 - 1)) * 256);
  };

  Loader8<S> ld;
  ld.uwave = uwave;
  ld.group_bytes = (uint32_t)steps * 2048u;
  const uint32_t outside = steps == 1 ? 0x80000000u : 0u;     // where it lies
  ld.row_step = ROW8 + outside;
  ld.group_step = 2048u + outside;
  ld.row_exps_step = 4u + outside;
  ld.group_exps_step = 64u + outside;
  Reader8 rd;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) rd.fa[kk] = line_frag_offset((wave >> 1) * (S::TM / 2), kk, lane);
  rd.fb = (uint32_t)((wave & 1) * 16384 + ((lane >> 4) & 1) * 2048 + (lane >> 5) * 256 + (lane & 15) * 16);
  rd.ea = (uint32_t)((wave >> 1) * (S::TM / 2) + (lane & 31)) * 4u;
  rd.eb = (uint32_t)((wave & 1) * (TB / 2) + (lane & 31)) * 4u;
  rd.shift = (lane >> 5) * 8;
  uint32_t chunk[2];                 // source chunk of the lane's 16 bytes in a row, even and odd load instructions
#pragma unroll
  for (int p = 0; p < 2; ++p) chunk[p] = (uint32_t)((lane & 7) ^ line_swz(p * 8 + (lane >> 3))) * 16u;
  const uint32_t whole = magic_a ? 0u : ~0u;
  auto source_row = [&](uint32_t slot) { return __umulhi(slot, magic_a) + (slot & whole); };
  auto setup_sources = [&](const Tile &t) {
    const auto p = args();
    const uint32_t pitch = (uint32_t)steps * ROW8;
    const bool gathered = p->a_map.o != nullptr;
    const uint32_t rows = gathered ? source_row((uint32_t)p->Tk) : (uint32_t)min(S::TM, t.row_end - t.row0);
    const size_t first = gathered ? 0 : (size_t)t.row0;
    ld.win_a = buffer_window(p->X.values + first * pitch, rows * pitch);
    ld.win_ea = buffer_window(p->X.exps + first * (pitch / BLOCK8), rows * (pitch / BLOCK8));
    const uint32_t per_expert = (uint32_t)(p->W.halves * 2 * ((p->W.d_out / p->W.halves + 31) / 32)) * ld.group_bytes;
    ld.win_b = buffer_window(p->W.values + (size_t)t.e * per_expert, per_expert);
    ld.win_eb = buffer_window(p->W.exps + (size_t)t.e * (per_expert / BLOCK8), per_expert / BLOCK8);
    if (S::ONCE) ld.again = t.row_end - __builtin_amdgcn_readfirstlane(s_off[t.e]) - S::TM;
    const int *idx = &s_idx[t.seq & 3][0];
    // rows past the segment read zeros: an offset outside the window at every stage (in a second stage of zeros it wraps into the window, where the
    // weights are the zeros)
    const uint32_t past = 0x80000000u;
#pragma unroll
    for (int I = 0; I < S::NLA; ++I) {
      const int r = (wave * S::NLA + I) * 8 + (lane >> 3);
      const uint32_t src = gathered ? source_row((uint32_t)idx[r]) : (uint32_t)r;
      ld.oa[I] = r < t.row_end - t.row0 ? src * pitch + chunk[I & 1] : past;
    }
    const int r = (wave & (S::TM / 64 - 1)) * 64 + lane;
    const uint32_t src = gathered ? source_row((uint32_t)idx[r]) : (uint32_t)r;
    ld.oea = r < t.row_end - t.row0 ? src * (pitch / BLOCK8) : past;
    // The wavefront loads four groups of 16 columns.  SwiGLU: a wavefront's 128 columns of the tile are 64 gates and their 64 ups.
    const int half_groups = (p->W.d_out / 2 + 31) / 32 * 2;
    const uint32_t group = OUT == OUT_SWIGLU ? (uint32_t)(t.n0 / 16 + (wave >> 1) * 4 + (wave & 1) * half_groups) : (uint32_t)(t.n0 / 16 + wave * 4);
    ld.ob = group * ld.group_bytes + lane * 16u;
    ld.oeb = group * (ld.group_bytes / BLOCK8) + (uint32_t)(lane >> 4) * (ld.group_bytes / BLOCK8) + (uint32_t)(lane & 15) * 4u;
  };

  // ---- open the first two tiles
  Tile lt{-1, 0, 0, 0, 0};
  if (!next_tile(lt)) return;
  Tile ct = lt, upcoming = lt;
  bool have_upcoming = next_tile(upcoming);
  fetch_rows(lt);
  if (have_upcoming) fetch_rows(upcoming);
  wait_loads<0>();
  __syncthreads();
  setup_sources(lt);
  ld.step = 0;
  bool loader_live = true;
  auto advance_loader = [&]() {
    if (!loader_live) return;
    if (++ld.step < ns) return;
    if (!have_upcoming) {
      loader_live = false;
      --ld.step;                    // stages past the end repeat the last one's addresses
      return;
    }
    lt = upcoming;
    ld.step = 0;
    have_upcoming = next_tile(upcoming);
    if (have_upcoming) fetch_rows(upcoming);
    setup_sources(lt);
  };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));
#pragma unroll 1
  for (int st = 0; st < 2; ++st) {
#pragma unroll
    for (int I = 0; I < S::NL; ++I) ld.load(I, lds0, st);
    advance_loader();
  }
  wait_loads<0>();
  __syncthreads();
  f32x16 acc[S::FM][FR];
  Frags8<S::FM> f[2];
  Exps8<S::FM> x;
#pragma unroll
  for (int i = 0; i < 2 * (FR + 1); ++i) rd.template read<S>(f[0], i, smem, 0, 0);
  rd.template read_exps<S>(x, smem, 0);
  rd.shift_exps(x);

  int cur = 0;
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  for (;;) {                        // one tile per trip
    if constexpr (EVEN) {
      if (ct.seq > 0) stage8<true, STORES, S>(ld, rd, f, x, acc, smem, lds0, I0{}, I1{});
      else stage8<true, 0, S>(ld, rd, f, x, acc, smem, lds0, I0{}, I1{});
      advance_loader();
      stage8<false, 0, S>(ld, rd, f, x, acc, smem, lds0, I1{}, I0{});
      advance_loader();
      for (int h = 2; h < ns; h += 2) {
        stage8<false, 0, S>(ld, rd, f, x, acc, smem, lds0, I0{}, I1{});
        advance_loader();
        stage8<false, 0, S>(ld, rd, f, x, acc, smem, lds0, I1{}, I0{});
        advance_loader();
      }
    } else {
      if (ct.seq > 0) stage8<true, STORES, S>(ld, rd, f, x, acc, smem, lds0, cur, cur ^ 1);
      else stage8<true, 0, S>(ld, rd, f, x, acc, smem, lds0, cur, cur ^ 1);
      advance_loader();
      cur ^= 1;
      for (int h = 1; h < ns; ++h) {
        stage8<false, 0, S>(ld, rd, f, x, acc, smem, lds0, cur, cur ^ 1);
        advance_loader();
        cur ^= 1;
      }
    }
    const int lane = lane_here(threadIdx.x & 63);
    char *patch = smem + S::OFF_PATCH + uwave * EPI_WAVE_BYTES;
    const auto p = args();
    const int N = p->W.d_out;
    const int rbase = ct.row0 + uwm * (S::TM / 2);            // the wavefront's first row
    const int left = max(min(S::TM / 2, ct.row_end - rbase), 0);
    const int *idx = &s_idx[ct.seq & 3][uwm * (S::TM / 2)];
    if constexpr (!HIDDEN) {
      constexpr int ES = 2, PER = 16 / ES;                           // bytes of an element, elements of a 16-byte chunk
      const int wcol = ct.n0 + uwn * (TB / 2);
      const window_t win = SCATTER ? make_window(p->C, (uint32_t)p->Tk * (uint32_t)N * ES)
                                   : make_window((const char *)p->C + (size_t)rbase * N * ES, (uint32_t)left * (uint32_t)N * ES);
      auto dest = [&](int fm, int block) {                           // 128 bytes of 32 rows
        BlockDest d{win, {}};
        const int col = wcol + (block * 8 + (lane & 7)) * PER;
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int r = fm * 32 + it * 8 + (lane >> 3);
          const uint32_t row = SCATTER ? (uint32_t)idx[r] : (uint32_t)r;
          d.off[it] = r < left && col < N ? (row * (uint32_t)N + (uint32_t)col) * ES : ~0u;
        }
        return d;
      };
      if constexpr (OUT == OUT_F16) {
        const int per_row = (N + 127) / 128;
        const window_t win_e = make_window(p->C_exps, (uint32_t)p->Tk * (uint32_t)per_row);
        store_wave_tile_f16(acc, patch, dest, [&](int fm, unsigned int e) {
          const int r = fm * 32 + (lane & 31);
          const uint32_t off = lane < 32 && r < left && wcol < N ? (uint32_t)idx[r] * (uint32_t)per_row + (uint32_t)(wcol / 128) : ~0u;
          __builtin_amdgcn_raw_buffer_store_b8((char)e, win_e, (int)off, 0, 0);
        }, lane);
      } else if constexpr (OUT == OUT_BF16_REST) {
        const window_t win_r = make_window(p->rest, (uint32_t)(p->Tk / p->sum_k) * (uint32_t)N * 2);
        store_wave_tile_rest(acc, patch, dest, [&](int fm, int block, i32x4 rest) {
          const int r = fm * 32 + (lane & 31), col = wcol + block * 64;
          const uint32_t row = (uint32_t)idx[r], t = magic_sum ? __umulhi(row, magic_sum) : row;
          const uint32_t off = lane < 32 && r < left && col < N ? (t * (uint32_t)N + (uint32_t)col) * 2 + (row - t * (uint32_t)p->sum_k) * 16 : ~0u;
          __builtin_amdgcn_raw_buffer_store_b128(rest, win_r, (int)off, 0, 0);
        }, lane);
      } else {
        store_wave_tile(acc, patch, dest, lane);
      }
    } else {
      // hidden rows: 64 (SwiGLU) or 128 units of the wavefront, blocks of 32
      constexpr int BLOCKS = OUT == OUT_SWIGLU ? 2 : 4, UNITS = BLOCKS * 32;
      const int half = N / p->W.halves, pitch = (half + ROW8 - 1) / ROW8 * ROW8, padded = (half + 31) / 32 * 32;
      const int unit0 = ct.n0 + uwn * UNITS;
      const window_t win = make_window(p->H.values + (size_t)rbase * pitch, (uint32_t)left * (uint32_t)pitch);
      const window_t win_e = make_window(p->H.exps + (size_t)rbase * (pitch / BLOCK8), (uint32_t)left * (uint32_t)(pitch / BLOCK8));
      acc_settle();
#pragma unroll
      for (int fm = 0; fm < S::FM; ++fm) {
        sched_fence();
        unsigned int bytes = 0;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          float h[16];
          unsigned int code[4];
          const bool exists = unit0 + b * 32 < padded;               // whole blocks; a half's padding has weights of zero
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float v = acc_read(acc[fm][b][i]);
            if constexpr (OUT == OUT_SWIGLU) {
              const float up = acc_read(acc[fm][2 + b][i]);
              h[i] = v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v)) * up;
            } else {
              h[i] = gelu_f(v);
            }
            if (!exists) h[i] = 0.f;
          }
          bytes |= pack_block(h, code) << (8 * b);
          // patch: rows of UNITS bytes, 16-byte chunks permuted by the row
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int c = b * 2 + (g >> 1);                          // the chunk of units 8 g + 4 (lane / 32) .. of the block
            const int row = lane & 31;
            const int at = OUT == OUT_SWIGLU ? row * 64 + ((c ^ ((row >> 1) & 3)) << 4) : row * 128 + ((c ^ (row & 7)) << 4);
            *reinterpret_cast<unsigned int *>(patch + at + (g & 1) * 8 + (lane >> 5) * 4) = code[g];
          }
        }
        sched_fence();
        constexpr int PER_ROW = UNITS / 16, ROWS = 64 / PER_ROW;     // lanes of a row, rows at a time
#pragma unroll
        for (int it = 0; it < 32 / ROWS; ++it) {
          const int row = it * ROWS + lane / PER_ROW, c = lane % PER_ROW;
          const int at = OUT == OUT_SWIGLU ? row * 64 + ((c ^ ((row >> 1) & 3)) << 4) : row * 128 + ((c ^ (row & 7)) << 4);
          const i32x4 v = *reinterpret_cast<const i32x4 *>(patch + at);
          const int col = unit0 + c * 16;
          const uint32_t off = fm * 32 + row < left && col < pitch ? (uint32_t)(fm * 32 + row) * (uint32_t)pitch + (uint32_t)col : ~0u;
          __builtin_amdgcn_raw_buffer_store_b128(v, win, (int)off, 0, 0);
        }
        const uint32_t off = lane < 32 && fm * 32 + lane < left && unit0 < pitch ? (uint32_t)(fm * 32 + lane) * (uint32_t)(pitch / BLOCK8) + (uint32_t)(unit0 / BLOCK8) : ~0u;
        if constexpr (OUT == OUT_SWIGLU) __builtin_amdgcn_raw_buffer_store_b16((short)bytes, win_e, (int)off, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b32((int)bytes, win_e, (int)off, 0, 0);
      }
    }
    if (!follow(ct)) break;
  }
  wait_loads<0>();
}

template <typename S, int OUT, bool SCATTER> int launch_as(hipStream_t s, const S2S8Args &a) {
  const int steps = ceil_div(a.W.d_in, ROW8), hidden = pitch8(a.W.d_out / a.W.halves);
  const int tiles_n = OUT == OUT_SWIGLU ? ceil_div(hidden, TB / 2) : OUT == OUT_GELU ? ceil_div(hidden, TB) : ceil_div(a.W.d_out, TB);
  const uint32_t magic = a.a_map.o ? division_magic(a.a_map.fan) : 0u;
  const dim3 grid(a.grid), block(NTHREADS);
  if (steps % 2 == 0 || steps == 1) hipLaunchKernelGGL((s2s8_stream_kernel<S, OUT, SCATTER, true>), grid, block, S::LDS_BYTES, s, a, tiles_n, a.group_m, magic, division_magic(a.sum_k));
  else hipLaunchKernelGGL((s2s8_stream_kernel<S, OUT, SCATTER, false>), grid, block, S::LDS_BYTES, s, a, tiles_n, a.group_m, magic, division_magic(a.sum_k));
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
template <typename S> int launch(hipStream_t s, const S2S8Args &a) {
  if (a.act == SMOE_ACT_SWIGLU) return launch_as<S, OUT_SWIGLU, false>(s, a);
  if (a.act == SMOE_ACT_GELU) return launch_as<S, OUT_GELU, false>(s, a);
  if (a.C_exps) return launch_as<S, OUT_F16, true>(s, a);
  if (a.rest) return launch_as<S, OUT_BF16_REST, true>(s, a);
  return a.c_map.o ? launch_as<S, OUT_BF16, true>(s, a) : launch_as<S, OUT_BF16, false>(s, a);
}
template <typename S, int OUT, bool SCATTER> int init_as() {
  int rc = set_lds_limit(s2s8_stream_kernel<S, OUT, SCATTER, true>, S::LDS_BYTES);
  return rc == SMOE_OK ? set_lds_limit(s2s8_stream_kernel<S, OUT, SCATTER, false>, S::LDS_BYTES) : rc;
}
template <typename S> int init() {
  int rc = init_as<S, OUT_SWIGLU, false>();
  if (rc == SMOE_OK) rc = init_as<S, OUT_GELU, false>();
  if (rc == SMOE_OK) rc = init_as<S, OUT_F16, true>();
  if (rc == SMOE_OK) rc = init_as<S, OUT_BF16_REST, true>();
  if (rc == SMOE_OK) rc = init_as<S, OUT_BF16, true>();
  if (rc == SMOE_OK) rc = init_as<S, OUT_BF16, false>();
  return rc;
}

}  // namespace

int init_stream8_kernels() {
  const int rc = init<Big8>();
  if (rc != SMOE_OK) return rc;
  const int half = init<Half8>();
  return half == SMOE_OK ? init<Half8Once>() : half;
}

// 32-bit offsets into the rows, an expert's weights and a scattered output; the fan-out's division.
bool s2s8_stream_supported(const S2S8Args &a) {
  if (a.Tk < 1 || a.W.E > MAX_E8 || a.grid < 8) return false;
  if (a.wide || ((a.C_exps || a.rest) && !a.c_map.o)) return false;
  const unsigned long long pitch = pitch8(a.W.d_in), rows = a.a_map.o ? a.Tk / a.a_map.fan : 256;
  if (rows * pitch > 0x7fff0000ULL || (unsigned long long)groups8(a.W.d_out, a.W.halves) * 16 * pitch + 32 * pitch * 16 > 0x7fff0000ULL) return false;
  if (!a.H.values && a.c_map.o && (unsigned long long)a.Tk * a.W.d_out * 2 > 0xfffffff0ULL) return false;
  if (256ULL * a.W.d_out * 2 > 0x7fff0000ULL) return false;
  if (a.a_map.o && (unsigned long long)a.Tk * a.a_map.fan >= 0x100000000ULL) return false;
  const long long m_tiles = (long long)a.Tk / 128 + a.W.E, n_tiles = ceil_div(a.W.d_out, 128);
  return m_tiles * n_tiles <= 0x7fffffffLL;
}
int launch_s2s8_stream(hipStream_t s, const S2S8Args &a) {
  if (!s2s8_stream_supported(a)) return SMOE_ERR_UNSUPPORTED;
  if (a.tile_shape != 1) return launch<Big8>(s, a);
  // see launch_as in gemm8_decode.hip; with a tile an expert on average the weights are read about once
  const bool once = a.call_weights > LAST_LEVEL_CACHE / 2 && (long long)a.Tk <= 128LL * a.W.E;
  return once ? launch<Half8Once>(s, a) : launch<Half8>(s, a);
}
