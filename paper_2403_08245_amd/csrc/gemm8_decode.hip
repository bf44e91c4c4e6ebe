// The products in 8 bits for a few rows per expert: a stream of the used experts' weights past a handful of rows.  Bound: HBM.
//
// A wavefront owns 64 columns (four groups of 16) of a tile of up to 32 rows of one expert, with the weights as the first operand, so that a lane ends
// up with four consecutive columns of one row.  Weights are laid out for it (smoe_weights8): a step of 128 of the contraction of a group is 2 KB, two
// loads of 16 bytes a lane, straight to registers; no LDS, no barrier in the loop.  Wavefronts of a block stand side by side (CW) or share the
// contraction (KW) and add their sums through LDS in a fixed order.
//
// Bare products: v_mfma_scale_f32_16x16x128_f8f6f4, lane (r, q) = (lane % 16, lane / 16) with elements 16 q .. 16 q + 15 and 64 + 16 q .. of row or column r, and
// the power of two of its elements 32 q .. 32 q + 31.  It adds its 128 products to about 2^-12 of the largest, far under the rounding of what is stored.
// Hidden rows, which are packed to codes of four bits, would feel that: 1.6e-3 (GELU) to 2.5e-3 (SwiGLU) of the codes came out on the other side of a border, a
// step of up to an eighth of a value each.  There the codes are widened to bf16, which holds them with their power of two exactly, and multiplied by
// v_mfma_f32_16x16x32_bf16: four times the matrix time, of which there is enough beside the weights' stream, and sums good to fp32 (under 1e-4 of the codes).
// Which eight of a lane's elements an instruction takes does not matter, as long as rows and columns give the same.
#include "block.h"
#include "mfma_common.h"
#include <type_traits>

namespace {

// Rows of a tile: one or two 16-row fragments.  (Four: 200 tokens on 8 experts, 1024 -> 2 x 2816 -> 1024, 35 -> 61 us: every wavefront reads its tile's
// rows from L2 for 64 columns, as many bytes as it reads of the weights.)
constexpr int DM = 32;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t window_t;

// 16-byte and 4-byte loads of a window: the lane's offset in a register, the rest of the address in a scalar one.  ONCE: kept by no cache.
template <bool ONCE> __device__ __forceinline__ i32x4 load16(window_t w, int lane_off, int off) {
  return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(w, lane_off, off, ONCE ? 2 : 0));
}
__device__ __forceinline__ unsigned int load4(window_t w, int lane_off, int off) { return (unsigned int)__builtin_amdgcn_raw_buffer_load_b32(w, lane_off, off, 0); }
__device__ __forceinline__ window_t window_of(const void *base, uint32_t bytes) {
  const unsigned long long p = (unsigned long long)base;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void *)(((unsigned long long)hi << 32) | lo), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}

struct Weights {                              // one step of the wavefront's four groups
  i32x8 v[4];
  unsigned int exps[4];
};
template <int F> struct Rows {                // one step of the tile's fragments
  i32x8 v[F];
  unsigned int exps[F];
};
__device__ __forceinline__ i32x8 joined(i32x4 lo, i32x4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// A lane's 32 elements of a step as the values they stand for; `exps`: the bytes of the step's four blocks of 32, the lane's are q / 2 and 2 + q / 2.
struct Wide {
  bf16x8 v[4];
};
__device__ __forceinline__ Wide widened(i32x8 codes, unsigned int exps, int q) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const unsigned int mine = exps >> (8 * (q >> 1));
  const float scale[2] = {__uint_as_float((mine & 0xffu) << 23), __uint_as_float((mine << 7) & 0x7f800000u)};
  Wide w;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bf16x2 lo = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale[i >> 2], false));
    const bf16x2 hi = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale[i >> 2], true));
    w.v[i >> 1][4 * (i & 1)] = lo[0];
    w.v[i >> 1][4 * (i & 1) + 1] = lo[1];
    w.v[i >> 1][4 * (i & 1) + 2] = hi[0];
    w.v[i >> 1][4 * (i & 1) + 3] = hi[1];
  }
  return w;
}

enum { ROWS_BF16, ROWS_F32, ROWS_F16 };       // ROWS_F16: with a power of two for 64 columns

// ACT: none (out: rows as OUT says), GELU or SwiGLU (out: packed hidden rows; a tile's columns are then 32 gates and their 32 ups)
template <int ACT, int OUT, int CW, int KW, bool ONCE>
__global__ void __launch_bounds__(64 * CW * KW, 2) s2s8_decode_kernel(S2S8Args a, int n_chunks, int groups, int steps, int pitch, int h_pitch) {
  __shared__ float s_part[KW > 1 ? KW - 1 : 1][CW][32][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int cw = wave % CW, kw = wave / CW;
  const int mt = (int)blockIdx.x / n_chunks, nc = (int)blockIdx.x - mt * n_chunks;
  int e, row0, row_end;
  if (!locate_rows<DM>(a.offsets, a.W.E, mt, lane, e, row0, row_end)) return;   // grid is an upper bound
  e = __builtin_amdgcn_readfirstlane(e);
  row0 = __builtin_amdgcn_readfirstlane(row0);
  row_end = __builtin_amdgcn_readfirstlane(row_end);
  const int r = lane & 15, q = lane >> 4;
  const int tile = nc * CW + cw;                     // the wavefront's columns, in units of 64 (SwiGLU: 32 hidden units)
  const int half_groups = groups / 2;
  auto group = [&](int j) { return ACT == SMOE_ACT_SWIGLU ? 2 * tile + (j & 1) + (j >> 1) * half_groups : 4 * tile + j; };
  auto exists = [&](int j) { return ACT == SMOE_ACT_SWIGLU ? 2 * tile + (j & 1) < half_groups : group(j) < groups; };
  // steps from .. to are this wavefront's: windows of its groups from the first of them on.  Groups that do not exist read zeros.
  const int from = steps * kw / KW, mine = steps * (kw + 1) / KW - from;
  window_t wv[4], we[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const size_t at = ((size_t)e * groups + group(j)) * steps + from;
    const bool have = exists(j);
    wv[j] = window_of(a.W.values + (have ? at * 2048 : 0), have ? (uint32_t)mine * 2048u : 0u);
    we[j] = window_of(a.W.exps + (have ? at * 64 : 0), have ? (uint32_t)mine * 64u : 0u);
  }

  // F fragments of rows
  auto run = [&](auto fragments, auto past_caches) {
    constexpr int F = decltype(fragments)::value;
    auto load_w = [&](int s) {
      Weights w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w.v[j] = joined(load16<decltype(past_caches)::value>(wv[j], lane * 16, s * 2048), load16<decltype(past_caches)::value>(wv[j], lane * 16 + 1024, s * 2048));
        w.exps[j] = load4(we[j], r * 4, s * 64);
      }
      return w;
    };
    const int second = mine > 1 ? 1 : 0;               // a share may be of one step or none: then products of zeros
    Weights w0 = load_w(0), w1 = load_w(second);
    const uint8_t *xv[F], *xe[F];                      // rows past the segment repeat its last row
#pragma unroll
    for (int m = 0; m < F; ++m) {
      const size_t src = map_row(a.a_map, min(row0 + m * 16 + r, row_end - 1));
      xv[m] = a.X.values + src * pitch + from * ROW8 + q * 16;
      xe[m] = a.X.exps + src * (pitch / BLOCK8) + from * 4;
    }
    auto load_x = [&](int s) {
      Rows<F> x;
#pragma unroll
      for (int m = 0; m < F; ++m) {
        x.v[m] = joined(*reinterpret_cast<const i32x4 *>(xv[m] + s * ROW8), *reinterpret_cast<const i32x4 *>(xv[m] + s * ROW8 + 64));
        x.exps[m] = *reinterpret_cast<const unsigned int *>(xe[m] + s * 4);
      }
      return x;
    };
    Rows<F> x0 = load_x(0), x1 = load_x(second);
    f32x4 acc[F][4];
#pragma unroll
    for (int m = 0; m < F; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Weights &w, const Rows<F> &x) {
      if constexpr (ACT == SMOE_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int m = 0; m < F; ++m)
            acc[m][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v[j], x.v[m], acc[m][j], 0, 0, 0,
                                                                         (int)(w.exps[j] >> (8 * q)), 0, (int)(x.exps[m] >> (8 * q)));
        return;
      }
      Wide xs[F];
#pragma unroll
      for (int m = 0; m < F; ++m) xs[m] = widened(x.v[m], x.exps[m], q);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Wide ws = widened(w.v[j], w.exps[j], q);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int m = 0; m < F; ++m) acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ws.v[i], xs[m].v[i], acc[m][j], 0, 0, 0);
      }
    };
    // the last steps stand by themselves, so that nothing is requested past the end
    int s = 0;
#pragma unroll 1
    for (; s + 4 <= mine; s += 2) {
      // fences: the compiler would request the next step in front of the products, into registers that there are not
      multiply(w0, x0);
      sched_fence();
      w0 = load_w(s + 2);
      x0 = load_x(s + 2);
      sched_fence();
      multiply(w1, x1);
      sched_fence();
      w1 = load_w(s + 3);
      x1 = load_x(s + 3);
      sched_fence();
    }
    multiply(w0, x0);
    if (s + 2 < mine) {
      sched_fence();
      w0 = load_w(s + 2);
      x0 = load_x(s + 2);
      sched_fence();
      multiply(w1, x1);
      multiply(w0, x0);
    } else if (s + 1 < mine) {
      multiply(w1, x1);
    }

    if constexpr (KW > 1) {                // sums over the contraction's shares, in their order
      if (kw > 0) {
#pragma unroll
        for (int m = 0; m < F; ++m)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) s_part[kw - 1][cw][m * 16 + j * 4 + i][lane] = acc[m][j][i];
      }
      __syncthreads();
      if (kw > 0) return;
#pragma unroll
      for (int p = 0; p < KW - 1; ++p)
#pragma unroll
        for (int m = 0; m < F; ++m)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] += s_part[p][cw][m * 16 + j * 4 + i][lane];
    }
    // lane (r, q): row r of the fragment, columns 4 q .. 4 q + 3 of each group
#pragma unroll
    for (int m = 0; m < F; ++m) {
      const int i = row0 + m * 16 + r;
      if constexpr (ACT == SMOE_ACT_NONE) {
        const size_t dst = i < row_end ? (size_t)map_row(a.c_map, i) : 0;
        float scale = 1.0f;
        if constexpr (OUT == ROWS_F16) {
          // The largest finite value of the row's 64 columns goes into [2^14, 2^15): exponents as in gemm8_stream.hip
          float most = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) most = fmaxf(most, finite_abs(acc[m][j][c]));
          most = fmaxf(most, __shfl_xor(most, 16, 64));
          most = fmaxf(most, __shfl_xor(most, 32, 64));
          const unsigned int e = max(__float_as_uint(most) >> 23, 15u);
          scale = __uint_as_float((268u - e) << 23);
          if (q == 0 && i < row_end && tile * 64 < a.W.d_out) a.C_exps[dst * ((a.W.d_out + 63) / 64) + tile] = (uint8_t)e;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = group(j) * 16 + 4 * q;
          if (i >= row_end || col >= a.W.d_out) continue;
          if constexpr (OUT == ROWS_F32) {
            *reinterpret_cast<f32x4 *>((float *)a.C + dst * a.W.d_out + col) = acc[m][j];
          } else if constexpr (OUT == ROWS_F16) {
            f16x4 v;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = (_Float16)(acc[m][j][c] * scale);
            *reinterpret_cast<f16x4 *>((_Float16 *)a.C + dst * a.W.d_out + col) = v;
          } else {
            bf16x4 v;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = (bf16_t)acc[m][j][c];
            *reinterpret_cast<bf16x4 *>((bf16_t *)a.C + dst * a.W.d_out + col) = v;
          }
        }
        if (OUT == ROWS_BF16 && a.rest) {
          const size_t t = (unsigned int)dst / (unsigned int)a.sum_k;
          unsigned int *to = reinterpret_cast<unsigned int *>(a.rest + t * a.W.d_out * 2 + (size_t)tile * 128 + (dst - t * a.sum_k) * 16);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            unsigned int word = 0;
#pragma unroll
            for (int j = 2 * h; j < 2 * h + 2; ++j)
#pragma unroll
              for (int c = 0; c < 4; ++c) word |= bf16_rest(acc[m][j][c]) << (8 * c + 4 * (j & 1));
            word <<= 2 * (q >> 1);
            word |= __shfl_xor(word, 32, 64);
            if (i < row_end && q < 2 && tile * 64 < a.W.d_out) to[2 * h + q] = word;
          }
        }
      } else {
        // two groups are a block of 32 hidden units, spread over the four lanes of a row
        constexpr int BLOCKS = ACT == SMOE_ACT_SWIGLU ? 1 : 2;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          float h[8], amax = 0.f;
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float v;
              if constexpr (ACT == SMOE_ACT_SWIGLU) {
                const float gate = acc[m][g][c];
                v = gate * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * gate)) * acc[m][2 + g][c];
              } else {
                v = gelu_f(acc[m][2 * b + g][c]);
              }
              h[g * 4 + c] = v;
              amax = fmaxf(amax, finite_abs(v));
            }
          amax = fmaxf(amax, __shfl_xor(amax, 16, 64));
          amax = fmaxf(amax, __shfl_xor(amax, 32, 64));
          const unsigned int byte = e4m3_byte(amax);
          const int col = ACT == SMOE_ACT_SWIGLU ? tile * 32 : tile * 64 + b * 32;
          if (i < row_end && col < h_pitch) {
            uint8_t *row = a.H.values + (size_t)i * h_pitch + col + 4 * q;
            *reinterpret_cast<unsigned int *>(row) = e4m3_four(h[0], h[1], h[2], h[3], byte);
            *reinterpret_cast<unsigned int *>(row + 16) = e4m3_four(h[4], h[5], h[6], h[7], byte);
            if (q == 0) a.H.exps[(size_t)i * (h_pitch / BLOCK8) + col / BLOCK8] = (uint8_t)byte;
          }
        }
      }
    }
  };
  auto by_rows = [&](auto past_caches) {
    if (row_end - row0 <= 16) run(std::integral_constant<int, 1>{}, past_caches);
    else run(std::integral_constant<int, 2>{}, past_caches);
  };
  // an expert with more rows than one tile has its weights read again, by other blocks, which should find them in the caches
  if (ONCE && row_end - __builtin_amdgcn_readfirstlane(a.offsets[e]) <= DM) {
    __asm__ volatile("" ::: "memory");   // keeps the two forms apart
    by_rows(std::true_type{});
  } else {
    by_rows(std::false_type{});
  }
}

template <int ACT, int OUT, int CW, int KW> int launch_as(hipStream_t s, const S2S8Args &a) {
  const int groups = groups8(a.W.d_out, a.W.halves), steps = ceil_div(a.W.d_in, ROW8), h_pitch = pitch8(a.W.d_out / a.W.halves);
  const int units = ACT == SMOE_ACT_SWIGLU ? h_pitch / 32 : ACT ? h_pitch / 64 : ceil_div(groups, 4);     // of a wavefront each
  const int n_chunks = ceil_div(units, CW);
  const long long blocks = ((long long)a.Tk / DM + a.W.E) * n_chunks;                       // >= sum_e ceil(n_e / DM)
  const dim3 grid((unsigned)blocks), block(64 * CW * KW);
  // Weights over half of the last-level cache are not there any more when the layer's turn comes again: read past it.  Three layers in turn, us, through /
  // past: 64 tokens on 64 experts, 2048 -> 2 x 512 -> 2048 (208 MB each) 47.8 / 45; 32 tokens on 16 experts, 4096 -> 2 x 1024 -> 4096 (208 MB) 45.5 / 42.8; 64
  // tokens on 8 experts, 1024 -> 2 x 2816 -> 1024 (71 MB) 27 / 30.
  if (a.call_weights > LAST_LEVEL_CACHE / 2)
    hipLaunchKernelGGL((s2s8_decode_kernel<ACT, OUT, CW, KW, true>), grid, block, 0, s, a, n_chunks, groups, steps, pitch8(a.W.d_in), h_pitch);
  else
    hipLaunchKernelGGL((s2s8_decode_kernel<ACT, OUT, CW, KW, false>), grid, block, 0, s, a, n_chunks, groups, steps, pitch8(a.W.d_in), h_pitch);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
// How the wavefronts of a block divide the work: side by side, or along the contraction where there are too few columns to fill the chip.  One product, weights from
// memory, us, 4 x 1 / 2 x 2 / 1 x 4: 64 tokens on 64 experts, k = 8, 512 -> 2048 13.6 / 15.7 / 18.9; 200 tokens on 8 experts, k = 2, 2816 -> 1024 22.6 / 14 / 10.3;
// four tokens on 64 experts, k = 8, 512 -> 2048 8.7 / 8 / 10.7; 16 tokens on 8 experts, k = 2, 14336 -> 4096 94 / 75 / 73.5.
// Groups of columns that lie an odd number of 32 KB apart (16 steps of the contraction, 48, ..) get in one another's way when 16 of them are read in step, with up to 16
// rows an expert, and so do some at odd numbers of 16 KB: 1 / 2 / 4 shares, T tokens on E experts, us:
//   2048 -> 8192 (64 on 64, k = 8) 203 / 188 / 173, -> 6144 157 / 150 / 136, -> 4096 108 / 105 / 94, -> 16384 (32 on 16, k = 2) 112 / 103 / 91, -> 8192 (64 on 32, k = 4) 109 / 105 / 95
//   1024 -> 8192 (64 on 64) 107 / 99 / 114, -> 4096 59 / 53 / 60, -> 16384 (32 on 16) 57 / 50 / 56, -> 20480 (32 on 8) 41 / 35 / 39, -> 8192 (64 on 32) 59 / 52 / 59
//   further odd numbers: 5120 -> 8192 (32 on 16) 121 / 115 / 117, 6144 -> 8192 136 / 136 / 137, 10240 -> 8192 231 / 234 / 226
//   others: 4096 -> 8192 96 / 111 / 103, 2560 -> 8192 62.6 / 62.5 / 62.7, 1536 -> 4096 (64 on 64) 77 / 78 / 81
// (Wavefronts that begin at different steps of the contraction gained 0 to 4 % and cost others up to 40 %.)
template <int ACT, int OUT> int launch(hipStream_t s, const S2S8Args &a) {
  const long long experts = a.Tk < a.W.E ? a.Tk : a.W.E, units = a.W.d_out / 64;
  const int steps = ceil_div(a.W.d_in, ROW8);
  const bool thin = a.Tk <= 16 * experts;
  int shares = experts * units >= 8 * a.grid ? 1 : experts * units >= 4 * a.grid ? 2 : 4;
  if (shares == 1 && thin) shares = steps % 32 == 16 ? 4 : steps % 16 == 8 ? 2 : 1;
  if (shares == 1) return launch_as<ACT, OUT, 4, 1>(s, a);
  if (shares == 2) return launch_as<ACT, OUT, 2, 2>(s, a);
  return launch_as<ACT, OUT, 1, 4>(s, a);
}

}  // namespace

int launch_s2s8_decode(hipStream_t s, const S2S8Args &a) {
  if (a.act == SMOE_ACT_SWIGLU) return launch<SMOE_ACT_SWIGLU, ROWS_BF16>(s, a);
  if (a.act == SMOE_ACT_GELU) return launch<SMOE_ACT_GELU, ROWS_BF16>(s, a);
  if (a.wide) return launch<SMOE_ACT_NONE, ROWS_F32>(s, a);
  return a.C_exps ? launch<SMOE_ACT_NONE, ROWS_F16>(s, a) : launch<SMOE_ACT_NONE, ROWS_BF16>(s, a);
}
