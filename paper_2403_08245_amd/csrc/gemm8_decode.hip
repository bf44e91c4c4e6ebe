// The products in 8 bits for a few rows per expert: a stream of the used experts' weights past a handful of rows.  Bound: HBM.
//
// A wavefront owns 64 columns (four groups of 16) of a 32-row tile of one expert: v_mfma_scale_f32_16x16x128_f8f6f4 with the weights as the first operand,
// so that a lane ends up with four consecutive columns of one row.  Weights are laid out as the instruction takes them (smoe_weights8): a
// step of 128 of the contraction of a group is 2 KB, two loads of 16 bytes a lane, straight to registers; no LDS, no barrier in the loop.
// Wavefronts of a block stand side by side (CW) or share the contraction (KW) and add their sums through LDS in a fixed order.
//
// Operands: lane (r, q) = (lane % 16, lane / 16) holds elements 16 q .. 16 q + 15 and 64 + 16 q .. of row or column r, and the power of two of
// its elements 32 q .. 32 q + 31.
#include "block.h"
#include "mfma_common.h"
#include <type_traits>

namespace {

constexpr int DM = 32;                        // rows of a tile: two 16-row fragments
constexpr int DEPTH = 2;                      // steps in flight per wavefront
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Weights {                              // one step of the wavefront's four groups
  i32x4 lo[4], hi[4];
  unsigned int exps[4];
};
struct Rows {                                 // one step of the tile's two fragments
  i32x4 lo[2], hi[2];
  unsigned int exps[2];
};
__device__ __forceinline__ i32x8 joined(i32x4 lo, i32x4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// ACT: none (out: bf16, or fp32 with WIDE), GELU or SwiGLU (out: packed hidden rows; a tile's columns are then 32 gates and their 32 ups)
template <int ACT, bool WIDE, int CW, int KW, bool ONCE>
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
  const bool two = row_end - row0 > 16;
  const int r = lane & 15, q = lane >> 4;
  const int tile = nc * CW + cw;                     // the wavefront's columns, in units of 64 (SwiGLU: 32 hidden units)
  const int half_groups = groups / 2;
  auto group = [&](int j) { return ACT == SMOE_ACT_SWIGLU ? 2 * tile + (j & 1) + (j >> 1) * half_groups : 4 * tile + j; };
  auto exists = [&](int j) { return ACT == SMOE_ACT_SWIGLU ? 2 * tile + (j & 1) < half_groups : group(j) < groups; };
  // groups that do not exist read one that does; their sums are not used
  const uint8_t *wv[4], *we[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const size_t at = ((size_t)e * groups + (exists(j) ? group(j) : 0)) * steps;
    wv[j] = a.W.values + at * 2048 + lane * 16;
    we[j] = a.W.exps + at * 64 + r * 4;
  }
  // steps from .. to are this wavefront's
  const int from = steps * kw / KW, to = steps * (kw + 1) / KW;
  const uint8_t *xv[2], *xe[2];                      // rows past the segment repeat its last row
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const size_t src = map_row(a.a_map, min(row0 + m * 16 + r, row_end - 1));
    xv[m] = a.X.values + src * pitch + q * 16;
    xe[m] = a.X.exps + src * (pitch / BLOCK8);
  }
  f32x4 acc[2][4];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto load_x = [&](int s) {
    Rows x;
#pragma unroll
    for (int m = 0; m < 2; ++m)
      if (m == 0 || two) {
        x.lo[m] = *reinterpret_cast<const i32x4 *>(xv[m] + s * ROW8);
        x.hi[m] = *reinterpret_cast<const i32x4 *>(xv[m] + s * ROW8 + 64);
        x.exps[m] = *reinterpret_cast<const unsigned int *>(xe[m] + s * 4);
      }
    return x;
  };
  auto multiply = [&](const Weights &w, const Rows &x) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
      if (m == 0 || two) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[m][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(joined(w.lo[j], w.hi[j]), joined(x.lo[m], x.hi[m]), acc[m][j], 0, 0, 0,
                                                                       (int)(w.exps[j] >> (8 * q)), 0, (int)(x.exps[m] >> (8 * q)));
      }
  };
  auto contract = [&](auto past_caches) {
    auto load_w = [&](int s) {
      Weights w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const i32x4 *src = reinterpret_cast<const i32x4 *>(wv[j] + (size_t)s * 2048);
        w.lo[j] = decltype(past_caches)::value ? __builtin_nontemporal_load(src) : *src;
        w.hi[j] = decltype(past_caches)::value ? __builtin_nontemporal_load(src + 64) : src[64];
        w.exps[j] = *reinterpret_cast<const unsigned int *>(we[j] + (size_t)s * 64);
      }
      return w;
    };
    Weights w[DEPTH];
    Rows x[DEPTH];
#pragma unroll
    for (int u = 0; u < DEPTH; ++u)
      if (from + u < to) {
        w[u] = load_w(from + u);
        x[u] = load_x(from + u);
      }
    int s = from;
#pragma unroll 1
    for (; s + 2 * DEPTH <= to; s += DEPTH) {
#pragma unroll
      for (int u = 0; u < DEPTH; ++u) {
        multiply(w[u], x[u]);
        w[u] = load_w(s + u + DEPTH);
        x[u] = load_x(s + u + DEPTH);
      }
    }
    // the last steps stand by themselves, so that nothing is requested past the end
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) {
      if (s + u < to) multiply(w[u], x[u]);
      if (s + u + DEPTH < to) {
        w[u] = load_w(s + u + DEPTH);
        x[u] = load_x(s + u + DEPTH);
      }
    }
#pragma unroll
    for (int u = 0; u < DEPTH - 1; ++u)
      if (s + u + DEPTH < to) multiply(w[u], x[u]);
  };
  // an expert with more rows than one tile has its weights read again, by other blocks, which should find them in the caches
  if (ONCE && row_end - __builtin_amdgcn_readfirstlane(a.offsets[e]) <= DM) {
    __asm__ volatile("" ::: "memory");   // keeps the two forms apart
    contract(std::true_type{});
  } else {
    contract(std::false_type{});
  }

  if constexpr (KW > 1) {                // sums over the contraction's shares, in their order
    if (kw > 0) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
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
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][j][i] += s_part[p][cw][m * 16 + j * 4 + i][lane];
  }
  // lane (r, q): row r of the fragment, columns 4 q .. 4 q + 3 of each group
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    if (m == 1 && !two) break;
    const int i = row0 + m * 16 + r;
    if constexpr (ACT == SMOE_ACT_NONE) {
      const size_t dst = i < row_end ? (size_t)map_row(a.c_map, i) : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = group(j) * 16 + 4 * q;
        if (i >= row_end || col >= a.W.d_out) continue;
        if constexpr (WIDE) {
          *reinterpret_cast<f32x4 *>((float *)a.C + dst * a.W.d_out + col) = acc[m][j];
        } else {
          bf16x4 v;
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] = (bf16_t)acc[m][j][c];
          *reinterpret_cast<bf16x4 *>((bf16_t *)a.C + dst * a.W.d_out + col) = v;
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
            h[g * 4 + c] = exists(2 * b) ? v : 0.f;
            amax = fmaxf(amax, finite_abs(h[g * 4 + c]));
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
}

template <int ACT, bool WIDE, int CW, int KW> int launch_as(hipStream_t s, const S2S8Args &a) {
  const int groups = groups8(a.W.d_out, a.W.halves), steps = ceil_div(a.W.d_in, ROW8), h_pitch = pitch8(a.W.d_out / a.W.halves);
  const int units = ACT == SMOE_ACT_SWIGLU ? h_pitch / 32 : ACT ? h_pitch / 64 : ceil_div(groups, 4);     // of a wavefront each
  const int n_chunks = ceil_div(units, CW);
  const long long blocks = ((long long)a.Tk / DM + a.W.E) * n_chunks;                       // >= sum_e ceil(n_e / 32)
  const dim3 grid((unsigned)blocks), block(64 * CW * KW);
  if (a.call_weights > LAST_LEVEL_CACHE)
    hipLaunchKernelGGL((s2s8_decode_kernel<ACT, WIDE, CW, KW, true>), grid, block, 0, s, a, n_chunks, groups, steps, pitch8(a.W.d_in), h_pitch);
  else
    hipLaunchKernelGGL((s2s8_decode_kernel<ACT, WIDE, CW, KW, false>), grid, block, 0, s, a, n_chunks, groups, steps, pitch8(a.W.d_in), h_pitch);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
template <int ACT, bool WIDE> int launch(hipStream_t s, const S2S8Args &a) {
  const long long experts = a.Tk < a.W.E ? a.Tk : a.W.E, units = ACT == SMOE_ACT_SWIGLU ? a.W.d_out / 64 : a.W.d_out / 64;
  if (experts * units >= 8 * a.grid) return launch_as<ACT, WIDE, 4, 1>(s, a);
  if (experts * units >= 4 * a.grid) return launch_as<ACT, WIDE, 2, 2>(s, a);
  return launch_as<ACT, WIDE, 1, 4>(s, a);
}

}  // namespace

int launch_s2s8_decode(hipStream_t s, const S2S8Args &a) {
  if (a.act == SMOE_ACT_SWIGLU) return launch<SMOE_ACT_SWIGLU, false>(s, a);
  if (a.act == SMOE_ACT_GELU) return launch<SMOE_ACT_GELU, false>(s, a);
  return a.wide ? launch<SMOE_ACT_NONE, true>(s, a) : launch<SMOE_ACT_NONE, false>(s, a);
}
