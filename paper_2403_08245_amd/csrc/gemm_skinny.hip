// Two dense products of the same few rows, P_w = X W_w for w = 0, 1, by shares of the contraction: the key and value projections of a decoding
// pass, whose consumer (rotary.hip) adds the shares.
//
// Bound by memory: every weight is read once for up to 64 rows.  A key or value projection is a few megabytes, and its columns alone, 128 to a
// wavefront as the loads want them, would keep a handful of compute units busy; so the contraction is cut into shares for as many blocks
// as the chip has units, and a block's four wavefronts share theirs again, adding up through LDS.  The weights go from memory straight to
// registers and through byte permutations into the matrix instructions, as in gemm_decode.hip.
#include "mfma_common.h"
#include "cache.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int COLS = 128;          // of a block
constexpr int SWAVES = 4;

// MT tiles of 16 rows.  Block: 128 columns of one of the two, one share; wavefront u of all the shares' takes steps u, u + all, ...
template <int MT> __global__ void __launch_bounds__(64 * SWAVES, 2) skinny_pair_kernel(const bf16_t *X, const bf16_t *W0, const bf16_t *W1, int M, int K, int N, int shares,
                                                                                     float *P) {
  __shared__ float s_part[SWAVES][32][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int chunks = (N + COLS - 1) / COLS;
  const int share = (int)blockIdx.x % shares, which = (int)blockIdx.x / shares, chunk = which % chunks, w = which / chunks;
  const int row0 = (int)blockIdx.y * MT * 16;
  const int c = lane & 15, q = lane >> 4, col = chunk * COLS + c * 8;
  const bool have = col < N;
  const bf16_t *W = (w ? W1 : W0) + (have ? col : 0) + (size_t)(8 * q) * N;
  const bf16_t *x_row[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x_row[m] = X + (size_t)min(row0 + m * 16 + c, M - 1) * K + 8 * q;   // rows past the last repeat it
  f32x4 acc[MT][8];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = K / HK, all = shares * SWAVES;
  auto load_w = [&](int s, u32x4 (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const u32x4 *>(W + ((size_t)s * HK + i) * N);
  };
  auto load_x = [&](int s, bf16x8 (&v)[MT]) {
#pragma unroll
    for (int m = 0; m < MT; ++m) v[m] = *reinterpret_cast<const bf16x8 *>(x_row[m] + s * HK);
  };
  auto use = [&](const u32x4 (&v)[8], const bf16x8 (&x)[MT]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4 f;
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] = __builtin_amdgcn_perm(v[2 * t + 1][j / 2], v[2 * t][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), x[m], acc[m][j], 0, 0, 0);
    }
  };
  int s = share * SWAVES + wave;
#pragma unroll 1
  for (; s + all < steps; s += 2 * all) {      // two at a time: both steps' requests go out before the first is used
    u32x4 a[8], b[8];
    bf16x8 xa[MT], xb[MT];
    load_w(s, a);
    load_x(s, xa);
    load_w(s + all, b);
    load_x(s + all, xb);
    use(a, xa);
    use(b, xb);
  }
  if (s < steps) {
    u32x4 a[8];
    bf16x8 xa[MT];
    load_w(s, a);
    load_x(s, xa);
    use(a, xa);
  }
  // The wavefronts' sums in their order.  Lane (c, q) holds row c of a tile and, in element r, columns 8 * (4 q + r) + j.
  float *out = P + ((size_t)share * 2 + w) * M * N;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (m) __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) s_part[wave][r * 8 + j][lane] = acc[m][j][r];
    __syncthreads();
    const int row = row0 + m * 16 + c, r = wave, first = chunk * COLS + 8 * (4 * q + r);
    f32x4 lo = f32x4{0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int p = 0; p < SWAVES; ++p) {
        lo[j] += s_part[p][r * 8 + j][lane];
        hi[j] += s_part[p][r * 8 + 4 + j][lane];
      }
    if (row < M && first < N) {
      *reinterpret_cast<f32x4 *>(out + (size_t)row * N + first) = lo;
      *reinterpret_cast<f32x4 *>(out + (size_t)row * N + first + 4) = hi;
    }
  }
}

}  // namespace

// The line at 512 rows: the attention layer's decoding pass in us, these kernels / the persistent ones (up to 32 rows the decoding ones), 2048
// wide, 16 experts, k = 4, 4 heads: 4 rows 41 / 59, 64 rows 58 / 76, 128 rows 76 / 93, 256 rows 126 / 140, 512 rows 120 / 135 (shorter
// contexts); 4096 wide, 64 experts, k = 8: 128 rows 163 / 176, 256 rows 223 / 239, 512 rows 218 / 230.  They win wherever tried; past that the shares
// outgrow their room and the large tiles fill the chip.
int skinny_shares(int M, int K, int N) {
  if (M < 1 || M > SKINNY_MAX_ROWS || K < HK || K % HK || N % 8) return 0;
  // a step or two for each wavefront, and about a block for each compute unit at most
  const int steps = K / HK, chunks = 2 * ceil_div(N, COLS) * ceil_div(M, 64);
  return std::max(1, std::min(ceil_div(steps, 2 * SWAVES), ceil_div(256, chunks)));
}

int launch_skinny_pair(hipStream_t s, const void *X, const void *W0, const void *W1, int M, int K, int N, int shares, float *P) {
  const int tiles = ceil_div(M, 16);
  auto go = [&](auto kernel, int mt) {
    kernel<<<dim3(2 * ceil_div(N, COLS) * shares, ceil_div(tiles, mt)), 64 * SWAVES, 0, s>>>((const bf16_t *)X, (const bf16_t *)W0, (const bf16_t *)W1, M, K, N, shares, P);
    return hipGetLastError() == hipSuccess ? SMOE_OK : SMOE_ERR_HIP;
  };
  return tiles == 1 ? go(skinny_pair_kernel<1>, 1) : tiles == 2 ? go(skinny_pair_kernel<2>, 2) : go(skinny_pair_kernel<4>, 4);
}
