// Rows in 8 bits: packing and unpacking them, and packing weights into the layout of the products.  Bound: HBM (8191 rows of 4096 from bf16 23 us, 102 MB,
// 4.4 TB/s, from fp32 31; to bf16 17, 5.9 TB/s).
#include "block.h"

namespace {

// Eight elements a thread, four threads a block of 32.  The row's padding is packed as zeros are.
template <typename T>
__global__ void __launch_bounds__(256) rows8_pack_kernel(const T *__restrict__ X, long long chunks, int per_row, int d, smoe_rows8 out) {
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (long long)gridDim.x * 256) {
    const long long row = i / per_row;
    const int c = (int)(i - row * per_row) * 8;
    const T *src = X + row * d + c;
    float y[8];
    if (d % 8 == 0 && c < d) {
#pragma unroll
      for (int q = 0; q < 8 * (int)sizeof(T) / 16; ++q) {
        const vec v = reinterpret_cast<const vec *>(src)[q];
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) y[q * (16 / (int)sizeof(T)) + j] = to_f32<T>(v[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = c + j < d ? to_f32<T>(src[j]) : 0.f;
    }
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = fmaxf(amax, finite_abs(y[j]));
    amax = fmaxf(amax, __shfl_xor(amax, 1, 64));
    amax = fmaxf(amax, __shfl_xor(amax, 2, 64));
    const unsigned int byte = e4m3_byte(amax);
    uint2 q;
    q.x = e4m3_four(y[0], y[1], y[2], y[3], byte);
    q.y = e4m3_four(y[4], y[5], y[6], y[7], byte);
    reinterpret_cast<uint2 *>(out.values)[i] = q;
    if (i % 4 == 0) out.exps[i / 4] = (uint8_t)byte;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) rows8_unpack_kernel(smoe_rows8 in, long long chunks, int per_row, int d, T *__restrict__ X) {
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (long long)gridDim.x * 256) {
    const long long row = i / per_row;
    const int c = (int)(i - row * per_row) * 8;
    if (c >= d) continue;
    const uint2 q = reinterpret_cast<const uint2 *>(in.values)[i];
    const unsigned int byte = in.exps[i / 4];
    float y[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      typedef float f2 __attribute__((ext_vector_type(2)));
      const int w = h ? (int)q.y : (int)q.x;
      const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
      y[4 * h] = a[0]; y[4 * h + 1] = a[1]; y[4 * h + 2] = b[0]; y[4 * h + 3] = b[1];
    }
    const float scale = __uint_as_float(byte << 23);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] *= scale;
    T *dst = X + row * d + c;
    if (d % 8 == 0) {
#pragma unroll
      for (int p = 0; p < 8 * (int)sizeof(T) / 16; ++p) {
        vec v;
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) v[j] = from_f32<T>(y[p * (16 / (int)sizeof(T)) + j]);
        reinterpret_cast<vec *>(dst)[p] = v;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < d) dst[j] = from_f32<T>(y[j]);
    }
  }
}

// The weighted sum of k slots' rows, eight columns a thread; up to K rows in flight, read past the caches (each once).
template <int K>
__global__ void __launch_bounds__(256) combine_f16_kernel(const uint4 *__restrict__ Yhat, const uint8_t *__restrict__ exps, const float *__restrict__ g, bf16_t *__restrict__ Y,
                                                          long long chunks, int k, int per_row, int exps_row, int exp_chunks) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
  typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (long long)gridDim.x * 256) {
    const long long t = i / per_row;
    const int c = (int)(i - t * per_row);
    const u32x4 *src = reinterpret_cast<const u32x4 *>(Yhat) + t * k * per_row + c;
    const uint8_t *e = exps + t * k * exps_row + c / exp_chunks;
    const float *w = g + t * k;
    float acc[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) acc[q] = 0.f;
    for (int j0 = 0; j0 < k; j0 += K) {
      u32x4 row[K];
      float scale[K];
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (j0 + j < k) {
          row[j] = __builtin_nontemporal_load(src + (long long)(j0 + j) * per_row);
          scale[j] = w[j0 + j] * __uint_as_float(((unsigned int)e[(long long)(j0 + j) * exps_row] - 14u) << 23);
        }
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (j0 + j < k) {
          const f16x8 v = __builtin_bit_cast(f16x8, row[j]);
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[q] = fmaf(scale[j], (float)v[q], acc[q]);
        }
    }
    bf16x8 o;
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (bf16_t)acc[q];
    reinterpret_cast<bf16x8 *>(Y)[i] = o;
  }
}

// The weighted sum of up to K slots' rows in bf16, to within an eighth of their last place, with what rounding took from them, which lies where the sums go: the eight
// threads of 64 columns, which are one wavefront's, read it in front of writing those.
template <int K>
__global__ void __launch_bounds__(256) combine_rest_kernel(const uint4 *__restrict__ Yhat, const float *__restrict__ g, uint4 *Y, long long chunks, int k, int per_row) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (long long)gridDim.x * 256) {
    const long long t = i / per_row;                                 // per_row: whole eights
    const int c = (int)(i - t * per_row), at = c & 7;
    const u32x4 *src = reinterpret_cast<const u32x4 *>(Yhat) + t * k * per_row + c;
    const uint2 *rest = reinterpret_cast<const uint2 *>(Y + (i - at)) + at / 4;
    u32x4 row[K];
    uint2 bits[K];
    float w[K];
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (j < k) {
        row[j] = __builtin_nontemporal_load(src + (long long)j * per_row);
        bits[j] = rest[2 * j];
        w[j] = g[t * k + j];
      }
    float acc[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) acc[q] = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (j < k) {
        const unsigned int first = bits[j].x >> (2 * (at & 3)), second = bits[j].y >> (2 * (at & 3));
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const unsigned int upper = q & 1 ? row[j][q / 2] & 0xffff0000u : row[j][q / 2] << 16;
          acc[q] = fmaf(w[j], bf16_with_rest(upper, ((q < 4 ? first : second) >> (8 * (q & 3))) & 3u), acc[q]);
        }
      }
    bf16x8 o;
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (bf16_t)acc[q];
    __builtin_amdgcn_wave_barrier();
    Y[i] = __builtin_bit_cast(uint4, o);
  }
}

// A block packs one step of 128 of the contraction of 64 columns: rows of W into LDS, a thread takes 32 elements of a column.
template <typename T>
__global__ void __launch_bounds__(256) weights8_pack_kernel(const T *__restrict__ W, smoe_weights8 out, int groups, int steps) {
  __shared__ float tile[ROW8][65];
  const int e = blockIdx.z, step = blockIdx.y, g0 = blockIdx.x * 4;
  const int half_groups = groups / out.halves, half = out.d_out / out.halves;
  // column of W that column n of the layout holds, or -1
  auto source = [&](int n) {
    const int h = n / (half_groups * 16), in = n - h * half_groups * 16;
    return h < out.halves && in < half ? h * half + in : -1;
  };
  const int c = threadIdx.x & 63;
  const int col = source(g0 * 16 + c);
  for (int r = threadIdx.x >> 6; r < ROW8; r += 4) {
    const int k = step * ROW8 + r;
    tile[r][c] = col >= 0 && k < out.d_in ? to_f32<T>(W[((size_t)e * out.d_in + k) * out.d_out + col]) : 0.f;
  }
  __syncthreads();
  const int b = threadIdx.x >> 6, g = g0 + c / 16, n = c % 16;      // block of 32, group and column in it
  if (g >= groups) return;
  float y[BLOCK8], amax = 0.f;
#pragma unroll
  for (int i = 0; i < BLOCK8; ++i) {
    y[i] = tile[b * BLOCK8 + i][c];
    amax = fmaxf(amax, finite_abs(y[i]));
  }
  const unsigned int byte = e4m3_byte(amax);
  const size_t at = ((size_t)e * groups + g) * steps + step;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 q;
    q.x = e4m3_four(y[16 * h], y[16 * h + 1], y[16 * h + 2], y[16 * h + 3], byte);
    q.y = e4m3_four(y[16 * h + 4], y[16 * h + 5], y[16 * h + 6], y[16 * h + 7], byte);
    q.z = e4m3_four(y[16 * h + 8], y[16 * h + 9], y[16 * h + 10], y[16 * h + 11], byte);
    q.w = e4m3_four(y[16 * h + 12], y[16 * h + 13], y[16 * h + 14], y[16 * h + 15], byte);
    *reinterpret_cast<uint4 *>(out.values + at * 2048 + (2 * b + h) * 256 + n * 16) = q;
  }
  out.exps[at * 64 + n * 4 + b] = (uint8_t)byte;
}

int row_blocks(long long chunks) {
  const long long n = (chunks + 255) / 256;
  return (int)(n < 16384 ? n : 16384);
}

}  // namespace

int launch_rows8_pack(hipStream_t s, smoe_dtype dt, const void *X, int rows, int d, const smoe_rows8 &out) {
  const int per_row = pitch8(d) / 8;
  const long long chunks = (long long)rows * per_row;
  if (dt == SMOE_BF16) hipLaunchKernelGGL((rows8_pack_kernel<bf16_t>), dim3(row_blocks(chunks)), dim3(256), 0, s, (const bf16_t *)X, chunks, per_row, d, out);
  else hipLaunchKernelGGL((rows8_pack_kernel<float>), dim3(row_blocks(chunks)), dim3(256), 0, s, (const float *)X, chunks, per_row, d, out);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
int launch_rows8_unpack(hipStream_t s, smoe_dtype dt, const smoe_rows8 &in, int rows, int d, void *X) {
  const int per_row = pitch8(d) / 8;
  const long long chunks = (long long)rows * per_row;
  if (dt == SMOE_BF16) hipLaunchKernelGGL((rows8_unpack_kernel<bf16_t>), dim3(row_blocks(chunks)), dim3(256), 0, s, in, chunks, per_row, d, (bf16_t *)X);
  else hipLaunchKernelGGL((rows8_unpack_kernel<float>), dim3(row_blocks(chunks)), dim3(256), 0, s, in, chunks, per_row, d, (float *)X);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
int launch_combine_f16(hipStream_t s, const void *Yhat, const uint8_t *exps, int exp_cols, const float *g, void *Y, int T, int k, int d) {
  const int per_row = d / 8;
  const long long chunks = (long long)T * per_row;
  const dim3 grid(row_blocks(chunks)), block(256);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, (const uint4 *)Yhat, exps, g, (bf16_t *)Y, chunks, k, per_row, ceil_div(d, exp_cols), exp_cols / 8); };
  if (k == 1) go(combine_f16_kernel<1>);
  else if (k == 2) go(combine_f16_kernel<2>);
  else if (k <= 4) go(combine_f16_kernel<4>);
  else go(combine_f16_kernel<8>);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
int launch_combine_rest(hipStream_t s, const void *Yhat, const float *g, void *Y, int T, int k, int d) {
  const int per_row = d / 8;
  const long long chunks = (long long)T * per_row;
  const dim3 grid(row_blocks(chunks)), block(256);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, (const uint4 *)Yhat, g, (uint4 *)Y, chunks, k, per_row); };
  if (k == 1) go(combine_rest_kernel<1>);
  else if (k == 2) go(combine_rest_kernel<2>);
  else if (k <= 4) go(combine_rest_kernel<4>);
  else go(combine_rest_kernel<REST_SLOTS>);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
int launch_weights8_pack(hipStream_t s, smoe_dtype dt, const void *W, const smoe_weights8 &out) {
  const int groups = groups8(out.d_out, out.halves), steps = ceil_div(out.d_in, ROW8);
  const dim3 grid(ceil_div(groups, 4), steps, out.E);
  if (dt == SMOE_BF16) hipLaunchKernelGGL((weights8_pack_kernel<bf16_t>), grid, dim3(256), 0, s, (const bf16_t *)W, out, groups, steps);
  else hipLaunchKernelGGL((weights8_pack_kernel<float>), grid, dim3(256), 0, s, (const float *)W, out, groups, steps);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
