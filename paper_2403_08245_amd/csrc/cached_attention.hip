// Attention of the last N positions of every sequence over the paged cache.
#include "cache.h"

namespace {

struct Dims {
  int N, G, shift;
};

// 8 stored elements of a row, as fp32
template <int FORMAT> __device__ __forceinline__ void stored8(const void *pages, const uint8_t *exps, size_t row, int d, int e0, float (&y)[8]) {
  if constexpr (FORMAT == SMOE_CACHE_BF16) {
    typedef bf16_t vec __attribute__((ext_vector_type(8)));
    const vec v = *reinterpret_cast<const vec *>((const bf16_t *)pages + row * d + e0);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (float)v[i];
  } else {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const uint2 q = *reinterpret_cast<const uint2 *>((const uint8_t *)pages + row * d + e0);
    const float scale = e4m3_scale(exps[row]);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, true);
    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, true);
    y[0] = a[0] * scale; y[1] = a[1] * scale; y[2] = b[0] * scale; y[3] = b[1] * scale;
    y[4] = c[0] * scale; y[5] = c[1] * scale; y[6] = e[0] * scale; y[7] = e[1] * scale;
  }
}

// One block of four wavefronts for each query row and head.  A wavefront takes every fourth 64 keys, one a lane; its lanes then
// hold d / 64 elements of the output each.
template <int D, int FORMAT>
__global__ void __launch_bounds__(256) cached_attention_kernel(const bf16_t *Q, smoe_cache c, smoe_places p, Dims dim, bf16_t *O, float *LSE) {
  __shared__ float q[D], part[4][D], top[4], sum[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, R = dim.N * dim.G;
  const size_t unit = blockIdx.x;              // ((b, n, g), head)
  const int hh = (int)(unit % c.h);
  const int b = (int)(unit / c.h / R), r = (int)(unit / c.h % R);
  const long long cap = (long long)p.width * c.page;
  const int len = (int)max(0ll, min((long long)p.lens[b], cap)), seen = len - dim.N + r / dim.G + 1;
  for (int i = threadIdx.x; i < D; i += 256) q[i] = (float)Q[unit * D + i];
  __syncthreads();
  constexpr int PER = D / 64;
  float m = -INFINITY, l = 0.f, acc[PER] = {};
  for (int k0 = wave * 64; k0 < seen; k0 += 256) {
    const int key = k0 + lane;
    const int id = key < seen ? find_page(p, c.pages, dim.shift, b, key) : -1;
    const size_t row = ((size_t)id * c.h + hh) * c.page + (key & (c.page - 1));
    float s = -INFINITY;
    if (id >= 0) {
      s = 0.f;
      for (int e = 0; e < D; e += 8) {
        float y[8];
        stored8<FORMAT>(c.K, c.K_exp, row, D, e, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(q[e + i], y[i], s);
      }
      s *= rsqrtf((float)D);
    }
    float mx = s;
    for (int x = 32; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
    const float m_new = fmaxf(m, mx), base = m_new == -INFINITY ? 0.f : m_new;
    const float w = expf(s - base), alpha = expf(m - base);
    l = l * alpha + w;
    m = m_new;
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] *= alpha;
    for (int kk = 0; kk < 64; ++kk) {
      const int idk = __shfl(id, kk, 64);
      const float wk = __shfl(w, kk, 64);
      if (idk < 0) continue;
      const size_t rk = ((size_t)idk * c.h + hh) * c.page + ((k0 + kk) & (c.page - 1));
      float y[8];
      stored8<FORMAT>(c.V, c.V_exp, rk, D, lane * PER & ~7, y);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        float v = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) v = ((lane * PER + i) & 7) == t ? y[t] : v;
        acc[i] = fmaf(wk, v, acc[i]);
      }
    }
  }
  for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x, 64);
  if (lane == 0) { top[wave] = m; sum[wave] = l; }
#pragma unroll
  for (int i = 0; i < PER; ++i) part[wave][lane * PER + i] = acc[i];
  __syncthreads();
  const float M = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), base = M == -INFINITY ? 0.f : M;
  float total = 0.f, scale[4];
  for (int i = 0; i < 4; ++i) { scale[i] = expf(top[i] - base); total += sum[i] * scale[i]; }
  for (int i = threadIdx.x; i < D; i += 256) {
    float o = 0.f;
    for (int k = 0; k < 4; ++k) o += part[k][i] * scale[k];
    O[unit * D + i] = (bf16_t)(total == 0.f ? 0.f : o / total);
  }
  if (threadIdx.x == 0) LSE[unit] = total == 0.f ? -INFINITY : M + logf(total);
}

}  // namespace

size_t cached_attention_workspace_bytes(int N, int G, int d_head) {
  (void)N; (void)G; (void)d_head;
  return 256;
}

int launch_cached_attention(hipStream_t s, const void *Q, int N, int G, const smoe_cache &c, const smoe_places &p, void *O, float *LSE, void *ws) {
  (void)ws;
  const Dims dim{N, G, __builtin_ctz((unsigned int)c.page)};
  const unsigned int blocks = (unsigned int)((size_t)p.sequences * N * G * c.h);
  auto go = [&](auto kernel) { kernel<<<blocks, 256, 0, s>>>((const bf16_t *)Q, c, p, dim, (bf16_t *)O, LSE); };
  if (c.d_head == 128) c.format == SMOE_CACHE_BF16 ? go(cached_attention_kernel<128, SMOE_CACHE_BF16>) : go(cached_attention_kernel<128, SMOE_CACHE_E4M3>);
  else c.format == SMOE_CACHE_BF16 ? go(cached_attention_kernel<64, SMOE_CACHE_BF16>) : go(cached_attention_kernel<64, SMOE_CACHE_E4M3>);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}
