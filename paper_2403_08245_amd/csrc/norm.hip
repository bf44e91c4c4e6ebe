// The root-mean-square norm of the residual stream with the addition in front of it, its gradient, and its output in 8 bits.
// Bound: HBM, each tensor read or written once; a row stays in registers between its sum and its output.  Rows of 2048 in bf16, 8192 of them: forward 22.5 us
// (134 MB, 6.0 TB/s), with 8 bits besides 27.5, 8 bits only 21, gradient 30 (4.5 TB/s); 8191 of 4096: 46, 57, 44, 51; 4000 of 5001, whose rows start off the
// 16-byte lines: 43 (3.7 TB/s), 46, 41, 75 (loads of single elements: 66, 80, 69, 85).
#include "block.h"
#include <algorithm>
#include <type_traits>

namespace {

// Eight elements of a row in memory.  WHOLE: rows are whole eights, on 16-byte lines; else a row starts on any element, and its last `n` may be fewer.
template <typename T, bool WHOLE> struct Chunks {
  static constexpr int PER = 16 / sizeof(T), N = 8 / PER;
  typedef T vec __attribute__((ext_vector_type(PER)));
  typedef T loose __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
  vec v[N];
  __device__ __forceinline__ void load(const T *p, int n) {
    if (WHOLE || n >= 8) {
#pragma unroll
      for (int q = 0; q < N; ++q) v[q] = WHOLE ? reinterpret_cast<const vec *>(p)[q] : *reinterpret_cast<const loose *>(p + q * PER);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i / PER][i % PER] = i < n ? p[i] : from_f32<T>(0.f);
    }
  }
  __device__ __forceinline__ void store(T *p, int n) const {
    if (WHOLE || n >= 8) {
#pragma unroll
      for (int q = 0; q < N; ++q) {
        if (WHOLE) reinterpret_cast<vec *>(p)[q] = v[q];
        else *reinterpret_cast<loose *>(p + q * PER) = v[q];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < n) p[i] = v[i / PER][i % PER];
    }
  }
};
// Eight elements as they are worked on
template <typename T, bool WHOLE> struct Pack {
  float v[8];
  __device__ __forceinline__ void load(const T *p, int n) {
    Chunks<T, WHOLE> x;
    x.load(p, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(x.v[i / x.PER][i % x.PER]);
  }
  __device__ __forceinline__ void store(T *p, int n) const {
    Chunks<T, WHOLE> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i / x.PER][i % x.PER] = from_f32<T>(v[i]);
    x.store(p, n);
  }
};
// the same, kept as they come
template <typename T, bool WHOLE> struct Raw : Chunks<T, WHOLE> {
  using C = Chunks<T, WHOLE>;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) C::v[i / C::PER][i % C::PER] = from_f32<T>(0.f);
  }
  __device__ __forceinline__ float get(int i) const { return to_f32<T>(C::v[i / C::PER][i % C::PER]); }
};

// sum over the TPR threads of a row, in all of them; `slot`: LDS of the row's wavefronts
template <int TPR> __device__ __forceinline__ float row_sum(float v, float *slot) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();                                   // the last sum has been read
    if ((threadIdx.x & 63) == 0) slot[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += slot[w];
  }
  return v;
}

// eight elements of a block of 32 per lane
__device__ __forceinline__ void store8(const float (&y)[8], uint8_t *values, uint8_t *exps, int col) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(y[i]));
  amax = fmaxf(amax, __shfl_xor(amax, 1, 64));
  amax = fmaxf(amax, __shfl_xor(amax, 2, 64));
  const unsigned int byte = e4m3_byte(amax);
  uint2 q;
  q.x = e4m3_four(y[0], y[1], y[2], y[3], byte);
  q.y = e4m3_four(y[4], y[5], y[6], y[7], byte);
  *reinterpret_cast<uint2 *>(values + col) = q;
  if (col % BLOCK8 == 0) exps[col / BLOCK8] = (uint8_t)byte;
}

// TPR threads a row, NV packs of eight elements each; rows wider than that are another instantiation's.
template <typename T, bool WHOLE, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 64 ? TPR : 256) norm_kernel(NormArgs a, int pitch) {
  constexpr int V = 8, ROWS = TPR > 64 ? 1 : 256 / TPR;
  __shared__ float s_sum[16];
  const int t = threadIdx.x % TPR;
  const long long row = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
  if (row >= a.rows) return;                           // with several rows a block each is one wavefront's
  const size_t at = (size_t)row * a.d;
  Pack<T, WHOLE> x[NV], w[NV];
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + t) * V;
#pragma unroll
    for (int q = 0; q < V; ++q) x[i].v[q] = w[i].v[q] = 0.f;
    if (c < a.d) {
      x[i].load((const T *)a.X + at + c, a.d - c);
      w[i].load((const T *)a.weight + c, a.d - c);
      if (a.R) {
        Pack<T, WHOLE> r;
        r.load((const T *)a.R + at + c, a.d - c);
#pragma unroll
        for (int q = 0; q < V; ++q) x[i].v[q] += r.v[q];
      }
    }
#pragma unroll
    for (int q = 0; q < V; ++q) sum = fmaf(x[i].v[q], x[i].v[q], sum);
  }
  sum = row_sum<TPR>(sum, s_sum);
  const float square = sum / (float)a.d + a.eps;
  float rstd = 1.0f / sqrtf(square), by = 1.0f;        // y = s by rstd weight
  // Squares past fp32's range, or so far under 1 that they lose bits or vanish, with an eps that does not hide that: the same of values `by` times as large.
  const bool large = !(square < INFINITY);
  if (__builtin_expect(large || (sum < (float)a.d * 0x1p-100f && a.eps < 0x1p-80f), 0)) {
    by = large ? 0x1p-70f : 0x1p100f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float y = x[i].v[q] * by;
        sum = fmaf(y, y, sum);
      }
    sum = row_sum<TPR>(sum, s_sum);
    rstd = 1.0f / sqrtf(sum / (float)a.d + a.eps * by * by);
  }
  if (a.rstd && t == 0) a.rstd[row] = by * rstd;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + t) * V;
    if (c < a.d) {
      if (a.S) x[i].store((T *)a.S + at + c, a.d - c);
#pragma unroll
      for (int q = 0; q < V; ++q) x[i].v[q] = x[i].v[q] * by * rstd * w[i].v[q];
      if (a.Y) x[i].store((T *)a.Y + at + c, a.d - c);
      if (!WHOLE && c + V > a.d) {                     // 0 by an rstd of NaN or infinity is no zero
#pragma unroll
        for (int q = 0; q < V; ++q) x[i].v[q] = c + q < a.d ? x[i].v[q] : 0.f;
      }
    }
    if (a.Y8.values && c < pitch) store8(x[i].v, a.Y8.values + (size_t)row * pitch, a.Y8.exps + (size_t)row * (pitch / BLOCK8), c);
  }
}

// Gradient.  A block's rows (ROWS at a time, TPR threads each) lie gridDim.x * ROWS apart; the next ones are requested before the present ones' sum is
// taken, so that HBM does not wait for it.  Up to 2048 elements a wavefront has a row to itself and no barrier stands in the loop (8192 rows of
// 2048 in bf16, with the sum of the parts: 256 threads a row, nothing requested ahead, 45 us; so 30, 134 MB at 4.9 TB/s in the larger kernel).  A block leaves its sum of dweight.
template <typename T, bool WHOLE, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) norm_bwd_kernel(NormBwdArgs a) {
  constexpr int V = 8, ROWS = TPR > 256 ? 1 : 256 / TPR;
  constexpr bool LEAN = TPR > 512;       // 128 registers a thread: neither the next row nor the weights are held
  __shared__ float s_sum[16];
  __shared__ float s_dw[ROWS > 1 ? NV * TPR * V : 1];
  const int t = threadIdx.x % TPR, mine = threadIdx.x / TPR;
  Pack<T, WHOLE> w[NV];
  float dw[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + t) * V;
#pragma unroll
    for (int q = 0; q < V; ++q) dw[i][q] = w[i].v[q] = 0.f;
    if (c < a.d && !LEAN) w[i].load((const T *)a.weight + c, a.d - c);
  }
  struct Row {
    Raw<T, WHOLE> s[NV], dy[NV], ds[NV];
    float rstd;
  };
  auto request = [&](long long row) {
    Row r;
    const size_t at = (size_t)row * a.d;
    r.rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + t) * V;
      if (c < a.d) {
        r.s[i].load((const T *)a.S + at + c, a.d - c);
        r.dy[i].load((const T *)a.dY + at + c, a.d - c);
        if (a.dS && !LEAN) r.ds[i].load((const T *)a.dS + at + c, a.d - c);
      } else {
        r.s[i].clear();
        r.dy[i].clear();
      }
    }
    return r;
  };
  const long long step = (long long)gridDim.x * ROWS;
  long long row = (long long)blockIdx.x * ROWS + mine;
  if (row < a.rows) {
    Row now = request(row);
    for (; row < a.rows; row += step) {
      // dX may be dS, S or dY: the next row is another one, and each element is read before it is written by the thread that reads it
      Row next;
      if constexpr (!LEAN) next = request(row + step < a.rows ? row + step : row);
      float u[NV][V], g[NV][V], dot = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < V; ++q) {
          u[i][q] = now.s[i].get(q) * now.rstd;
          g[i][q] = now.dy[i].get(q);
          dw[i][q] = fmaf(g[i][q], u[i][q], dw[i][q]);
        }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * V;
        if (LEAN && c < a.d) w[i].load((const T *)a.weight + c, a.d - c);
#pragma unroll
        for (int q = 0; q < V; ++q) {
          g[i][q] *= w[i].v[q];
          dot = fmaf(g[i][q], u[i][q], dot);
        }
      }
      const float mean = row_sum<TPR>(dot, s_sum) / (float)a.d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * V;
        if (c < a.d) {
          Pack<T, WHOLE> o;
          if (LEAN && a.dS) now.ds[i].load((const T *)a.dS + (size_t)row * a.d + c, a.d - c);
#pragma unroll
          for (int q = 0; q < V; ++q) o.v[q] = now.rstd * (g[i][q] - u[i][q] * mean) + (a.dS ? now.ds[i].get(q) : 0.f);
          o.store((T *)a.dX + (size_t)row * a.d + c, a.d - c);
        }
      }
      if constexpr (!LEAN) now = next;
      else if (row + step < a.rows) now = request(row + step);
    }
  }
  // the block's sum, in the order of its wavefronts
  if constexpr (ROWS > 1) {
#pragma unroll
    for (int m = 0; m < ROWS - 1; ++m) {
      if (mine == m) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int q = 0; q < V; ++q) s_dw[(i * V + q) * TPR + t] = dw[i][q];
      }
      __syncthreads();
      if (mine == m + 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int q = 0; q < V; ++q) dw[i][q] += s_dw[(i * V + q) * TPR + t];
      }
      __syncthreads();
    }
    if (mine != ROWS - 1) return;
  }
  float *part = a.part + (size_t)blockIdx.x * a.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + t) * V;
    if (c < a.d) {
#pragma unroll
      for (int q = 0; q < V; ++q)
        if (WHOLE || c + q < a.d) part[c + q] = dw[i][q];
    }
  }
}

// dweight = the sum of the parts: 16 columns a block, each in 64 shares that are added in a fixed order.  In 64 bits: up to 512 parts of either sign, whose sum is often smaller than
// they are (1999 rows of 999 in fp32: error against 64 bits 1.24e-7 in 32 bits, 0.77e-7 so, 0.61e-7 a sum in 64 bits throughout)
template <typename T> __global__ void __launch_bounds__(1024) norm_dweight_kernel(const float *__restrict__ part, int parts, int d, T *__restrict__ dweight) {
  __shared__ double s_part[64][16];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), share = threadIdx.x >> 4;
  double sum = 0.0;
  if (c < d) {
#pragma unroll 8
    for (int p = share; p < parts; p += 64) sum += (double)part[(size_t)p * d + c];
  }
  s_part[share][threadIdx.x & 15] = sum;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  sum = 0.0;
#pragma unroll
  for (int q = 0; q < 16; ++q) sum += s_part[(threadIdx.x >> 4) * 16 + q][threadIdx.x & 15];
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (threadIdx.x < 16 && c < d) dweight[c] = from_f32<T>((float)sum);
}

// The shape for rows of d elements: threads a row, packs a thread.
template <typename F> struct Shapes {
  int d;
  F f;
  template <int TPR, int NV> void go() const {
    if (d % 8 == 0) f(std::true_type{}, std::integral_constant<int, TPR>{}, std::integral_constant<int, NV>{});
    else f(std::false_type{}, std::integral_constant<int, TPR>{}, std::integral_constant<int, NV>{});
  }
};
// Two wavefronts a row in fp32, whose packs are two loads each, where in bf16 one holds a row's two packs.  Rows of x and r in us, one / two: fp32, 1999 of 999 9.4 / 9.1 (x
// alone 6.1 / 5.7), 200 of 700 4.2 / 3.5, 8192 of 1024 24.4 / 23; bf16, 16384 of 777 21.1 / 23.2, 2000 of 1024 4.8 / 4.8.
template <typename T, typename F> void by_shape(int d, F f) {
  const int packs = ceil_div(pitch8(d), 8);
  const Shapes<F> s{d, f};
  if (packs <= 64) s.template go<64, 1>();
  else if (packs <= 128 && sizeof(T) == 4) s.template go<128, 1>();
  else if (packs <= 128) s.template go<64, 2>();
  else if (packs <= 256) s.template go<256, 1>();
  else if (packs <= 512) s.template go<256, 2>();
  else if (packs <= 1024) s.template go<256, 4>();
  else if (packs <= 2048) s.template go<1024, 2>();
  else s.template go<1024, 4>();
}
// Of the gradient, whose registers hold two rows and the sums: a wavefront a row up to 2048 elements, two packs a thread from there on (4096 rows of 8192 in bf16, 256
// threads of four packs, one block a compute unit: 70 us; 512 of two 65).
template <typename F> void by_bwd_shape(int d, F f) {
  const int packs = ceil_div(pitch8(d), 8);
  const Shapes<F> s{d, f};
  if (packs <= 64) s.template go<64, 1>();
  else if (packs <= 128) s.template go<64, 2>();
  else if (packs <= 256) s.template go<64, 4>();
  else if (packs <= 512) s.template go<256, 2>();
  else if (packs <= 1024) s.template go<512, 2>();
  else if (packs <= 2048) s.template go<1024, 2>();
  else s.template go<1024, 4>();
}
constexpr int BWD_BLOCKS = 512;
constexpr int LAUNCH_ROWS = 1 << 21;       // a launch has fewer than 2^32 threads

template <typename T> int launch_norm_as(hipStream_t s, const NormArgs &all) {
  for (long long first = 0; first < all.rows; first += LAUNCH_ROWS) {
    NormArgs a = all;
    const size_t skip = (size_t)first * all.d;
    const int pitch = pitch8(all.d);
    a.rows = (int)std::min<long long>(all.rows - first, LAUNCH_ROWS);
    a.X = (const T *)all.X + skip;
    if (a.R) a.R = (const T *)all.R + skip;
    if (a.S) a.S = (T *)all.S + skip;
    if (a.Y) a.Y = (T *)all.Y + skip;
    if (a.rstd) a.rstd += first;
    if (a.Y8.values) {
      a.Y8.values += (size_t)first * pitch;
      a.Y8.exps += (size_t)first * (pitch / BLOCK8);
    }
    by_shape<T>(a.d, [&](auto whole, auto tpr, auto nv) {
      constexpr int TPR = decltype(tpr)::value, ROWS = TPR > 64 ? 1 : 256 / TPR;
      hipLaunchKernelGGL((norm_kernel<T, decltype(whole)::value, TPR, decltype(nv)::value>), dim3(ceil_div(a.rows, ROWS)), dim3(TPR > 64 ? TPR : 256), 0, s, a,
                         pitch);
    });
    SMOE_LAUNCH_CHECK();
  }
  return SMOE_OK;
}
template <typename T> int launch_norm_bwd_as(hipStream_t s, const NormBwdArgs &a) {
  const int parts = norm_bwd_parts(SMOE_BF16, a.rows, a.d);
  if (a.rows > 0) {
    by_bwd_shape(a.d, [&](auto whole, auto tpr, auto nv) {
      constexpr int TPR = decltype(tpr)::value;
      hipLaunchKernelGGL((norm_bwd_kernel<T, decltype(whole)::value, TPR, decltype(nv)::value>), dim3(parts), dim3(TPR > 256 ? TPR : 256), 0, s, a);
    });
    SMOE_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL((norm_dweight_kernel<T>), dim3(ceil_div(a.d, 16)), dim3(1024), 0, s, a.part, a.rows > 0 ? parts : 0, a.d, (T *)a.dweight);
  SMOE_LAUNCH_CHECK();
  return SMOE_OK;
}

}  // namespace

int launch_norm(hipStream_t s, smoe_dtype dt, const NormArgs &a) { return dt == SMOE_BF16 ? launch_norm_as<bf16_t>(s, a) : launch_norm_as<float>(s, a); }
int norm_bwd_parts(smoe_dtype, int rows, int d) {
  int per = 1;                   // rows a block has at a time
  by_bwd_shape(d, [&](auto, auto tpr, auto) { per = decltype(tpr)::value > 256 ? 1 : 256 / decltype(tpr)::value; });
  const int blocks = ceil_div(rows, per);
  return blocks < BWD_BLOCKS ? blocks : BWD_BLOCKS;
}
int launch_norm_bwd(hipStream_t s, smoe_dtype dt, const NormBwdArgs &a) {
  return dt == SMOE_BF16 ? launch_norm_bwd_as<bf16_t>(s, a) : launch_norm_bwd_as<float>(s, a);
}
