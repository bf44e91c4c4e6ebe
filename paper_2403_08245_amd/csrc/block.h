// The block around the experts (smoe_block.h): what api_block.hip and its kernels share.
#pragma once
#include "common.h"
#include "smoe_block.h"

// ---- gate.hip
constexpr int GATE_MAX_T = (1 << 26) - 64;      // a wavefront a token, in one launch
int launch_score_gate(hipStream_t s, const float *logits, const float *bias, int T, int E, int k, const smoe_gate_rule &rule, int32_t *idx, float *gates);
int launch_score_gate_bwd(hipStream_t s, const float *logits, const int32_t *idx, const float *dgates, int T, int E, int k, const smoe_gate_rule &rule,
                          float *dlogits);

// ---- norm.hip
constexpr int NORM_MAX_D = 32768, NORM_MAX_ROWS = 0x7fffffff - 63;
struct NormArgs {
  const void *X, *R, *weight;
  int rows, d;
  float eps;
  void *S, *Y;
  smoe_rows8 Y8;      // values NULL: none
  float *rstd;
};
struct NormBwdArgs {
  const void *dY, *dS, *S, *weight;
  const float *rstd;
  int rows, d;
  void *dX, *dweight;
  float *part;        // [norm_bwd_parts][d]
};
int launch_norm(hipStream_t s, smoe_dtype dt, const NormArgs &a);
int norm_bwd_parts(smoe_dtype dt, int rows, int d);
int launch_norm_bwd(hipStream_t s, smoe_dtype dt, const NormBwdArgs &a);

// ---- rows8.hip
constexpr int ROW8 = 128;      // rows of 8-bit elements are whole 128s: the contraction step of a matrix instruction and a cache line
constexpr int BLOCK8 = 32;     // elements that share a power of two
static inline int pitch8(int d) { return ceil_div(d, ROW8) * ROW8; }
static inline int groups8(int d_out, int halves) { return halves * 2 * ceil_div(d_out / halves, 32); }
int launch_rows8_pack(hipStream_t s, smoe_dtype dt, const void *X, int rows, int d, const smoe_rows8 &out);
int launch_rows8_unpack(hipStream_t s, smoe_dtype dt, const smoe_rows8 &in, int rows, int d, void *X);
// Y[t] = sum_j g[t k + j] Yhat[t k + j] of rows as S2S8Args has them with C_exps, rounded to bf16 once
// (exp_cols: the columns that share a power of two, 64 or 128)
int launch_combine_f16(hipStream_t s, const void *Yhat, const uint8_t *exps, int exp_cols, const float *g, void *Y, int T, int k, int d);
// The same of rows in bf16 and what rounding took from them (S2S8Args::rest), which lies in Y and makes way for the sums
constexpr int REST_SLOTS = 8;
int launch_combine_rest(hipStream_t s, const void *Yhat, const float *g, void *Y, int T, int k, int d);
int launch_weights8_pack(hipStream_t s, smoe_dtype dt, const void *W, const smoe_weights8 &out);

// ---- products (gemm8_decode.hip, gemm8_stream.hip)
// For sorted rows i: out[i or o[i]] = X[in(i)] W[e(i)], or the activation of it as packed rows [Tk, d_out / halves].
struct S2S8Args {
  smoe_rows8 X;
  smoe_weights8 W;
  RowMap a_map, c_map;
  const int32_t *offsets;
  int Tk;
  // [*, d_out] bf16; few rows, with `wide`: fp32; with C_exps [Tk, ceil(d_out / n)]: fp16 times 2^(exponent - 141), one for n columns of a row, n = 64 for few
  // rows and 128 for many
  void *C = nullptr;
  bool wide = false;
  uint8_t *C_exps = nullptr;
  // C in bf16 for sums of up to REST_SLOTS rows each, d_out a multiple of 64: what rounding took from a row goes where the sums will be, in two bits an element.
  // The place of 64 columns' sums, 128 bytes, has 16 for each row i % sum_k: words [32 columns][odd or even four of them], byte b, bits 2 g and 2 g + 1 for
  // column 8 g + 4 odd + b.  NULL: not kept.
  uint8_t *rest = nullptr;
  int sum_k = 1;
  smoe_rows8 H{nullptr, nullptr};  // in C's place: expert-sorted
  int act = SMOE_ACT_NONE;
  size_t call_weights = 0;         // bytes of all the weights that the call may read: past the last-level cache they are read past it
  int grid = 256, group_m = 4;     // of the persistent kernels (smoe_ctx)
  int tile_shape = 0;              // 0 chosen by size, 1 128 x 256 only, 2 256 x 256 only (smoe_ctx)
};
bool s2s8_stream_supported(const S2S8Args &a);
int launch_s2s8_stream(hipStream_t s, const S2S8Args &a);
int init_stream8_kernels();        // with the context's device current
int launch_s2s8_decode(hipStream_t s, const S2S8Args &a);

#if defined(__HIPCC__)
// The byte of the power of two of a block whose largest finite |x| is amax: e + 127 for the smallest e with amax 2^-e <= 448 = 1.75 * 2^8, i.e. the
// exponent of amax less 8, one more where its fraction is past 1.75.
__device__ __forceinline__ unsigned int e4m3_byte(float amax) {
  const unsigned int bits = __float_as_uint(amax);
  return (unsigned int)max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
}
// |x| where it is finite, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// x as it is rounded to e4m3 in a block of that byte (multiplying by 2^-e is exact but for values far below the smallest of e4m3)
__device__ __forceinline__ float e4m3_scaled(float x, unsigned int byte) {
  float y = x * __uint_as_float((254u - byte) << 23);
  if (byte == 247u) y = fabsf(y) > 240.f ? copysignf(240.f, y) : y;      // e = 120: the code above 240 would stand for 2^128
  return fabsf(x) < INFINITY ? y : NAN;
}
// Where x lies between the halves of steps around the bf16 number nearest to it, in quarters of a step: 0 .. 3, in bits 14 and 15
__device__ __forceinline__ unsigned int bf16_rest_at_14(float x) {
  const unsigned int u = __float_as_uint(x);
  return u + 0x7fffu + ((u >> 16) & 1u);
}
__device__ __forceinline__ unsigned int bf16_rest(float x) { return (bf16_rest_at_14(x) >> 14) & 3u; }
// The number back, in the middle of its quarter, from the upper half of its bits; zeros, infinities and NaN, and those under 2^-126, as they are
__device__ __forceinline__ float bf16_with_rest(unsigned int upper, unsigned int rest) {
  const bool plain = ((upper + 0x800000u) & 0x7f000000u) == 0u;      // exponents 0 and 255
  return __uint_as_float(plain ? upper : upper + (rest << 14) - 0x6000u);
}
__device__ __forceinline__ unsigned int e4m3_four(float a, float b, float c, float d, unsigned int byte) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_scaled(a, byte), e4m3_scaled(b, byte), 0, false);
  return (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_scaled(c, byte), e4m3_scaled(d, byte), lo, true);
}
#endif
