/*
 * smoe_block.h -- C ABI of libsmoe, a transformer block around its experts: the router's gate by scores, the root-mean-square norm of the
 * residual stream with the addition in front of it, and the experts' products (Alg. 1 and Alg. 3 forward) on activations and weights in 8 bits.
 *
 * The conventions are those of smoe.h: device pointers on the context's device, contiguous row-major tensors, int32 indices, no allocation,
 * no synchronisation and no host copies, workspaces from the caller, errors found before anything is enqueued, outputs overwritten,
 * identical calls give identical bits.  Every tensor starts on a 16-byte line.
 */
#ifndef SMOE_BLOCK_H_
#define SMOE_BLOCK_H_

#include "smoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- routing by scores --------------------------------------------------------------------------------------------------
 * The gate of Sec. 3.1 step 1 with scores of all experts, s = softmax(x) over the row's E logits or s = sigmoid(x) of each:
 *   1. rank[e] = s[e] + bias[e] (bias NULL: s[e]); the bias moves the choice, not the weights.
 *   2. With groups > 1, the experts are `groups` runs of E / groups; a group counts as the sum of its group_best largest ranks (of all it has,
 *      where it has fewer), and the kept_groups largest stay, ties to the lower group.
 *   3. The k largest ranks of the experts in them are kept, ties to the lower expert id, slots by descending rank.
 *   4. gates[t,j] = scale * s[e_j], divided by the sum of the k kept scores with `renormalise`.
 * Ranks that are scores alone (no bias, and groups that count by one expert or all stay) are compared as the exact scores are, which is as the logits are;
 * others, and sums of two, as 64-bit numbers, in which scores may be equal whose logits are not (sigmoids of logits over 37 are 1).  Gates are fp32.  A masked expert, whose logit is NaN or -inf, has score 0 and comes behind
 * every other of the kept groups, whatever its bias; so does one whose rank is NaN or -inf.  Such experts count nothing towards their
 * group, and a group of nothing else comes last.  Logits of +inf share the softmax equally, as do the logits of a row that are all masked; kept scores that
 * are all 0 share `scale` equally under `renormalise`.  Every slot of every token is written. */
typedef enum { SMOE_SCORE_SOFTMAX = 0, SMOE_SCORE_SIGMOID = 1 } smoe_score;
typedef struct {
  int32_t score;         /* smoe_score */
  int32_t groups;        /* 1 .. 64, divides E */
  int32_t kept_groups;   /* 1 .. groups; k <= kept_groups * E / groups */
  int32_t group_best;    /* 1 or 2 */
  int32_t renormalise;   /* 0 or 1 */
  float scale;           /* finite */
} smoe_gate_rule;

/* logits [T,E] fp32, bias [E] fp32 or NULL (in); expert_idxs [T*k] int32, gates [T*k] fp32 (out).  E <= 1024 and k <= 64, else
 * SMOE_ERR_UNSUPPORTED, as are more than 2^26 - 64 tokens.  T = 0 is a no-op. */
int smoe_score_gate(smoe_ctx *ctx, void *stream, const float *logits, const float *bias, int T, int E, int k, const smoe_gate_rule *rule,
                    int32_t *expert_idxs, float *gates);
/* Gradient of the gates with respect to the logits (the choice is piecewise constant, the bias has none):
 *   dlogits [T,E] fp32 (out, every entry written) from logits, expert_idxs and dgates [T*k].  An expert named by several slots of a token
 * gets the sum of their gradients; slots that name none in [0,E) have gate 0 and get none.  Masked experts have gradient 0.  dlogits may be the
 * logits themselves. */
int smoe_score_gate_bwd(smoe_ctx *ctx, void *stream, const float *logits, const int32_t *expert_idxs, const float *dgates, int T, int E, int k,
                        const smoe_gate_rule *rule, float *dlogits);

/* ---- rows in 8 bits --------------------------------------------------------------------------------------------------------
 * A row of d elements as e4m3 (4 exponent and 3 mantissa bits, largest value 448, no infinities) with a power of two for every 32 of them: x is
 * stored as round(x 2^-e) to the nearest, ties to even, and stands for it times 2^e; e is the smallest whole number >= -126 for which the
 * block's largest finite |x| 2^-e is at most 448, stored as e + 127.  Infinities and NaN are stored as NaN; finite values that would come out as
 * 2^128 (from 1.9375 * 2^127 on) are stored as 240 * 2^120.
 * Rows are as wide as whole 128s: values [rows, P] and exps [rows, P / 32] with P = 128 * ceil(d / 128); what lies behind the d elements
 * is stored as zeros are, and the products need it so. */
typedef struct {
  uint8_t *values, *exps;
} smoe_rows8;

/* X [rows, d] (F32 or BF16) -> out. */
int smoe_rows8_pack(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *X, int rows, int d, const smoe_rows8 *out);
/* The values that rows stand for -> X [rows, d]; those that bf16 does not hold (under 2^-133) are rounded. */
int smoe_rows8_unpack(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const smoe_rows8 *in, int rows, int d, void *X);

/* Weights W [E, d_in, d_out] in 8 bits, blocks of 32 along d_in (the contraction), laid out for the products: made once, by
 * smoe_weights8_pack, from F32 or BF16 weights.  halves = 2: the columns are [gate | up] (SWIGLU); else 1.
 * values takes smoe_weights8_bytes, exps a 32nd of it.  (Layout: each half's columns in groups of 16, padded with zeros to an even number of groups,
 * d_in in steps of 128, padded; values [E, groups, steps, 8, 16, 16]: 16 elements of the contraction of 16 columns, eight times; exps
 * [E, groups, steps, 16, 4].) */
typedef struct {
  uint8_t *values, *exps;
  int32_t E, d_in, d_out, halves;
} smoe_weights8;
size_t smoe_weights8_bytes(int E, int d_in, int d_out, int halves);   /* 0: bad sizes */
int smoe_weights8_pack(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *W, const smoe_weights8 *out);

/* ---- the norm of the residual stream -----------------------------------------------------------------------------------------
 * s = x + r;  rstd = 1 / sqrt(mean(s^2) + eps) over a row's d elements;  y = s rstd weight.
 *   X, R [rows, d], weight [d] of one dtype (F32 or BF16; R NULL: s = x).  Sums are fp32, and y is made from the unrounded s.
 *   S [rows, d] (out, nullable): s rounded once, the stream that goes on.  Y [rows, d] and Y8 (out, either may be NULL, not both): y in the
 *   dtype, and in 8 bits (packed from the unrounded y).  rstd [rows] fp32 (out, nullable): kept for the backward pass.
 * Squares that leave fp32's range at either end are no loss: y is that of the formula for every finite s and every eps, 0 included (rows of zeros are then 0 / 0); an rstd past
 * fp32's range, of rows under 2^-127, is kept as infinity, and the backward pass of such rows is not finite.
 * S and Y may be X or R themselves; any other overlap of an output with an input or output is SMOE_ERR_INVALID_ARG.  1 <= d <= 32768, else
 * SMOE_ERR_UNSUPPORTED; eps >= 0. */
int smoe_add_norm_fwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *X, const void *R, const void *weight, int rows, int d, float eps,
                      void *S, void *Y, const smoe_rows8 *Y8, float *rstd);
/* Gradients from dY, and from dS, that of S where the stream goes on (nullable): dX [rows, d] (that of R is the same) and dweight [d]:
 *   g = dY weight, u = s rstd;  dX = rstd (g - u mean(g u)) + dS;  dweight = sum over the rows of dY u.
 * S: the forward's (X itself where R was NULL).  dX may be dY, S or dS itself; any other overlap is SMOE_ERR_INVALID_ARG.  rows = 0 gives dweight = 0. */
size_t smoe_add_norm_bwd_workspace_bytes(smoe_dtype dtype, int rows, int d);
int smoe_add_norm_bwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *dY, const void *dS, const void *S, const void *weight,
                      const float *rstd, int rows, int d, void *dX, void *dweight, void *ws, size_t ws_bytes);

/* ---- the experts' products in 8 bits ---------------------------------------------------------------------------------------------
 * smoe_plinear_fwd on rows and weights in 8 bits, bf16 out: X [x_rows, d_in] and W (halves = 1) as packed, the other arguments as there;
 * d_out a multiple of 8.  No workspace.  Products are summed in fp32 over the contraction; the matrix instructions add each 64 or 128 of
 * them with an error of about 2^-12 of the largest (1.5e-5 of the sum for normal values), under the output's rounding.  With gates, Y is the sum
 * of the rows of Yhat as they were to within 2^-10 before their rounding to bf16, for gates_k up to 8 and d_out of whole 64s; else of the rounded ones.  Kernel modes 1 and 2 of
 * smoe_set_kernel_mode force the kernels for few rows, 3 and 4 the 128 x 256 / 256 x 256 tiles. */
int smoe_plinear8_fwd(smoe_ctx *ctx, void *stream, const smoe_rows8 *X, int x_rows, int d_in, const smoe_weights8 *W, int d_out, const smoe_routing *r,
                      int k, const float *gates, int gates_k, int grouped_in, int grouped_out, void *Yhat, void *Y);
/* The SMoE MLP (Alg. 3) forward: X [T, d_model] rows, W1 (halves = 2 for SWIGLU, else 1) and W2 (halves = 1) packed, gates [T*k] fp32,
 * Y [T, d_model] bf16 (out).  The hidden rows are packed to 8 bits from fp32 in the first product's epilogue, and a hidden value within the product's error of
 * a border between two codes may take either.  The kernels for few rows make that product from bf16 in fp32 (under 1e-4 of the codes differ from the definition's,
 * and Y is as near to it as its rounding allows); those for many rows by the 8-bit instructions (2e-3 of the codes, and Y's error in the root mean square is 1.2 to
 * 1.7 times its rounding's, with most of it in the few tokens whose largest hidden values are concerned).  The second product's rows are summed from fp32 or fp16 with
 * a power of two for 64 or 128 columns.  d_model a multiple of 8, d_expert any. */
size_t smoe_mlp8_fwd_workspace_bytes(smoe_act act, int T, int k, int d_model, int d_expert);
int smoe_mlp8_fwd(smoe_ctx *ctx, void *stream, smoe_act act, const smoe_rows8 *X, int T, int d_model, int d_expert, const smoe_weights8 *W1,
                  const smoe_weights8 *W2, const smoe_routing *r, int k, const float *gates, void *Y, void *ws, size_t ws_bytes);

#ifdef __cplusplus
}
#endif
#endif /* SMOE_BLOCK_H_ */
