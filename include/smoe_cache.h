/*
 * smoe_cache.h -- C ABI of libsmoe, positions and serving: rotary positions of queries and keys, a paged cache of keys
 * and values, attention of new tokens over it, and the decoding pass of the SMoE attention layer (Alg. 4) that runs them.
 *
 * The conventions are those of smoe.h: device pointers (unless said otherwise) on the context's device, contiguous
 * row-major tensors, int32 indices, no allocation, no synchronisation and no host copies, workspaces from the caller,
 * errors found before anything is enqueued, outputs overwritten, identical calls give identical bits.  Every tensor starts on a
 * 16-byte line.  Outputs and workspaces that lie over a cache's pages are SMOE_ERR_INVALID_ARG.  The contents of index arrays live on
 * the device: values out of range never lead to an access out of bounds; what they do instead is said at each entry point.
 */
#ifndef SMOE_CACHE_H_
#define SMOE_CACHE_H_

#include "smoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions ------------------------------------------------------------------------------------------
 * A row of d_head elements at position p has its first `rot` elements taken as rot / 2 pairs (a, b), and pair i turned by the
 * angle w = 2 pi p f_i, f_i turns per position:
 *     a' = m (a cos w - b sin w),   b' = m (a sin w + b cos w);      elements from `rot` on are copied.
 * Pair i is elements (i, i + rot / 2), or (2 i, 2 i + 1) when interleaved.  m (`amplitude`) is 1 unless the scaling says so.
 *
 * The frequencies are kept as 64-bit fractions of a turn: p f_i modulo one turn is then one integer product that wraps, exact at
 * every position int32 holds, where a product of 32-bit floating numbers is off by 2 pi p f_i 2^-24 (0.06 at a million). */
typedef struct {
  const uint64_t *turns; /* [rot / 2] device: frac(f_i) * 2^64 */
  int32_t rot;           /* even, 2 .. d_head */
  int32_t interleaved;   /* 0 or 1 */
  float amplitude;       /* m */
} smoe_rotary;

/* How the frequencies are stretched for contexts longer than the `trained_length` positions of training, by `factor` s >= 1:
 *   NONE    2 pi f_i = base^(-2 i / rot)
 *   LINEAR  the same, divided by s (positions interpolated)
 *   BASE    of the longer base `base s^(rot / (rot - 2))`: the fastest pair as it was, the slowest s times slower
 *   BLEND   pairs that turn 32 times or more within trained_length as they were, those that turn once or less divided by s, in
 *           between by their number of turns; m = 1 + 0.1 ln s */
typedef enum { SMOE_ROTARY_NONE = 0, SMOE_ROTARY_LINEAR = 1, SMOE_ROTARY_BASE = 2, SMOE_ROTARY_BLEND = 3 } smoe_rotary_scaling;

/* Fills the HOST arrays turns[rot / 2] and amplitude[1] (host call; the caller copies turns to the device once).
 * rot even and positive, base > 1, factor >= 1, trained_length > 0 (read by BLEND only). */
int smoe_rotary_frequencies(int rot, double base, int scaling, double factor, double trained_length, uint64_t *turns,
                            float *amplitude);

/* Turns the rows of Q [rows, hq, d_head] and K [rows, hk, d_head] into Qr and Kr of the same shapes and dtype (F32 or BF16;
 * computed in fp32, rounded once).  Row i's position is positions[i], any int32, or i % T when positions is NULL (T >= 1).
 * K may be NULL (hk = 0, Kr = NULL).  Qr = Q and Kr = K turn in place; any other overlap of an output with an input or
 * output is SMOE_ERR_INVALID_ARG.  d_head a multiple of 8, at most 512, else SMOE_ERR_UNSUPPORTED.  rows = 0 is a no-op. */
int smoe_rotary_fwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *Q, int hq, const void *K, int hk, int rows,
                    int d_head, int T, const int32_t *positions, const smoe_rotary *rotary, void *Qr, void *Kr);
/* The gradient: dQ and dK from the upstream dQr and dKr (turned back by the same angles, times m). */
int smoe_rotary_bwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *dQr, int hq, const void *dKr, int hk, int rows,
                    int d_head, int T, const int32_t *positions, const smoe_rotary *rotary, void *dQ, void *dK);

/* ---- paged cache --------------------------------------------------------------------------------------------------
 * Keys and values of h heads live in `pages` pages of `page` positions each, as K, V [pages, h, page, d_head].
 *   BF16  the rows as they are.
 *   E4M3  8-bit floating point (4 exponent and 3 mantissa bits, largest value 448, no infinities) with one power of two for each row
 *         and head: x is stored as round(x 2^-e) to the nearest, ties to even, and stands for it times 2^e; e is the smallest
 *         whole number >= -126 for which the row's largest finite |x| 2^-e is at most 448, kept as e + 127 in K_exp, V_exp
 *         [pages, h, page].  Powers of two cost a floating format no precision.  Infinities and NaN are stored as NaN; finite values that
 *         would come out as 2^128 (from 1.9375 * 2^127 on) are stored as 240 * 2^120.  The stored values are exact in bf16 for
 *         e >= -124, and for the rows of smaller e that were bf16 when they were stored; a key turned or projected as it is stored
 *         (in fp32) may hold steps under bf16's least there, and is read rounded to the nearest.
 * page is a power of two, 16 .. 65536; d_head 64 or 128; K_exp and V_exp are NULL for BF16.  Calls that write to a cache refuse one whose
 * arrays share memory. */
typedef enum { SMOE_CACHE_BF16 = 0, SMOE_CACHE_E4M3 = 1 } smoe_cache_format;
typedef struct {
  void *K, *V;             /* bf16 or e4m3 */
  uint8_t *K_exp, *V_exp;
  int32_t pages, page, h, d_head;
  int32_t format;          /* smoe_cache_format */
} smoe_cache;

/* Which place in the cache the rows of a call mean.  block_table [sequences, width]: the page that holds positions
 * j * page .. j * page + page - 1 of a sequence.  Either
 *   seqs [rows], positions [rows] given, lens NULL: row i is that position of that sequence, in any order; or
 *   lens [sequences] given, seqs and positions NULL: rows = sequences * N, and row b * N + n is position
 *     lens[b] - N + n (at least -2^31) of sequence b: the last N positions of every sequence.
 * A row whose sequence is outside [0, sequences), whose position is negative or past the table's width * page positions, or whose
 * page is outside [0, pages) has no place (padding). */
typedef struct {
  const int32_t *block_table;
  int32_t sequences, width;
  const int32_t *seqs, *positions, *lens;
} smoe_places;

/* Writes the rows K, V [rows, h, d_head] (bf16) to their places; rows without one are left out.  Two rows with the same place in
 * one call leave a mixture of the two there.  With `rotary`, K is turned by its position first, in fp32 and rounded once
 * as it is stored, and the rows of Q [rows, hq, d_head] are turned into Qr (Q NULL: keys only; Qr = Q in place; rows without a place
 * are turned by whatever their position says).  rotary NULL: Q and Qr NULL. */
int smoe_cache_append(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const smoe_cache *cache, const smoe_places *places,
                      const void *K, const void *V, int rows, const smoe_rotary *rotary, const void *Q, int hq, void *Qr);

/* Reads the rows' places back into K, V [rows, h, d_head] (bf16); rows without one become zeros.  K and V do not overlap. */
int smoe_cache_read(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const smoe_cache *cache, const smoe_places *places, int rows,
                    void *K, void *V);

/* ---- attention of new tokens over the cache ---------------------------------------------------------------------------
 * The decoding form of smoe_attention_fwd: softmax(q k^T / sqrt(d_head)) v of the last N positions of every sequence over the keys and
 * values in the cache, their own (written before) among them.  Q and O [B, N, G, h, d_head] bf16 (B sequences, G = k slots per token,
 * h heads per expert), head hh of every slot on key/value head hh; LSE [B, N, G, h] fp32, the log-sum-exp.
 * lens [B] counts the new positions in: query n sits at position p = lens[b] - N + n and attends positions 0 .. p.
 * A query with p < 0, or whose visible scores are all -infinity, attends nothing: O = 0, LSE = -infinity.  What lies in the cache at
 * positions that a query does not see never reaches it, NaN and infinities included.  Lengths count as at most width * page, and
 * positions on pages outside [0, pages) are not seen.
 * The places' seqs and positions are not read (NULL).  N >= 1, G >= 1.  O may be Q; else Q, O, LSE and the workspace do not overlap.  The workspace holds the partial sums of sequences that
 * several blocks share; none is needed (0, ws may be NULL) where the table holds at most 512 positions.  The query looks at sizes only, and
 * gives 0 for sizes that the call refuses, too. */
size_t smoe_cached_attention_workspace_bytes(const smoe_cache *cache, const smoe_places *places, int N, int G);
int smoe_cached_attention_fwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *Q, int N, int G, const smoe_cache *cache,
                              const smoe_places *places, void *O, float *LSE, void *ws, size_t ws_bytes);

/* ---- decoding pass of the SMoE attention layer, Alg. 4 --------------------------------------------------------------
 * smoe_momha_fwd for the last N positions of every sequence, over a cache that holds the earlier ones:
 *   K = X W_K, V = X W_V and Q = ParallelLinear(X, W_Q, o), Q and K turned (rotary, or NULL), K and V appended, attention over the cache,
 *   O = ParallelLinear(Ohat, W_O, o, p).
 * What the layer's tensors are rounded to follows from the batch: up to 512 rows, d_model a multiple of 32 and 32 rows an expert or fewer on
 * average, K and V are rounded once, as they are stored, Ohat once, and Q and the slots' outputs are fp32; past that Q and the slots'
 * outputs are bf16, and past 512 rows or off the multiple of 32 so are K and V before they are turned.  (Error of O against 64 bits,
 * root mean square: 1.6e-3 to 2.4e-3, and 3.0e-3 to 3.7e-3.)
 * X, O [B * N, d_model] in sequence order; weights, r, k and gates as in smoe_momha_fwd with T = N (h_expert and d_head
 * are the cache's).  lens counts the new positions in; rows past the table's end or with lens[b] < N are computed but not stored.
 * O may be X; the workspace lies apart from X, gates and O, and O from gates (else SMOE_ERR_INVALID_ARG). */
size_t smoe_momha_decode_workspace_bytes(int B, int N, int k, int d_model, int h_expert, int d_head);
int smoe_momha_decode(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *X, int N, int d_model, const void *W_K,
                      const void *W_V, const void *W_Q, const void *W_O, const smoe_routing *r, int k, const float *gates,
                      const smoe_cache *cache, const smoe_places *places, const smoe_rotary *rotary, void *O, void *ws,
                      size_t ws_bytes);

#ifdef __cplusplus
}
#endif
#endif /* SMOE_CACHE_H_ */
