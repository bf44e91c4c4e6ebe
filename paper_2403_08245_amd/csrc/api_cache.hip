// C ABI of libsmoe, positions and serving (smoe_cache.h): argument checks and launches.  The decoding pass of the attention layer is in
// api.hip, beside the layer's other passes.
#include "cache.h"
#include <cmath>

int cache_args_ok(const smoe_cache *c) {
  if (!c || !c->K || !c->V || c->pages < 1 || c->page < 1 || c->h < 1 || c->d_head < 1) return SMOE_ERR_INVALID_ARG;
  if (c->format != SMOE_CACHE_BF16 && c->format != SMOE_CACHE_E4M3) return SMOE_ERR_INVALID_ARG;
  if ((c->format == SMOE_CACHE_E4M3) != (c->K_exp != nullptr) || (c->K_exp != nullptr) != (c->V_exp != nullptr)) return SMOE_ERR_INVALID_ARG;
  if (c->page < 16 || c->page > 65536 || (c->page & (c->page - 1)) || (c->d_head != 64 && c->d_head != 128) || c->h > 65535) return SMOE_ERR_UNSUPPORTED;
  if (!aligned16(c->K) || !aligned16(c->V) || !aligned16(c->K_exp) || !aligned16(c->V_exp)) return SMOE_ERR_UNSUPPORTED;
  return SMOE_OK;
}
// the table, and positions that stay within 31 bits
static int table_ok(const smoe_cache *c, const smoe_places *p) {
  if (!p || !p->block_table || p->sequences < 1 || p->width < 1) return SMOE_ERR_INVALID_ARG;
  if ((long long)p->width * c->page > 0x7fff0000LL) return SMOE_ERR_UNSUPPORTED;
  return SMOE_OK;
}
int lengths_ok(const smoe_cache *c, const smoe_places *p) {
  int rc = table_ok(c, p);
  if (rc != SMOE_OK) return rc;
  return p->lens && !p->seqs && !p->positions ? SMOE_OK : SMOE_ERR_INVALID_ARG;
}
static int places_ok(const smoe_cache *c, const smoe_places *p, int rows) {
  int rc = table_ok(c, p);
  if (rc != SMOE_OK) return rc;
  if (p->lens) return !p->seqs && !p->positions && rows % p->sequences == 0 ? SMOE_OK : SMOE_ERR_INVALID_ARG;
  return rows == 0 || (p->seqs && p->positions) ? SMOE_OK : SMOE_ERR_INVALID_ARG;
}
int rotary_args_ok(const smoe_rotary *r, int d_head) {
  if (!r || !r->turns || r->rot < 2 || (r->rot & 1) || r->rot > d_head || (r->interleaved != 0 && r->interleaved != 1)) return SMOE_ERR_INVALID_ARG;
  if (((uintptr_t)r->turns & 7) || !std::isfinite(r->amplitude)) return SMOE_ERR_INVALID_ARG;
  return SMOE_OK;
}
bool over_pages(const smoe_cache *c, const void *p, size_t bytes) {
  const size_t rows = (size_t)c->pages * c->h * c->page, stored = rows * c->d_head * (c->format == SMOE_CACHE_BF16 ? 2 : 1);
  return overlap(p, bytes, c->K, stored) || overlap(p, bytes, c->V, stored) || overlap(p, bytes, c->K_exp, rows) || overlap(p, bytes, c->V_exp, rows);
}
bool pages_apart(const smoe_cache *c) {
  const size_t rows = (size_t)c->pages * c->h * c->page, stored = rows * c->d_head * (c->format == SMOE_CACHE_BF16 ? 2 : 1);
  return !overlap(c->K, stored, c->V, stored) && !overlap(c->K_exp, rows, c->V_exp, rows) && !overlap(c->K, stored, c->K_exp, rows) &&
         !overlap(c->K, stored, c->V_exp, rows) && !overlap(c->V, stored, c->K_exp, rows) && !overlap(c->V, stored, c->V_exp, rows);
}

extern "C" {

int smoe_rotary_frequencies(int rot, double base, int scaling, double factor, double trained_length, uint64_t *turns, float *amplitude) {
  if (rot < 2 || (rot & 1) || !turns || !amplitude || !(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor)) return SMOE_ERR_INVALID_ARG;
  if (scaling < SMOE_ROTARY_NONE || scaling > SMOE_ROTARY_BLEND) return SMOE_ERR_INVALID_ARG;
  if (scaling == SMOE_ROTARY_BLEND && (!(trained_length > 0.0) || !std::isfinite(trained_length))) return SMOE_ERR_INVALID_ARG;
  constexpr double TWO_PI = 6.283185307179586476925286766559;
  constexpr double FEW = 1.0, MANY = 32.0;      // turns within the trained length under which a pair is slow, over which it is fast
  if (scaling == SMOE_ROTARY_BASE && rot > 2) base *= std::pow(factor, rot / (rot - 2.0));
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot);
    if (scaling == SMOE_ROTARY_LINEAR) f /= factor;
    if (scaling == SMOE_ROTARY_BLEND) {
      const double keep = std::fmin(std::fmax((trained_length * f / TWO_PI - FEW) / (MANY - FEW), 0.0), 1.0);
      f = f / factor * (1.0 - keep) + f * keep;
    }
    turns[i] = (uint64_t)std::ldexp(f / TWO_PI, 64);   // f <= 1 radian, so under a sixth of a turn
  }
  *amplitude = scaling == SMOE_ROTARY_BLEND ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return SMOE_OK;
}

static int turn(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *Q, int hq, const void *K, int hk, int rows, int d, int T,
                const int32_t *positions, const smoe_rotary *rotary, void *Qr, void *Kr, bool back) {
  if (!ctx || (dtype != SMOE_F32 && dtype != SMOE_BF16) || rows < 0 || hq < 1 || hk < 0 || d < 1 || (!positions && T < 1)) return SMOE_ERR_INVALID_ARG;
  int rc = rotary_args_ok(rotary, d);
  if (rc != SMOE_OK) return rc;
  if (rows == 0) return SMOE_OK;
  if (!Q || !Qr || (hk > 0) != (K != nullptr) || (hk > 0) != (Kr != nullptr)) return SMOE_ERR_INVALID_ARG;
  if (d % 8 || d > 512 || hq > 65535 || hk > 65535) return SMOE_ERR_UNSUPPORTED;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Qr) || !aligned16(Kr)) return SMOE_ERR_UNSUPPORTED;
  const size_t q = (size_t)rows * hq * d * dtype_size(dtype), k = (size_t)rows * hk * d * dtype_size(dtype);
  if ((Qr != Q && overlap(Qr, q, Q, q)) || (Kr != K && overlap(Kr, k, K, k)) || overlap(Qr, q, K, k) || overlap(Kr, k, Q, q) || overlap(Qr, q, Kr, k))
    return SMOE_ERR_INVALID_ARG;
  TurnArgs a;
  a.Q = Q; a.K = K; a.Qr = Qr; a.Kr = Kr;
  a.hq = hq; a.hk = hk; a.rows = rows; a.d = d;
  a.T = positions ? 1 : T;
  a.positions = positions;
  a.rotary = *rotary;
  a.back = back;
  return launch_turn((hipStream_t)stream, dtype, a);
}

int smoe_rotary_fwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *Q, int hq, const void *K, int hk, int rows, int d_head, int T,
                    const int32_t *positions, const smoe_rotary *rotary, void *Qr, void *Kr) {
  return turn(ctx, stream, dtype, Q, hq, K, hk, rows, d_head, T, positions, rotary, Qr, Kr, false);
}
int smoe_rotary_bwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *dQr, int hq, const void *dKr, int hk, int rows, int d_head, int T,
                    const int32_t *positions, const smoe_rotary *rotary, void *dQ, void *dK) {
  return turn(ctx, stream, dtype, dQr, hq, dKr, hk, rows, d_head, T, positions, rotary, dQ, dK, true);
}

int smoe_cache_append(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const smoe_cache *cache, const smoe_places *places, const void *K,
                      const void *V, int rows, const smoe_rotary *rotary, const void *Q, int hq, void *Qr) {
  if (!ctx || rows < 0) return SMOE_ERR_INVALID_ARG;
  int rc = cache_args_ok(cache);
  if (rc == SMOE_OK) rc = places_ok(cache, places, rows);
  if (rc == SMOE_OK && rotary) rc = rotary_args_ok(rotary, cache->d_head);
  if (rc != SMOE_OK) return rc;
  if ((Q != nullptr) != (Qr != nullptr) || (Q && !rotary) || (Q && hq < 1)) return SMOE_ERR_INVALID_ARG;
  if (dtype != SMOE_BF16 || (Q && hq > 65535)) return SMOE_ERR_UNSUPPORTED;
  if (rows == 0) return SMOE_OK;
  if (!K || !V) return SMOE_ERR_INVALID_ARG;
  if (!aligned16(K) || !aligned16(V) || !aligned16(Q) || !aligned16(Qr)) return SMOE_ERR_UNSUPPORTED;
  const int d = cache->d_head;
  const size_t q = (size_t)rows * hq * d * 2, k = (size_t)rows * cache->h * d * 2;
  if (Q && ((Qr != Q && overlap(Qr, q, Q, q)) || overlap(Qr, q, K, k) || overlap(Qr, q, V, k) || over_pages(cache, Qr, q))) return SMOE_ERR_INVALID_ARG;
  if (!pages_apart(cache)) return SMOE_ERR_INVALID_ARG;
  TurnArgs a;
  a.Q = Q; a.K = K; a.V = V; a.Qr = Qr;
  a.hq = Q ? hq : 0; a.hk = cache->h; a.rows = rows; a.d = d;
  if (rotary) a.rotary = *rotary;
  return launch_cache_append((hipStream_t)stream, a, *cache, *places);
}

int smoe_cache_read(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const smoe_cache *cache, const smoe_places *places, int rows, void *K, void *V) {
  if (!ctx || rows < 0) return SMOE_ERR_INVALID_ARG;
  int rc = cache_args_ok(cache);
  if (rc == SMOE_OK) rc = places_ok(cache, places, rows);
  if (rc != SMOE_OK) return rc;
  if (dtype != SMOE_BF16) return SMOE_ERR_UNSUPPORTED;
  if (rows == 0) return SMOE_OK;
  if (!K || !V) return SMOE_ERR_INVALID_ARG;
  if (!aligned16(K) || !aligned16(V)) return SMOE_ERR_UNSUPPORTED;
  const size_t bytes = (size_t)rows * cache->h * cache->d_head * 2;
  if (overlap(K, bytes, V, bytes) || over_pages(cache, K, bytes) || over_pages(cache, V, bytes)) return SMOE_ERR_INVALID_ARG;
  return launch_cache_read((hipStream_t)stream, *cache, *places, rows, K, V);
}

size_t smoe_cached_attention_workspace_bytes(const smoe_cache *cache, const smoe_places *places, int N, int G) {
  if (cache_args_ok(cache) != SMOE_OK || table_ok(cache, places) != SMOE_OK || N < 1 || G < 1 || !cached_attention_fits(places->sequences, N, G, cache->h)) return 0;
  return cached_attention_workspace_bytes(N, G, cache->d_head, places->width * cache->page);
}

int smoe_cached_attention_fwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *Q, int N, int G, const smoe_cache *cache,
                              const smoe_places *places, void *O, float *LSE, void *ws, size_t ws_bytes) {
  if (!ctx || !Q || !O || !LSE || N < 1 || G < 1) return SMOE_ERR_INVALID_ARG;
  int rc = cache_args_ok(cache);
  if (rc == SMOE_OK) rc = lengths_ok(cache, places);
  if (rc != SMOE_OK) return rc;
  if (dtype != SMOE_BF16 || !cached_attention_fits(places->sequences, N, G, cache->h)) return SMOE_ERR_UNSUPPORTED;
  if (!aligned16(Q) || !aligned16(O)) return SMOE_ERR_UNSUPPORTED;
  const size_t need = cached_attention_workspace_bytes(N, G, cache->d_head, places->width * cache->page);
  if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)) return SMOE_ERR_WORKSPACE;
  const size_t bytes = (size_t)places->sequences * N * G * cache->h * cache->d_head * 2;
  const size_t lse = (size_t)places->sequences * N * G * cache->h * sizeof(float);
  if ((O != Q && overlap(O, bytes, Q, bytes)) || overlap(LSE, lse, Q, bytes) || overlap(LSE, lse, O, bytes)) return SMOE_ERR_INVALID_ARG;
  if (need && (overlap(ws, need, Q, bytes) || overlap(ws, need, O, bytes) || overlap(ws, need, LSE, lse))) return SMOE_ERR_INVALID_ARG;
  if (over_pages(cache, O, bytes) || over_pages(cache, LSE, lse) || (need && over_pages(cache, ws, need))) return SMOE_ERR_INVALID_ARG;
  return launch_cached_attention((hipStream_t)stream, Q, false, N, G, *cache, *places, O, LSE, ws);
}

}  // extern "C"
