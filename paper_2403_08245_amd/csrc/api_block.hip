// C ABI of libsmoe, the block around the experts (smoe_block.h): argument checks, workspace layout and launches.
#include "block.h"
#include <cmath>

namespace {
bool dtype_ok(int dt) { return dt == SMOE_F32 || dt == SMOE_BF16; }
bool aligned(const void *p) { return aligned16(p); }
template <typename... Rest> bool aligned(const void *p, Rest... rest) { return aligned16(p) && aligned(rest...); }

// An array of a call, to tell whether two share memory.
struct Span {
  const void *p;
  size_t bytes;
};
bool apart(const Span &a, const Span &b) { return !overlap(a.p, a.bytes, b.p, b.bytes); }
bool same_or_apart(const Span &a, const Span &b) { return a.p == b.p || apart(a, b); }

int rule_ok(const smoe_gate_rule *r, int E, int k) {
  if (!r || (r->score != SMOE_SCORE_SOFTMAX && r->score != SMOE_SCORE_SIGMOID) || (r->renormalise != 0 && r->renormalise != 1)) return SMOE_ERR_INVALID_ARG;
  if (!std::isfinite(r->scale) || r->groups < 1 || E % r->groups || r->kept_groups < 1 || r->kept_groups > r->groups) return SMOE_ERR_INVALID_ARG;
  if (r->group_best < 1 || (long long)k > (long long)r->kept_groups * (E / r->groups)) return SMOE_ERR_INVALID_ARG;
  if (r->groups > 64 || r->group_best > 2 || E > 1024 || k > 64) return SMOE_ERR_UNSUPPORTED;
  return SMOE_OK;
}
int gate_args_ok(smoe_ctx *ctx, int T, int E, int k, const smoe_gate_rule *rule) {
  if (!ctx || T < 0 || E < 1 || k < 1 || k > E) return SMOE_ERR_INVALID_ARG;
  int rc = rule_ok(rule, E, k);
  if (rc != SMOE_OK) return rc;
  return T > GATE_MAX_T || (long long)T * k > 0x7fffffffLL ? SMOE_ERR_UNSUPPORTED : SMOE_OK;
}

bool routing_ok(const smoe_routing *r) {
  if (!r || r->Tk < 0 || r->E < 1 || !r->expert_offsets) return false;
  return r->Tk == 0 || (r->sorted_expert_idxs && r->sorted_scattered_idxs);
}
size_t rows8_bytes(int rows, int d) { return (size_t)rows * pitch8(d); }

// weights of E experts, d_in -> d_out, and sizes that the kernels' grids and addresses hold
int weights8_ok(const smoe_weights8 *w) {
  if (!w || !w->values || !w->exps || w->E < 1 || w->d_in < 1 || w->d_out < 1 || (w->halves != 1 && w->halves != 2) || w->d_out % w->halves) return SMOE_ERR_INVALID_ARG;
  if (w->E > 65535 || w->d_in > (1 << 22) || w->d_out > (1 << 22) || !aligned(w->values, w->exps)) return SMOE_ERR_UNSUPPORTED;
  return SMOE_OK;
}
int weights8_fit(const smoe_weights8 *w, int E, int d_in, int d_out, int halves) {
  int rc = weights8_ok(w);
  if (rc != SMOE_OK) return rc;
  return w->E == E && w->d_in == d_in && w->d_out == d_out && w->halves == halves ? SMOE_OK : SMOE_ERR_INVALID_ARG;
}
// blocks of the decoding kernels' grids, at most
bool grid_fits(int Tk, int E, int d_out) { return ((long long)Tk / 32 + E) * (ceil_div(d_out, 32) + 4) * 256 <= 0xffffffffLL; }

size_t weights8_size(int E, int d_in, int d_out, int halves) { return (size_t)E * groups8(d_out, halves) * ceil_div(d_in, ROW8) * 2048; }

// Which kernels a product takes, by an estimate of their times in us (the rows of each expert are on the device: they are taken as even).  Fitted to 91
// products, seven layers at 8 to 2000 rows an expert, each timed on all three kernels; what the rule picks takes 0.6 % more than the fastest on
// average, 36 % at worst (32 experts of 300 rows, 1280 -> 1280: 39 us for 29).  Some of them, few rows / 128 x 256 / 256 x 256:
//   64 experts, 2048 -> 1024: 8 rows 33 / 32 / 35, 32 rows 45 / 34 / 36, 200 rows 126 / 50 / 45, 2000 rows - / 350 / 287
//   8 experts, 2816 -> 1024: 8 rows 9 / 26 / 32, 128 rows 21 / 25 / 35, 300 rows 36 / 27 / 36, 2000 rows - / 55 / 51
//   16 experts, 2048 -> 1536: 8 rows 12 / 22 / 26, 64 rows 24 / 23 / 28, 200 rows 52 / 22 / 32, 1200 rows - / 80 / 63
double few_rows_time(const S2S8Args &a) {
  const double expert = (double)groups8(a.W.d_out, a.W.halves) * ceil_div(a.W.d_in, ROW8) * 2048e-6, used = a.Tk < a.W.E ? a.Tk : a.W.E;      // MB of weights
  // tiles of 32 rows read them from the caches, once from memory, and write rows in pieces of 32 bytes (14756 rows on 48 experts, 128 -> 3712: 90 us)
  return 4.0 + (a.Tk / 32.0 + 0.5 * used) * expert / 8.2 + used * expert * 0.08 + (a.act ? 0.0 : (double)a.Tk * a.W.d_out * 1e-6);
}
double tiles_time(const S2S8Args &a, int rows, double stage, double lone_stage, double epilogue) {
  const double used = a.Tk < a.W.E ? a.Tk : a.W.E, each = a.Tk / used / rows;
  const double m_tiles = used * (each <= 0.8 ? 1.0 : each + 0.5), tiles = m_tiles * ceil_div(a.W.d_out, 256);
  const double rounds = std::fmax(1.0, std::ceil(tiles / a.grid - 0.05)), steps = a.W.d_in <= ROW8 ? 2 : ceil_div(a.W.d_in, ROW8);
  const double from_memory = m_tiles < 1.6 * used ? 1.6 * std::fmin(1.0, tiles / a.grid) : 0.0;      // a stage of weights that only this tile reads
  if (a.act) epilogue *= 1.8;
  return 4.5 + rounds * (steps * std::fmax(tiles > 128 ? stage : lone_stage, from_memory) + epilogue);
}
// what every launch takes from the context; true: the kernels for few rows
bool set_launch(const smoe_ctx *ctx, S2S8Args &a) {
  a.grid = ctx->stream_grid;
  a.group_m = ctx->group_m;
  a.tile_shape = ctx->tile_shape;
  if (ctx->kernel_mode || !s2s8_stream_supported(a)) return true;
  if (!a.tile_shape) {
    const double few = few_rows_time(a), half = tiles_time(a, 128, 1.03, 0.92, 3.0), big = tiles_time(a, 256, 1.58, 1.2, 4.5);
    if (few <= half && few <= big) return true;
    a.tile_shape = half <= big ? 1 : 2;
  }
  return false;
}
int product8(smoe_ctx *ctx, hipStream_t s, S2S8Args a) { return set_launch(ctx, a) ? launch_s2s8_decode(s, a) : launch_s2s8_stream(s, a); }

// Workspace of the MLP: hidden rows and their exponents, and the second product's rows [Tk, d_model], 2 bytes an element and their exponents, or fp32.
struct Mlp8Layout {
  size_t h, h_exps, yhat, y_exps, total;
};
// Rows of the second product in fp32, where the kernels for few rows make them, up to here: they are few, and in the caches.
constexpr int WIDE_ROWS = 8192;
Mlp8Layout mlp8_layout(int Tk, int d_model, int d_expert) {
  Mlp8Layout l;
  l.h = 0;
  l.h_exps = align256(rows8_bytes(Tk, d_expert));
  l.yhat = l.h_exps + align256(rows8_bytes(Tk, d_expert) / BLOCK8);
  l.y_exps = l.yhat + align256((size_t)Tk * d_model * (Tk <= WIDE_ROWS ? 4 : 2));
  l.total = l.y_exps + align256((size_t)Tk * ceil_div(d_model, 64));
  return l;
}
}  // namespace

extern "C" {

int smoe_score_gate(smoe_ctx *ctx, void *stream, const float *logits, const float *bias, int T, int E, int k, const smoe_gate_rule *rule,
                    int32_t *expert_idxs, float *gates) {
  int rc = gate_args_ok(ctx, T, E, k, rule);
  if (rc != SMOE_OK || T == 0) return rc;
  if (!logits || !expert_idxs || !gates) return SMOE_ERR_INVALID_ARG;
  if (!aligned(logits, bias, expert_idxs, gates)) return SMOE_ERR_UNSUPPORTED;
  const Span x{logits, (size_t)T * E * 4}, b{bias, (size_t)E * 4}, i{expert_idxs, (size_t)T * k * 4}, g{gates, (size_t)T * k * 4};
  if (!apart(i, x) || !apart(g, x) || !apart(i, b) || !apart(g, b) || !apart(i, g)) return SMOE_ERR_INVALID_ARG;
  return launch_score_gate((hipStream_t)stream, logits, bias, T, E, k, *rule, expert_idxs, gates);
}

int smoe_score_gate_bwd(smoe_ctx *ctx, void *stream, const float *logits, const int32_t *expert_idxs, const float *dgates, int T, int E, int k,
                        const smoe_gate_rule *rule, float *dlogits) {
  int rc = gate_args_ok(ctx, T, E, k, rule);
  if (rc != SMOE_OK || T == 0) return rc;
  if (!logits || !expert_idxs || !dgates || !dlogits) return SMOE_ERR_INVALID_ARG;
  if (!aligned(logits, expert_idxs, dgates, dlogits)) return SMOE_ERR_UNSUPPORTED;
  const Span o{dlogits, (size_t)T * E * 4}, x{logits, (size_t)T * E * 4}, i{expert_idxs, (size_t)T * k * 4}, g{dgates, (size_t)T * k * 4};
  if (!same_or_apart(o, x) || !apart(o, i) || !apart(o, g)) return SMOE_ERR_INVALID_ARG;
  return launch_score_gate_bwd((hipStream_t)stream, logits, expert_idxs, dgates, T, E, k, *rule, dlogits);
}

int smoe_rows8_pack(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *X, int rows, int d, const smoe_rows8 *out) {
  if (!ctx || !dtype_ok(dtype) || rows < 0 || d < 1 || !out) return SMOE_ERR_INVALID_ARG;
  if (rows == 0) return SMOE_OK;
  if (!X || !out->values || !out->exps) return SMOE_ERR_INVALID_ARG;
  if (d > (1 << 22) || !aligned(X, out->values, out->exps)) return SMOE_ERR_UNSUPPORTED;
  const Span x{X, (size_t)rows * d * dtype_size(dtype)}, v{out->values, rows8_bytes(rows, d)}, e{out->exps, rows8_bytes(rows, d) / BLOCK8};
  if (!apart(x, v) || !apart(x, e) || !apart(v, e)) return SMOE_ERR_INVALID_ARG;
  return launch_rows8_pack((hipStream_t)stream, dtype, X, rows, d, *out);
}

int smoe_rows8_unpack(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const smoe_rows8 *in, int rows, int d, void *X) {
  if (!ctx || !dtype_ok(dtype) || rows < 0 || d < 1 || !in) return SMOE_ERR_INVALID_ARG;
  if (rows == 0) return SMOE_OK;
  if (!X || !in->values || !in->exps) return SMOE_ERR_INVALID_ARG;
  if (d > (1 << 22) || !aligned(X, in->values, in->exps)) return SMOE_ERR_UNSUPPORTED;
  const Span x{X, (size_t)rows * d * dtype_size(dtype)}, v{in->values, rows8_bytes(rows, d)}, e{in->exps, rows8_bytes(rows, d) / BLOCK8};
  if (!apart(x, v) || !apart(x, e)) return SMOE_ERR_INVALID_ARG;
  return launch_rows8_unpack((hipStream_t)stream, dtype, *in, rows, d, X);
}

size_t smoe_weights8_bytes(int E, int d_in, int d_out, int halves) {
  if (E < 1 || d_in < 1 || d_out < 1 || (halves != 1 && halves != 2) || d_out % halves || E > 65535 || d_in > (1 << 22) || d_out > (1 << 22)) return 0;
  return weights8_size(E, d_in, d_out, halves);
}

int smoe_weights8_pack(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *W, const smoe_weights8 *out) {
  if (!ctx || !dtype_ok(dtype) || !W) return SMOE_ERR_INVALID_ARG;
  int rc = weights8_ok(out);
  if (rc != SMOE_OK) return rc;
  if (!aligned(W)) return SMOE_ERR_UNSUPPORTED;
  const size_t bytes = weights8_size(out->E, out->d_in, out->d_out, out->halves);
  const Span w{W, (size_t)out->E * out->d_in * out->d_out * dtype_size(dtype)}, v{out->values, bytes}, e{out->exps, bytes / BLOCK8};
  if (!apart(w, v) || !apart(w, e) || !apart(v, e)) return SMOE_ERR_INVALID_ARG;
  return launch_weights8_pack((hipStream_t)stream, dtype, W, *out);
}

static int norm_sizes_ok(smoe_ctx *ctx, smoe_dtype dtype, int rows, int d) {
  if (!ctx || !dtype_ok(dtype) || rows < 0 || d < 1) return SMOE_ERR_INVALID_ARG;
  return d > NORM_MAX_D || rows > NORM_MAX_ROWS ? SMOE_ERR_UNSUPPORTED : SMOE_OK;
}

int smoe_add_norm_fwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *X, const void *R, const void *weight, int rows, int d, float eps,
                      void *S, void *Y, const smoe_rows8 *Y8, float *rstd) {
  int rc = norm_sizes_ok(ctx, dtype, rows, d);
  if (rc != SMOE_OK) return rc;
  if (!(eps >= 0.f) || !std::isfinite(eps) || (!Y && !Y8)) return SMOE_ERR_INVALID_ARG;
  if (rows == 0) return SMOE_OK;
  if (!X || !weight || (Y8 && (!Y8->values || !Y8->exps))) return SMOE_ERR_INVALID_ARG;
  if (!aligned(X, R, weight, S, Y, rstd, Y8 ? Y8->values : nullptr, Y8 ? Y8->exps : nullptr)) return SMOE_ERR_UNSUPPORTED;
  const size_t n = (size_t)rows * d * dtype_size(dtype);
  const Span ins[] = {{X, n}, {R, n}, {weight, (size_t)d * dtype_size(dtype)}};
  const Span outs[] = {{S, n}, {Y, n}, {rstd, (size_t)rows * 4}, {Y8 ? Y8->values : nullptr, rows8_bytes(rows, d)}, {Y8 ? Y8->exps : nullptr, rows8_bytes(rows, d) / BLOCK8}};
  for (int o = 0; o < 5; ++o) {
    for (int i = 0; i < 3; ++i)
      if (o < 2 && i < 2 ? !same_or_apart(outs[o], ins[i]) : !apart(outs[o], ins[i])) return SMOE_ERR_INVALID_ARG;
    for (int p = 0; p < o; ++p)
      if (!apart(outs[o], outs[p])) return SMOE_ERR_INVALID_ARG;
  }
  NormArgs a{X, R, weight, rows, d, eps, S, Y, Y8 ? *Y8 : smoe_rows8{nullptr, nullptr}, rstd};
  return launch_norm((hipStream_t)stream, dtype, a);
}

size_t smoe_add_norm_bwd_workspace_bytes(smoe_dtype dtype, int rows, int d) {
  if (!dtype_ok(dtype) || rows < 0 || rows > NORM_MAX_ROWS || d < 1 || d > NORM_MAX_D) return 0;
  return align256((size_t)norm_bwd_parts(dtype, rows, d) * d * sizeof(float));
}

int smoe_add_norm_bwd(smoe_ctx *ctx, void *stream, smoe_dtype dtype, const void *dY, const void *dS, const void *S, const void *weight, const float *rstd,
                      int rows, int d, void *dX, void *dweight, void *ws, size_t ws_bytes) {
  int rc = norm_sizes_ok(ctx, dtype, rows, d);
  if (rc != SMOE_OK) return rc;
  if (!dweight || (rows > 0 && (!dY || !S || !weight || !rstd || !dX))) return SMOE_ERR_INVALID_ARG;
  if (!aligned(dY, dS, S, weight, rstd, dX, dweight)) return SMOE_ERR_UNSUPPORTED;
  const size_t need = smoe_add_norm_bwd_workspace_bytes(dtype, rows, d);
  if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)) return SMOE_ERR_WORKSPACE;
  const size_t n = (size_t)rows * d * dtype_size(dtype), w = (size_t)d * dtype_size(dtype);
  const Span ins[] = {{dY, n}, {dS, n}, {S, n}, {weight, w}, {rstd, (size_t)rows * 4}};
  const Span outs[] = {{dX, n}, {dweight, w}, {ws, need}};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 5; ++i)
      if (o == 0 && i < 3 ? !same_or_apart(outs[o], ins[i]) : !apart(outs[o], ins[i])) return SMOE_ERR_INVALID_ARG;
    for (int p = 0; p < o; ++p)
      if (!apart(outs[o], outs[p])) return SMOE_ERR_INVALID_ARG;
  }
  NormBwdArgs a{dY, dS, S, weight, rstd, rows, d, dX, dweight, (float *)ws};
  return launch_norm_bwd((hipStream_t)stream, dtype, a);
}

int smoe_plinear8_fwd(smoe_ctx *ctx, void *stream, const smoe_rows8 *X, int x_rows, int d_in, const smoe_weights8 *W, int d_out, const smoe_routing *r,
                      int k, const float *gates, int gates_k, int grouped_in, int grouped_out, void *Yhat, void *Y) {
  if (!ctx || !X || !routing_ok(r) || d_in < 1 || d_out < 1 || k < 1 || x_rows < 0) return SMOE_ERR_INVALID_ARG;
  const int Tk = r->Tk;
  if (grouped_in ? (k != 1 || x_rows != Tk) : ((long long)x_rows * k != Tk)) return SMOE_ERR_INVALID_ARG;
  if (gates ? (grouped_out || gates_k < 1 || Tk % gates_k || !Y) : Y != nullptr) return SMOE_ERR_INVALID_ARG;
  int rc = weights8_fit(W, r->E, d_in, d_out, 1);
  if (rc != SMOE_OK) return rc;
  if (d_out % 8 || !grid_fits(Tk, r->E, d_out)) return SMOE_ERR_UNSUPPORTED;
  if (Tk == 0) return SMOE_OK;
  if (!X->values || !X->exps || !Yhat) return SMOE_ERR_INVALID_ARG;
  if (!aligned(X->values, X->exps, gates, Yhat, Y)) return SMOE_ERR_UNSUPPORTED;
  const size_t stored = weights8_size(r->E, d_in, d_out, 1), rows = rows8_bytes(x_rows, d_in);
  const Span ins[] = {{X->values, rows}, {X->exps, rows / BLOCK8}, {W->values, stored}, {W->exps, stored / BLOCK8}, {gates, (size_t)Tk * 4},
                      {r->sorted_scattered_idxs, (size_t)Tk * 4}, {r->expert_offsets, ((size_t)r->E + 1) * 4}};
  const Span outs[] = {{Yhat, (size_t)Tk * d_out * 2}, {Y, gates ? (size_t)(Tk / gates_k) * d_out * 2 : 0}};
  for (const Span &o : outs)
    for (const Span &i : ins)
      if (!apart(o, i)) return SMOE_ERR_INVALID_ARG;
  if (!apart(outs[0], outs[1])) return SMOE_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  S2S8Args a;
  a.X = *X; a.W = *W;
  a.a_map = RowMap{grouped_in ? nullptr : r->sorted_scattered_idxs, grouped_in ? 1 : k};
  a.c_map = RowMap{grouped_out ? nullptr : r->sorted_scattered_idxs, 1};
  a.offsets = r->expert_offsets;
  a.Tk = Tk;
  a.C = Yhat;
  a.call_weights = stored;
  // Sums of rows rounded to bf16 would err by 2.35e-3, so what rounding took from them is kept beside them, where the sums will be (1.7e-3).  That has room for eight rows, in places of 64 columns.
  const bool rest = gates && gates_k <= REST_SLOTS && d_out % 64 == 0 && (long long)Tk * gates_k < 0x100000000LL;
  if (rest) {
    a.rest = (uint8_t *)Y;
    a.sum_k = gates_k;
  }
  rc = product8(ctx, s, a);
  if (rc != SMOE_OK || !gates) return rc;
  const int T = Tk / gates_k;
  return rest ? launch_combine_rest(s, Yhat, gates, Y, T, gates_k, d_out) : launch_combine(s, SMOE_BF16, Yhat, gates, Y, T, gates_k, d_out);
}

size_t smoe_mlp8_fwd_workspace_bytes(smoe_act act, int T, int k, int d_model, int d_expert) {
  if ((act != SMOE_ACT_GELU && act != SMOE_ACT_SWIGLU) || T < 0 || k < 1 || d_model < 1 || d_expert < 1 || (long long)T * k > 0x7fffffffLL) return 0;
  return mlp8_layout(T * k, d_model, d_expert).total;
}

int smoe_mlp8_fwd(smoe_ctx *ctx, void *stream, smoe_act act, const smoe_rows8 *X, int T, int d_model, int d_expert, const smoe_weights8 *W1,
                  const smoe_weights8 *W2, const smoe_routing *r, int k, const float *gates, void *Y, void *ws, size_t ws_bytes) {
  if (!ctx || !X || !routing_ok(r) || T < 0 || d_model < 1 || d_expert < 1 || k < 1 || (act != SMOE_ACT_GELU && act != SMOE_ACT_SWIGLU && act != SMOE_ACT_NONE))
    return SMOE_ERR_INVALID_ARG;
  if (act == SMOE_ACT_NONE) return SMOE_ERR_UNSUPPORTED;
  const int Tk = r->Tk, halves = act == SMOE_ACT_SWIGLU ? 2 : 1;
  if ((long long)T * k != Tk) return SMOE_ERR_INVALID_ARG;
  if (d_expert > (1 << 21)) return SMOE_ERR_UNSUPPORTED;
  int rc = weights8_fit(W1, r->E, d_model, d_expert * halves, halves);
  if (rc == SMOE_OK) rc = weights8_fit(W2, r->E, d_expert, d_model, 1);
  if (rc != SMOE_OK) return rc;
  if (d_model % 8 || !grid_fits(Tk, r->E, d_expert * halves) || !grid_fits(Tk, r->E, d_model)) return SMOE_ERR_UNSUPPORTED;
  if (Tk == 0) return SMOE_OK;
  if (!X->values || !X->exps || !gates || !Y) return SMOE_ERR_INVALID_ARG;
  if (!aligned(X->values, X->exps, gates, Y)) return SMOE_ERR_UNSUPPORTED;
  const Mlp8Layout l = mlp8_layout(Tk, d_model, d_expert);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < l.total) return SMOE_ERR_WORKSPACE;
  const size_t first = weights8_size(r->E, d_model, d_expert * halves, halves), second = weights8_size(r->E, d_expert, d_model, 1), rows = rows8_bytes(T, d_model);
  const Span ins[] = {{X->values, rows}, {X->exps, rows / BLOCK8}, {W1->values, first}, {W1->exps, first / BLOCK8}, {W2->values, second}, {W2->exps, second / BLOCK8},
                      {gates, (size_t)Tk * 4}, {r->sorted_scattered_idxs, (size_t)Tk * 4}, {r->expert_offsets, ((size_t)r->E + 1) * 4}};
  const Span outs[] = {{Y, (size_t)T * d_model * 2}, {ws, l.total}};
  for (const Span &o : outs)
    for (const Span &i : ins)
      if (!apart(o, i)) return SMOE_ERR_INVALID_ARG;
  if (!apart(outs[0], outs[1])) return SMOE_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  char *at = (char *)ws;
  S2S8Args a;
  a.X = *X; a.W = *W1;
  a.a_map = RowMap{r->sorted_scattered_idxs, k};
  a.c_map = RowMap{nullptr, 1};
  a.offsets = r->expert_offsets;
  a.Tk = Tk;
  a.H = smoe_rows8{(uint8_t *)at + l.h, (uint8_t *)at + l.h_exps};
  a.act = act;
  a.call_weights = first + second;
  rc = product8(ctx, s, a);
  if (rc != SMOE_OK) return rc;
  a.X = a.H; a.W = *W2;
  a.H = smoe_rows8{nullptr, nullptr};
  a.act = SMOE_ACT_NONE;
  a.a_map = RowMap{nullptr, 1};
  a.c_map = RowMap{r->sorted_scattered_idxs, 1};
  a.C = at + l.yhat;
  // a few rows are summed from fp32, others from fp16 with exponents: rounded to bf16 before the sum, Y would err by 2.35e-3 instead of 1.66e-3
  a.C_exps = (uint8_t *)at + l.y_exps;
  const bool few = set_launch(ctx, a);
  a.wide = few && Tk <= WIDE_ROWS;
  rc = few ? launch_s2s8_decode(s, a) : launch_s2s8_stream(s, a);
  if (rc != SMOE_OK) return rc;
  return a.wide ? launch_combine_wide(s, (const float *)a.C, gates, Y, T, k, d_model) : launch_combine_f16(s, a.C, a.C_exps, few ? 64 : 128, gates, Y, T, k, d_model);
}

}  // extern "C"
