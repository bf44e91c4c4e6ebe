// Rotary positions, the paged key-value cache and attention over it: what api_cache.hip, api.hip and the kernels share.
#pragma once
#include "common.h"
#include "smoe_cache.h"
#include <algorithm>

// Rows of Q, K and V of one launch that turns rows by their positions and, for a cache, stores those of K and V.
struct TurnArgs {
  const void *Q = nullptr, *K = nullptr, *V = nullptr;
  void *Qr = nullptr, *Kr = nullptr;      // Kr: without a cache
  int hq = 0, hk = 0, rows = 0, d = 0;
  int T = 1;                              // without a cache: the position of row i is positions[i], or i % T
  const int32_t *positions = nullptr;
  smoe_rotary rotary{nullptr, 0, 0, 1.f}; // turns NULL: nothing is turned
  bool back = false;                      // by the opposite angle
  // With a cache: K and V as fp32 shares [shares][2][rows][hk * d] that add up to them (launch_skinny_pair), in the place of bf16 rows.
  const float *parts = nullptr;
  int shares = 0;
  bool wide = false;                      // with shares: Q and Qr are fp32
};
int launch_turn(hipStream_t s, smoe_dtype dt, const TurnArgs &a);
bool cache_append_fits(int rows, int hq, int hk, int d);   // into one launch, however the rows come
int launch_cache_append(hipStream_t s, const TurnArgs &a, const smoe_cache &c, const smoe_places &p);
int launch_cache_read(hipStream_t s, const smoe_cache &c, const smoe_places &p, int rows, void *K, void *V);

// Two dense products X [M, K] W [K, N] of few rows, left as shares of the contraction, P [shares][2][M][N] fp32 (gemm_skinny.hip).
constexpr int SKINNY_MAX_ROWS = 512;
int skinny_shares(int M, int K, int N);      // 0: not for this kernel
int launch_skinny_pair(hipStream_t s, const void *X, const void *W0, const void *W1, int M, int K, int N, int shares, float *P);

bool cached_attention_fits(int B, int N, int G, int h);   // into one launch
size_t cached_attention_workspace_bytes(int N, int G, int d_head, int positions);   // positions the table holds
// wide: Q is fp32 (and not O), and meets the keys as two bf16 numbers
int launch_cached_attention(hipStream_t s, const void *Q, bool wide, int N, int G, const smoe_cache &c, const smoe_places &p, void *O, float *LSE, void *ws);

// What the entry points ask of a cache, its places and a rotary table, before anything is enqueued (host).
int cache_args_ok(const smoe_cache *c);
int lengths_ok(const smoe_cache *c, const smoe_places *p);   // the form with lens
int rotary_args_ok(const smoe_rotary *r, int d_head);
bool over_pages(const smoe_cache *c, const void *p, size_t bytes);   // does an array share memory with the cache's?
bool pages_apart(const smoe_cache *c);                               // do its own arrays lie apart, as who writes to it needs?

// The page of a sequence's position, or -1.
__device__ __forceinline__ int find_page(const smoe_places &p, int pages, int page_shift, int seq, int pos) {
  if ((unsigned)seq >= (unsigned)p.sequences || pos < 0 || (pos >> page_shift) >= p.width) return -1;
  const int id = p.block_table[(size_t)seq * p.width + (pos >> page_shift)];
  return (unsigned)id < (unsigned)pages ? id : -1;
}
// Sequence and position that a row of a call means; N = rows / sequences in the form with lens.
__device__ __forceinline__ void find_place(const smoe_places &p, int N, int row, int &seq, int &pos) {
  if (p.lens) {
    seq = row / N;
    const int back = N - (row - seq * N);
    pos = max(p.lens[seq], (int)0x80000000 + back) - back;      // a length whose position would pass the least int32 has that one: no place
  } else {
    seq = p.seqs[row];
    pos = p.positions[row];
  }
}
// the scale 2^e of a row in e4m3, from the byte that holds e + 127 (1 .. 254)
__device__ __forceinline__ float e4m3_scale(unsigned int byte) { return __uint_as_float(byte << 23); }
