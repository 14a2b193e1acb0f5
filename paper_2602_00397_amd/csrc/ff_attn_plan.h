// How a call of attention is cut: plain arithmetic, the same on the GPU (ff_attention.hip) and on the host (ff_launch_checks.hip).
// Lengths, starts and tables come from the caller's device memory: whatever they hold, what these functions give lies within
// the tensors.
#pragma once

#include "ff_internal.h"

#define ATTN_FN __host__ __device__ __forceinline__

constexpr int kTileKeys = 64;        // keys of one step; pieces of a split row are multiples of it

// r / d for 0 <= r < 2^31 and a divisor d up to 2^16 that the host knows: a product instead of a division's forty instructions
// (mul = floor(2^(31 + s) / d) + 1 with s = ceil(log2 d): its excess over 2^(31 + s) / d times r stays below 2^(31 + s) / d).
struct FastDiv {
  uint32_t mul = 0;
  int32_t shift = -1;      // s - 1; -1: d = 1
  ATTN_FN int operator()(int r) const { return shift < 0 ? r : (int)((uint32_t)(((uint64_t)(uint32_t)r * mul) >> 32) >> shift); }
};
inline FastDiv fast_div(int d) {
  FastDiv f;
  int s = 0;
  while ((1 << s) < d) ++s;
  if (s == 0) return f;
  f.mul = (uint32_t)((1ull << (31 + s)) / (unsigned)d + 1);
  f.shift = s - 1;
  return f;
}

struct AttnParams {
  const bf16_t *q, *k, *v;       // k, v: rows of a prompt, or pages
  bf16_t *o;
  float *lse;                    // [T][n_heads] or nullptr
  const int32_t *starts;         // [n_seqs + 1]
  const int32_t *lens;           // [n_seqs], or nullptr: a sequence's keys are its own rows
  const int32_t *table;          // [n_seqs][table_stride], or nullptr
  int64_t q_stride, k_stride, v_stride, o_stride;
  int32_t T, n_seqs, n_heads, n_kv, group, causal, window;
  FastDiv by_group, by_kv;
  int32_t table_stride, page_shift, n_pages;
  float scale_log2;              // scale * log2(e)
  // room for pieces of rows split along the keys
  float *part = nullptr;
  size_t part_bytes = 0;
  int32_t *counters = nullptr;   // [kAttnCounters], zero: how many pieces of a tile have ended; zero again when the call has
};
constexpr int kAttnCounters = 16384, kAttnSeqs = 16384;   // most sequences of a call
constexpr int kMostItems = 1 << 24;      // a sequence's (tile, piece), and all of a call's, are counted up to this number
// One kernel's share of a call: the sequences with rows (new tokens times heads of a group) in (rows_above, rows_upto], in tiles of
// tile_rows, split along the keys into about `target` pieces of at least min_steps times 64 keys (0: not split).  join_here: a tile's last piece
// joins them, no launch of its own.  by_tile: the tiles of all sequences by their number, the last first.
struct AttnPlan {
  int64_t rows_above = 0, rows_upto = -1;
  int32_t tile_rows = 1, target = 0, min_steps = 1, max_items = 0, join_here = 0, by_tile = 0;
  size_t part_at = 0;
  float *part = nullptr;
};
size_t ff_attention_part_bytes(int n_heads, int n_kv, int head_dim, int n_tokens, int n_seqs);
size_t ff_attention_need(const AttnParams &p, int head_dim, int max_chunk);   // what this call takes
hipError_t ff_attention_init();   // raises the kernels' dynamic-LDS limits
hipError_t ff_launch_attention(const AttnParams &p, int head_dim, int max_chunk, hipStream_t s);
// flag[0] is set to 1 + a sequence whose start, length or page is out of range.  The caller zeroes flag[0] first.
hipError_t ff_launch_validate_pages(const AttnParams &p, int32_t *flag, hipStream_t s);

ATTN_FN int attn_min(int a, int b) { return a < b ? a : b; }
ATTN_FN int attn_max(int a, int b) { return a > b ? a : b; }
ATTN_FN int attn_clamp(int v, int lo, int hi) { return attn_min(attn_max(v, lo), hi); }

constexpr int kMaxKeys = 1 << 30;    // of a sequence: positions and their sums with a piece or a window stay below 2^31
ATTN_FN long most_keys(const AttnParams &p) { return ((long)p.table_stride << p.page_shift) < kMaxKeys ? ((long)p.table_stride << p.page_shift) : (long)kMaxKeys; }

struct Seq { int t0, n, keys; };
ATTN_FN Seq seq_of(const AttnParams &p, int s) {
  Seq q;
  q.t0 = attn_clamp(p.starts[s], 0, p.T);
  q.n = attn_clamp(p.starts[s + 1], q.t0, p.T) - q.t0;
  q.keys = q.n;
  if (p.lens) {
    q.keys = attn_clamp(p.lens[s], 0, (int)most_keys(p));
  }
  return q;
}
// most keys that one row tile of the sequence needs, counted from a multiple of kTileKeys
ATTN_FN int span_of(const AttnParams &p, int keys, int tile_rows) {
  const int more = p.by_group(tile_rows) + 1 + kTileKeys;
  return p.window > 0 && p.window < keys - more ? p.window + more : keys;
}
ATTN_FN int tiles_of(const AttnParams &p, const AttnPlan &pl, int n) {
  const long rows = (long)n * p.group;
  return rows > pl.rows_above && rows <= pl.rows_upto ? (int)((rows + pl.tile_rows - 1) / pl.tile_rows) : 0;
}

// What a sequence adds to the price of a call, in steps of kTileKeys keys for one row tile and one key head, and how long a piece of
// a split row is then: the call comes to about pl.target pieces.  (Prices: fp32 is plenty.)
ATTN_FN float price_of(const AttnParams &p, const AttnPlan &pl, const Seq &q) {
  return (float)tiles_of(p, pl, q.n) * (float)((span_of(p, q.keys, pl.tile_rows) + kTileKeys - 1) / kTileKeys);
}
ATTN_FN int piece_keys_for(const AttnParams &p, const AttnPlan &pl, float steps) {
  const float per = ceilf(steps * (float)p.n_kv / (float)pl.target);
  return attn_max(pl.min_steps, per < (float)(kMaxKeys / kTileKeys) ? (int)per : kMaxKeys / kTileKeys) * kTileKeys;
}
constexpr int kUnsplit = kMaxKeys;
// pieces that every tile of the sequence is given (a tile with fewer keys leaves its last ones empty)
ATTN_FN int seq_pieces(const AttnParams &p, const AttnPlan &pl, const Seq &q, int keys_per_piece) {
  return attn_max(0, span_of(p, q.keys, pl.tile_rows) - 1) / keys_per_piece + 1;
}

// keys [lo, hi) that some row of the tile sees, lo a multiple of kTileKeys
struct Range { int lo, hi; };
ATTN_FN Range tile_range(const AttnParams &p, const Seq &q, int tile, int tile_rows) {
  Range r = {0, q.keys};
  if (p.causal) {
    const int rows = q.n * p.group;
    const int tok_lo = p.by_group(tile * tile_rows), tok_hi = p.by_group(attn_min((tile + 1) * tile_rows, rows) - 1);
    r.hi = attn_max(0, q.keys - q.n + tok_hi + 1);
    if (p.window > 0) r.lo = attn_max(0, q.keys - q.n + tok_lo + 1 - attn_min(p.window, kMaxKeys)) & ~(kTileKeys - 1);
  }
  return r;
}
// keys [lo, hi) that row r of the sequence sees
ATTN_FN Range row_range(const AttnParams &p, const Seq &q, int r) {
  Range g = {0, q.keys};
  if (p.causal) {
    g.hi = attn_max(0, q.keys - q.n + p.by_group(r) + 1);
    if (p.window > 0) g.lo = attn_max(0, g.hi - attn_min(p.window, kMaxKeys));
  }
  return g;
}
ATTN_FN int pieces_of(const Range &r, int keys_per_piece) {
  return r.hi > r.lo ? (r.hi - r.lo - 1) / keys_per_piece + 1 : 1;
}
