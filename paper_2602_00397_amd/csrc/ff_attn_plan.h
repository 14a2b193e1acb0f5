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
  // the table of sequence s and key head h starts at s * seq_tables + h * head_tables
  int64_t seq_tables = 0;
  int32_t head_tables = 0;
  // pages in 8 bits: k and v are codes, with a scale for every 2^scale_shift keys of a page and head; nullptr: bf16
  const float *k_scale = nullptr, *v_scale = nullptr;
  int32_t scale_shift = 0;
  int32_t selected = 0;          // the tables are of selected pages: no sequence has many keys
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
// flag[0] is set to 1 + a sequence whose start, length or (if there is a table) page is out of range.  The caller zeroes flag[0] first.
hipError_t ff_launch_validate_pages(const AttnParams &p, int32_t *flag, hipStream_t s);

// The write of new tokens into pages in 8 bits: seqs has starts, lens, tables and the pages' shape (scale_shift with it).
// Of a scale that the write gives.  Its codes' values are normal bf16 numbers, and attention's sums, of up to 2^30 of them with weights up to
// 2^8 (a row's maximum may lag that far), stay below 2^(9 + 80 + 30 + 8).
constexpr int kLeastExp8 = -110, kMostExp8 = 80;
constexpr int kMaxScaleTokens = 128;
struct Append8Params {
  AttnParams seqs;
  const bf16_t *k, *v;
  int64_t k_stride, v_stride;
  uint8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
};
hipError_t ff_launch_append8(const Append8Params &a, int head_dim, hipStream_t s);

// Which pages blocks of new tokens read.  seqs has starts, lens, tables and the pages' shape; for the means also the cache.
struct SelectParams {
  AttnParams seqs;
  float *means;                  // [n_pages][n_kv][head_dim]; written by the first, read by the others
  int32_t query_block, keep, first, n_blocks, width;
  double *scores;                // [n_blocks][n_kv][table_stride]
  int32_t *starts, *lens, *tables;
};
hipError_t ff_launch_page_means(const SelectParams &a, int head_dim, hipStream_t s);
hipError_t ff_launch_select_pages(const SelectParams &a, int head_dim, hipStream_t s);

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

// ---- new tokens by the runs of positions and by the blocks that they lie in
// They stand at the positions keys - n .. keys - 1 of their sequence, as far as these are not negative.
// The sequence as the calls see it that write something for new tokens: those behind the table's end have no place and are left out, so that none
// stands on an earlier token's (which other rows may share).  (Lengths from 2^30 on, which no sequence has, are cut as everywhere.)
ATTN_FN Seq placed_seq(const AttnParams &p, int s) {
  Seq q = seq_of(p, s);
  const int keys = p.lens[s];
  if (keys > q.keys && keys < kMaxKeys) q.n = attn_max(0, q.n - (keys - q.keys));
  return q;
}
ATTN_FN int first_new(const Seq &q) { return q.keys > q.n ? q.keys - q.n : 0; }
// how many runs of 2^shift positions have new tokens
ATTN_FN int runs_of(const Seq &q, int shift) {
  return q.n > 0 && q.keys > 0 ? ((q.keys - 1) >> shift) - (first_new(q) >> shift) + 1 : 0;
}
// A call's runs are numbered so that the sequence of a number is found from the starts alone: those of sequence s from run_base on, with a gap
// up to run_base of the next.  A run has a token, and all of a sequence's but two are full; where there are fewer tokens than that makes,
// the numbers are the tokens'.
ATTN_FN bool runs_by_token(long n_tokens, long n_seqs, int shift) { return n_tokens <= (n_tokens >> shift) + 2 * n_seqs; }
ATTN_FN int run_base(int t0, int s, int shift, bool by_token) { return by_token ? t0 : (t0 >> shift) + 2 * s; }
// how many numbers there are
inline long most_runs(long n_tokens, long n_seqs, int shift) {
  return runs_by_token(n_tokens, n_seqs, shift) ? n_tokens : (n_tokens >> shift) + 2 * n_seqs;
}
ATTN_FN int blocks_of(const Seq &q, int query_block) { return (int)(((long)q.n + query_block - 1) / query_block); }
// Block number `at` of sequence s: its rows, how many pages lie in front of the one that its first token is in, how many from that one to the
// last token's, and the keys of as many of the former as are kept and of the latter, up to the last token.
struct Block { int s, t0, n, earlier, own, keys; };
ATTN_FN Block block_at(const Seq &q, int s, int at, int query_block, int keep, int page_shift) {
  Block b = {s, 0, 0, 0, 0, 0};
  const int t = at * query_block;
  b.t0 = q.t0 + t;
  b.n = attn_min(query_block, q.n - t);
  const int last = q.keys - q.n + t + b.n - 1;              // (below 0: its tokens see nothing)
  if (last < 0) return b;
  b.earlier = attn_max(last - b.n + 1, 0) >> page_shift;
  b.own = (last >> page_shift) - b.earlier + 1;
  // (its own pages are the last of the list, and the last of those ends with the block's last token)
  b.keys = ((attn_min(keep, b.earlier) + b.own - 1) << page_shift) + (last & ((1 << page_shift) - 1)) + 1;
  return b;
}
