// Attention on bf16 MFMA: o_t = sum_j p_j v_j, p = softmax_j(scale q_t . k_j), one pass over the keys with the running maximum
// and sum of each row's softmax, over a prompt's own keys or over keys in pages.
//
// Rows.  The n_heads / n_kv heads that share a key head are rows of one tile, beside the tokens: row r of a sequence is token
// r / group, head r % group.  A key tile is fetched once for all of them, and a chunk of a few tokens fills a tile.
//
// Products.  Both are formed transposed: S^T = K Q^T has a row's keys in the registers of the lanes that own the row, so the
// softmax needs one exchange between lanes per tile, and O^T = V^T P^T takes those registers, rounded to bf16 and paired, as its
// operand without any exchange: the order of the keys inside one MFMA is free, and V's operand is read in S's order.  K and V lie
// in LDS as they lie in memory, 16-byte chunks swizzled; V^T comes from transposing LDS reads.
//
// Softmax.  fp32 throughout, base 2 (the scale and log2 e are one factor of the exponent's fma).  A row's maximum is only replaced
// when it has grown by more than 2^8: the exponentials stay below 256, far from fp32's and bf16's limits, and most tiles
// leave the sums as they are.  P is rounded to bf16 because the MFMA takes no wider operand; its row sum is kept in fp32 of the unrounded values.
#include "ff_attn_plan.h"
#include "ff_fp8.h"
#include "ff_wave.h"

#include <algorithm>
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(2))) int32_t i32x2_t;

constexpr float kNoMax = -3.0e38f;   // a row's maximum before its first key: finite, so no difference of two is a NaN
constexpr float kLazy = 8.0f;

__device__ __forceinline__ f32x16_t mfma32(const u32x4_t &a, const u32x4_t &b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma16(const u32x4_t &a, const u32x4_t &b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ u32x4_t lds_read16(uint32_t addr) {
  return *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t *>(addr);
}
// 16 lanes read four rows of 16 values of 16 bits (lane i the 8 bytes at quarter i % 4 of row i / 4); lane i gets the rows' value i
__device__ __forceinline__ u32x2_t lds_read_tr(uint32_t addr) {
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4_t *>(addr)));
}
// 16 lanes read eight rows of 16 bytes (lane i the 8 bytes at half i % 2 of row i / 2); lane i gets the rows' byte i
__device__ __forceinline__ u32x2_t lds_read_tr8(uint32_t addr) {
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<__attribute__((address_space(3))) i32x2_t *>(addr)));
}
// asynchronous copy of 16 bytes per lane to LDS from a wave-uniform base and a 32-bit offset (see gload_lds16)
__device__ __forceinline__ void gload_lds16_at(const void *base, uint32_t offset, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(offset), "s"(base), "s"(lds_addr)
               : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}

// A tile in LDS is a run of 256-byte rows: one key of head_dim 128, two of 64.  Chunk c of row r lies at place c ^ swizzle(r):
// the 16 lanes that read chunk c of 16 keys, and the 16 or 32 that read 32 or 64 bytes of 8 or 4 neighbouring keys, meet all banks.
template <int HD>
__device__ __forceinline__ int swizzle(int r) {
  return HD == 128 ? ((r & 1) << 3) | ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3) : ((r & 1) << 2) | (r & 2) | ((r & 4) >> 2);
}
// byte offset of chunk c of a key in its tile
template <int HD>
__device__ __forceinline__ uint32_t chunk_at(int key, int c) {
  if (HD == 128) return (uint32_t)(key * 256 + ((c ^ swizzle<HD>(key)) << 4));
  return (uint32_t)((key >> 1) * 256 + (((((key & 1) << 3) | c) ^ swizzle<HD>(key >> 1)) << 4));
}
// what lane l of the copy of 1 KB number i brings: key and chunk
template <int HD>
__device__ __forceinline__ void copied(int i, int lane, int &key, int &chunk) {
  const int r = i * 4 + (lane >> 4);
  const int c = (lane & 15) ^ swizzle<HD>(r);
  if (HD == 128) { key = r; chunk = c; }
  else { key = 2 * r + (c >> 3); chunk = c & 7; }
}

// ---- which part of which sequence a workgroup computes -----------------------------------------------------------------

// Sequence number lane + s0, which the first 64 lanes of a call's sequences keep in `first`.
__device__ __forceinline__ Seq lane_seq(const AttnParams &p, int s0, const Seq &first) {
  const int s = s0 + (threadIdx.x & 63);
  if (s0 == 0) return first;
  return s < p.n_seqs ? seq_of(p, s) : Seq{0, 0, 0};
}
// More than 64 sequences are looked at by 64, a wavefront of the workgroup to each 64, and the sums go through LDS; then a workgroup finds
// an item's sequence in those and one look more.  (2048 single tokens over 200 keys: 652 us with a look at every sequence for every
// item, 311 so.)
constexpr int kGroups = kAttnSeqs / 64;
struct Sums { int items[kGroups]; };      // (tile, piece) of each 64 sequences
// (tile, piece) of this lane's sequence.  Sums of 64 of these and of the sums stay in 32 bits, whatever the lengths are.
__device__ __forceinline__ int lane_items(const AttnParams &p, const AttnPlan &pl, const Seq &q, int keys) {
  return (int)min((long)tiles_of(p, pl, q.n) * seq_pieces(p, pl, q, keys), (long)kMostItems);
}
// all (tile, piece) of the call, and with more than 64 sequences each 64's in `sums` (a barrier before and behind)
template <int W>
__device__ __forceinline__ int count_items(const AttnParams &p, const AttnPlan &pl, int keys, const Seq &first, Sums &sums) {
  if (__builtin_expect(p.n_seqs <= 64, 1)) return last_lane(lane_sums(lane_items(p, pl, first, keys)));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n_groups = (p.n_seqs + 63) >> 6;
  __syncthreads();
  for (int g = wave; g < n_groups; g += W) {
    const int sum = lane_sums(lane_items(p, pl, lane_seq(p, g * 64, first), keys));
    if (lane == 63) sums.items[g] = min(sum, kMostItems);
  }
  __syncthreads();
  int all = 0;
  for (int g = lane; g < n_groups; g += 64) all += sums.items[g];
  return last_lane(lane_sums(min(all, kMostItems)));
}
// (rounded: the kernels of one call find the same, whatever the compiler could fuse the product with)
__device__ __forceinline__ float lane_price(const AttnParams &p, const AttnPlan &pl, const Seq &q) {
  float price = price_of(p, pl, q);
  asm("" : "+v"(price));
  return price;
}
// How long a piece is and how many (tile, piece) there are, from the work of the whole call; every wavefront of W finds the same.
struct Cut { int keys, items; Seq first; };
template <int W>
__device__ __forceinline__ Cut cut_of(const AttnParams &p, const AttnPlan &pl, Sums &sums) {
  Cut c = {kUnsplit, 0, {0, 0, 0}};
  const int lane = threadIdx.x & 63;
  if (lane < p.n_seqs) c.first = seq_of(p, lane);
  if (pl.target > 0) {
    float steps;
    if (__builtin_expect(p.n_seqs <= 64, 1)) {
      steps = last_lane(lane_sums(lane_price(p, pl, c.first)));
    } else {
      // (by 64 and then over those, so that kernels of more and of fewer wavefronts find the same sum in fp32)
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_groups = (p.n_seqs + 63) >> 6;
      for (int g = wave; g < n_groups; g += W) {
        const float sum = lane_sums(lane_price(p, pl, lane_seq(p, g * 64, c.first)));
        if (lane == 63) sums.items[g] = __builtin_bit_cast(int, sum);
      }
      __syncthreads();
      float mine = 0.f;
      for (int g = lane; g < n_groups; g += 64) mine += __builtin_bit_cast(float, sums.items[g]);
      steps = last_lane(lane_sums(mine));
    }
    c.keys = __builtin_amdgcn_readfirstlane(piece_keys_for(p, pl, steps));
  }
  c.items = count_items<W>(p, pl, c.keys, c.first, sums);
  return c;
}

struct Item {
  int s, tile, piece, kvh;   // piece of tile of sequence s, key head kvh
  int n_tiles, n_pieces;     // of the sequence (a tile may have fewer pieces)
  int first;                 // number of the sequence's first (tile, piece)
  Seq seq;
};
// The sequence of (tile, piece) number x, counted over the sequences in pieces of `keys`, or, with BY_SEQ, sequence x.
template <bool BY_SEQ>
__device__ __forceinline__ Item find_seq(const AttnParams &p, const AttnPlan &pl, int keys, const Seq &first, const Sums &sums, int x) {
  const int lane = threadIdx.x & 63;
  Item it = {};
  int base = 0, s0 = 0;                    // 64 sequences from s0 on, with `base` items before
  if (__builtin_expect(p.n_seqs > 64, 0)) {
    const int n_groups = (p.n_seqs + 63) >> 6;
    bool found = false;
    for (int g0 = 0; g0 < n_groups && !found; g0 += 64) {
      const int mine = g0 + lane < n_groups ? sums.items[g0 + lane] : 0, incl = lane_sums(mine);
      const int excl = base + incl - mine;
      const unsigned long long hit = __ballot(BY_SEQ ? g0 + lane == x >> 6 : x >= excl && x < excl + mine);
      found = hit != 0;
      if (found) {
        const int l = __builtin_ctzll(hit);
        s0 = (g0 + l) * 64;
        base = __builtin_amdgcn_readlane(excl, l);
      } else {
        base += last_lane(incl);
      }
    }
    if (!found) return it;
  }
  const Seq q = lane_seq(p, s0, first);
  const int tiles = tiles_of(p, pl, q.n), pieces = seq_pieces(p, pl, q, keys);
  const int mine = lane_items(p, pl, q, keys), excl = base + lane_sums(mine) - mine;
  const unsigned long long hit = __ballot(BY_SEQ ? s0 + lane == x : x >= excl && x < excl + mine);
  if (!hit) return it;
  const int l = __builtin_ctzll(hit);
  it.s = s0 + l;
  it.first = __builtin_amdgcn_readlane(excl, l);
  it.n_tiles = __builtin_amdgcn_readlane(tiles, l);
  it.n_pieces = __builtin_amdgcn_readlane(pieces, l);
  it.seq.t0 = __builtin_amdgcn_readlane(q.t0, l);
  it.seq.n = __builtin_amdgcn_readlane(q.n, l);
  it.seq.keys = __builtin_amdgcn_readlane(q.keys, l);
  return it;
}
// Item number -> what to compute.  Key heads go innermost (workgroups id mod 8 share an XCD, so its L2 keeps one head's keys where
// there are eight), then the tiles of one piece, the last first: under a causal mask those have the most keys.
__device__ __forceinline__ Item work_of(const AttnParams &p, const AttnPlan &pl, const Cut &cut, const Sums &sums, int id) {
  const int x = p.by_kv(id);
  Item it = find_seq<false>(p, pl, cut.keys, cut.first, sums, x);
  const int local = x - it.first;
  it.kvh = id - x * p.n_kv;
  if (it.n_tiles == 0) return it;       // (no such item)
  it.piece = local / it.n_tiles;
  it.tile = it.n_tiles - 1 - (local - it.piece * it.n_tiles);
  return it;
}
// The same for tiles that are not split, of at most 64 sequences, with the last tiles of all of them first, then those before, so that
// none of the longest begins when the others end.  There are sum max(0, tiles - t) tiles from number t on: it is found bit by bit.
__device__ __forceinline__ Item work_by_tile(const AttnParams &p, const AttnPlan &pl, const Cut &cut, int id) {
  const int x = p.by_kv(id), tiles = tiles_of(p, pl, cut.first.n), lane = threadIdx.x & 63;
  int t = 0;                             // the largest number from which on there are more than x tiles
  for (int bit = 1 << (31 - __builtin_clz(cut.items)); bit; bit >>= 1)
    if (last_lane(lane_sums(max(0, tiles - t - bit))) > x) t += bit;
  const int before = last_lane(lane_sums(max(0, tiles - t - 1)));
  const unsigned long long has = __ballot(tiles > t);
  const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(has >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)has, 0));
  const unsigned long long hit = __ballot(tiles > t && rank == x - before);
  Item it = {};
  if (!hit) return it;
  const int l = __builtin_ctzll(hit);
  it.s = l;
  it.tile = t;
  it.kvh = id - x * p.n_kv;
  it.n_tiles = __builtin_amdgcn_readlane(tiles, l);
  it.n_pieces = 1;
  it.seq.t0 = __builtin_amdgcn_readlane(cut.first.t0, l);
  it.seq.n = __builtin_amdgcn_readlane(cut.first.n, l);
  it.seq.keys = __builtin_amdgcn_readlane(cut.first.keys, l);
  return it;
}
__device__ __forceinline__ int items_of(const AttnParams &p, const AttnPlan &pl, const Cut &cut) {
  // (chunks that overlap may have more than there is room for: nothing is computed, and no counter is left behind)
  const long n = (long)cut.items * p.n_kv;
  return n <= pl.max_items ? (int)n : 0;
}

// Partial sums of a piece: tile_rows times HD sums, then tile_rows pairs of maximum and sum.  The few-row kernel's sums lie by rows,
// the other's as its lanes hold them: 1 KB for four values of each lane, 32 rows together.
template <int HD>
__device__ __forceinline__ float *part_of(const AttnPlan &pl, int x, int kvh, int n_kv) {
  return pl.part + ((size_t)x * n_kv + kvh) * ((size_t)pl.tile_rows * (HD + 2));
}

// the token and the head that row r of a sequence is
__device__ __forceinline__ int64_t row_token(const AttnParams &p, const Seq &q, int r) { return q.t0 + p.by_group(r); }
__device__ __forceinline__ int row_head(const AttnParams &p, int kvh, int r) { return kvh * p.group + r - p.by_group(r) * p.group; }

// the lane's number, found again where it is asked for: none of the registers of the loops before holds it
__device__ __forceinline__ int fresh_lane() {
  int none = 0;
  asm volatile("" : "+v"(none));
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

// where keys lie: rows of a prompt, pages in bf16, pages in 8 bits
enum Source { kRows, kPages, kPages8 };
__device__ __forceinline__ const int32_t *table_of(const AttnParams &p, const Item &it) {
  return p.table + it.s * p.seq_tables + (size_t)it.kvh * p.head_tables;
}
template <bool PAGED>
struct KeySource {
  const bf16_t *k, *v;          // PAGED: the head's part of page 0; else the head's part of the sequence's first row
  const int32_t *table;         // the sequence's
  uint32_t page_elems, k_pitch, v_pitch;   // elements of a page (all heads), bytes from key to key
  int shift, n_pages;
};
template <int HD, bool PAGED>
__device__ __forceinline__ KeySource<PAGED> key_source(const AttnParams &p, const Item &it) {
  KeySource<PAGED> ks;
  if (PAGED) {
    ks.shift = p.page_shift;
    ks.k = p.k + (((size_t)it.kvh << p.page_shift) * HD);
    ks.v = p.v + (((size_t)it.kvh << p.page_shift) * HD);
    ks.page_elems = (uint32_t)((p.n_kv << p.page_shift) * HD);
    ks.table = table_of(p, it);
    ks.n_pages = p.n_pages;
    ks.k_pitch = ks.v_pitch = HD * 2;
  } else {
    ks.k = p.k + (size_t)it.seq.t0 * p.k_stride + it.kvh * HD;
    ks.v = p.v + (size_t)it.seq.t0 * p.v_stride + it.kvh * HD;
    ks.k_pitch = (uint32_t)p.k_stride * 2;
    ks.v_pitch = (uint32_t)p.v_stride * 2;
    ks.table = nullptr; ks.page_elems = 0; ks.shift = 0; ks.n_pages = 0;
  }
  return ks;
}
// Copies `first` to `first` + NI - 1 of a tile of TILE keys, 1 KB each, as one wavefront makes them.  The keys of one copy (4 or 8,
// aligned) are in one page.
template <int HD, bool PAGED, int NI, int TILE>
struct Copier {
  static constexpr int KPI = 512 / HD;
  KeySource<PAGED> ks;
  int first, end;
  uint32_t k_off[NI], v_off[NI];     // of this lane, from the copy's first key
  __device__ __forceinline__ Copier(const KeySource<PAGED> &src, int first_copy, int end_key, int lane) : ks(src), first(first_copy), end(end_key) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int key, chunk;
      copied<HD>(first + i, lane, key, chunk);
      k_off[i] = (uint32_t)(key - (first + i) * KPI) * ks.k_pitch + chunk * 16;
      v_off[i] = PAGED ? k_off[i] : (uint32_t)(key - (first + i) * KPI) * ks.v_pitch + chunk * 16;
    }
  }
  // where a key's value lies (a wave-uniform key below `end`)
  __device__ __forceinline__ const bf16_t *value(int key) const {
    if (!PAGED) return reinterpret_cast<const bf16_t *>(reinterpret_cast<const uint8_t *>(ks.v) + (uint64_t)(uint32_t)key * ks.v_pitch);
    const int page = ks.table[key >> ks.shift];
    return ks.v + (size_t)((unsigned)page < (unsigned)ks.n_pages ? page : 0) * ks.page_elems + (key & ((1 << ks.shift) - 1)) * HD;
  }
  // the tile that starts at key j, a multiple of 32; keys from `end` on are replaced by the last one
  template <bool VALUES>
  __device__ __forceinline__ void copy(int j, uint32_t lds, int lane) const {
    const bf16_t *src = VALUES ? ks.v : ks.k;
    const uint32_t pitch = VALUES ? ks.v_pitch : ks.k_pitch;
    const bool full = j + TILE <= end;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key0 = full ? j + (first + i) * KPI : min(j + (first + i) * KPI, end - 1);
      uint32_t off = VALUES ? v_off[i] : k_off[i];
      if (!full) {
        int key, chunk;
        copied<HD>(first + i, lane, key, chunk);
        off = (uint32_t)(min(j + key, end - 1) - key0) * pitch + chunk * 16;
      }
      const uint8_t *base;
      if (PAGED) {
        int page = scalar_load(ks.table + (key0 >> ks.shift));
        page = __builtin_amdgcn_readfirstlane((unsigned)page < (unsigned)ks.n_pages ? page : 0);
        base = reinterpret_cast<const uint8_t *>(src + (size_t)page * ks.page_elems) + (uint32_t)(key0 & ((1 << ks.shift) - 1)) * (HD * 2);
      } else {
        base = reinterpret_cast<const uint8_t *>(src) + (uint64_t)(uint32_t)key0 * pitch;
      }
      gload_lds16_at(base, off, lds + (first + i) * 1024);
    }
  }
};

// infinities and NaN of a pair of bf16 values set to 0; `any` collects whether there were some
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, uint32_t &any) {
  const uint32_t n = ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;     // an exponent of all ones carries into its half's top bit
  any |= n;
  return w & ~((n - (n >> 15)) | n);
}
__device__ __forceinline__ void bf16x4(const u32x2_t &w, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// Pages in 8 bits: codes become bf16 on their way to the matrix unit, and the rest is as for pages in bf16.
struct Source8 {
  const uint8_t *k, *v;        // the head's part of page 0
  const float *ks, *vs;
  const int32_t *table;
  uint32_t page_bytes, page_scales;      // of all heads
  int shift, scale_shift, n_pages;
};
template <int HD>
__device__ __forceinline__ Source8 source8(const AttnParams &p, const Item &it) {
  Source8 s;
  s.shift = p.page_shift;
  s.scale_shift = p.scale_shift;
  s.k = reinterpret_cast<const uint8_t *>(p.k) + ((size_t)it.kvh << p.page_shift) * HD;
  s.v = reinterpret_cast<const uint8_t *>(p.v) + ((size_t)it.kvh << p.page_shift) * HD;
  s.ks = p.k_scale + ((size_t)it.kvh << (p.page_shift - p.scale_shift));
  s.vs = p.v_scale + ((size_t)it.kvh << (p.page_shift - p.scale_shift));
  s.page_bytes = (uint32_t)((p.n_kv << p.page_shift) * HD);
  s.page_scales = (uint32_t)(p.n_kv << (p.page_shift - p.scale_shift));
  s.table = table_of(p, it);
  s.n_pages = p.n_pages;
  return s;
}
// page and place of a wave-uniform key
__device__ __forceinline__ int page_of(const Source8 &s, int key, int &place) {
  const int page = scalar_load(s.table + (key >> s.shift));
  place = key & ((1 << s.shift) - 1);
  return __builtin_amdgcn_readfirstlane((unsigned)page < (unsigned)s.n_pages ? page : 0);
}
template <bool VALUES>
__device__ __forceinline__ float scale8(const Source8 &s, int page, int place) {
  return scalar_load((VALUES ? s.vs : s.ks) + (size_t)page * s.page_scales + (place >> s.scale_shift));
}
// Codes in LDS: 256-byte rows of 2 keys of head_dim 128 or 4 of 64, 16-byte chunks swizzled.  The places are different ones for chunk c
// of the keys 8 a + b + {0 .. 3}, a = 0 .. 3, b = 0 or 4, which 16 lanes read for K, and of 16 neighbouring keys, which 32 lanes read for V.
template <int HD>
__device__ __forceinline__ int swizzle8(int r) {
  return HD == 128 ? (r & 5) | ((r ^ (r >> 2)) & 2) : ((r ^ (r >> 2)) & 1) | (r & 2);
}
template <int HD>
__device__ __forceinline__ uint32_t chunk8_at(int key, int c) {
  constexpr int S = HD == 128 ? 1 : 2;            // log2 of the keys of a row
  return (uint32_t)((key >> S) * 256 + (((((key & ((1 << S) - 1)) << (4 - S)) | c) ^ swizzle8<HD>(key >> S)) << 4));
}
// The copies of KEYS (32 or 64) keys in 8 bits to LDS, as one wavefront makes them, 1 KB each, and their scales, one for each 8 keys.
// Scalar arithmetic is what these cost (a lookup of page and scale for each KB: some 750 scalar instructions a step, 48 tokens 67 us), so keys
// that are all there and in one page have one lookup, and others one for each 16; the values lie where their keys do.
template <int HD, int KEYS>
struct Copier8 {
  static constexpr int S = HD == 128 ? 1 : 2, KPI = 1024 / HD, NI = KEYS / KPI;   // log2 of the keys of a row, keys of a copy
  Source8 src;
  int end;
  // of the last keys that were asked for, from page 0 of the head's codes and scales on
  uint64_t codes_at[KEYS / 16], scales_at[KEYS / 16];
  // key and offset of this lane's 16 bytes of copy i, from the copy's first key
  static __device__ __forceinline__ int key_of(int i, int lane) { return ((i * 4 + (lane >> 4)) << S | (lane & 15) >> (4 - S)) - i * KPI; }
  static __device__ __forceinline__ int chunk_of(int i, int lane) { return ((lane & 15) ^ swizzle8<HD>(i * 4 + (lane >> 4))) & ((1 << (4 - S)) - 1); }
  __device__ __forceinline__ void look(int g, int key) {
    int place;
    const int page = page_of(src, key, place);
    codes_at[g] = (uint64_t)page * src.page_bytes + (uint32_t)place * HD;
    scales_at[g] = (uint64_t)page * src.page_scales + (uint32_t)((place & -16) >> src.scale_shift);
  }
  // keys, or the values of the keys that were asked for last
  template <bool VALUES>
  __device__ __forceinline__ void copy(int j, uint32_t lds, int lane, f32x4_t (&scale)[KEYS / 32]) {
    const uint8_t *const codes = VALUES ? src.v : src.k;
    const float *const scales = VALUES ? src.vs : src.ks;
    if (j + KEYS <= end && (1 << src.shift) >= KEYS) {
      if (!VALUES) look(0, j);
      const uint8_t *base = codes + codes_at[0];
#pragma unroll
      for (int i = 0; i < NI; ++i) gload_lds16_at(base + i * 1024, (uint32_t)(key_of(i, lane) * HD + chunk_of(i, lane) * 16), lds + i * 1024);
      const float *from = scales + scales_at[0];
      if ((1 << src.scale_shift) >= KEYS) {
        const float one = scalar_load(from);
#pragma unroll
        for (int b = 0; b < KEYS / 8; ++b) scale[b >> 2][b & 3] = one;
      } else {
#pragma unroll
        for (int b = 0; b < KEYS / 8; ++b) scale[b >> 2][b & 3] = scalar_load(from + (b * 8 >> src.scale_shift));
      }
      return;
    }
#pragma unroll
    for (int g = 0; g < KEYS / 16; ++g) {
      // (behind the end: the last key again, with some scale of its page; no row sees them)
      const int key0 = min(j + g * 16, end - 1);
      if (!VALUES) look(g, key0);
      const uint8_t *base = codes + codes_at[g];
#pragma unroll
      for (int i = g * 16 / KPI; i < (g + 1) * 16 / KPI; ++i) {
        const int key = min(j + i * KPI + key_of(i, lane), end - 1) - key0;
        gload_lds16_at(base, (uint32_t)(key * HD + chunk_of(i, lane) * 16), lds + i * 1024);
      }
      const float *from = scales + scales_at[g];
      scale[g >> 1][g % 2 * 2] = scalar_load(from);
      scale[g >> 1][g % 2 * 2 + 1] = scalar_load(from + (8 >> src.scale_shift));
    }
  }
};
// The keys and values of a tile of 64 on their way from pages in 8 bits to bf16 in LDS, as one of RW wavefronts brings them: NU times 16
// channels of a key to a lane (8 of head_dim 64), 8 keys at a time, which share a page and a scale.  Pages are looked up a tile ahead, and
// the values' are those that the keys had, so that no wavefront waits for a table where its matrix instructions could start.
template <int HD, int RW>
struct Stager8 {
  static constexpr int CPL = HD == 128 ? 16 : 8, NU = HD / (CPL * RW), KPC = 64 * CPL / HD, W = CPL / 8;
  Source8 src;
  int first, end, step;                       // tiles from one to the next of the same wavefronts: `step` keys
  uint32_t code[2][NU][CPL / 4];
  float scale[2][NU];
  int next[NU], keys[NU], values[NU];         // pages of the next tile, of the last keys that were asked for, of the values that are next
  __device__ __forceinline__ int key0(int j, int i) const { return min(j + (first + i) * KPC, end - 1); }
  __device__ __forceinline__ void look(int j) {
#pragma unroll
    for (int i = 0; i < NU; ++i) next[i] = scalar_load(src.table + (key0(j, i) >> src.shift));
  }
  // (`look` has been called for j)
  __device__ __forceinline__ void load_keys(int j, int lane) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      values[i] = keys[i];
      keys[i] = __builtin_amdgcn_readfirstlane((unsigned)next[i] < (unsigned)src.n_pages ? next[i] : 0);
    }
    load<false>(j, lane, keys);
    if (j + step < end) look(j + step);
  }
  // `after`: the next tile's keys have been asked for in between
  __device__ __forceinline__ void load_values(int j, int lane, bool after) {
#pragma unroll
    for (int i = 0; i < NU; ++i)
      if (!after) values[i] = keys[i];
    load<true>(j, lane, values);
  }
  template <bool VALUES>
  __device__ __forceinline__ void load(int j, int lane, const int (&pages)[NU]) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int from = key0(j, i), key = min(j + (first + i) * KPC + lane / (HD / CPL), end - 1) - from, place = from & ((1 << src.shift) - 1);
      const uint8_t *base = (VALUES ? src.v : src.k) + (size_t)pages[i] * src.page_bytes + (uint32_t)place * HD;
      const uint8_t *at = base + (uint32_t)(key * HD + lane % (HD / CPL) * CPL);
      if constexpr (CPL == 16) __builtin_memcpy(code[VALUES][i], __builtin_assume_aligned(at, 16), 16);
      else __builtin_memcpy(code[VALUES][i], __builtin_assume_aligned(at, 8), 8);
      scale[VALUES][i] = scale8<VALUES>(src, pages[i], place);
    }
  }
  // `edge`: infinities and NaN become 0; returns whether there were some
  template <bool VALUES>
  __device__ __forceinline__ bool store(uint32_t lds, int lane, bool edge) const {
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int h = 0; h < W; ++h) {
        u32x4_t w = decode8(code[VALUES][i][2 * h], code[VALUES][i][2 * h + 1], scale[VALUES][i]);
        if (edge)
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = finite_pair(w[e], odd);
        const int key = (first + i) * KPC + lane / (HD / CPL);
        *reinterpret_cast<__attribute__((address_space(3))) u32x4_t *>(lds + chunk_at<HD>(key, lane % (HD / CPL) * W + h)) = w;
      }
    return odd != 0;
  }
};

// The largest of a lane's scores.  v_max3 takes two at a time, where fmaxf first quiets each of its arguments.  The compiler does not
// count the wait states between an MFMA and inline asm that reads what it wrote (18 after the longest): the first asm has them, and
// the others depend on it.
__device__ __forceinline__ float max16(const f32x16_t &s) {
  float mx;
  asm("s_nop 15\n\ts_nop 3\n\tv_max3_f32 %0, %1, %2, %3" : "=v"(mx) : "v"(s[0]), "v"(s[1]), "v"(s[2]));
#pragma unroll
  for (int i = 3; i < 15; i += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(mx) : "v"(s[i]), "v"(s[i + 1]));
  asm("v_max_f32 %0, %0, %1" : "+v"(mx) : "v"(s[15]));
  return mx;
}
__device__ __forceinline__ float max_score(const f32x16_t (&s)[2]) { return fmaxf(max16(s[0]), max16(s[1])); }
// What lane l ^ 32, or l ^ 16, holds beside this lane's value, by the vector unit (a shuffle goes through LDS).
__device__ __forceinline__ f32x2_t with_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f32x2_t{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ f32x2_t with_row(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f32x2_t{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float larger(const f32x2_t &v) { return fmaxf(v[0], v[1]); }
// natural log of the sum that belongs to a maximum (in powers of two of the scaled products) and a sum
__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.f || l != l ? (m + __log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// ---- few rows: single tokens of a generation step ------------------------------------------------------------------------
// HBM-bound: every key is read once for at most 16 NB rows.  Four wavefronts, each with keys of its own (32 at a time, every
// fourth 32 of the piece), its own 32 keys of LDS and its own softmax state, without barriers until they join at the end: K of the
// next keys is on its way while V of these is waited for, and the other way round.  Workgroups take pieces in turn, two of them
// on a CU, so one streams while the other starts or joins.  The last piece of a tile to end joins all of them, in order, if the rows
// are few (pl.join_here), else another launch does.  48 tokens of 32 heads over 8 key heads of 128 and up to 16384 keys: 94 us, 4.7 TB/s.
// One token over 8191 keys: 16 us for 6.8 of bytes, bound by its chain of latencies (cut of the call, page, key, value, sums, join).
constexpr int kFewWaves = 4, kFewGrid = 512;

// The sums of a piece go past this XCD's L2 (relaxed atomics of device scope: a release fence would write back all of it).
__device__ __forceinline__ void part_store(float *at, float a, float b) {
  const f32x2_t v = {a, b};
  __hip_atomic_store(reinterpret_cast<uint64_t *>(at), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2_t part_load(const float *at) {
  return __builtin_bit_cast(f32x2_t, __hip_atomic_load(reinterpret_cast<const uint64_t *>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Pages in 8 bits (EIGHT) come 64 keys at a time, as many bytes (32 where two sets' registers would not fit).  Lane (l16, quad) holds 16 channels of a key for two MFMAs, whose
// channels are in that order in Q too, and eight neighbouring keys of a channel for V^T, by one transposing read.
template <int HD, int NB, bool EIGHT>
__global__ __launch_bounds__(64 * kFewWaves, 2) void ff_attn_few_kernel(AttnParams p, AttnPlan pl) {
  constexpr int KS = HD / 32, DB = HD / 16, SETS = EIGHT && !(HD == 128 && NB == 2) ? 2 : 1, KEYS = 32 * SETS;   // of a step, 32 to a set
  constexpr int NI = KEYS * HD * (EIGHT ? 1 : 2) / 1024;
  constexpr uint32_t kHalf = 32 * HD * 2, kSet = 32 * HD;
  constexpr int kRows = 16 * NB, kPitch = HD + 4, kBatch = 16;
  extern __shared__ __align__(256) uint8_t lds[];
  __shared__ int last_s;
  __shared__ Sums sums_s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l16 = lane & 15, quad = lane >> 4;
  const uint32_t k_at = lds_addr_of(lds) + wave * 2 * kHalf, v_at = k_at + kHalf;
  // where this lane's operands lie in a tile (the swizzle repeats after 16 keys, that of codes after 32)
  uint32_t k_off[KS], v_off[DB];
#pragma unroll
  for (int c = 0; c < KS; ++c) {
    if (EIGHT) k_off[c] = k_at + chunk8_at<HD>((l16 >> 2) * 8 + (l16 & 3) + (c & 1) * 4, (c >> 1) * 4 + quad);      // chunk c / 2 of the two keys
    else k_off[c] = k_at + chunk_at<HD>(l16, c * 4 + quad);
  }
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    if (EIGHT) v_off[d] = v_at + chunk8_at<HD>(quad * 8 + (l16 >> 1), d) + (l16 & 1) * 8;
    else v_off[d] = v_at + chunk_at<HD>(quad * 4 + (l16 >> 2), d * 2 + ((l16 & 3) >> 1)) + (l16 & 1) * 8;
  }
  // key x of this lane's eight scores of a set
  const auto key_of = [&](int set, int x) { return EIGHT ? set * 32 + quad * 8 + x : (x >> 2) * 16 + quad * 4 + (x & 3); };

  const Cut cut = cut_of<kFewWaves>(p, pl, sums_s);
  const int n_items = items_of(p, pl, cut);
  for (int id = blockIdx.x; id < n_items; id += gridDim.x) {
    const Item it = work_of(p, pl, cut, sums_s, id);
    if (it.n_tiles == 0) continue;
    const int n_rows = it.seq.n * p.group, row0 = it.tile * kRows;
    const Range range = tile_range(p, it.seq, it.tile, kRows);
    const int n_pieces = pieces_of(range, cut.keys);
    if (it.piece >= n_pieces) continue;
    const int beg = range.lo + it.piece * cut.keys, end = range.hi - beg > cut.keys ? beg + cut.keys : range.hi;
    std::conditional_t<EIGHT, Copier8<HD, KEYS>, const Copier<HD, true, NI, 32>> copier = [&] {
      if constexpr (EIGHT) return Copier8<HD, KEYS>{source8<HD>(p, it), end, {}, {}};
      else return Copier<HD, true, NI, 32>(key_source<HD, true>(p, it), 0, end, lane);
    }();
    [[maybe_unused]] f32x4_t k_scale[SETS], v_scale[SETS];        // of each eight keys on their way
    const auto copy_k = [&](int j) __attribute__((always_inline)) {
      if constexpr (EIGHT) copier.template copy<false>(j, k_at, lane, k_scale);
      else copier.template copy<false>(j, k_at, lane);
    };
    const auto copy_v = [&](int j) __attribute__((always_inline)) {
      if constexpr (EIGHT) copier.template copy<true>(j, v_at, lane, v_scale);
      else copier.template copy<true>(j, v_at, lane);
    };
    // of those, that of the eight keys that are number b of a set
    const auto pick = [](f32x4_t scale, int b) __attribute__((always_inline)) {
      const float lo = b & 1 ? scale[1] : scale[0], hi = b & 1 ? scale[3] : scale[2];
      return b & 2 ? hi : lo;
    };

    // the rows' own limits, and the part of the tile's keys that all of them see
    Range see[NB];
    u32x4_t q[NB][KS];
    int all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = min(row0 + b * 16 + l16, n_rows - 1);
      see[b] = row_range(p, it.seq, r);
      see[b].hi = min(see[b].hi, end);
      all_lo = max(all_lo, see[b].lo);
      all_hi = min(all_hi, see[b].hi);
      const bf16_t *src = p.q + row_token(p, it.seq, r) * p.q_stride + row_head(p, it.kvh, r) * HD;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        q[b][s] = *reinterpret_cast<const u32x4_t *>(src + (EIGHT ? (s >> 1) * 64 + quad * 16 + (s & 1) * 8 : s * 32 + quad * 8));
    }
    int j = beg + wave * KEYS;
    if (j < end) copy_k(j);
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) {
      all_lo = max(all_lo, __shfl_xor(all_lo, off));
      all_hi = min(all_hi, __shfl_xor(all_hi, off));
    }
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[b][s]));   // (arrived: no wait for it among the copies' later on)
    if (j < end) copy_v(j);

    f32x4_t o[NB][DB];
    float m[NB], l[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      m[b] = kNoMax;
      l[b] = 0.f;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[b][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    for (; j < end; j += KEYS * kFewWaves) {
      const bool more = j + KEYS * kFewWaves < end;
      wait_copies<NI>();                    // K is here, V on its way
      // S^T: the keys of each set, 16 and 16, by the rows
      f32x4_t s[NB][SETS][2];
      u32x4_t kf[SETS][2][EIGHT ? KS / 2 : KS];
#pragma unroll
      for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int c = 0; c < (EIGHT ? KS / 2 : KS); ++c)
            kf[set][kt][c] = EIGHT ? lds_read16(k_off[c * 2 + kt] + set * kSet) : lds_read16(k_off[c] + kt * 16 * HD * 2);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K is in registers: its place is free
      float ks[SETS];
      if constexpr (EIGHT)
#pragma unroll
        for (int set = 0; set < SETS; ++set) ks[set] = pick(k_scale[set], l16 >> 2);
      if (more) copy_k(j + KEYS * kFewWaves);
#pragma unroll
      for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
          for (int b = 0; b < NB; ++b) s[b][set][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < KS; ++c) {
            const u32x4_t f = kf[set][kt][EIGHT ? c / 2 : c];
            const u32x4_t a = EIGHT ? decode8(f[c % 2 * 2], f[c % 2 * 2 + 1], ks[set]) : f;
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b][set][kt] = mfma16(a, q[b][c], s[b][set][kt]);
          }
        }
      const bool masked = j < all_lo || j + KEYS > all_hi;
      u32x4_t pk[NB][SETS];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float mx = -INFINITY;
#pragma unroll
        for (int set = 0; set < SETS; ++set) {
          if (masked) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              const int key = j + key_of(set, x);
              s[b][set][x >> 2][x & 3] = key >= see[b].lo && key < see[b].hi ? s[b][set][x >> 2][x & 3] : -INFINITY;
            }
          }
          const float most = fmaxf(fmaxf(fmaxf(s[b][set][0][0], s[b][set][0][1]), fmaxf(s[b][set][0][2], s[b][set][0][3])),
                                   fmaxf(fmaxf(s[b][set][1][0], s[b][set][1][1]), fmaxf(s[b][set][1][2], s[b][set][1][3])));
          mx = set == 0 ? most : fmaxf(mx, most);
        }
        mx = larger(with_half(larger(with_row(mx)))) * p.scale_log2;
        if (__any(mx > m[b] + kLazy)) {
          const float m_new = fmaxf(m[b], mx), a = __builtin_amdgcn_exp2f(m[b] - m_new);
          m[b] = m_new;
          l[b] *= a;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[b][d][i] *= a;
        }
#pragma unroll
        for (int set = 0; set < SETS; ++set) {
          float e[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            e[x] = __builtin_amdgcn_exp2f(fmaf(s[b][set][x >> 2][x & 3], p.scale_log2, -m[b]));
            l[b] += e[x];
          }
          pk[b][set] = u32x4_t{pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])};
        }
      }
      if (more) wait_copies<NI>();          // V is here, the next K on its way
      else wait_copies<0>();
      // O^T += V^T P^T
      [[maybe_unused]] float vs[SETS];
      if constexpr (EIGHT)
#pragma unroll
        for (int set = 0; set < SETS; ++set) vs[set] = pick(v_scale[set], quad);
      const auto values = [&](int set, int d) __attribute__((always_inline)) {
        if constexpr (EIGHT) {
          const u32x2_t v = lds_read_tr8(v_off[d] + set * kSet);
          return decode8(v[0], v[1], vs[set]);
        } else {
          const u32x2_t v0 = lds_read_tr(v_off[d]), v1 = lds_read_tr(v_off[d] + 16 * HD * 2);
          return u32x4_t{v0[0], v0[1], v1[0], v1[1]};
        }
      };
      if (!masked) {
#pragma unroll
        for (int set = 0; set < SETS; ++set)
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const u32x4_t vf = values(set, d);
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b][d] = mfma16(vf, pk[b][set], o[b][d]);
          }
      } else {
        uint32_t odd = 0;
#pragma unroll
        for (int set = 0; set < SETS; ++set)
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            u32x4_t vf = values(set, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[e] = finite_pair(vf[e], odd);
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b][d] = mfma16(vf, pk[b][set], o[b][d]);
          }
        if (__any(odd != 0)) {
          // infinities and NaN among the values (0 in the product): they reach the rows that see their key, and no other
#pragma unroll 1
          for (int x = 0; x < KEYS; ++x) {
            [[maybe_unused]] float scale = 1.f;
            if constexpr (EIGHT) {
              int place;
              const int page = page_of(copier.src, min(j + x, end - 1), place);
              scale = scale8<true>(copier.src, page, place);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
              float v[4];
              u32x2_t w;
              if constexpr (EIGHT) {
                const uint32_t codes = *reinterpret_cast<const __attribute__((address_space(3))) uint32_t *>(v_at + chunk8_at<HD>(x, d) + quad * 4);
                w = decode4(codes, scale);
              } else {
                w = *reinterpret_cast<const __attribute__((address_space(3))) u32x2_t *>(v_at + chunk_at<HD>(x, d * 2 + (quad >> 1)) + (quad & 1) * 8);
              }
              bf16x4(w, v);
#pragma unroll
              for (int b = 0; b < NB; ++b)
                if (j + x >= see[b].lo && j + x < see[b].hi)
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    if (!(fabsf(v[i]) < INFINITY)) o[b][d][i] += v[i];
            }
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V is in registers
      if (more) copy_v(j + KEYS * kFewWaves);
    }

    // join the four wavefronts' sums
    float *joined = reinterpret_cast<float *>(lds);                        // [4][kRows][kPitch]
    float *ml = joined + kFewWaves * kRows * kPitch;                       // [4][kRows][2]
    __syncthreads();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32x2_t both = with_row(l[b]);
      both = with_half(both[0] + both[1]);
      l[b] = both[0] + both[1];
      const int r = b * 16 + l16;
#pragma unroll
      for (int d = 0; d < DB; ++d)
        *reinterpret_cast<f32x4_t *>(joined + (wave * kRows + r) * kPitch + d * 16 + quad * 4) = o[b][d];
      if (quad == 0) {
        ml[(wave * kRows + r) * 2] = m[b];
        ml[(wave * kRows + r) * 2 + 1] = l[b];
      }
    }
    __syncthreads();
    const int rows_here = min(kRows, n_rows - row0);
    const bool whole = n_pieces == 1;
    // (tile, piece) numbers of this tile: x0, x0 + n_tiles, ...
    const int x0 = it.first + it.n_tiles - 1 - it.tile;
    const auto out = [&](int r, int c, float a, float b, float top, float sum) __attribute__((always_inline)) {
      const int row = row0 + r;
      const int64_t t = row_token(p, it.seq, row);
      const int head = row_head(p, it.kvh, row);
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      *reinterpret_cast<uint32_t *>(p.o + t * p.o_stride + head * HD + c) = pack_bf16x2(a * inv, b * inv);
      if (c == 0 && p.lse) p.lse[t * p.n_heads + head] = lse_of(top, sum);
    };
    float *part = whole ? nullptr : part_of<HD>(pl, x0 + it.piece * it.n_tiles, it.kvh, p.n_kv);
    for (int i = threadIdx.x; i < rows_here * (HD / 2); i += 64 * kFewWaves) {
      const int r = i / (HD / 2), c = (i % (HD / 2)) * 2;
      float mw[kFewWaves], top = kNoMax, sum = 0.f, a = 0.f, b = 0.f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        mw[w] = ml[(w * kRows + r) * 2];
        top = fmaxf(top, mw[w]);
      }
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(mw[w] - top);
        sum = fmaf(ml[(w * kRows + r) * 2 + 1], f, sum);
        const f32x2_t x = *reinterpret_cast<const f32x2_t *>(joined + (w * kRows + r) * kPitch + c);
        a = fmaf(x[0], f, a);
        b = fmaf(x[1], f, b);
      }
      if (whole) {
        out(r, c, a, b, top, sum);
      } else {
        part_store(part + r * HD + c, a, b);
        if (c == 0) part_store(part + kRows * HD + r * 2, top, sum);
      }
    }
    if (!whole && pl.join_here) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // this wavefront's sums have arrived
      __syncthreads();
      int *counter = p.counters + x0 * p.n_kv + it.kvh;
      if (threadIdx.x == 0) {
        last_s = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n_pieces - 1;
        if (last_s) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as the next call expects it
      }
      __syncthreads();
      if (last_s) {
        const size_t step = (size_t)it.n_tiles * p.n_kv * ((size_t)kRows * (HD + 2));
        const float *src = part_of<HD>(pl, x0, it.kvh, p.n_kv);
        for (int i = threadIdx.x; i < rows_here * (HD / 2); i += 64 * kFewWaves) {
          const int r = i / (HD / 2), c = (i % (HD / 2)) * 2;
          // kBatch pieces' loads on their way at a time; their sums in a running maximum's scale, in the pieces' order
          float top = kNoMax, sum = 0.f, a = 0.f, b = 0.f;
          for (int k0 = 0; k0 < n_pieces; k0 += kBatch) {
            f32x2_t x[kBatch], w[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
              const float *from = src + (size_t)min(k0 + k, n_pieces - 1) * step;
              w[k] = part_load(from + kRows * HD + r * 2);
              x[k] = part_load(from + r * HD + c);
            }
            float higher = top;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) higher = fmaxf(higher, w[k][0]);
            const float f0 = __builtin_amdgcn_exp2f(top - higher);
            sum *= f0; a *= f0; b *= f0;
            top = higher;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
              const bool is = k0 + k < n_pieces;       // (not by a factor of 0: the sums may be infinite)
              const float f = __builtin_amdgcn_exp2f(w[k][0] - top);
              sum = is ? fmaf(w[k][1], f, sum) : sum;
              a = is ? fmaf(x[k][0], f, a) : a;
              b = is ? fmaf(x[k][1], f, b) : b;
            }
          }
          out(r, c, a, b, top, sum);
        }
      }
    }
    __syncthreads();                        // nothing of this piece is still being read when the next one's copies land
  }
}

// ---- many rows: prompts and chunks of them --------------------------------------------------------------------------------
// MFMA-bound.  RW wavefronts of 32 rows share the key tiles of 64; with KW = 2 there are two such groups of wavefronts, which take
// every other tile, for half as many rows, and join at the end.  Two stages of LDS for K and two for V: in step i, Q K of tile i
// and P V of tile i - 1 are one run of MFMAs, whose operands are read four MFMAs ahead, and the softmax of tile i follows, while the
// copies of K of tile i + 1 and V of tile i land.  One barrier a step.  A SIMD's two wavefronts take turns: in eight wavefronts of 128
// channels the second four make the softmax of tile i at the start of step i + 1, so their exponentials go through the vector unit while
// the matrix pipe works for the first four, and the other way round (8192 tokens of 32 heads over 8 key heads of 128, causal, 520 us
// without turns, 500 with); elsewhere they drift apart by themselves, and MFMAs have priority.
// Pages in 8 bits go through registers: asked for at a step's start, turned into bf16 and written to their place in LDS at its end.
template <int HD, int RW, int KW, Source SRC>
__global__ __launch_bounds__(RW * KW * 64, HD == 64 && (SRC != kRows || KW == 1) ? 4 : 2) void ff_attn_tile_kernel(AttnParams p, AttnPlan pl) {
  constexpr bool PAGED = SRC != kRows, EIGHT = SRC == kPages8;
  constexpr int KS = HD / 16, DB = HD / 32, NI = kTileKeys * HD * 2 / 1024 / RW;
  constexpr uint32_t kHalf = kTileKeys * HD * 2;
  constexpr int kRows = 32 * RW, kStep = kTileKeys * KW;
  extern __shared__ __align__(256) uint8_t lds[];
  __shared__ int odd_s[KW][2];
  __shared__ Sums sums_s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % RW, kw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / RW;
  const int lane = threadIdx.x & 63;
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15, grp = lane >> 4;
  const Cut cut = cut_of<RW * KW>(p, pl, sums_s);
  const int id = blockIdx.y * gridDim.x + blockIdx.x;
  if (id >= items_of(p, pl, cut)) return;
  const Item it = !PAGED && pl.by_tile ? work_by_tile(p, pl, cut, id) : work_of(p, pl, cut, sums_s, id);
  if (it.n_tiles == 0) return;
  const int kpp = cut.keys;
  const int n_rows = it.seq.n * p.group, row0 = it.tile * kRows + wave * 32;
  const Range range = tile_range(p, it.seq, it.tile, kRows);
  const int n_pieces = pieces_of(range, kpp);
  if (it.piece >= n_pieces) return;
  const int beg = range.lo + it.piece * kpp, end = range.hi - beg > kpp ? beg + kpp : range.hi;
  std::conditional_t<EIGHT, Stager8<HD, RW>, const Copier<HD, PAGED, NI, kTileKeys>> copier = [&] {
    if constexpr (EIGHT) {
      Stager8<HD, RW> s8;
      s8.src = source8<HD>(p, it);
      s8.first = wave * Stager8<HD, RW>::NU;
      s8.end = end;
      s8.step = kStep;
      return s8;
    }
    else return Copier<HD, PAGED, NI, kTileKeys>(key_source<HD, PAGED>(p, it), wave * NI, end, lane);
  }();
  const auto copy_k = [&](int j, uint32_t to) __attribute__((always_inline)) {
    if constexpr (EIGHT) copier.load_keys(j, lane);
    else copier.template copy<false>(j, to, lane);
  };
  // (in 8 bits: behind the next tile's keys, if there is one)
  const auto copy_v = [&](int j, uint32_t to) __attribute__((always_inline)) {
    if constexpr (EIGHT) copier.load_values(j, lane, j + kStep < end);
    else copier.template copy<true>(j, to, lane);
  };
  const uint32_t ring_k = lds_addr_of(lds) + kw * 4 * kHalf, ring_v = ring_k + 2 * kHalf;

  // (out before the rows' own arithmetic and loads)
  if (beg + kw * kTileKeys < end) {
    if constexpr (EIGHT) copier.look(beg + kw * kTileKeys);
    copy_k(beg + kw * kTileKeys, ring_k);
  }
  Range see;
  u32x4_t q[KS];
  {
    const int row = min(row0 + l32, n_rows - 1);
    see = row_range(p, it.seq, row);
    see.hi = min(see.hi, end);
    const bf16_t *src = p.q + row_token(p, it.seq, row) * p.q_stride + row_head(p, it.kvh, row) * HD + half * 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u32x4_t *>(src + s * 16);
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[s]));   // (arrived: no wait for it among the copies' later on)
  }
  // (limits grow with the row: the first and the last row have the extremes)
  const int lo_first = __builtin_amdgcn_readlane(see.lo, 0);
  const int hi_last = row0 < n_rows ? __builtin_amdgcn_readlane(see.hi, 31) : 0;     // (no rows: no tile is seen)

  f32x16_t o[DB];
  u32x4_t pk[4];
  float m = kNoMax, l = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // Tiles that not all rows of the workgroup see whole: their values are looked through for infinities and NaN when they have landed, by
  // the wavefront that copied them, which puts 0 in their place and leaves the tile's key in the stage's flag if there are any.
  const int edge_lo = row_range(p, it.seq, min((it.tile + 1) * kRows, n_rows) - 1).lo, edge_hi = min(row_range(p, it.seq, it.tile * kRows).hi, end);
  const auto is_edge = [&](int j) { return j < edge_lo || j + kTileKeys > edge_hi; };
  volatile int *const odd_tile = odd_s[kw];

  // Where this lane's operands lie in a tile: chunk 0 of the key that is its row of K, and 8 bytes of each of two keys for V^T.  Chunk c
  // is 16 c away by exclusive or (the swizzle is one), the other keys' operands are 32 and 16 keys further (it repeats after 16).
  const uint32_t k_off = chunk_at<HD>(l32, half);
  uint32_t v_off[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) v_off[r] = chunk_at<HD>(half * 4 + (l16 >> 2) + 8 * r, (grp & 1) * 2 + ((l16 & 3) >> 1)) + (l16 & 1) * 8;

  // scores of the tile at key j -> weights, in the rows' running maximum's scale
  // (see.lo <= see.hi also where the piece's end cuts the latter: a piece is longer than the limits of a tile's rows are apart)
  auto weights = [&](f32x16_t (&s)[2], int j, auto masked) __attribute__((always_inline)) {
    if (masked) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = j + half * 4 - see.lo + (kb * 32 + (i & 3) + 8 * (i >> 2));
          s[kb][i] = (unsigned)key < (unsigned)(see.hi - see.lo) ? s[kb][i] : -INFINITY;
        }
    }
    const float mx = larger(with_half(max_score(s))) * p.scale_log2;
    if (__any(mx > m + kLazy)) {
      const float m_new = fmaxf(m, mx), a = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= a;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= a;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[x >> 1][(x & 1) * 8 + i], p.scale_log2, -m));
        l += e[i];
      }
      pk[x] = u32x4_t{pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])};
    }
  };
  // The infinities and NaN among the values of the tile at key j, which are 0 in LDS: they reach the rows that see their key, and no other.
  auto add_odd = [&](int j) __attribute__((always_inline)) {
    const int far = fresh_lane() >> 5;
#pragma unroll 1
    for (int key = j; key < min(j + kTileKeys, end); ++key) {
      const bool seen = key >= see.lo && key < see.hi;
      [[maybe_unused]] const bf16_t *src = nullptr;
      [[maybe_unused]] const uint8_t *codes = nullptr;
      [[maybe_unused]] float scale = 1.f;
      if constexpr (EIGHT) {
        int place;
        const int page = page_of(copier.src, key, place);
        scale = scale8<true>(copier.src, page, place);
        codes = copier.src.v + (size_t)page * copier.src.page_bytes + (uint32_t)place * HD + far * 4;
      } else {
        src = copier.value(key) + far * 4;
      }
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float v[4];
          if constexpr (EIGHT) {
            bf16x4(decode4(*reinterpret_cast<const uint32_t *>(codes + d * 32 + g * 8), scale), v);
          } else {
            bf16x4(*reinterpret_cast<const u32x2_t *>(src + d * 32 + g * 8), v);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (seen && !(fabsf(v[i]) < INFINITY)) o[d][g * 4 + i] += v[i];
          __builtin_amdgcn_sched_barrier(0);       // (a few registers at a time)
        }
    }
  };
  // P V of the tile whose values are in LDS at `v_at` and Q K of the one whose keys are at `k_at`, or either, in one run: each operand
  // is read D MFMAs before its own
  auto products = [&](f32x16_t (&s)[2], uint32_t v_at, uint32_t k_at, auto with_v, auto with_k) __attribute__((always_inline)) {
    constexpr int NV = with_v ? 4 * DB : 0, N = NV + (with_k ? 2 * KS : 0), D = 4;
    u32x4_t f[D];
    auto load = [&](int n) __attribute__((always_inline)) {
      if (n < NV) {
        const u32x2_t v0 = lds_read_tr(((v_at + v_off[0]) ^ (n % DB * 64)) + (n / DB) * 16 * HD * 2);
        const u32x2_t v1 = lds_read_tr(((v_at + v_off[1]) ^ (n % DB * 64)) + (n / DB) * 16 * HD * 2);
        f[n % D] = u32x4_t{v0[0], v0[1], v1[0], v1[1]};
      } else {
        f[n % D] = lds_read16(((k_at + k_off) ^ ((n - NV) / 2 * 32)) + (n - NV) % 2 * 32 * HD * 2);
      }
    };
#pragma unroll
    for (int n = 0; n < D; ++n) load(n);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (n < NV) {
        o[n % DB] = mfma32(f[n % D], pk[n / DB], o[n % DB]);
      } else {
        const int kb = (n - NV) % 2, c = (n - NV) / 2;
        if (c == 0)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
        s[kb] = mfma32(f[n % D], q[c], s[kb]);
      }
      if (n + D < N) load(n + D);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto is_seen = [&](int j) { return j < hi_last && j + kTileKeys > lo_first; };

  if (beg < end) {
    // Step i: K of tile i is in stage i % 2, V of tile i - 1 in the other.  The copies that go out at its start fill the stages that
    // step i - 1 read, and have landed when it ends.  (Past the end there are none, but a tile that ends behind it is copied whole:
    // the last key again.)
    const auto begin = [&](int j, uint32_t at) __attribute__((always_inline)) {
      if (j + kStep < end) copy_k(j + kStep, ring_k + (kHalf - at));
      if (j < end) copy_v(j, ring_v + at);
    };
    const auto step_end = [&](int j, uint32_t at) __attribute__((always_inline)) {
      if constexpr (EIGHT) {
        if (j + kStep < end) copier.template store<false>(ring_k + (kHalf - at), lane, false);
        if (j < end && copier.template store<true>(ring_v + at, lane, is_edge(j))) odd_tile[at != 0] = j;
      } else if (is_edge(j) && j < end) {
        wait_copies<0>();
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint32_t mine = ring_v + at + (wave * NI + i) * 1024 + lane * 16;
          u32x4_t v = lds_read16(mine);
          uint32_t odd = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = finite_pair(v[e], odd);
          if (odd) {
            *reinterpret_cast<__attribute__((address_space(3))) u32x4_t *>(mine) = v;
            odd_tile[at != 0] = j;
          }
        }
      }
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    const auto is_odd = [&](int j, uint32_t at) { return is_edge(j) && __builtin_amdgcn_readfirstlane(odd_tile[at != 0]) == j; };
    const int start = beg + kw * kTileKeys;
    // (all wavefronts make the same number of steps)
    const int last = beg + (end - beg + kStep - 1) / kStep * kStep + kw * kTileKeys;
    uint32_t at = 0;
    if (threadIdx.x < 2 * KW) odd_s[threadIdx.x >> 1][threadIdx.x & 1] = -1;
    if constexpr (EIGHT)
      if (start < end) copier.template store<false>(ring_k, lane, false);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const auto is_inner = [&](int j) { return j > start && !is_edge(j - kStep) && !is_edge(j) && j + kStep < end; };
    for (int j = start;; j += kStep, at = kHalf - at) {
      // both products in one run: of tiles that every row of the workgroup sees whole, then of tiles that some see in part
      if (is_inner(j)) {
        f32x16_t s[2];
        const bool late = HD == 128 && RW == 8 && wave >= 4;
        bool have = false;
        do {
          copy_k(j + kStep, ring_k + (kHalf - at));
          copy_v(j, ring_v + at);
          if (late && have) weights(s, j, std::false_type());
          have = true;
          __builtin_amdgcn_s_setprio(1);
          products(s, ring_v + kHalf - at, ring_k + at, std::true_type(), std::true_type());
          __builtin_amdgcn_s_setprio(0);
          if (!late) weights(s, j, std::false_type());
          if constexpr (EIGHT) {
            copier.template store<false>(ring_k + (kHalf - at), lane, false);
            copier.template store<true>(ring_v + at, lane, false);
          }
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          j += kStep;
          at = kHalf - at;
        } while (is_inner(j));
        if (late) weights(s, j, std::false_type());
      }
      for (; j > start && j < last && !is_inner(j) && is_seen(j - kStep) && is_seen(j); j += kStep, at = kHalf - at) {
        f32x16_t s[2];
        begin(j, at);
        products(s, ring_v + kHalf - at, ring_k + at, std::true_type(), std::true_type());
        if (is_odd(j - kStep, kHalf - at)) add_odd(j - kStep);
        weights(s, j, std::true_type());
        step_end(j, at);
      }
      f32x16_t s[2];
      const bool seen = j < last && is_seen(j);
      begin(j, at);
      if (j > start && is_seen(j - kStep)) {
        products(s, ring_v + kHalf - at, 0, std::true_type(), std::false_type());
        if (is_odd(j - kStep, kHalf - at)) add_odd(j - kStep);
      }
      if (seen) {
        products(s, 0, ring_k + at, std::false_type(), std::true_type());
        weights(s, j, std::true_type());
      }
      step_end(j, at);
      if (j >= last) break;
    }
  }
  const f32x2_t both = with_half(l);
  l = both[0] + both[1];
  const int end_lane = fresh_lane(), end_row = end_lane & 31, end_half = end_lane >> 5;
  if (KW > 1) {
    // the second group's sums, through LDS, into the first's
    constexpr int kPitch = HD + 4;
    float *other = reinterpret_cast<float *>(lds) + (wave * 32 + end_row) * kPitch;
    float *ml = reinterpret_cast<float *>(lds) + kRows * kPitch + (wave * 32 + end_row) * 2;
    __syncthreads();
    if (kw == 1) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4_t *>(other + d * 32 + g * 8 + end_half * 4) = f32x4_t{o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]};
      if (end_half == 0) {
        ml[0] = m;
        ml[1] = l;
      }
    }
    __syncthreads();
    if (kw == 1) return;
    const float top = fmaxf(m, ml[0]), a = __builtin_amdgcn_exp2f(m - top), b = __builtin_amdgcn_exp2f(ml[0] - top);
    m = top;
    l = l * a + ml[1] * b;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(other + d * 32 + g * 8 + end_half * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][g * 4 + i] = fmaf(o[d][g * 4 + i], a, x[i] * b);
      }
  }
  if (n_pieces == 1) {
    if (row0 + end_row >= n_rows) return;
    const int row = row0 + end_row;
    const int head = row_head(p, it.kvh, row);
    const int64_t t = row_token(p, it.seq, row);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    bf16_t *dst = p.o + t * p.o_stride + head * HD;
    // (a lane has four channels of each eight and the lane 32 further the others: they trade, for 16 bytes of one eight each)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        u32x4_t v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const auto r = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[d][g * 4 + 2 * i] * inv, o[d][g * 4 + 2 * i + 1] * inv),
                                                          pack_bf16x2(o[d][g * 4 + 4 + 2 * i] * inv, o[d][g * 4 + 5 + 2 * i] * inv), false, false);
          v[i] = r[0];
          v[2 + i] = r[1];
        }
        *reinterpret_cast<u32x4_t *>(dst + d * 32 + (g + end_half) * 8) = v;
      }
    if (end_half == 0 && p.lse) p.lse[t * p.n_heads + head] = lse_of(m, l);
  } else {
    float *part = part_of<HD>(pl, it.first + it.piece * it.n_tiles + it.n_tiles - 1 - it.tile, it.kvh, p.n_kv);
    const int r = wave * 32 + end_row;
    float *mine = part + wave * 32 * HD + end_lane * 4;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4_t *>(mine + (d * 4 + g) * 256) = f32x4_t{o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]};
    if (end_half == 0) *reinterpret_cast<f32x2_t *>(part + kRows * HD + r * 2) = f32x2_t{m, l};
  }
}

// ---- rows split along the keys: their pieces joined, in order ------------------------------------------------------------
// The split tile with number x, counted as tiles would be without pieces: which it is, how many pieces it has (1: nothing to join) and
// where the first one's sums lie.
struct Split { Seq seq; int tile, n; size_t step; const float *src; };
template <int HD>
__device__ __forceinline__ Split find_split(const AttnParams &p, const AttnPlan &pl, Sums &sums, int x, int kvh) {
  Split r = {};
  const Cut cut = cut_of<4>(p, pl, sums);
  count_items<4>(p, pl, kUnsplit, cut.first, sums);
  const Item whole = find_seq<false>(p, pl, kUnsplit, cut.first, sums, x);
  count_items<4>(p, pl, cut.keys, cut.first, sums);
  if (whole.n_tiles == 0) return r;
  r.seq = whole.seq;
  r.tile = x - whole.first;
  r.n = pieces_of(tile_range(p, whole.seq, r.tile, pl.tile_rows), cut.keys);
  const Item it = find_seq<true>(p, pl, cut.keys, cut.first, sums, whole.s);
  const int x0 = it.first + it.n_tiles - 1 - r.tile;
  // (chunks that overlap may have more pieces than there is room for)
  if (x0 < 0 || ((long)x0 + (long)(r.n - 1) * it.n_tiles + 1) * p.n_kv > pl.max_items) r.n = 0;
  r.step = (size_t)it.n_tiles * p.n_kv * ((size_t)pl.tile_rows * (HD + 2));
  r.src = part_of<HD>(pl, x0, kvh, p.n_kv);
  return r;
}
// Sums of C channels of row r over its pieces, `at` floats into each; eight pieces' loads on their way at a time
template <int HD, int C>
__device__ __forceinline__ void join_pieces(const Split &sp, int tile_rows, int r, int at, float &top, float &sum, float (&acc)[C]) {
  top = kNoMax;
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < C; ++e) acc[e] = 0.f;
  for (int k0 = 0; k0 < sp.n; k0 += 8) {
    float v[8][C];
    f32x2_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float *from = sp.src + (size_t)min(k0 + k, sp.n - 1) * sp.step;
      w[k] = *reinterpret_cast<const f32x2_t *>(from + tile_rows * HD + r * 2);
#pragma unroll
      for (int e = 0; e < C; ++e) v[k][e] = from[at + e];
    }
    float higher = top;
#pragma unroll
    for (int k = 0; k < 8; ++k) higher = fmaxf(higher, w[k][0]);
    const float f0 = __builtin_amdgcn_exp2f(top - higher);
    top = higher;
    sum *= f0;
#pragma unroll
    for (int e = 0; e < C; ++e) acc[e] *= f0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool is = k0 + k < sp.n;                  // (not by a factor of 0: the sums may be infinite)
      const float f = __builtin_amdgcn_exp2f(w[k][0] - top);
      sum = is ? fmaf(w[k][1], f, sum) : sum;
#pragma unroll
      for (int e = 0; e < C; ++e) acc[e] = is ? fmaf(v[k][e], f, acc[e]) : acc[e];
    }
  }
}
// The tile kernel's: one wavefront to 1 KB of every piece, 32 rows of eight channels.
template <int HD>
__global__ __launch_bounds__(256) void ff_attn_join_kernel(AttnParams p, AttnPlan pl) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int runs = pl.tile_rows / 32 * (HD / 8);                // of 1 KB in a tile
  const int id = (int)blockIdx.x * 4 / runs, run = (int)blockIdx.x * 4 % runs + wave;
  const int x = p.by_kv(id), kvh = id - x * p.n_kv;
  __shared__ Sums sums_s;
  const Split sp = find_split<HD>(p, pl, sums_s, x, kvh);
  if (sp.n <= 1) return;
  const int r = run / (HD / 8) * 32 + (lane & 31), c = run % (HD / 8) * 8 + (lane >> 5) * 4;
  const int row = sp.tile * pl.tile_rows + r;
  if (row >= sp.seq.n * p.group) return;
  float top, sum, acc[4];
  join_pieces<HD, 4>(sp, pl.tile_rows, r, run * 256 + lane * 4, top, sum, acc);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const int64_t t = row_token(p, sp.seq, row);
  const int head = row_head(p, kvh, row);
  *reinterpret_cast<u32x2_t *>(p.o + t * p.o_stride + head * HD + c) =
      u32x2_t{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
  if (c == 0 && p.lse) p.lse[t * p.n_heads + head] = lse_of(top, sum);
}
// The few-row kernel's, where one workgroup would have many rows to join: one wavefront to a row.
template <int HD>
__global__ __launch_bounds__(256) void ff_attn_join_rows_kernel(AttnParams p, AttnPlan pl) {
  constexpr int C = HD / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = (int)blockIdx.x * 4 / pl.tile_rows, r = (int)blockIdx.x * 4 % pl.tile_rows + wave;
  const int x = p.by_kv(id), kvh = id - x * p.n_kv;
  __shared__ Sums sums_s;
  const Split sp = find_split<HD>(p, pl, sums_s, x, kvh);
  const int row = sp.tile * pl.tile_rows + r;
  if (sp.n <= 1 || row >= sp.seq.n * p.group) return;
  float top, sum, acc[C];
  join_pieces<HD, C>(sp, pl.tile_rows, r, r * HD + lane * C, top, sum, acc);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const int64_t t = row_token(p, sp.seq, row);
  const int head = row_head(p, kvh, row);
  bf16_t *dst = p.o + t * p.o_stride + head * HD + lane * C;
  if (C == 2) *reinterpret_cast<uint32_t *>(dst) = pack_bf16x2(acc[0] * inv, acc[C - 1] * inv);
  else *dst = f32_to_bf16(acc[0] * inv);
  if (lane == 0 && p.lse) p.lse[t * p.n_heads + head] = lse_of(top, sum);
}

// one wavefront per sequence and table
__global__ __launch_bounds__(64) void ff_attn_validate_kernel(AttnParams p, int32_t *flag) {
  const int s = blockIdx.x, lane = threadIdx.x;
  const int a = p.starts[s], b = p.starts[s + 1];
  bool bad = a < 0 || b < a || b > p.T || p.lens[s] < 0 || p.lens[s] > most_keys(p);
  const Seq q = seq_of(p, s);
  const int first = p.window > 0 ? max(0, q.keys - q.n + 1 - min(p.window, kMaxKeys)) >> p.page_shift : 0;
  const int pages = p.table && q.n > 0 ? (int)(((long)q.keys + (1 << p.page_shift) - 1) >> p.page_shift) : 0;
  for (int i = first + lane; i < pages; i += 64) {
    const int page = p.table[s * p.seq_tables + (size_t)blockIdx.y * p.head_tables + i];
    bad = bad || page < 0 || page >= p.n_pages;
  }
  if (__any(bad) && lane == 0) atomicMax(flag, s + 1);
}

size_t few_lds(int hd, int nb) {
  const size_t ring = (size_t)kFewWaves * 2 * 32 * hd * 2;
  const size_t join = (size_t)kFewWaves * 16 * nb * (hd + 4 + 2) * 4;
  return std::max(ring, join);
}
size_t tile_lds(int hd, int rw, int kw) {
  const size_t ring = (size_t)kw * 4 * kTileKeys * hd * 2;
  const size_t join = kw > 1 ? (size_t)32 * rw * (hd + 4 + 2) * 4 : 0;
  return std::max(ring, join);
}

template <int HD>
hipError_t raise_limits() {
  hipError_t e = hipSuccess;
  auto raise = [&](const void *fn, size_t lds) {
    if (e == hipSuccess) e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  };
  const auto few = [&](auto eight) {
    raise(reinterpret_cast<const void *>(ff_attn_few_kernel<HD, 1, eight()>), few_lds(HD, 1));
    raise(reinterpret_cast<const void *>(ff_attn_few_kernel<HD, 2, eight()>), few_lds(HD, 2));
  };
  const auto tile = [&](auto src) {
    raise(reinterpret_cast<const void *>(ff_attn_tile_kernel<HD, 4, 2, src()>), tile_lds(HD, 4, 2));
    raise(reinterpret_cast<const void *>(ff_attn_tile_kernel<HD, 8, 1, src()>), tile_lds(HD, 8, 1));
  };
  few(std::false_type());
  few(std::true_type());
  tile(std::integral_constant<Source, kRows>());
  tile(std::integral_constant<Source, kPages>());
  tile(std::integral_constant<Source, kPages8>());
  return e;
}

// One token's keys go to a piece for every CU, and no more: its pieces are joined by one workgroup.  Many tokens' are cut finer, for
// their lengths differ.  (Heads of 128, us with 256 / 512 / 1024 pieces: 8 key heads, one token over
// 8191 keys, whose pieces were 256 / 128 / 64 keys long for it, 15.7 / 19.9 / 33.8, over 32768 28.6 / 32.0 / 44.3; 48 tokens over up to 16384 137 / 97 / 94.)
// Over keys in 8 bits, which come in half the time, to fewer: with 512 / 768 / 1024 pieces 8 key heads of 128, 48 tokens over up to 16384 keys
// 49.7 / 46.5 / 50.4, all over 16384 303 / 281 / 291, 96 over up to 8192 60.9 / 53.6 / 52.3, 200 over up to 2000 49.5 / 52.2 / 52.0; 4 key heads, 48
// tokens 40.2 / 38.4 / 46.7; heads of 64 27.3 / 28.2 / 31.2.
// Selected pages are few for every token, long context or short, so they are not cut finer than for one token.  256 / 512 / 1024 pieces over 8 bits: 8
// key heads of 128, 48 tokens with 32 pages of 64 kept, all of which have 2112 keys, 39.0 / 48.9 / 46.2, of contexts of up to 32768 (15 have some
// 2100 keys, 22 fewer than 256) 26.3 / 29.7 / 32.8; 100 tokens with 16 kept, equal 44.8 / 44.8 / 63.0, ragged 31.4 / 29.5 / 35.7; 4 key heads, 48
// equal 35.9 / 37.7 / 33.8, ragged 20.6 / 26.9 / 25.8; heads of 64 23.6 / 27.4 / 29.9, ragged 20.0 / 17.7 / 19.8.
int few_target(long tiles, int n_kv, bool eight, bool selected) {
  if (selected || tiles * n_kv < 128) return kFewGrid / 2;
  return eight ? 3 * kFewGrid / 2 : 2 * kFewGrid;
}
int most_few_target(long tiles, int n_kv) { return few_target(tiles, n_kv, false, false); }
// Items that a plan can have at most: about `target` pieces and one more for each of the tiles and key heads.
long most_items(long tiles, int n_kv, int target) { return tiles * n_kv + target + 16; }
// (More items than counters: not split.  32768 keys among sequences of 200, 8 key heads of 128: 1400 tokens 273 us, 1600 670.)
size_t item_bytes(int tile_rows, int head_dim) { return (size_t)tile_rows * (head_dim + 2) * sizeof(float); }
// Chunks with fewer (128-row tile, key head) than this are split along the keys (see choose).
long few_items(long n_seqs) { return n_seqs == 1 ? 192 : 384; }
int tile_target(long n_seqs, int head_dim) { return n_seqs > 1 && head_dim == 64 ? 512 : 256; }

// How the call is cut.  rows of a sequence = new tokens times heads of a group.
struct Choice {
  AttnPlan few, tile;
  int nb = 0, rw = 0;             // 0: that kernel is not launched
  long tiles = 0, few_tiles = 0;  // most tiles of each
  size_t bytes = 0;
};
// `even`: a prompt's last tiles have not many more keys than the others.
Choice choose(int n_heads, int n_kv, int head_dim, int n_tokens, int n_seqs, int max_chunk, bool paged, bool even, bool eight, bool selected) {
  Choice c;
  const int group = n_heads / n_kv;
  const long rows = (long)n_tokens * group, chunk_rows = (long)max_chunk * group, seqs = std::min(n_seqs, n_tokens);
  constexpr long kAll = 0x7fffffffffffL;
  const auto set = [&](AttnPlan &pl, int tile_rows, long tiles, long above, long upto, int target, int min_steps) {
    pl.tile_rows = tile_rows;
    pl.rows_above = above;
    pl.rows_upto = upto;
    pl.min_steps = min_steps;
    pl.target = most_items(tiles, n_kv, target) <= kAttnCounters ? target : 0;
    pl.max_items = (int)std::min<long>(most_items(tiles, n_kv, pl.target), 0x7fffffff);   // (the price of a call is summed in fp32)
    pl.part_at = c.bytes / sizeof(float);
    if (pl.target > 0) c.bytes += pl.max_items * item_bytes(tile_rows, head_dim);
  };
  // One workgroup joins a tile's pieces where these have few rows in all; a launch more costs 1 to 3 us, and many rows several times
  // that.  (us joined by the last piece and by a launch: 8 key heads, one token of 4 rows over 8191 keys 15.4 and 16.5, 32768 28.2 and
  // 31.1; 4 key heads, one token of 7 rows over 16384 keys 24.1 and 20.5, four tokens 56 and 24.)
  const auto joins_here = [&](long tile_rows, long tiles) { return tile_rows <= 8 && tile_rows * few_target(tiles, n_kv, eight, selected) <= 256 * tiles * n_kv; };
  // (the rows' own tiles and a part-filled one for each sequence; a call with more of them than are counted has longer chunks than the host
  // knows)
  if (paged && chunk_rows <= 32 && rows / 16 + seqs <= kMostItems) {
    c.nb = chunk_rows <= 16 ? 1 : 2;
    c.few_tiles = rows / (16 * c.nb) + seqs;
    set(c.few, 16 * c.nb, c.few_tiles, 0, kAll, few_target(c.few_tiles, n_kv, eight, selected), 4);
    c.few.join_here = joins_here(chunk_rows, c.few_tiles);
    return c;
  }
  // sequences that generate one token beside chunks; blocks over selected pages that are mostly full have no more of them than a
  // prompt's last, whose tile takes no longer than the others' (8192 tokens in blocks of 128: 4.7 us less without a launch for them)
  const bool both = paged && n_seqs > 1 && group <= 16 && !(selected && 2l * n_tokens >= (long)n_seqs * max_chunk);
  // 256 rows, or 128 rows and two groups of keys: half as many steps for the longest tile, but twice the tiles, and steps that take 1.4
  // times as long.  256 rows where the others would be more than a tile for every CU, and where one causal prompt's longest tile takes as long as the
  // launch, where they are themselves.  (us with 128 and 256 rows, 8 key heads of 128 / 64.  One causal prompt of 2048 tokens, 256
  // tiles of 256 rows: 49 and 55 / 34 and 45, of 2560, 320 tiles, 79 and 70 / 53 and 54, of 4096 157 and 131 / 104 and 93.  In a window of
  // 512, 1700 tokens, 208 tiles: 37 and 25 / 27 and 20.  Prompts of 512 tokens, two of them, 128 tiles: 18 and 22 / 12 and 16, six 42 and
  // 31 / 27 and 19; 12 of 120, 176 tiles, 19 and 13 / 13 and 10; 100 and 1500 together, 200 tiles, which the host does not know, 35 and 41 / 25 and 34.
  // Chunks over longer contexts, which are split along the keys below 192 or 384 tiles of 128 rows: heads of 128, three chunks of 900 tokens, 337
  // tiles of 256, 79 and 70, two of 1100, 275 tiles, 106 and 97, six of 500, 375 tiles, 158 and 163; heads of 64, whose workgroups are two to a CU,
  // three of 900 over 9000 keys 121 and 179.)
  c.rw = rows / 256 * n_kv > (paged ? (head_dim == 128 ? 264 : 384) : even ? 128 : 264) ? 8 : 4;
  const int tile_rows = 32 * c.rw;
  c.tiles = rows / tile_rows + seqs;
  // Split into a piece for every CU where whole rows would leave many idle: partial sums written and joined cost some 6 us, and as much
  // again for twice as many.  With sequences of different lengths the longest may take the launch's whole time, so those are split
  // up to twice as many items.  (us in 256 pieces and whole, 8 key heads of 128: one chunk of 512 tokens over 8192 keys, 128 items,
  // 90 and 133; 1024 tokens, 256 items, 157 and 148.  Chunks of up to 500 of 8 heads of 64 with single tokens, 336 items, 76 and 85;
  // 24 sequences of up to 300 tokens, 590 items, 101 and 84.)
  const long items = rows / 128 * n_kv;
  const bool split = paged && items < few_items(n_seqs);
  set(c.tile, tile_rows, c.tiles, both ? 16 : 0, kAll, split ? tile_target(n_seqs, head_dim) : 0, 4);
  if (both) {
    c.nb = 1;
    c.few_tiles = seqs;
    set(c.few, 16, seqs, 0, 16, few_target(seqs, n_kv, eight, selected), 4);
    c.few.join_here = joins_here(group, seqs);
  }
  return c;
}

template <int HD>
hipError_t launch(const AttnParams &p, Choice &c, hipStream_t s) {
  if (c.bytes > p.part_bytes) return hipErrorInvalidValue;
  c.few.part = p.part + c.few.part_at;
  c.tile.part = p.part + c.tile.part_at;
  if (c.nb) {
    // (four workgroups of narrow heads in 8 bits on a CU, which have half the bytes on their way that the others have: 48 tokens of 8 key heads of
    // 64 over up to 16384 keys in pages of 16 / 64 47.3 / 33.4 us with two, 32.6 / 28.5 with four)
    const int most = HD == 64 && p.k_scale ? 2 * kFewGrid : kFewGrid;
    const dim3 grid((unsigned)std::min(c.few.max_items, most)), block(64 * kFewWaves);
    const size_t lds = few_lds(HD, c.nb);
    const auto few = [&](auto eight) {
      if (c.nb == 1) hipLaunchKernelGGL((ff_attn_few_kernel<HD, 1, eight()>), grid, block, lds, s, p, c.few);
      else hipLaunchKernelGGL((ff_attn_few_kernel<HD, 2, eight()>), grid, block, lds, s, p, c.few);
    };
    if (p.k_scale) few(std::true_type());
    else few(std::false_type());
    if (c.few.target > 0 && !c.few.join_here)
      hipLaunchKernelGGL((ff_attn_join_rows_kernel<HD>), dim3((unsigned)(c.few_tiles * p.n_kv * (c.few.tile_rows / 4))), dim3(256), 0, s, p, c.few);
  }
  if (c.rw) {
    // (a launch's dimension has 32 bits of threads)
    const unsigned items = (unsigned)c.tile.max_items, across = std::min(items, 1u << 20);
    const dim3 grid(across, (items + across - 1) / across), block(512);
    const size_t lds = tile_lds(HD, c.rw, 8 / c.rw);
    const auto tile = [&](auto src) {
      if (c.rw == 4) hipLaunchKernelGGL((ff_attn_tile_kernel<HD, 4, 2, src()>), grid, block, lds, s, p, c.tile);
      else hipLaunchKernelGGL((ff_attn_tile_kernel<HD, 8, 1, src()>), grid, block, lds, s, p, c.tile);
    };
    if (p.k_scale) tile(std::integral_constant<Source, kPages8>());
    else if (p.table) tile(std::integral_constant<Source, kPages>());
    else tile(std::integral_constant<Source, kRows>());
    if (c.tile.target > 0)
      hipLaunchKernelGGL((ff_attn_join_kernel<HD>), dim3((unsigned)(c.tiles * p.n_kv * (c.tile.tile_rows / 32 * (HD / 8) / 4))), dim3(256), 0, s, p, c.tile);
  }
  return hipGetLastError();
}

}  // namespace

// The most that any call of up to n_tokens tokens and n_seqs sequences takes, whatever its longest chunk is: more tokens or sequences
// never have less, although a call of very many takes none (choose gives up its split where the items would be more than the counters).
size_t ff_attention_part_bytes(int n_heads, int n_kv, int head_dim, int n_tokens, int n_seqs) {
  const int group = n_heads / n_kv;
  const long rows = (long)n_tokens * group, seqs = std::min(n_seqs, n_tokens);
  // (a plan that is split has no more items than counters, and a call of fewer tiles no more than one of more)
  const auto bytes = [&](long tiles, int target, int tile_rows) {
    return std::min<long>(most_items(tiles, n_kv, target), kAttnCounters) * item_bytes(tile_rows, head_dim);
  };
  const auto few = [&](long tiles, int tile_rows) { return bytes(tiles, most_few_target(tiles, n_kv), tile_rows); };
  // tiles of 128 rows, the only ones of calls that are split, beside sequences of at most 16 rows
  const long whole = std::min(rows / 128, (few_items(n_seqs) - 1) / n_kv);
  size_t most = bytes(whole + seqs, tile_target(n_seqs, head_dim), 128) + (n_seqs > 1 && group <= 16 ? few(seqs, 16) : 0);
  if (group <= 16) most = std::max(most, few(rows / 16 + seqs, 16));
  if (group <= 32) most = std::max(most, few(rows / 32 + seqs, 32));
  return most;
}

static Choice choose(const AttnParams &p, int head_dim, int max_chunk) {
  const bool even = !p.causal || p.n_seqs > 1 || (p.window > 0 && p.window < p.T);
  return choose(p.n_heads, p.n_kv, head_dim, p.T, p.n_seqs, max_chunk, p.table != nullptr, even, p.k_scale != nullptr, p.selected);
}

size_t ff_attention_need(const AttnParams &p, int head_dim, int max_chunk) {
  return choose(p, head_dim, max_chunk).bytes;
}

hipError_t ff_attention_init() {
  hipError_t e = raise_limits<128>();
  return e == hipSuccess ? raise_limits<64>() : e;
}

hipError_t ff_launch_attention(const AttnParams &p, int head_dim, int max_chunk, hipStream_t s) {
  Choice c = choose(p, head_dim, max_chunk);
  // Prompts' longest tiles first while a CU has a few tiles; with many, tiles of one sequence side by side share its keys in L2.  (us by
  // length and by sequence, causal, 8 key heads of 64 / 128: 13 prompts of up to 861 tokens, 616 tiles, 25.7 and 31.0 / 39.6 and
  // 45.7; 16 of 1024, 2176 tiles, 95 and 109 / 204 and 205; 32 of 1024, 4352 tiles, 210 and 214 / 406 and 397.  In a window of 300 the
  // last tiles are no longer than others: 16 of 1024 76 and 81 / 171 and 159.)
  c.tile.by_tile = !p.table && p.causal && p.window == 0 && p.n_seqs > 1 && p.n_seqs <= 64 && c.tiles * p.n_kv <= 12 * 256;
  return head_dim == 128 ? launch<128>(p, c, s) : launch<64>(p, c, s);
}

hipError_t ff_launch_validate_pages(const AttnParams &p, int32_t *flag, hipStream_t s) {
  hipLaunchKernelGGL(ff_attn_validate_kernel, dim3(p.n_seqs, p.head_tables ? p.n_kv : 1), dim3(64), 0, s, p, flag);
  return hipGetLastError();
}
