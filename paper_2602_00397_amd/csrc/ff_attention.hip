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

#include <algorithm>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

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

// How long a piece is, from the work of the whole call; every wavefront finds the same.
__device__ __forceinline__ int piece_keys(const AttnParams &p, const AttnPlan &pl) {
  if (pl.target <= 0) return kUnsplit;
  const int lane = threadIdx.x & 63;
  float steps = 0.f;
  for (int s0 = 0; s0 < p.n_seqs; s0 += 64)
    if (s0 + lane < p.n_seqs) steps += price_of(p, pl, seq_of(p, s0 + lane));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) steps += __shfl_xor(steps, off);
  return __builtin_amdgcn_readfirstlane(piece_keys_for(p, pl, steps));
}

struct Item {
  bool found;
  int s, tile, piece, kvh;   // piece of tile of sequence s, key head kvh
  int n_tiles, n_pieces;     // of the sequence (a tile may have fewer pieces)
  int first;                 // number of the sequence's first (tile, piece)
  Seq seq;
};
// The (tile, piece) number x, counted over the sequences, or, with by_seq, the first one of sequence x.
__device__ __forceinline__ Item find_item(const AttnParams &p, const AttnPlan &pl, int keys_per_piece, int x, bool by_seq) {
  const int lane = threadIdx.x & 63;
  Item it;
  it.found = false;
  int base = 0;
  for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
    Seq q = {0, 0, 0};
    int tiles = 0, pieces = 1;
    if (s0 + lane < p.n_seqs) {
      q = seq_of(p, s0 + lane);
      tiles = tiles_of(p, pl, q.n);
      pieces = seq_pieces(p, pl, q, keys_per_piece);
    }
    const int mine = tiles * pieces;
    int incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(incl, d);
      if (lane >= d) incl += up;
    }
    const int excl = base + incl - mine;
    const unsigned long long hit = __ballot(by_seq ? s0 + lane == x : x >= excl && x < excl + mine);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      it.found = true;
      it.s = s0 + l;
      it.first = __builtin_amdgcn_readlane(excl, l);
      it.n_tiles = __builtin_amdgcn_readlane(tiles, l);
      it.n_pieces = __builtin_amdgcn_readlane(pieces, l);
      it.seq.t0 = __builtin_amdgcn_readlane(q.t0, l);
      it.seq.n = __builtin_amdgcn_readlane(q.n, l);
      it.seq.keys = __builtin_amdgcn_readlane(q.keys, l);
      return it;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return it;
}
// Workgroup number -> item.  Key heads go innermost (workgroups id mod 8 share an XCD, so its L2 keeps one head's keys where there
// are eight), then the tiles of one piece, the last first: under a causal mask those have the most keys.
__device__ __forceinline__ Item work_of(const AttnParams &p, const AttnPlan &pl, int keys_per_piece, int id) {
  const int x = id / p.n_kv;
  Item it = find_item(p, pl, keys_per_piece, x, false);
  if (it.found) {
    const int local = x - it.first;
    it.kvh = id - x * p.n_kv;
    it.piece = local / it.n_tiles;
    it.tile = it.n_tiles - 1 - (local - it.piece * it.n_tiles);
  }
  return it;
}

// partial sums of a piece: tile_rows rows of HD sums, then tile_rows pairs of maximum and sum
template <int HD>
__device__ __forceinline__ float *part_of(const AttnPlan &pl, int x, int kvh, int n_kv) {
  return pl.part + ((size_t)x * n_kv + kvh) * ((size_t)pl.tile_rows * (HD + 2));
}

// where keys lie
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
    ks.table = p.table + (size_t)it.s * p.table_stride;
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
// Copies number i of the tile that starts at key j (a multiple of 32) to LDS: 1 KB of K and 1 KB of V.  Keys from `end` on are
// replaced by the last one.  The keys of one copy (4 or 8, aligned) are in one page.
template <int HD, bool PAGED>
__device__ __forceinline__ void copy_keys(const KeySource<PAGED> &ks, int i, int j, int end, uint32_t lds_k, uint32_t lds_v, int lane) {
  constexpr int KPI = 512 / HD;
  int key, chunk;
  copied<HD>(i, lane, key, chunk);
  const int first = min(j + i * KPI, end - 1);      // (wave-uniform)
  const int mine = min(j + key, end - 1);
  if (PAGED) {
    // (by a scalar load: the wait for it is not one for the copies before it)
    int page = *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(ks.table + (first >> ks.shift)));
    page = __builtin_amdgcn_readfirstlane((unsigned)page < (unsigned)ks.n_pages ? page : 0);
    const size_t at = (size_t)page * ks.page_elems;
    const uint32_t off = (uint32_t)(((mine & ((1 << ks.shift) - 1)) * HD + chunk * 8) * 2);
    gload_lds16_at(ks.k + at, off, lds_k + i * 1024);
    gload_lds16_at(ks.v + at, off, lds_v + i * 1024);
  } else {
    const uint8_t *kb = reinterpret_cast<const uint8_t *>(ks.k) + (size_t)first * ks.k_pitch;
    const uint8_t *vb = reinterpret_cast<const uint8_t *>(ks.v) + (size_t)first * ks.v_pitch;
    gload_lds16_at(kb, (uint32_t)(mine - first) * ks.k_pitch + chunk * 16, lds_k + i * 1024);
    gload_lds16_at(vb, (uint32_t)(mine - first) * ks.v_pitch + chunk * 16, lds_v + i * 1024);
  }
}

// infinities and NaN of a pair of bf16 values set to 0; `any` collects whether there were some
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, uint32_t &any) {
  const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
  any |= lo | hi;
  return w & ~(lo | hi);
}
__device__ __forceinline__ float lds_bf16(uint32_t addr) {
  return __uint_as_float((uint32_t)(*reinterpret_cast<const __attribute__((address_space(3))) uint16_t *>(addr)) << 16);
}

// natural log of the sum that belongs to a maximum (in powers of two of the scaled products) and a sum
__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.f || l != l ? (m + __log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// ---- few rows: single tokens of a generation step ------------------------------------------------------------------------
// HBM-bound: every key is read once for at most 16 NB rows.  Four wavefronts, each with keys of its own (32 at a time, every
// fourth 32 of the piece), its own two stages of LDS and its own softmax state, without barriers until they join at the end.
template <int HD, int NB>
__global__ __launch_bounds__(256) void ff_attn_few_kernel(AttnParams p, AttnPlan pl) {
  constexpr int KS = HD / 32, DB = HD / 16, NI = 32 * HD * 2 / 1024;
  constexpr uint32_t kHalf = 32 * HD * 2, kStage = 2 * kHalf;
  constexpr int kRows = 16 * NB, kPitch = HD + 4;
  extern __shared__ __align__(256) uint8_t lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l16 = lane & 15, quad = lane >> 4;
  const int kpp = piece_keys(p, pl);
  const Item it = work_of(p, pl, kpp, blockIdx.x);
  if (!it.found) return;
  const int n_rows = it.seq.n * p.group, row0 = it.tile * kRows;
  const Range range = tile_range(p, it.seq, it.tile, kRows);
  const int n_pieces = pieces_of(range, kpp);
  if (it.piece >= n_pieces) return;
  const int beg = range.lo + it.piece * kpp, end = min(range.hi, beg + kpp);
  const KeySource<true> ks = key_source<HD, true>(p, it);
  const uint32_t ring = lds_addr_of(lds) + wave * 2 * kStage;

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
    const bf16_t *src = p.q + (int64_t)(it.seq.t0 + r / p.group) * p.q_stride + (it.kvh * p.group + r % p.group) * HD + quad * 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[b][s] = *reinterpret_cast<const u32x4_t *>(src + s * 32);
  }
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) {
    all_lo = max(all_lo, __shfl_xor(all_lo, off));
    all_hi = min(all_hi, __shfl_xor(all_hi, off));
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);

  f32x4_t o[NB][DB];
  float m[NB], l[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    m[b] = kNoMax;
    l[b] = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[b][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  auto copy_tile = [&](int j, uint32_t stage) {
#pragma unroll
    for (int i = 0; i < NI; ++i) copy_keys<HD, true>(ks, i, j, end, stage, stage + kHalf, lane);
  };
  int j = beg + wave * 32;
  uint32_t stage = ring;
  wait_copies<0>();                       // (q is here: only copies are counted from now on)
  if (j < end) copy_tile(j, stage);
  for (; j < end; j += 128) {
    const bool more = j + 128 < end;
    if (more) {
      copy_tile(j + 128, stage ^ ring ^ (ring + kStage));
      wait_copies<2 * NI>();
    } else {
      wait_copies<0>();
    }
    // S^T: 32 keys by the rows
    f32x4_t s[NB][2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      u32x4_t kf[KS];
#pragma unroll
      for (int c = 0; c < KS; ++c) kf[c] = lds_read16(stage + chunk_at<HD>(kt * 16 + l16, c * 4 + quad));
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        s[b][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KS; ++c) s[b][kt] = mfma16(kf[c], q[b][c], s[b][kt]);
      }
    }
    const bool masked = j < all_lo || j + 32 > all_hi;
    u32x4_t pk[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (masked) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = j + kt * 16 + quad * 4 + i;
            s[b][kt][i] = key >= see[b].lo && key < see[b].hi ? s[b][kt][i] : -INFINITY;
          }
      }
      float mx = fmaxf(fmaxf(fmaxf(s[b][0][0], s[b][0][1]), fmaxf(s[b][0][2], s[b][0][3])),
                       fmaxf(fmaxf(s[b][1][0], s[b][1][1]), fmaxf(s[b][1][2], s[b][1][3])));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * p.scale_log2;
      if (__any(mx > m[b] + kLazy)) {
        const float m_new = fmaxf(m[b], mx), a = __builtin_amdgcn_exp2f(m[b] - m_new);
        m[b] = m_new;
        l[b] *= a;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[b][d][i] *= a;
      }
      float e[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        e[x] = __builtin_amdgcn_exp2f(fmaf(s[b][x >> 2][x & 3], p.scale_log2, -m[b]));
        l[b] += e[x];
      }
      pk[b] = u32x4_t{pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])};
    }
    // O^T += V^T P^T
    uint32_t odd = 0;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      const int c = d * 2 + ((l16 & 3) >> 1);
      u32x2_t v0 = lds_read_tr(stage + kHalf + chunk_at<HD>(quad * 4 + (l16 >> 2), c) + (l16 & 1) * 8);
      u32x2_t v1 = lds_read_tr(stage + kHalf + chunk_at<HD>(16 + quad * 4 + (l16 >> 2), c) + (l16 & 1) * 8);
      u32x4_t vf = {v0[0], v0[1], v1[0], v1[1]};
      if (masked) {
#pragma unroll
        for (int x = 0; x < 4; ++x) vf[x] = finite_pair(vf[x], odd);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) o[b][d] = mfma16(vf, pk[b], o[b][d]);
    }
    if (masked && __any(odd != 0)) {
      // infinities and NaN among the values (0 in the product): they reach the rows that see their key, and no other
#pragma unroll 1
      for (int x = 0; x < 32; ++x) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int ch = d * 16 + quad * 4 + i;
            const float v = lds_bf16(stage + kHalf + chunk_at<HD>(x, ch >> 3) + (ch & 7) * 2);
            if (!(fabsf(v) < INFINITY))
#pragma unroll
              for (int b = 0; b < NB; ++b)
                if (j + x >= see[b].lo && j + x < see[b].hi) o[b][d][i] += v;
          }
      }
    }
    stage = stage ^ ring ^ (ring + kStage);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // nothing of this stage is still being read when it is filled again
  }

  // join the four wavefronts' sums
  float *joined = reinterpret_cast<float *>(lds);                        // [4][kRows][kPitch]
  float *ml = joined + 4 * kRows * kPitch;                               // [4][kRows][2]
  __syncthreads();
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    l[b] += __shfl_xor(l[b], 16);
    l[b] += __shfl_xor(l[b], 32);
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
  const bool whole = n_pieces == 1;
  float *part = whole ? nullptr : part_of<HD>(pl, it.first + it.piece * it.n_tiles + it.n_tiles - 1 - it.tile, it.kvh, p.n_kv);
  for (int i = threadIdx.x; i < kRows * (HD / 4); i += 256) {
    const int r = i / (HD / 4), c = (i % (HD / 4)) * 4;
    if (row0 + r >= n_rows) break;
    float mw[4], top = kNoMax, sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      mw[w] = ml[(w * kRows + r) * 2];
      top = fmaxf(top, mw[w]);
    }
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = __builtin_amdgcn_exp2f(mw[w] - top);
      sum = fmaf(ml[(w * kRows + r) * 2 + 1], a, sum);
      const f32x4_t x = *reinterpret_cast<const f32x4_t *>(joined + (w * kRows + r) * kPitch + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(x[e], a, acc[e]);
    }
    if (whole) {
      const int row = row0 + r;
      const int64_t t = it.seq.t0 + row / p.group;
      const int head = it.kvh * p.group + row % p.group;
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      *reinterpret_cast<u32x2_t *>(p.o + t * p.o_stride + head * HD + c) =
          u32x2_t{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
      if (c == 0 && p.lse) p.lse[t * p.n_heads + head] = lse_of(top, sum);
    } else {
      *reinterpret_cast<f32x4_t *>(part + r * HD + c) = acc;
      if (c == 0) {
        part[kRows * HD + r * 2] = top;
        part[kRows * HD + r * 2 + 1] = sum;
      }
    }
  }
}

// ---- many rows: prompts and chunks of them --------------------------------------------------------------------------------
// MFMA-bound.  WAVES wavefronts of 32 rows each share the key tiles of 64 in two stages of LDS.
template <int HD, int WAVES, bool PAGED>
__global__ __launch_bounds__(WAVES * 64) void ff_attn_tile_kernel(AttnParams p, AttnPlan pl) {
  constexpr int KS = HD / 16, DB = HD / 32, NI = kTileKeys * HD * 2 / 1024 / WAVES;
  constexpr uint32_t kHalf = kTileKeys * HD * 2, kStage = 2 * kHalf;
  constexpr int kRows = 32 * WAVES;
  extern __shared__ __align__(256) uint8_t lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15, grp = lane >> 4;
  const int kpp = piece_keys(p, pl);
  const Item it = work_of(p, pl, kpp, blockIdx.x);
  if (!it.found) return;
  const int n_rows = it.seq.n * p.group, row0 = it.tile * kRows + wave * 32;
  const Range range = tile_range(p, it.seq, it.tile, kRows);
  const int n_pieces = pieces_of(range, kpp);
  if (it.piece >= n_pieces) return;
  const int beg = range.lo + it.piece * kpp, end = min(range.hi, beg + kpp);
  const KeySource<PAGED> ks = key_source<HD, PAGED>(p, it);
  const uint32_t ring = lds_addr_of(lds);

  const int row = min(row0 + l32, n_rows - 1);
  Range see = row_range(p, it.seq, row);
  see.hi = min(see.hi, end);
  const int head = it.kvh * p.group + row % p.group;
  const int64_t t = it.seq.t0 + row / p.group;
  u32x4_t q[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u32x4_t *>(p.q + t * p.q_stride + head * HD + s * 16 + half * 8);
  // (limits grow with the row: the first and the last row of the wavefront have the extremes)
  const int lo_first = __builtin_amdgcn_readlane(see.lo, 0), lo_last = __builtin_amdgcn_readlane(see.lo, 31);
  const int hi_first = __builtin_amdgcn_readlane(see.hi, 0), hi_last = __builtin_amdgcn_readlane(see.hi, 31);

  f32x16_t o[DB];
  float m = kNoMax, l = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  auto copy_tile = [&](int j, uint32_t stage) {
#pragma unroll
    for (int i = 0; i < NI; ++i) copy_keys<HD, PAGED>(ks, wave * NI + i, j, end, stage, stage + kHalf, lane);
  };
  uint32_t stage = ring;
  wait_copies<0>();
  if (beg < end) copy_tile(beg, stage);
  for (int j = beg; j < end; j += kTileKeys) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // this tile is here, and nobody reads the other stage any more
    if (j + kTileKeys < end) copy_tile(j + kTileKeys, stage ^ ring ^ (ring + kStage));
    if (j < hi_last && j + kTileKeys > lo_first && row0 < n_rows) {
      f32x16_t s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
        for (int c = 0; c < KS; ++c) s[kb] = mfma32(lds_read16(stage + chunk_at<HD>(kb * 32 + l32, c * 2 + half)), q[c], s[kb]);
      }
      const bool masked = j < lo_last || j + kTileKeys > hi_first;
      if (masked) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = j + kb * 32 + half * 4 + (i & 3) + 8 * (i >> 2);
            s[kb][i] = key >= see.lo && key < see.hi ? s[kb][i] : -INFINITY;
          }
      }
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[0][i]);
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[1][i]);
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * p.scale_log2;
      if (__any(mx > m + kLazy)) {
        const float m_new = fmaxf(m, mx), a = __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= a;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= a;
      }
      u32x4_t pk[4];
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
      uint32_t odd = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const int c = d * 4 + (grp & 1) * 2 + ((l16 & 3) >> 1), key = x * 16 + half * 4 + (l16 >> 2);
          const u32x2_t v0 = lds_read_tr(stage + kHalf + chunk_at<HD>(key, c) + (l16 & 1) * 8);
          const u32x2_t v1 = lds_read_tr(stage + kHalf + chunk_at<HD>(key + 8, c) + (l16 & 1) * 8);
          u32x4_t vf = {v0[0], v0[1], v1[0], v1[1]};
          if (masked) {
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[e] = finite_pair(vf[e], odd);
          }
          o[d] = mfma32(vf, pk[x], o[d]);
        }
      if (masked && __any(odd != 0)) {
        // infinities and NaN among the values (0 in the product): they reach the rows that see their key, and no other
#pragma unroll 1
        for (int x = 0; x < kTileKeys; ++x) {
          const bool seen = j + x >= see.lo && j + x < see.hi;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int ch = d * 32 + half * 4 + (i & 3) + 8 * (i >> 2);
              const float v = lds_bf16(stage + kHalf + chunk_at<HD>(x, ch >> 3) + (ch & 7) * 2);
              if (seen && !(fabsf(v) < INFINITY)) o[d][i] += v;
            }
        }
      }
    }
    stage = stage ^ ring ^ (ring + kStage);
  }

  l += __shfl_xor(l, 32);
  if (row0 + l32 >= n_rows) return;
  if (n_pieces == 1) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    bf16_t *dst = p.o + t * p.o_stride + head * HD;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<u32x2_t *>(dst + d * 32 + g * 8 + half * 4) =
            u32x2_t{pack_bf16x2(o[d][g * 4] * inv, o[d][g * 4 + 1] * inv), pack_bf16x2(o[d][g * 4 + 2] * inv, o[d][g * 4 + 3] * inv)};
    if (half == 0 && p.lse) p.lse[t * p.n_heads + head] = lse_of(m, l);
  } else {
    float *part = part_of<HD>(pl, it.first + it.piece * it.n_tiles + it.n_tiles - 1 - it.tile, it.kvh, p.n_kv);
    const int r = wave * 32 + l32;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4_t *>(part + r * HD + d * 32 + g * 8 + half * 4) =
            f32x4_t{o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]};
    if (half == 0) {
      part[kRows * HD + r * 2] = m;
      part[kRows * HD + r * 2 + 1] = l;
    }
  }
}

// ---- rows split along the keys: their pieces joined, in order ------------------------------------------------------------
// One wavefront to a (token, head).
template <int HD>
__global__ __launch_bounds__(256) void ff_attn_join_kernel(AttnParams p, AttnPlan few, AttnPlan tile) {
  const int lane = threadIdx.x & 63;
  const long id = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = (int)(id / p.n_heads), head = (int)(id % p.n_heads);
  if (t >= p.T) return;
  // the sequence whose rows hold the token
  int s = -1;
  for (int s0 = 0; s0 < p.n_seqs && s < 0; s0 += 64) {
    bool mine = false;
    if (s0 + lane < p.n_seqs) {
      const Seq q = seq_of(p, s0 + lane);
      mine = t >= q.t0 && t < q.t0 + q.n;
    }
    const unsigned long long hit = __ballot(mine);
    if (hit) s = s0 + __builtin_ctzll(hit);
  }
  if (s < 0) return;
  const Seq q = seq_of(p, s);
  const bool is_few = tiles_of(p, few, q.n) > 0;
  const AttnPlan &pl = is_few ? few : tile;
  if (pl.target <= 0) return;
  const int kpp = piece_keys(p, pl);
  const Item it = find_item(p, pl, kpp, s, true);
  const int kvh = head / p.group, row = (t - it.seq.t0) * p.group + head % p.group;
  const int tl = row / pl.tile_rows, r = row - tl * pl.tile_rows;
  const int n = pieces_of(tile_range(p, it.seq, tl, pl.tile_rows), kpp);
  const int x0 = it.first + it.n_tiles - 1 - tl;
  // (chunks that overlap may have more pieces than there were workgroups and room for)
  if (n <= 1 || it.n_tiles == 0 || ((long)x0 + (long)(n - 1) * it.n_tiles + 1) * p.n_kv > pl.max_items) return;
  float top = kNoMax;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, part_of<HD>(pl, x0 + i * it.n_tiles, kvh, p.n_kv)[pl.tile_rows * HD + r * 2]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  float sum = 0.f, acc[HD / 64] = {};
  for (int i = 0; i < n; ++i) {
    const float *part = part_of<HD>(pl, x0 + i * it.n_tiles, kvh, p.n_kv);
    const float a = __builtin_amdgcn_exp2f(part[pl.tile_rows * HD + r * 2] - top);
    sum = fmaf(part[pl.tile_rows * HD + r * 2 + 1], a, sum);
#pragma unroll
    for (int e = 0; e < HD / 64; ++e) acc[e] = fmaf(part[r * HD + lane * (HD / 64) + e], a, acc[e]);
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  bf16_t *dst = p.o + (int64_t)t * p.o_stride + head * HD;
  if (HD == 128) *reinterpret_cast<uint32_t *>(dst + lane * 2) = pack_bf16x2(acc[0] * inv, acc[HD / 64 - 1] * inv);
  else dst[lane] = f32_to_bf16(acc[0] * inv);
  if (lane == 0 && p.lse) p.lse[(int64_t)t * p.n_heads + head] = lse_of(top, sum);
}

// one wavefront per sequence
__global__ __launch_bounds__(64) void ff_attn_validate_kernel(AttnParams p, int32_t *flag) {
  const int s = blockIdx.x, lane = threadIdx.x;
  const int a = p.starts[s], b = p.starts[s + 1];
  bool bad = a < 0 || b < a || b > p.T || p.lens[s] < 0 || p.lens[s] > most_keys(p);
  const Seq q = seq_of(p, s);
  const int first = p.window > 0 ? max(0, q.keys - q.n + 1 - p.window) >> p.page_shift : 0;
  const int pages = q.n > 0 ? (int)(((long)q.keys + (1 << p.page_shift) - 1) >> p.page_shift) : 0;
  for (int i = first + lane; i < pages; i += 64) {
    const int page = p.table[(size_t)s * p.table_stride + i];
    bad = bad || page < 0 || page >= p.n_pages;
  }
  if (__any(bad) && lane == 0) atomicMax(flag, s + 1);
}

constexpr int kFewWaves = 4;
size_t few_lds(int hd, int nb) {
  const size_t ring = (size_t)kFewWaves * 2 * 2 * 32 * hd * 2;
  const size_t join = (size_t)kFewWaves * 16 * nb * (hd + 4 + 2) * 4;
  return std::max(ring, join);
}
size_t tile_lds(int hd) { return (size_t)2 * 2 * kTileKeys * hd * 2; }

template <int HD>
hipError_t raise_limits() {
  hipError_t e = hipSuccess;
  auto raise = [&](const void *fn, size_t lds) {
    if (e == hipSuccess) e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  };
  raise(reinterpret_cast<const void *>(ff_attn_few_kernel<HD, 1>), few_lds(HD, 1));
  raise(reinterpret_cast<const void *>(ff_attn_few_kernel<HD, 2>), few_lds(HD, 2));
  raise(reinterpret_cast<const void *>(ff_attn_few_kernel<HD, 4>), few_lds(HD, 4));
  raise(reinterpret_cast<const void *>(ff_attn_tile_kernel<HD, 4, true>), tile_lds(HD));
  raise(reinterpret_cast<const void *>(ff_attn_tile_kernel<HD, 8, true>), tile_lds(HD));
  raise(reinterpret_cast<const void *>(ff_attn_tile_kernel<HD, 4, false>), tile_lds(HD));
  raise(reinterpret_cast<const void *>(ff_attn_tile_kernel<HD, 8, false>), tile_lds(HD));
  return e;
}

// How the call is cut.  rows of a sequence = new tokens times heads of a group.
struct Choice {
  AttnPlan few, tile;
  int nb = 0, waves = 0;          // 0: that kernel is not launched
  size_t bytes = 0;
};
// Items that a plan can have at most: about `target` pieces and one more for each (tile, key head).  Their tiles: the rows' own and
// one part-filled tile for each sequence.
long tiles_bound(long rows, int n_seqs, int n_tokens, int tile_rows) { return rows / tile_rows + std::min(n_seqs, n_tokens); }

Choice choose(int n_heads, int n_kv, int head_dim, int n_tokens, int n_seqs, int max_chunk, bool paged) {
  Choice c;
  const int group = n_heads / n_kv;
  const long rows = (long)n_tokens * group, chunk_rows = (long)max_chunk * group;
  const auto set = [&](AttnPlan &pl, int tile_rows, long above, long upto, int target, int min_steps) {
    const long tiles = tiles_bound(rows, n_seqs, n_tokens, tile_rows);
    pl.tile_rows = tile_rows;
    pl.rows_above = above;
    pl.rows_upto = upto;
    pl.min_steps = min_steps;
    // rows enough for every CU are not split: whole rows need no second pass
    pl.target = paged && rows / tile_rows * n_kv < 512 ? target : 0;
    pl.max_items = (int)std::min<long>(tiles * n_kv + pl.target + 16, 0x7fffffff);   // (the price of a call is summed in fp32)
    pl.part_at = c.bytes / sizeof(float);
    if (pl.target > 0) c.bytes += (size_t)pl.max_items * tile_rows * (head_dim + 2) * sizeof(float);
  };
  const long all = 0x7fffffffffffL;
  if (paged && chunk_rows <= 64) {
    c.nb = chunk_rows <= 16 ? 1 : (chunk_rows <= 32 ? 2 : 4);
    set(c.few, 16 * c.nb, 0, all, 1024, 4);
    return c;
  }
  c.waves = chunk_rows <= 128 ? 4 : 8;
  const bool both = paged && n_seqs > 1 && group <= 16;     // sequences that generate one token beside chunks
  set(c.tile, 32 * c.waves, both ? 16 : 0, all, 256, 4);
  if (both) {
    c.nb = 1;
    set(c.few, 16, 0, 16, 1024, 4);
  }
  return c;
}

template <int HD>
hipError_t launch(const AttnParams &p, Choice &c, hipStream_t s) {
  if (c.bytes > p.part_bytes) return hipErrorInvalidValue;
  c.few.part = p.part + c.few.part_at;
  c.tile.part = p.part + c.tile.part_at;
  if (c.nb) {
    const dim3 grid((unsigned)c.few.max_items), block(64 * kFewWaves);
    const size_t lds = few_lds(HD, c.nb);
    if (c.nb == 1) hipLaunchKernelGGL((ff_attn_few_kernel<HD, 1>), grid, block, lds, s, p, c.few);
    else if (c.nb == 2) hipLaunchKernelGGL((ff_attn_few_kernel<HD, 2>), grid, block, lds, s, p, c.few);
    else hipLaunchKernelGGL((ff_attn_few_kernel<HD, 4>), grid, block, lds, s, p, c.few);
  }
  if (c.waves) {
    const dim3 grid((unsigned)c.tile.max_items), block(64 * c.waves);
    const size_t lds = tile_lds(HD);
    if (p.table) {
      if (c.waves == 4) hipLaunchKernelGGL((ff_attn_tile_kernel<HD, 4, true>), grid, block, lds, s, p, c.tile);
      else hipLaunchKernelGGL((ff_attn_tile_kernel<HD, 8, true>), grid, block, lds, s, p, c.tile);
    } else {
      if (c.waves == 4) hipLaunchKernelGGL((ff_attn_tile_kernel<HD, 4, false>), grid, block, lds, s, p, c.tile);
      else hipLaunchKernelGGL((ff_attn_tile_kernel<HD, 8, false>), grid, block, lds, s, p, c.tile);
    }
  }
  if (c.few.target > 0 || c.tile.target > 0) {
    const long waves = (long)p.T * p.n_heads;
    hipLaunchKernelGGL((ff_attn_join_kernel<HD>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, p, c.few, c.tile);
  }
  return hipGetLastError();
}

}  // namespace

// (whatever the longest chunk is: the most that any choice takes)
size_t ff_attention_part_bytes(int n_heads, int n_kv, int head_dim, int n_tokens, int n_seqs) {
  const int group = n_heads / n_kv;
  size_t most = 0;
  for (int rows : {16, 32, 64, 128, 129})
    most = std::max(most, choose(n_heads, n_kv, head_dim, n_tokens, n_seqs, std::max(1, (rows + (rows > 128 ? group - 1 : 0)) / group), true).bytes);
  return most;
}

size_t ff_attention_need(const AttnParams &p, int head_dim, int max_chunk) {
  return choose(p.n_heads, p.n_kv, head_dim, p.T, p.n_seqs, max_chunk, p.table != nullptr).bytes;
}

hipError_t ff_attention_init() {
  hipError_t e = raise_limits<128>();
  return e == hipSuccess ? raise_limits<64>() : e;
}

hipError_t ff_launch_attention(const AttnParams &p, int head_dim, int max_chunk, hipStream_t s) {
  Choice c = choose(p.n_heads, p.n_kv, head_dim, p.T, p.n_seqs, max_chunk, p.table != nullptr);
  return head_dim == 128 ? launch<128>(p, c, s) : launch<64>(p, c, s);
}

hipError_t ff_launch_validate_pages(const AttnParams &p, int32_t *flag, hipStream_t s) {
  hipLaunchKernelGGL(ff_attn_validate_kernel, dim3(p.n_seqs), dim3(64), 0, s, p, flag);
  return hipGetLastError();
}
