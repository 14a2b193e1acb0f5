// What the wavefronts of several kernels do alike: sums over lanes, and which sequence of a call an item belongs to.
#pragma once

#include "ff_attn_plan.h"

// Running sums over the 64 lanes (lane 63: all of them), by DPP: some 8 cycles a step, where a shuffle through LDS takes over 100.
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T dpp(T v) {
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
template <class T>
__device__ __forceinline__ T lane_sums(T v) {
  v += dpp<0x111, 0xf>(v);     // the lane before in the row of 16, then 2, 4 and 8 before
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);     // rows 1 and 3: the last lane of the row before
  v += dpp<0x143, 0xc>(v);     // rows 2 and 3: lane 31
  return v;
}
// the largest of the lanes' values, none of them below 0 (in all lanes)
__device__ __forceinline__ float lane_max(float v) {
  v = fmaxf(v, dpp<0x111, 0xf>(v));
  v = fmaxf(v, dpp<0x112, 0xf>(v));
  v = fmaxf(v, dpp<0x114, 0xf>(v));
  v = fmaxf(v, dpp<0x118, 0xf>(v));
  v = fmaxf(v, dpp<0x142, 0xa>(v));
  v = fmaxf(v, dpp<0x143, 0xc>(v));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ float last_lane(float v) { return __builtin_bit_cast(float, last_lane(__builtin_bit_cast(int, v))); }
// a wave-uniform value by a scalar load: the wait for it is not one for the copies before it
template <class T>
__device__ __forceinline__ T scalar_load(const T *at) {
  return *reinterpret_cast<const __attribute__((address_space(4))) T *>(reinterpret_cast<uintptr_t>(at));
}

// Items are counted over the sequences: `get` gives a sequence, `count` its items.  Item number x (the same in all lanes) is number `at` of sequence s;
// s < 0: there are fewer.  64 sequences are looked at together, so a call of up to 64 takes one look.
struct Found { int s, at; Seq seq; };
template <class Get, class Count>
__device__ __forceinline__ Found find_item(const AttnParams &p, long x, Get get, Count count) {
  const int lane = threadIdx.x & 63;
  Found f = {-1, 0, {0, 0, 0}};
  for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
    const Seq q = s0 + lane < p.n_seqs ? get(p, s0 + lane) : Seq{0, 0, 0};
    // (a call's tokens keep the sums in 32 bits; starts that do not ascend may not: nothing is found then, or another item)
    const int mine = count(q), upto = lane_sums(mine);
    const unsigned long long hit = __ballot(x < (long)(unsigned)upto);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int n = __builtin_amdgcn_readlane(mine, l), at = (int)x - (__builtin_amdgcn_readlane(upto, l) - n);
      if ((unsigned)at < (unsigned)n)
        f = {s0 + l, at, {__builtin_amdgcn_readlane(q.t0, l), __builtin_amdgcn_readlane(q.n, l), __builtin_amdgcn_readlane(q.keys, l)}};
      return f;
    }
    x -= (unsigned)last_lane(upto);
  }
  return f;
}
// The same for runs of 2^shift positions that new tokens have a place in (runs_of, placed_seq), of which a call of more than 64 sequences has
// numbers with gaps: then the last sequence that begins at or before number x is found by steps of 64th parts, three looks at most, where
// counting looks at all.  (1024 and 16384 single tokens of 8 key heads are written in 24 and 344 us, in 35 and 3390 by counting.)
__device__ __forceinline__ Found find_run(const AttnParams &p, int x, int shift) {
  if (p.n_seqs <= 64) return find_item(p, x, placed_seq, [&](const Seq &q) { return runs_of(q, shift); });
  const Found none = {-1, 0, {0, 0, 0}};
  const int lane = threadIdx.x & 63;
  const bool by_token = runs_by_token(p.T, p.n_seqs, shift);
  int s = 0, to = p.n_seqs, step;
  do {
    step = (to - s + 63) >> 6;
    const int at = s + lane * step;
    const unsigned long long hit = __ballot(at < to && run_base(attn_clamp(p.starts[attn_min(at, to - 1)], 0, p.T), at, shift, by_token) <= x);
    if (!hit) return none;
    s += (63 - __builtin_clzll(hit)) * step;
    to = attn_min(to, s + step);
  } while (step > 1);
  const Seq q = placed_seq(p, s);
  const int at = x - run_base(q.t0, s, shift, by_token);
  if (at < 0 || at >= runs_of(q, shift)) return none;
  return {s, at, q};
}
