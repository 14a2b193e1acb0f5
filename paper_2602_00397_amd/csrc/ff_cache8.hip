// Keys and values of new tokens into a cache in 8 bits: e4m3 codes with a power of two for every block of tokens and head.
//
// A block's scale 2^e is the least for which its largest finite value stays within 448, e4m3's largest: the codes then have all of
// e4m3's range for the block, and, the scale being a power of two, a value is rounded once, to four bits of mantissa or to 2^-9 of
// the scale.  A block that tokens are added to keeps its scale unless it has to grow; then its older codes are divided by
// the factor, which rounds only those that come below e4m3's normal range.
//
// HBM-bound for prompts: values are read once, held in registers while their largest is found, and written at half the size.
#include <algorithm>

#include "ff_fp8.h"
#include "ff_wave.h"

namespace {

// 448 * 2^e >= top > 448 * 2^(e - 1), within [kLeast, kMost]
__device__ __forceinline__ int exponent_for(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000);
  return min(max(e, kLeastExp8), kMostExp8);
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// A unit is a block's part of this call for one head of k or v.  W wavefronts share it, 32 tokens to each at most, so that the new
// values stay in registers between the search for the largest and the conversion.
constexpr int kThreads = 256;
template <int HD, int W>
__global__ __launch_bounds__(kThreads) void ff_append8_kernel(Append8Params a, long n_items) {
  constexpr int LPK = HD / 8, TPW = 64 / LPK, PASSES = 32 / TPW, UNITS = 4 / W;   // lanes of a token, tokens of a wavefront's load
  __shared__ float top_s[4];
  const AttnParams &p = a.seqs;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int token = (wave % W) * TPW + lane / LPK, channel = lane % LPK * 8;       // of a pass: W * TPW tokens
  for (long id = blockIdx.x; id * UNITS < n_items; id += gridDim.x) {
    const long unit = id * UNITS + wave / W;
    // (all of a workgroup's wavefronts pass the barrier below the same number of times)
    // k and v of a head side by side, then the heads, then the blocks (of runs and heads there are fewer than 2^31)
    const bool is_v = unit & 1;
    const int pair = (int)(unit >> 1), run = p.by_kv(pair), kvh = pair - run * p.n_kv;
    const Found f = unit < n_items ? find_run(p, run, p.scale_shift) : Found{-1, 0, {0, 0, 0}};
    const int first = first_new(f.seq), block = (first >> p.scale_shift) + f.at;
    const int from = max(first, block << p.scale_shift);
    const int n = f.s < 0 ? 0 : (int)min((long)f.seq.keys, (long)(block + 1) << p.scale_shift) - from;
    // token number i of the unit is row t0 of the call + i.  (Its values are on their way while the page is looked up.)
    const int64_t t0 = (int64_t)f.seq.t0 + (from - (f.seq.keys - f.seq.n));
    const bf16_t *src = (is_v ? a.v + t0 * a.v_stride : a.k + t0 * a.k_stride) + kvh * HD + channel;
    const int64_t stride = is_v ? a.v_stride : a.k_stride;
    int page = -1;
    if (f.s >= 0) page = p.table[f.s * p.seq_tables + (from >> p.page_shift)];
    u32x4_t x[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int t = i * W * TPW + token;
      x[i] = u32x4_t{0, 0, 0, 0};
      if (i * W * TPW < n && t < n) x[i] = *reinterpret_cast<const u32x4_t *>(src + t * stride);
    }
    const bool here = n > 0 && (unsigned)page < (unsigned)p.n_pages;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = fabsf(__uint_as_float(x[i][e] << 16)), hi = fabsf(__uint_as_float(x[i][e] & 0xffff0000u));
        if (lo < INFINITY) top = fmaxf(top, lo);
        if (hi < INFINITY) top = fmaxf(top, hi);
      }
    top = lane_max(top);
    if (W > 1) {
      if (lane == 0) top_s[wave] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, top_s[wave / W * W + w]);
    }
    const int place = from & ((1 << p.page_shift) - 1), in_block = place & ((1 << p.scale_shift) - 1);
    const size_t head = (size_t)(here ? page : 0) * p.n_kv + kvh;
    float *const scale = (is_v ? a.v_scale : a.k_scale) + (head << (p.page_shift - p.scale_shift)) + (place >> p.scale_shift);
    int e = exponent_for(top);
    if (here) {
      uint8_t *codes = (is_v ? a.v_codes : a.k_codes) + ((head << p.page_shift) + place) * HD + channel;
      if (in_block > 0) {
        const int old = min(max((int)(__float_as_uint(*scale) >> 23 & 255) - 127, kLeastExp8), kMostExp8);
        // (2^-126 is the least power that the conversion takes: codes times less are 0 all the same)
        const float factor = power(max(old - e, -126));
        if (old < e)
          for (int t = token - in_block; t < 0; t += W * TPW) {
            u32x2_t *at = reinterpret_cast<u32x2_t *>(codes + (int64_t)t * HD);
            u32x2_t w = *at;
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = encode4(decode2<false>(w[i], factor), decode2<true>(w[i], factor), 1.f);
            *at = w;
          }
        e = max(e, old);
      }
      const float inverse = power(-e);
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int t = i * W * TPW + token;
        if (i * W * TPW < n && t < n) {
          u32x2_t w;
#pragma unroll
          for (int j = 0; j < 2; ++j) w[j] = encode4(x[i][2 * j], x[i][2 * j + 1], inverse);
          *reinterpret_cast<u32x2_t *>(codes + t * HD) = w;
        }
      }
    }
    if (W > 1) __syncthreads();      // all of the unit's wavefronts have read the old scale, and top_s
    if (here && lane == 0 && wave % W == 0) *scale = power(e);
  }
}

template <int HD>
hipError_t launch(const Append8Params &a, hipStream_t s) {
  const int tokens = 1 << a.seqs.scale_shift, w = tokens > 64 ? 4 : tokens > 32 ? 2 : 1;
  const long items = most_runs(a.seqs.T, a.seqs.n_seqs, a.seqs.scale_shift) * 2 * a.seqs.n_kv;
  // (a workgroup takes units in turn where there are very many)
  const dim3 grid((unsigned)std::min<long>((items * w + 3) / 4, 1 << 20)), block(kThreads);
  if (w == 1) hipLaunchKernelGGL((ff_append8_kernel<HD, 1>), grid, block, 0, s, a, items);
  else if (w == 2) hipLaunchKernelGGL((ff_append8_kernel<HD, 2>), grid, block, 0, s, a, items);
  else hipLaunchKernelGGL((ff_append8_kernel<HD, 4>), grid, block, 0, s, a, items);
  return hipGetLastError();
}

}  // namespace

hipError_t ff_launch_append8(const Append8Params &a, int head_dim, hipStream_t s) {
  return head_dim == 128 ? launch<128>(a, s) : launch<64>(a, s);
}
