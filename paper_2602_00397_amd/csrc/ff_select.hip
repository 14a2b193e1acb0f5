// Sparse attention's choice: which pages of its sequence's cache a block of new tokens reads, for each key head.
//
// A page is scored by its mean key: s = (sum of the block's queries of the key head) . mean, what the block's logits over the page
// add up to, over the page's length.  Scores are float64, as the FFN predictor's are: the list does not depend on the
// order of a sum, and the best pages are exactly the best, ties to the earlier page.  The means are kept by the caller and made anew for
// pages that new tokens come to.
#include <algorithm>

#include "ff_fp8.h"
#include "ff_wave.h"

namespace {

constexpr int kThreads = 256, kBatch = 8;     // loads of a lane on their way

// ---- mean keys of the pages that have new tokens ------------------------------------------------------------------------------
// A workgroup to a page and key head: HD / 8 lanes to a key, float64 sums (of up to 4096 bf16 numbers, nearly always exact), one rounding.
template <int HD, bool EIGHT>
__global__ __launch_bounds__(kThreads) void ff_page_means_kernel(SelectParams a, long n_items) {
  constexpr int LPK = HD / 8, GROUPS = kThreads / LPK;
  __shared__ double sums[GROUPS][HD];
  const AttnParams &p = a.seqs;
  const int group = threadIdx.x / LPK, channel = threadIdx.x % LPK * 8;
  for (long id = blockIdx.x; id < n_items; id += gridDim.x) {
    const int run = p.by_kv((int)id), kvh = (int)id - run * p.n_kv;       // (fewer than 2^31)
    const Found f = find_run(p, run, p.page_shift);
    if (f.s < 0) continue;
    const int number = (first_new(f.seq) >> p.page_shift) + f.at, page = p.table[f.s * p.seq_tables + number];
    if ((unsigned)page >= (unsigned)p.n_pages) continue;
    const int live = (int)min((long)f.seq.keys - ((long)number << p.page_shift), 1L << p.page_shift);
    const size_t head = (size_t)page * p.n_kv + kvh;
    double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int j = group; j < live; j += GROUPS) {
      const size_t at = ((head << p.page_shift) + j) * HD + channel;
      u32x4_t x;
      if (EIGHT) {
        const u32x2_t codes = *reinterpret_cast<const u32x2_t *>(reinterpret_cast<const uint8_t *>(p.k) + at);
        x = decode8(codes[0], codes[1], p.k_scale[(head << (p.page_shift - p.scale_shift)) + (j >> p.scale_shift)]);
      } else {
        x = *reinterpret_cast<const u32x4_t *>(p.k + at);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[2 * e] += (double)__uint_as_float(x[e] << 16);
        acc[2 * e + 1] += (double)__uint_as_float(x[e] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[group][channel + e] = acc[e];
    __syncthreads();
    if (threadIdx.x < HD) {
      double sum = 0;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) sum += sums[g][threadIdx.x];
      a.means[head * HD + threadIdx.x] = (float)(sum / live);
    }
    __syncthreads();
  }
}

// ---- blocks of new tokens -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ Block block_of(const SelectParams &a, int x) {
  const Found f = find_item(a.seqs, x, seq_of, [&](const Seq &q) { return blocks_of(q, a.query_block); });
  return f.s < 0 ? Block{-1, 0, 0, 0, 0, 0} : block_at(f.seq, f.s, f.at, a.query_block, a.keep, a.seqs.page_shift);
}

// ---- the best pages, in order ---------------------------------------------------------------------------------------------------
// A workgroup to a block and key head scores the earlier pages and lists the best; where there are few blocks, several score and the last
// of them to end lists.  It is a chain of latencies (one token over 2047 pages, 48 over up to 512, 8192 in blocks of 128, each call repeated on one
// state: 12.0, 10.5 and 17.3 us with 512 threads, 13.8, 13.3 and 16.1 with 256; as two launches, scores and lists, 15.3, 16.1 and 24.0; on three
// states in turn, as traced, 13.6, 15.1 and 22.5).  Blocks with no more earlier pages than are kept need no scores.
//
// The list: the scores' range is cut into 1024 parts; those above the part that holds
// the last page wanted are taken, and of that part's few the best, by counting for each how many are better.  (2047 pages of which 64
// are kept 14.1 us by whole numbers alone, as below, 9.4 so.)
// Where that part has too many, or scores are not finite, the scores are compared as whole numbers in their order: the range of those is
// cut in 1024 until the part with the last one wanted has no more than are wanted of it, or is one number (then its first pages are); each
// cut is ten bits of it, so there are at most seven.  So are scores of more pages than are held, which are read again for each cut (one token over 4096
// pages 15 us, 8192 44, 65536 272).
constexpr int kSelectThreads = 512;
constexpr int kBins = 1024, kHeld = 4096, kFew = 64;     // parts; scores that are held in LDS (of more pages they are read again); candidates of a part
__device__ __forceinline__ uint64_t order_of(double s) {      // (-0 as +0; NaN by its bits)
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
// (of plain min and max, mixed 64-bit types take the double one)
__device__ __forceinline__ uint64_t lower(uint64_t a, uint64_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint64_t higher(uint64_t a, uint64_t b) { return a < b ? b : a; }
struct SelectShared {
  double held[kHeld];
  double extreme[2][kSelectThreads / 64];
  int bins[kBins], sums[kSelectThreads / 64], sums2[kSelectThreads / 64], odd[kSelectThreads / 64], found[3], n_few;
  double few[kFew], last;
  int few_at[kFew], last_at;
};
// The part, counted from the highest, in which the running count reaches `want`: found = part, how many are above it, how many in it.
__device__ __forceinline__ void find_part(SelectShared &sh, int want) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  constexpr int PER = kBins / kSelectThreads;
  const int top = kBins - 1 - PER * (int)threadIdx.x;
  int c[PER], mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    c[i] = sh.bins[top - i];
    mine += c[i];
  }
  const int upto = lane_sums(mine);
  if (lane == 63) sh.sums[wave] = upto;
  __syncthreads();
  int above = upto - mine;
#pragma unroll
  for (int w = 0; w < kSelectThreads / 64; ++w) above += w < wave ? sh.sums[w] : 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (above < want && want <= above + c[i]) {
      sh.found[0] = top - i;
      sh.found[1] = above;
      sh.found[2] = c[i];
    }
    above += c[i];
  }
  __syncthreads();
}
// The pages that `taken` says, in order, and of those that `tied` says the first `ties`: a run of pages to a thread.
template <class Taken, class Tied>
__device__ __forceinline__ void write_list(SelectShared &sh, int n, int ties, const int32_t *table, int32_t *list, Taken taken, Tied tied) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int per = (n + kSelectThreads - 1) / kSelectThreads, from = min(n, (int)threadIdx.x * per), to = min(n, from + per);
  int t = 0, e = 0;
  for (int i = from; i < to; ++i) {
    t += taken(i);
    e += tied(i);
  }
  const int t_upto = lane_sums(t), e_upto = lane_sums(e);
  if (lane == 63) {
    sh.sums[wave] = t_upto;
    sh.sums2[wave] = e_upto;
  }
  __syncthreads();
  int at = t_upto - t, before = e_upto - e;
#pragma unroll
  for (int w = 0; w < kSelectThreads / 64; ++w) {
    at += w < wave ? sh.sums[w] : 0;
    before += w < wave ? sh.sums2[w] : 0;
  }
  for (int i = from; i < to; ++i) {
    const bool is = taken(i), tie = tied(i);
    if (is || (tie && before < ties)) list[at + min(before, ties)] = table[i];
    at += is;
    before += tie;
  }
}
template <class Get>
__device__ __forceinline__ void list_by_numbers(SelectShared &sh, int n, int kept, const int32_t *table, int32_t *list, Get number) {
  uint64_t lo = 0, hi = ~0ull;
  int want = kept;               // of those in [lo, hi]; all above are taken
  for (;;) {
    const int shift = max(0, 64 - (int)__clzll((long long)(hi - lo | 1)) - 10);
    __syncthreads();             // (what the last use of the counts read)
    for (int i = threadIdx.x; i < kBins; i += kSelectThreads) sh.bins[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kSelectThreads) {
      const uint64_t u = number(i);
      if (u >= lo && u <= hi) atomicAdd(&sh.bins[(u - lo) >> shift], 1);
    }
    __syncthreads();
    find_part(sh, want);
    lo += (uint64_t)sh.found[0] << shift;
    hi = lo + lower(hi - lo, ((uint64_t)1 << shift) - 1);
    want -= sh.found[1];
    if (shift == 0 || sh.found[2] == want) break;
  }
  __syncthreads();
  write_list(sh, n, want, table, list, [&](int i) { return number(i) > hi; }, [&](int i) { const uint64_t u = number(i); return u >= lo && u <= hi; });
}
__device__ __forceinline__ void score_store(double *at, double v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double score_load(const double *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
constexpr int kRun = kSelectThreads / 2;        // pages that a workgroup scores at a time, four lanes to two of them
template <int HD>
__global__ __launch_bounds__(kSelectThreads) void ff_select_pages_kernel(SelectParams a) {
  constexpr int LPR = HD / 8, GROUPS = kSelectThreads / LPR;
  static_assert(GROUPS * HD <= kHeld, "the groups' sums lie where the scores come afterwards");
  __shared__ SelectShared sh;
  __shared__ double sum[HD];
  const AttnParams &p = a.seqs;
  const int x = blockIdx.y, kvh = blockIdx.x, piece = blockIdx.z;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Block b = block_of(a, x);
  int32_t *list = a.tables + ((size_t)x * p.n_kv + kvh) * a.width;
  const int32_t *table = p.table + (b.s < 0 ? 0 : b.s * p.seq_tables);
  const int n = b.earlier, kept = min(a.keep, n);
  if (piece == 0) {
    if (kvh == 0 && threadIdx.x == 0) {
      const int end = attn_clamp(p.starts[p.n_seqs], 0, p.T);
      a.starts[x] = b.s < 0 ? end : b.t0;
      a.lens[x] = b.keys;
      if (x == a.n_blocks - 1) a.starts[a.n_blocks] = b.s < 0 ? end : b.t0 + b.n;
    }
    for (int i = kept + threadIdx.x; i < a.width; i += kSelectThreads) list[i] = i < kept + b.own ? table[n + i - kept] : -1;
    if (n <= a.keep)
      for (int i = threadIdx.x; i < n; i += kSelectThreads) list[i] = table[i];
  }
  const int pieces = min((int)gridDim.z, (n + kRun - 1) / kRun);
  if (n <= a.keep || piece >= pieces) return;

  // the block's queries of the key head, summed
  const int group = threadIdx.x / LPR, channel = threadIdx.x % LPR * 8, rows = b.n * p.group;
  double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int r0 = group; r0 < rows; r0 += GROUPS * kBatch) {
    u32x4_t w[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = min(r0 + i * GROUPS, rows - 1), t = p.by_group(r);
      w[i] = *reinterpret_cast<const u32x4_t *>(p.q + (int64_t)(b.t0 + t) * p.q_stride + (kvh * p.group + r - t * p.group) * HD + channel);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const bool is = r0 + i * GROUPS < rows;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t v = is ? w[i][e] : 0;
        acc[2 * e] += (double)__uint_as_float(v << 16);
        acc[2 * e + 1] += (double)__uint_as_float(v & 0xffff0000u);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) sh.held[group * HD + channel + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < HD) {
    double s = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) s += sh.held[g * HD + threadIdx.x];
    sum[threadIdx.x] = s;
  }
  for (int i = threadIdx.x; i < kBins; i += kSelectThreads) sh.bins[i] = 0;
  if (threadIdx.x == 0) sh.n_few = 0;
  __syncthreads();

  // scores
  const bool hold = n <= kHeld, alone = pieces == 1;
  double *scores = a.scores + ((size_t)x * p.n_kv + kvh) * p.table_stride;
  const int quarter = threadIdx.x & 3;
  for (int j0 = piece * kRun; j0 < n; j0 += pieces * kRun) {
    float4 m[2][HD / 16];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int page = table[min(j0 + u * (kRun / 2) + (int)(threadIdx.x >> 2), n - 1)];
      page = (unsigned)page < (unsigned)p.n_pages ? page : 0;
      const float *mean = a.means + ((size_t)page * p.n_kv + kvh) * HD + quarter * 4;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) m[u][i] = *reinterpret_cast<const float4 *>(mean + i * 16);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int j = j0 + u * (kRun / 2) + (threadIdx.x >> 2);
      double s = 0;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const double *q = sum + i * 16 + quarter * 4;
        s += (double)m[u][i].x * q[0] + (double)m[u][i].y * q[1] + (double)m[u][i].z * q[2] + (double)m[u][i].w * q[3];
      }
      s += __shfl_xor(s, 1);
      s += __shfl_xor(s, 2);
      if (quarter == 0 && j < n) {
        if (alone && hold) sh.held[j] = s;
        else score_store(scores + j, s);
      }
    }
  }
  if (!alone) {
    // the last workgroup of the block and key head to end goes on
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // this wavefront's scores have arrived
    __syncthreads();
    int *counter = p.counters + x * p.n_kv + kvh;
    if (threadIdx.x == 0) {
      sh.found[0] = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pieces - 1;
      if (sh.found[0]) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as the next call expects it
    }
    __syncthreads();
    if (!sh.found[0]) return;
  } else if (!hold) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  if (hold && !alone) {
    for (int i0 = threadIdx.x; i0 < n; i0 += kSelectThreads * kBatch) {
      double s[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) s[i] = score_load(scores + min(i0 + i * kSelectThreads, n - 1));
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (i0 + i * kSelectThreads < n) sh.held[i0 + i * kSelectThreads] = s[i];
    }
  }
  __syncthreads();
  const int first = a.first, want = kept - first;
  bool by_numbers = !hold;
  double lo = INFINITY, hi = -INFINITY, scale = 0;
  if (hold) {
    bool odd = false;
    for (int i = first + threadIdx.x; i < n; i += kSelectThreads) {
      const double s = sh.held[i];
      odd = odd || !(fabs(s) < INFINITY);
      lo = fmin(lo, s);
      hi = fmax(hi, s);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      lo = fmin(lo, __shfl_xor(lo, off));
      hi = fmax(hi, __shfl_xor(hi, off));
    }
    const bool any_odd = __any(odd);
    if (lane == 0) {
      sh.extreme[0][wave] = lo;
      sh.extreme[1][wave] = hi;
      sh.odd[wave] = any_odd;
    }
    __syncthreads();
    by_numbers = want == 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 64; ++w) {
      lo = fmin(lo, sh.extreme[0][w]);
      hi = fmax(hi, sh.extreme[1][w]);
      by_numbers = by_numbers || sh.odd[w];
    }
    const double range = hi - lo;
    by_numbers = by_numbers || !(range > 1e-290 && range < 1e290);
    scale = (kBins - 1) / range;
  }
  const auto part_of = [&](double s) { return min((int)((s - lo) * scale), kBins - 1); };       // (rounded, but never out of order)
  int part = 0, need = 0, c = 0;
  if (!by_numbers) {
    for (int i = first + threadIdx.x; i < n; i += kSelectThreads) atomicAdd(&sh.bins[part_of(sh.held[i])], 1);
    __syncthreads();
    find_part(sh, want);
    part = sh.found[0];
    need = want - sh.found[1];
    c = sh.found[2];
    by_numbers = c > kFew;
  }
  if (by_numbers) {
    list_by_numbers(sh, n, kept, table, list, [&](int i) { return i < first ? ~0ull : order_of(hold ? sh.held[i] : score_load(scores + i)); });
    return;
  }
  for (int i = first + threadIdx.x; i < n; i += kSelectThreads)
    if (part_of(sh.held[i]) == part) {
      const int k = atomicAdd(&sh.n_few, 1);
      sh.few[k] = sh.held[i];
      sh.few_at[k] = i;
    }
  __syncthreads();
  if ((int)threadIdx.x < c) {
    const double s = sh.few[threadIdx.x];
    const int at = sh.few_at[threadIdx.x];
    int better = 0;
    for (int k = 0; k < c; ++k) better += sh.few[k] > s || (sh.few[k] == s && sh.few_at[k] < at);
    if (better == need - 1) {
      sh.last = s;
      sh.last_at = at;
    }
  }
  __syncthreads();
  const double last = sh.last;
  const int last_at = sh.last_at;
  const auto taken = [&](int i) {
    const double s = sh.held[i];
    const int its = part_of(s);
    return i < first || its > part || (its == part && (s > last || (s == last && i <= last_at)));
  };
  write_list(sh, n, 0, table, list, taken, [](int) { return false; });
}

template <int HD>
hipError_t means(const SelectParams &a, hipStream_t s) {
  const long items = most_runs(a.seqs.T, a.seqs.n_seqs, a.seqs.page_shift) * a.seqs.n_kv;
  const dim3 grid((unsigned)std::min<long>(items, 1 << 20)), block(kThreads);
  if (a.seqs.k_scale) hipLaunchKernelGGL((ff_page_means_kernel<HD, true>), grid, block, 0, s, a, items);
  else hipLaunchKernelGGL((ff_page_means_kernel<HD, false>), grid, block, 0, s, a, items);
  return hipGetLastError();
}

}  // namespace

hipError_t ff_launch_page_means(const SelectParams &a, int head_dim, hipStream_t s) {
  return head_dim == 128 ? means<128>(a, s) : means<64>(a, s);
}

hipError_t ff_launch_select_pages(const SelectParams &a, int head_dim, hipStream_t s) {
  const AttnParams &p = a.seqs;
  // (a sequence's pages are shared out where there are few blocks; then there are counters for all of them)
  const long units = (long)a.n_blocks * p.n_kv;
  const long pieces = std::max(1l, std::min((p.table_stride + kRun - 1l) / kRun, 512 / units));
  const dim3 grid(p.n_kv, a.n_blocks, (unsigned)pieces);
  if (head_dim == 128) hipLaunchKernelGGL((ff_select_pages_kernel<128>), grid, dim3(kSelectThreads), 0, s, a);
  else hipLaunchKernelGGL((ff_select_pages_kernel<64>), grid, dim3(kSelectThreads), 0, s, a);
  return hipGetLastError();
}
