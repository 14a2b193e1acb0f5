// Pages of a cache shared by the rows of a table.  The counts, tables and lengths stay on the GPU: one workgroup plans what a call
// does (which pages are free, which move where), in the order of the entries and of the pages, so that the result does not depend on
// any timing; a second launch changes the tables and copies pages, whose contents no other part of the launch touches.
#include "ff_pages.h"

#include <algorithm>

#include "ff_wave.h"

namespace {

constexpr int kPlanThreads = 1024, kThreads = 256;

__device__ __forceinline__ int pages_of(const PoolParams &p, int len) {
  const long most = (long)p.table_stride << p.page_shift, n = len < 0 ? 0 : (long)len < most ? (long)len : most;
  return (int)((n + (1 << p.page_shift) - 1) >> p.page_shift);
}
__device__ __forceinline__ int clamped_len(const PoolParams &p, int len) {
  const long most = (long)p.table_stride << p.page_shift;
  return len < 0 ? 0 : (long)len < most ? len : (int)most;
}
__device__ __forceinline__ bool is_page(const PoolParams &p, int page) { return (unsigned)page < (unsigned)p.n_pages; }
__device__ __forceinline__ bool is_row(const PoolParams &p, int row) { return (unsigned)row < (unsigned)p.n_rows; }

// Workspace: what a plan says, then arrays.  Fork and grow: each entry's first number among the pages that the call takes (kSkip: the
// entry is none), these pages, the last entry of each row; fork also the rows that are read and their lengths, as they were.
// Compact: the free pages among the first `live`, and where each page behind those goes.
constexpr int kHeader = 64, kSkip = -2;
struct Work {
  int *ok, *moves;                                    // whether there are pages enough; how many pages move
  int *first, *lens, *winner, *pages, *rows;          // n, n, n_rows, ..., n * table_stride
};
__host__ __device__ inline Work work_of(const PoolParams &p) {
  Work w;
  w.ok = p.ws;
  w.moves = p.ws + 1;
  w.first = p.ws + kHeader;
  w.lens = w.first + p.n;
  w.winner = w.lens + p.n;
  w.rows = w.winner + p.n_rows;                       // (of a fork; its pages are at most n)
  w.pages = w.rows;
  return w;
}

// Running sum over the workgroup's threads in front of this one's; `all` of them together (two barriers).
__device__ __forceinline__ int sums_before(int v, int &all) {
  __shared__ int wave_sums[kPlanThreads / 64];
  const int wave = threadIdx.x >> 6, upto = lane_sums(v);
  if ((threadIdx.x & 63) == 63) wave_sums[wave] = upto;
  __syncthreads();
  int before = upto - v;
  all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const int s = wave_sums[w];
    if (w < wave) before += s;
    all += s;
  }
  __syncthreads();
  return before;
}
// what another thread of the workgroup wrote, not what this CU's cache held before
__device__ __forceinline__ int fresh(const int *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(int *at, int v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// (those stores have arrived where the loads above look: no write-back of a cache is needed, which a fence would make)
__device__ __forceinline__ void written() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Of several entries of one row the last counts: every row that is listed is marked with the number of its last entry, in LDS where there is
// room for all rows.
constexpr int kRowsHeld = 4096;
struct Winners {
  int held[kRowsHeld];
};
__device__ __forceinline__ void find_winners(const PoolParams &p, const Work &w, Winners &in) {
  const bool hold = p.n_rows <= kRowsHeld;
  for (int i = threadIdx.x; i < p.n; i += kPlanThreads) {
    const int row = p.to[i];
    if (!is_row(p, row)) continue;
    if (hold) in.held[row] = 0;
    else put(&w.winner[row], 0);
  }
  written();
  __syncthreads();
  for (int i = threadIdx.x; i < p.n; i += kPlanThreads) {
    const int row = p.to[i];
    if (!is_row(p, row)) continue;
    if (hold) atomicMax(&in.held[row], i + 1);
    else __hip_atomic_fetch_max(&w.winner[row], i + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  written();
  __syncthreads();
}
__device__ __forceinline__ bool wins(const PoolParams &p, const Work &w, const Winners &in, int i) {
  const int row = p.to[i];
  return (p.n_rows <= kRowsHeld ? in.held[row] : fresh(&w.winner[row])) == i + 1;
}
// The first `want` free pages, in order, to `sink` with their numbers; how many there are of them.
template <class Sink>
__device__ __forceinline__ int find_free(const PoolParams &p, int want, Sink sink) {
  int found = 0;
  for (int j0 = 0; j0 < p.n_pages && found < want; j0 += 4 * kPlanThreads) {
    const int j = j0 + 4 * (int)threadIdx.x;
    int r[4];
    if (j + 4 <= p.n_pages) {
      const int4 v = *reinterpret_cast<const int4 *>(p.refs + j);
      r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = j + e < p.n_pages ? p.refs[j + e] : 1;
    }
    int mine = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += r[e] <= 0;
    int at = found + sums_before(mine, all);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r[e] <= 0) {
        if (at < want) sink(at, j + e);
        ++at;
      }
    found += all;
  }
  return min(found, want);
}

// ---- copies -----------------------------------------------------------------------------------------------------------------------
// HBM-bound: 16 KB of a page's part to a workgroup at a time, four loads of a lane on their way.  What is written goes past the
// caches, and so does what is read if it is read once (2.2 GB of pages read and written 434 us, 5.1 TB/s; both through the caches 454, reads
// alone 446; 64 pages' sequences each in three more 66, through the caches 75, with reads past them 74).  (With 4096 workgroups 453, a million 462;
// 8 KB at a time 435 but the 64 sequences 76, 32 KB 435 and 71.)
constexpr int kPiece = 16384;
struct Parts {
  int n, pieces;                       // pieces of a page in all parts
  uint8_t *data[kPartsAtOnce];
  int64_t bytes[kPartsAtOnce];
  int upto[kPartsAtOnce];              // pieces of a page in this part and those before it
};
// ONCE: no page is read twice.
template <bool ONCE, class T>
__device__ __forceinline__ void copy_as(uint8_t *to, const uint8_t *from, int bytes) {
  const int n = bytes / (int)sizeof(T);
  const T *src = reinterpret_cast<const T *>(from);
  T *dst = reinterpret_cast<T *>(to);
  for (int i = threadIdx.x; i < n; i += 4 * kThreads) {
    T v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e * kThreads < n) v[e] = ONCE ? __builtin_nontemporal_load(src + i + e * kThreads) : src[i + e * kThreads];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e * kThreads < n) __builtin_nontemporal_store(v[e], dst + i + e * kThreads);
  }
}
// piece number x of a page
template <bool ONCE>
__device__ void copy_piece(const Parts &parts, int x, int64_t from, int64_t to) {
  // (a lane to a part)
  const int lane = threadIdx.x & 63;
  const int k = __popcll(__ballot(lane < parts.n - 1 && x >= parts.upto[lane]));
  const int64_t bytes = parts.bytes[k], at = (int64_t)(x - (k ? parts.upto[k - 1] : 0)) * kPiece;
  const int n = (int)(bytes - at < kPiece ? bytes - at : kPiece);
  const uint8_t *src = parts.data[k] + from * bytes + at;
  uint8_t *dst = parts.data[k] + to * bytes + at;
  if (bytes % 16 == 0) copy_as<ONCE, u32x4_t>(dst, src, n);
  else if (bytes % 4 == 0) copy_as<ONCE, uint32_t>(dst, src, n);
  else copy_as<ONCE, uint8_t>(dst, src, n);
}
__global__ __launch_bounds__(kThreads) void ff_pages_copy_kernel(Parts parts, int n_pages, int n, const int32_t *from, const int32_t *to) {
  for (long id = blockIdx.x; id < (long)n * parts.pieces; id += gridDim.x) {
    const int i = (int)(id / parts.pieces), a = from[i], b = to[i];
    if (a != b && (unsigned)a < (unsigned)n_pages && (unsigned)b < (unsigned)n_pages) copy_piece<false>(parts, (int)(id - (long)i * parts.pieces), a, b);
  }
}

// ---- fork -------------------------------------------------------------------------------------------------------------------------
// Workgroup 0 plans; the others keep the rows that are read as they are now.
__global__ __launch_bounds__(kPlanThreads) void ff_pages_fork_plan_kernel(PoolParams p) {
  const Work w = work_of(p);
  int *const pages = w.rows + (size_t)p.n * p.table_stride;
  if (blockIdx.x > 0) {
    for (int i = blockIdx.x - 1; i < p.n; i += gridDim.x - 1) {
      if (!is_row(p, p.from[i])) continue;
      const int *row = p.table + (size_t)p.from[i] * p.table_stride;
      const int len = p.lens[p.from[i]];
      if (threadIdx.x == 0) w.lens[i] = clamped_len(p, len);
      for (int j = threadIdx.x; j < pages_of(p, len); j += kPlanThreads) w.rows[(size_t)i * p.table_stride + j] = row[j];
    }
    return;
  }
  __shared__ Winners in;
  find_winners(p, w, in);
  int want = 0;
  for (int i0 = 0; i0 < p.n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int first = kSkip, needs = 0;
    if (i < p.n && is_row(p, p.to[i]) && is_row(p, p.from[i]) && wins(p, w, in, i)) {
      const int len = clamped_len(p, p.lens[p.from[i]]);
      if ((len & ((1 << p.page_shift) - 1)) != 0) {
        const int last = p.table[(size_t)p.from[i] * p.table_stride + (len >> p.page_shift)];
        // (a row that stays where it is keeps its last page unless others hold it)
        needs = is_page(p, last) && (p.from[i] != p.to[i] || p.refs[last] > 1);
      }
      if (needs || p.from[i] != p.to[i]) first = 0;
    }
    int all;
    const int before = sums_before(needs, all);
    if (i < p.n) w.first[i] = first == kSkip ? kSkip : needs ? want + before : -1;
    want += all;
  }
  const int found = find_free(p, want, [&](int at, int page) { pages[at] = page; });
  if (threadIdx.x == 0) {
    *w.ok = found == want;
    *p.result = want - found;
  }
}
// The first `n_apply` workgroups change the rows, the others copy the part-filled pages.
__global__ __launch_bounds__(kThreads) void ff_pages_fork_kernel(PoolParams p, Parts parts, int n_apply) {
  const Work w = work_of(p);
  const int *const pages = w.rows + (size_t)p.n * p.table_stride;
  if (!*w.ok) return;
  if ((int)blockIdx.x >= n_apply) {
    const int n_copy = gridDim.x - n_apply;
    for (long id = blockIdx.x - n_apply; id < (long)p.n * parts.pieces; id += n_copy) {
      const int i = (int)(id / parts.pieces), first = w.first[i];
      if (first < 0) continue;
      const int page = w.rows[(size_t)i * p.table_stride + (w.lens[i] >> p.page_shift)];
      copy_piece<false>(parts, (int)(id - (long)i * parts.pieces), page, pages[first]);
    }
    return;
  }
  for (int i = blockIdx.x; i < p.n; i += n_apply) {
    const int first = w.first[i];
    if (first == kSkip) continue;
    int *row = p.table + (size_t)p.to[i] * p.table_stride;
    const int *src = w.rows + (size_t)i * p.table_stride;
    const int len = w.lens[i], had = pages_of(p, p.lens[p.to[i]]), gets = pages_of(p, len), full = len >> p.page_shift;
    for (int j = threadIdx.x; j < max(had, gets); j += kThreads) {
      if (j < had && is_page(p, row[j])) atomicSub(&p.refs[row[j]], 1);
      int page = j < gets ? src[j] : -1;
      if (j == full && first >= 0) page = pages[first];
      if (is_page(p, page)) atomicAdd(&p.refs[page], 1);
      row[j] = page;
    }
    __syncthreads();               // (the old length has been read)
    if (threadIdx.x == 0) p.lens[p.to[i]] = len;
  }
}

// ---- grow, free -------------------------------------------------------------------------------------------------------------------
// One workgroup.  With up to 1024 entries that take up to 4096 pages the plan stays in LDS, and rows that change by a few pages, as they do
// when tokens are generated, have a thread each (256 rows of a page at most 24.9 us with a wavefront each and fences, 5.7 so).
constexpr int kHeldPages = 4096, kFewPages = 8;
__global__ __launch_bounds__(kPlanThreads) void ff_pages_grow_kernel(PoolParams p) {
  __shared__ Winners in;
  __shared__ int firsts[kPlanThreads], held[kHeldPages];
  const Work w = work_of(p);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  find_winners(p, w, in);
  long wanted = 0;
  bool long_change = false;
  int first = kSkip;
  for (int i0 = 0; i0 < p.n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    const bool is = i < p.n && is_row(p, p.to[i]) && wins(p, w, in, i);
    const int change = is ? pages_of(p, p.new_lens[i]) - pages_of(p, p.lens[p.to[i]]) : 0;
    int all;
    const int before = sums_before(max(change, 0), all);            // (of 1024 rows of at most 2^20 pages)
    first = is ? (int)min(wanted + before, 0x7fffffffL) : kSkip;
    if (p.n > kPlanThreads && i < p.n) put(&w.first[i], first);
    long_change = long_change || change > kFewPages || change < -kFewPages;
    wanted += all;
  }
  const bool in_lds = p.n <= kPlanThreads && wanted <= kHeldPages;
  if (p.n <= kPlanThreads) firsts[threadIdx.x] = first;
  const int want = (int)min(wanted, (long)p.n_pages + 1);
  const int found = find_free(p, want, [&](int at, int page) {
    if (in_lds) held[at] = page;
    else put(&w.pages[at], page);
  });
  if (threadIdx.x == 0) *p.result = (int)min(wanted - found, 0x7fffffffL);
  if (found < want) return;
  written();
  const bool by_wave = __syncthreads_or(long_change) || p.n > kPlanThreads;
  const auto apply = [&](int i, int at, int step, int begin) __attribute__((always_inline)) {
    if (begin == kSkip) return;
    int *row = p.table + (size_t)p.to[i] * p.table_stride;
    const int len = clamped_len(p, p.new_lens[i]), had = pages_of(p, p.lens[p.to[i]]), gets = pages_of(p, len);
    for (int j = had + at; j < gets; j += step) {
      const int page = in_lds ? held[begin + j - had] : fresh(&w.pages[begin + j - had]);
      row[j] = page;
      p.refs[page] = 1;
    }
    for (int j = gets + at; j < had; j += step) {
      if (is_page(p, row[j])) atomicSub(&p.refs[row[j]], 1);
      row[j] = -1;
    }
    if (at == 0) p.lens[p.to[i]] = len;
  };
  if (!by_wave) {
    if ((int)threadIdx.x < p.n) apply(threadIdx.x, 0, 1, first);
    return;
  }
  for (int i = wave; i < p.n; i += kPlanThreads / 64) apply(i, lane, 64, p.n <= kPlanThreads ? firsts[i] : fresh(&w.first[i]));
}

__global__ __launch_bounds__(kThreads) void ff_pages_validate_kernel(PoolParams p, int32_t *flag) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < p.n && is_row(p, p.to[i]) && p.new_lens[i] != clamped_len(p, p.new_lens[i])) atomicMax(flag, i + 1);
}

// (a row that is listed twice: whoever takes an entry gives its page back)
__global__ __launch_bounds__(kThreads) void ff_pages_free_kernel(PoolParams p) {
  for (int i = blockIdx.x; i < p.n; i += gridDim.x) {
    const int r = p.to[i];
    if (!is_row(p, r)) continue;
    const int had = pages_of(p, fresh(&p.lens[r]));
    for (int j = threadIdx.x; j < had; j += kThreads) {
      const int page = atomicExch(&p.table[(size_t)r * p.table_stride + j], -1);
      if (is_page(p, page)) atomicSub(&p.refs[page], 1);
    }
    __syncthreads();               // (the length has been read)
    if (threadIdx.x == 0) p.lens[r] = 0;
  }
}

// ---- compact ----------------------------------------------------------------------------------------------------------------------
// Page number k of those in use at or behind `live` goes to free page number k in front of it: there are as many.
struct Compact { int *moves, *live, *holes, *origin, *target; };
__host__ __device__ inline Compact compact_of(const PoolParams &p) {
  Compact c;
  c.moves = p.ws;
  c.live = p.ws + 1;
  c.holes = p.ws + kHeader;
  c.origin = c.holes + p.n_pages;
  c.target = c.origin + p.n_pages;
  return c;
}
__global__ __launch_bounds__(kPlanThreads) void ff_pages_compact_plan_kernel(PoolParams p) {
  const Compact c = compact_of(p);
  int live = 0;
  for (int j = threadIdx.x; j < p.n_pages; j += kPlanThreads) live += p.refs[j] > 0;
  int all;
  sums_before(live, all);
  live = all;
  int holes = 0, moves = 0;
  for (int j0 = 0; j0 < p.n_pages; j0 += kPlanThreads) {
    const int j = j0 + threadIdx.x, r = j < p.n_pages ? p.refs[j] : 0;
    const bool is_hole = j < live && r <= 0, is_move = j >= live && r > 0;
    // (a run of pages may have both: the two counts go together, 11 bits are enough for each)
    int both;
    const int before = sums_before((int)is_hole | (int)is_move << 12, both);
    if (is_hole) put(&c.holes[holes + (before & 0xfff)], j);
    if (is_move) put(&c.origin[moves + (before >> 12)], j);
    if (j < p.n_pages && j >= live && !is_move) c.target[j] = -1;
    holes += both & 0xfff;
    moves += both >> 12;
  }
  written();
  __syncthreads();
  for (int k = threadIdx.x; k < moves; k += kPlanThreads) {
    const int a = fresh(&c.origin[k]), b = fresh(&c.holes[k]);
    c.target[a] = b;
    p.refs[b] = p.refs[a];
    p.refs[a] = 0;
  }
  if (threadIdx.x == 0) {
    *c.moves = moves;
    *c.live = *p.result = live;
  }
}
__global__ __launch_bounds__(kThreads) void ff_pages_compact_kernel(PoolParams p, Parts parts, int n_apply) {
  const Compact c = compact_of(p);
  const int moves = *c.moves, live = *c.live;
  if ((int)blockIdx.x >= n_apply) {
    const int n_copy = gridDim.x - n_apply;
    for (long id = blockIdx.x - n_apply; id < (long)moves * parts.pieces; id += n_copy) {
      const int k = (int)(id / parts.pieces);
      copy_piece<true>(parts, (int)(id - (long)k * parts.pieces), c.origin[k], c.holes[k]);
    }
    return;
  }
  for (int r = blockIdx.x; r < p.n_rows; r += n_apply) {
    int *row = p.table + (size_t)r * p.table_stride;
    for (int j = threadIdx.x; j < pages_of(p, p.lens[r]); j += kThreads) {
      const int page = row[j];
      if (is_page(p, page) && page >= live && c.target[page] >= 0) row[j] = c.target[page];
    }
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------------
Parts parts_of(const ff_page_part *parts, int n) {
  Parts q = {};
  q.n = n;
  for (int k = 0; k < n; ++k) {
    q.data[k] = static_cast<uint8_t *>(parts[k].data);
    q.bytes[k] = parts[k].page_bytes;
    q.pieces += (int)((parts[k].page_bytes + kPiece - 1) / kPiece);
    q.upto[k] = q.pieces;
  }
  return q;
}
constexpr long kCopyGrid = 16384;
int copy_grid(const Parts &q, long moves) { return (int)std::min<long>(moves * q.pieces, kCopyGrid); }

}  // namespace

size_t ff_pages_ints(int64_t n, int32_t n_pages, int32_t n_rows, int32_t table_stride) {
  const size_t fork = kHeader + 2 * (size_t)n + n_rows + (size_t)n * table_stride + (size_t)n;
  const size_t grow = kHeader + 2 * (size_t)n + n_rows + (size_t)n_pages + 1;
  const size_t compact = kHeader + 3 * (size_t)n_pages;
  return std::max(std::max(fork, grow), compact);
}

hipError_t ff_launch_pages_copy(const ff_page_part *parts, int n_parts, int32_t n_pages, int32_t n, const int32_t *from, const int32_t *to, hipStream_t s) {
  for (int k = 0; k < n_parts; k += kPartsAtOnce) {
    const Parts q = parts_of(parts + k, std::min(kPartsAtOnce, n_parts - k));
    hipLaunchKernelGGL(ff_pages_copy_kernel, dim3(copy_grid(q, n)), dim3(kThreads), 0, s, q, n_pages, n, from, to);
  }
  return hipGetLastError();
}

// (parts beyond those of the first launch are copied before the rows change: the plan has what they need)
hipError_t ff_launch_pages_fork(const PoolParams &p, const ff_page_part *parts, int n_parts, hipStream_t s) {
  hipLaunchKernelGGL(ff_pages_fork_plan_kernel, dim3(1 + std::min(p.n, 1024)), dim3(kPlanThreads), 0, s, p);
  int k = 0;
  do {
    const Parts q = parts_of(parts + k, std::min(kPartsAtOnce, n_parts - k));
    k += q.n;
    const int apply = k >= n_parts ? std::min(p.n, 1024) : 0;
    hipLaunchKernelGGL(ff_pages_fork_kernel, dim3(apply + copy_grid(q, p.n)), dim3(kThreads), 0, s, p, q, apply);
  } while (k < n_parts);
  return hipGetLastError();
}

hipError_t ff_launch_pages_grow(const PoolParams &p, hipStream_t s) {
  hipLaunchKernelGGL(ff_pages_grow_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
  return hipGetLastError();
}

hipError_t ff_launch_validate_grow(const PoolParams &p, int32_t *flag, hipStream_t s) {
  hipLaunchKernelGGL(ff_pages_validate_kernel, dim3((p.n + kThreads - 1) / kThreads), dim3(kThreads), 0, s, p, flag);
  return hipGetLastError();
}

hipError_t ff_launch_pages_free(const PoolParams &p, hipStream_t s) {
  hipLaunchKernelGGL(ff_pages_free_kernel, dim3(std::min(p.n, 4096)), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

hipError_t ff_launch_pages_compact(const PoolParams &p, const ff_page_part *parts, int n_parts, hipStream_t s) {
  hipLaunchKernelGGL(ff_pages_compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
  int k = 0;
  do {
    const Parts q = parts_of(parts + k, std::min(kPartsAtOnce, n_parts - k));
    k += q.n;
    const int apply = k >= n_parts ? std::min(p.n_rows, 1024) : 0;
    hipLaunchKernelGGL(ff_pages_compact_kernel, dim3(apply + copy_grid(q, p.n_pages)), dim3(kThreads), 0, s, p, q, apply);
  } while (k < n_parts);
  return hipGetLastError();
}
