// Pages of a cache, shared by the rows of a table: parameters of the kernels that fork, grow, free and compact them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastforward.h"

constexpr int kPartsAtOnce = 64;      // of one launch

struct PoolParams {
  int32_t *refs, *table, *lens;
  int32_t n_pages, page_shift, n_rows, table_stride;
  // entries of the call: rows that are read and written (fork), rows and lengths (grow), rows (free)
  int32_t n;
  const int32_t *from, *to, *new_lens;
  int32_t *result;               // pages that were missing, or pages in use
  int32_t *ws;                   // see ff_pages_ints
};
// 32-bit numbers of workspace that a call with n entries takes at most; grow and compact, which keep no row's pages, with a table_stride of 0
size_t ff_pages_ints(int64_t n, int32_t n_pages, int32_t n_rows, int32_t table_stride);

hipError_t ff_launch_pages_copy(const ff_page_part *parts, int n_parts, int32_t n_pages, int32_t n, const int32_t *from, const int32_t *to, hipStream_t s);
hipError_t ff_launch_pages_fork(const PoolParams &p, const ff_page_part *parts, int n_parts, hipStream_t s);
hipError_t ff_launch_pages_grow(const PoolParams &p, hipStream_t s);
// flag[0] is set to 1 + an entry of a grow whose length its row cannot have.  The caller zeroes flag[0] first.
hipError_t ff_launch_validate_grow(const PoolParams &p, int32_t *flag, hipStream_t s);
hipError_t ff_launch_pages_free(const PoolParams &p, hipStream_t s);
hipError_t ff_launch_pages_compact(const PoolParams &p, const ff_page_part *parts, int n_parts, hipStream_t s);
