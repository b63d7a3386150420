// What the kernels on paged caches share: the rows of a sequence, its length and its pages, each checked before it forms an
// address, and the words that they report to.
#pragma once

#include <limits.h>

#include "cascade_internal.cuh"

namespace cascade {

// A load of what the kernel in front may have written: an ordinary one.  These kernels start as programmatic dependents, before that one
// is done, so what they read is not constant for as long as they run, which a load through the read-only path (__ldg) asks for.
template <typename T>
__device__ __forceinline__ T fresh(const T* p) {
  return *p;
}

// Words 0 .. kStatusWords - 1: a bounded wait that gave up, as in a plan (WaitCtx).  Then a bad index: its code, the sequence (or
// pair) and the value.
enum PagedStatus { kBadIndexWord = 32, kPagedStatusWords = 36 };
enum PagedBad {
  kBadRowStart = 121,  // row_start falls, or leaves [0, n_rows]
  kBadLength = 122,    // kv_len below 0, or more rows than the table has pages for
  kBadPage = 123,      // a page id outside [0, n_pages)
  kBadPosition = 124,  // a position outside the rotary table
  kBadPair = 125,      // a page pair outside [0, n_pages)
  kBadRows = 126       // a sequence has more rows than max_rows
};

__device__ __forceinline__ void paged_report(int32_t* status, int code, int where, int value) {
  if (atomicCAS(status + kBadIndexWord, 0, code) == 0) {
    status[kBadIndexWord + 1] = where;
    status[kBadIndexWord + 2] = value;
  }
}

// First row and number of rows of sequence b; none where row_start makes no sense.
__device__ __forceinline__ int2 paged_rows(const PagedDev& g, int b) {
  const int first = fresh(g.row_start + b), end = fresh(g.row_start + b + 1);
  if (first < 0 || end < first || end > g.n_rows) {
    paged_report(g.status, kBadRowStart, b, first);
    return make_int2(0, 0);
  }
  return make_int2(first, end - first);
}
// Cache rows of sequence b, as many as its row of the table can hold.
__device__ __forceinline__ int paged_len(const PagedDev& g, int b) {
  const int len = fresh(g.kv_len + b);
  const int64_t most = (int64_t)g.max_pages * g.page_size;
  if (len >= 0 && len <= most) return len;
  paged_report(g.status, kBadLength, b, len);
  return len < 0 ? 0 : (int)most;
}
// Id of page i of sequence b (i below max_pages); page 0 in the place of a bad one, which is reported.
__device__ __forceinline__ int paged_checked(const PagedDev& g, int b, int id) {
  if ((unsigned)id < (unsigned)g.n_pages) return id;
  paged_report(g.status, kBadPage, b, id);
  return 0;
}
__device__ __forceinline__ int paged_page(const PagedDev& g, int b, int i) {
  return paged_checked(g, b, fresh(g.table + (int64_t)b * g.table_stride + i));
}
// Cache rows that row i of the n of a sequence sees; `row` is its place among all rows.
__device__ __forceinline__ int paged_seen(const PagedDev& g, bool causal, int n, int len, int i, int row) {
  if (g.visible) return max(0, min(len, fresh(g.visible + row)));
  return causal ? max(0, len - n + i + 1) : len;
}

// Sequence and tile of tile number t, of those of `per_tile` rows each that the sequences of least .. most rows have: of 32
// sequences at a time the one with the longest cache first, and of a sequence its last tile (which sees most), so that the last
// tiles to start are short ones.  {sequence, tile}, or {-1, 0} past the last.  All lanes of a warp.
__device__ __forceinline__ int2 paged_tile(const PagedDev& g, int t, int per_tile, int lane) {
  int before = 0;
  for (int b0 = 0; b0 < g.batch; b0 += 32) {
    const int b = b0 + lane;
    const int n = b < g.batch ? paged_rows(g, b).y : 0;
    const int tiles = n >= g.least && n <= g.most ? (n + per_tile - 1) / per_tile : 0;
    const int total = __reduce_add_sync(0xffffffffu, tiles);
    if (t < before + total) {
      const int len = tiles > 0 ? fresh(g.kv_len + b) : INT_MIN;
      int first = before;  // tiles of the sequences that come before this lane's
      for (int j = 0; j < min(32, g.batch - b0); ++j) {
        const int other = __shfl_sync(0xffffffffu, len, j), n_other = __shfl_sync(0xffffffffu, tiles, j);
        if (other > len || (other == len && j < lane)) first += n_other;
      }
      const int who = __ffs(__ballot_sync(0xffffffffu, t >= first && t < first + tiles)) - 1;
      return make_int2(b0 + who, __shfl_sync(0xffffffffu, first + tiles, who) - 1 - t);
    }
    before += total;
  }
  return make_int2(-1, 0);
}

}  // namespace cascade
