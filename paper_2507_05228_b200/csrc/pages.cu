// Page tables of a paged cache on the device: a step of the tables (fork, free, room for new rows), compaction, and the copies of
// pages that both ask for.  Nothing is decided on the host, so a decode loop that forks its sequences stays a graph.
//
// Fork and compaction are chains of small steps over the tables and the pages (count the holders of every page, rank the free
// ones, hand them out), each of which needs all of the one before: latency, not bytes.  One cluster of CTAs does the whole chain
// in one launch, with the cluster's hardware barrier between the steps and the few totals that the CTAs exchange in distributed
// shared memory.  A page is free when no sequence holds it, so the holders are counted anew every time and no list of free pages
// has to be kept.  No list is written either: whoever ranks a free page looks up who takes the page of that rank.  Where the holders
// fit in the shared memory of one CTA (kOne), that CTA does it alone, without a barrier or a trip to L2 between the steps (64
// sequences, 1800 pages: a fork with its copies 17.2 us by a cluster, so 14.5).
// Copying is bound by HBM: twice the bytes of the pages.
#include <limits.h>

#include "paged.cuh"

namespace cascade {

namespace {

constexpr int kPagesThreads = 1024, kMaxPagesCluster = 16;
constexpr int kMaxForkSeqs = 8192;  // six words each in shared memory
static_assert(kMaxForkSeqs <= 32 * kPagesThreads, "a bit for each of a thread's sequences");

// (all threads of the cluster; orders their accesses to global and shared memory)
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// s_all[rank] of every CTA of the cluster becomes `value` (one thread calls it; visible after the next cluster_sync)
__device__ __forceinline__ void tell_cluster(int* s_all, int rank, int n_cta, int value) {
  const uint32_t local = (uint32_t)__cvta_generic_to_shared(s_all + rank);
  for (int to = 0; to < n_cta; ++to) {
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(local), "r"(to));
    asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(value) : "memory");
  }
}

// Rank of this thread's flag among those of the block before it, and the number of all; s_warp: one word a warp
__device__ __forceinline__ int block_rank(bool flag, int* s_warp, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t m = __ballot_sync(0xffffffffu, flag);
  __syncthreads();
  if (lane == 0) s_warp[warp] = __popc(m);
  __syncthreads();
  const int mine = s_warp[lane];  // as many warps as lanes
  const int before = __reduce_add_sync(0xffffffffu, lane < warp ? mine : 0);
  total = __reduce_add_sync(0xffffffffu, mine);
  return before + __popc(m & ((1u << lane) - 1u));
}
static_assert(kPagesThreads == 32 * 32, "a word for every warp");

// Number of pages with pred(page) in [first, end), the same for all threads
template <typename F>
__device__ __forceinline__ int count_pages(int first, int end, int* s_warp, F pred) {
  int mine = 0;
  for (int p = first + (int)threadIdx.x; p < end; p += kPagesThreads) mine += pred(p) ? 1 : 0;
  mine = __reduce_add_sync(0xffffffffu, mine);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = mine;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, s_warp[threadIdx.x & 31]);
}
// f(page, rank) for every page with pred(page) in [first, end), ranks from `rank0` on in the order of the pages
template <typename P, typename F>
__device__ __forceinline__ void rank_pages(int first, int end, int rank0, int* s_warp, P pred, F f) {
  for (int p0 = first; p0 < end; p0 += kPagesThreads) {
    const int p = p0 + (int)threadIdx.x;
    const bool is = p < end && pred(p);
    int total;
    const int r = block_rank(is, s_warp, total);
    if (is) f(p, rank0 + r);
    rank0 += total;
  }
}

// Holders of the pages: in p.refs, for all CTAs of the cluster, or (kOne) in shared memory until the end.
template <bool kOne>
struct Holders {
  int* refs;
  __device__ __forceinline__ int get(int page) const { return kOne ? refs[page] : __ldcg(refs + page); }
};
template <bool kOne>
__device__ __forceinline__ void sync_all() {
  if constexpr (kOne) __syncthreads();
  else cluster_sync();
}

// Entries of row `row` of the table that are pages of it; a bad length has none.
__device__ __forceinline__ int pages_of(int rows, const PagesParams& p) {
  return rows < 0 || rows > (int64_t)p.width * p.page_size ? -1 : (rows + p.page_size - 1) / p.page_size;
}

// f(sequence, column, entry) for this thread's share of the table
template <typename F>
__device__ __forceinline__ void for_entries(int n, int width, int64_t mine, int all, F f) {
  const int64_t entries = (int64_t)n * width;
  if (entries <= INT_MAX - all) {  // (a 64-bit division takes as long as a trip to L2)
#pragma unroll 4
    for (int e = (int)mine; e < (int)entries; e += all) f(e / width, e % width, (int64_t)e);
  } else {
    for (int64_t e = mine; e < entries; e += all) f((int)(e / width), (int)(e % width), e);
  }
}

template <bool kOne>
__global__ void __launch_bounds__(kPagesThreads) pages_fork_kernel(const __grid_constant__ PagesParams p) {
  extern __shared__ int s_dyn[];
  __shared__ int s_warp[32], s_all[kMaxPagesCluster], s_bad, s_long, s_carry, s_ids;
  const int n = p.n_seqs, P = p.page_size;
  int* s_at = s_dyn;           // pages that the sequences before take
  int* s_last = s_dyn + n;     // page that the sequence goes on writing, -1: none
  int* s_had = s_dyn + 2 * n;  // rows it has
  int* s_src = s_dyn + 3 * n;  // the sequence it continues
  int* s_add = s_dyn + 4 * n;  // rows it gets
  int* s_own = s_dyn + 5 * n;  // 1: it gets a copy of that page
  const Holders<kOne> holders{kOne ? s_dyn + 6 * n : p.refs};
  const int n_cta = kOne ? 1 : gridDim.x, rank = kOne ? 0 : blockIdx.x, tid = threadIdx.x;
  const int gt = rank * kPagesThreads + tid, all = n_cta * kPagesThreads;
  grid_go();
  grid_wait();
  if (tid == 0) s_bad = s_long = s_carry = s_ids = 0;
  __syncthreads();
  for (int i = gt; i < p.n_pages; i += all) holders.refs[i] = 0;
  if (gt < 4) p.report[gt] = 0;
  for (int i = tid; i < n; i += kPagesThreads) {
    const int src = fresh(p.source + i), add = fresh(p.add + i);
    int had = 0, last = -1;
    if (src < -1 || src >= n || add < 0) {
      atomicAdd(&s_bad, 1);
    } else if (src >= 0) {
      had = fresh(p.kv_in + src);
      if (pages_of(had, p) < 0) {
        had = 0;
        atomicAdd(&s_bad, 1);
      } else if (add > 0 && had % P > 0) {
        last = fresh(p.table_in + (int64_t)src * p.width + had / P);
      }
    }
    if ((int64_t)had + max(add, 0) > (int64_t)p.width * P) atomicAdd(&s_long, 1);
    s_had[i] = had;
    s_last[i] = last;
    s_src[i] = src;
    s_add[i] = max(0, add);
  }
  sync_all<kOne>();
  // holders of every page
  for_entries(n, p.width, gt, all, [&](int i, int c, int64_t) {
    if ((int64_t)c * P < s_had[i]) {
      const int page = fresh(p.table_in + (int64_t)s_src[i] * p.width + c);
      if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(holders.refs + page, 1);
      else atomicAdd(kOne ? &s_ids : p.report + 2, 1);
    }
  });
  sync_all<kOne>();
  // A sequence that goes on writing a page that others hold, too, gets a copy of its own: except the first of them where all
  // would write it (they leave, it stays alone with it).  A reader among them sees the rows that it has and no more, but may write
  // there itself one day.
  // Every CTA works this out for all sequences.  Few of them go through all others each.  Of more, the writers of every such page are
  // counted, and the first of them is found, in a hash table of a cell a sequence (s_at: the page, s_own: the number, then the first); neither
  // depends on the order of the atomics.  (us, all from one prompt, each through all | hash table: 16 sequences 5.2 | 6.8, 64: 7.6 | 8.6,
  // 256: 15.6 | 15.6, 1024: 42 | 23, 8192: 1495 | 78.)
  uint32_t mine = 0;  // which of this thread's sequences write a page that is held more than once
  for (int i = tid, k = 0; i < n; i += kPagesThreads, ++k) {
    const int last = s_last[i];
    s_own[i] = 0;
    s_at[i] = -1;
    if ((unsigned)last < (unsigned)p.n_pages && holders.get(last) > 1) mine |= 1u << k;
  }
  if (n <= 256) {
    if (mine) {  // (256 threads have a sequence)
      int writers = 0, first = n;
      for (int j = n - 1; j >= 0; --j)
        if (s_last[j] == s_last[tid]) {
          ++writers;
          first = j;
        }
      s_own[tid] = !(writers == holders.get(s_last[tid]) && first == tid);
    }
  } else if (__syncthreads_or(mine != 0)) {
    auto each = [&](uint32_t which, auto f) {
      for (int i = tid, k = 0; i < n; i += kPagesThreads, ++k)
        if (which >> k & 1) f(i, k);
    };
    auto cell_of = [&](int i) {  // (no more pages than cells, so there is one)
      const int page = s_last[i];
      int c = (int)((unsigned)page * 2654435769u % (unsigned)n);
      for (;;) {
        const int there = atomicCAS(&s_at[c], -1, page);
        if (there == -1 || there == page) return c;
        c = c + 1 == n ? 0 : c + 1;
      }
    };
    uint32_t by_all = 0, own = 0;
    each(mine, [&](int i, int) { atomicAdd(&s_own[cell_of(i)], 1); });
    __syncthreads();
    each(mine, [&](int i, int k) { by_all |= (uint32_t)(s_own[cell_of(i)] == holders.get(s_last[i])) << k; });
    __syncthreads();
    each(~0u, [&](int i, int) { s_own[i] = n; });
    __syncthreads();
    each(by_all, [&](int i, int) { atomicMin(&s_own[cell_of(i)], i); });
    __syncthreads();
    each(mine, [&](int i, int k) { own |= (uint32_t)!(by_all >> k & 1 && s_own[cell_of(i)] == i) << k; });
    __syncthreads();
    each(~0u, [&](int i, int k) { s_own[i] = own >> k & 1; });
  }
  __syncthreads();
  // pages that every sequence takes, and how many those before it take
  auto takes = [&](int i) { return (int)(((int64_t)s_had[i] + s_add[i] + P - 1) / P) - (s_had[i] + P - 1) / P + s_own[i]; };
  for (int i0 = 0; i0 < n; i0 += kPagesThreads) {
    const int i = i0 + tid, mine = i < n ? takes(i) : 0, lane = tid & 31;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) s_warp[tid >> 5] = incl;
    __syncthreads();
    const int of = s_warp[lane], before = __reduce_add_sync(0xffffffffu, lane < (tid >> 5) ? of : 0);
    const int total = __reduce_add_sync(0xffffffffu, of), carry = s_carry;
    if (i < n) s_at[i] = carry + before + incl - mine;
    __syncthreads();
    if (tid == 0) s_carry = carry + total;
    __syncthreads();
  }
  const int need = s_carry, chunk = (p.n_pages + n_cta - 1) / n_cta;
  const int first = min(p.n_pages, rank * chunk), end = min(p.n_pages, first + chunk);
  auto is_free = [&](int page) { return holders.get(page) == 0; };
  int n_free = count_pages(first, end, s_warp, is_free), rank0 = 0;
  if constexpr (!kOne) {
    if (tid == 0) tell_cluster(s_all, rank, n_cta, n_free);
    cluster_sync();
    n_free = 0;
    for (int r = 0; r < n_cta; ++r) {
      if (r < rank) rank0 += s_all[r];
      n_free += s_all[r];
    }
  }
  const int bad_ids = kOne ? s_ids : __ldcg(p.report + 2);
  if (s_bad + s_long + bad_ids > 0 || need > n_free) {  // nothing is done (the same decision in every CTA)
    sync_all<kOne>();
    for (int i = gt; i < p.n_pages; i += all) holders.refs[i] = 0;
    for (int i = gt; i < n; i += all) {
      *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
      p.kv_out[i] = fresh(p.kv_in + i);
    }
    sync_all<kOne>();
    for_entries(n, p.width, gt, all, [&](int i, int c, int64_t e) {
      const int page = fresh(p.table_in + e);
      p.table_out[e] = page;
      if (c < pages_of(fresh(p.kv_in + i), p) && (unsigned)page < (unsigned)p.n_pages) atomicAdd(holders.refs + page, 1);
    });
    sync_all<kOne>();
    const int left = count_pages(first, end, s_warp, is_free);
    if (tid == 0) atomicAdd(p.report + 3, left);
    if (gt == 0) {
      p.report[0] = max(0, need - n_free);
      p.report[1] = s_long;
      p.report[2] = bad_ids + s_bad;
    }
    if constexpr (kOne)
      for (int i = tid; i < p.n_pages; i += kPagesThreads) p.refs[i] = holders.refs[i];
    return;
  }
  // The page of rank r goes to the last sequence whose first rank is not above r (one that takes none shares its first rank with
  // the next).
  rank_pages(first, end, rank0, s_warp, is_free, [&](int page, int r) {
    if (r >= need) return;
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_at[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    const int off = r - s_at[lo], old = (s_had[lo] + P - 1) / P, own = s_own[lo];
    if (own && off == 0) *reinterpret_cast<int2*>(p.pairs + 2 * lo) = make_int2(s_last[lo], page);
    p.table_out[(int64_t)lo * p.width + old + off - own] = page;
    holders.refs[page] = 1;
  });
  for_entries(n, p.width, gt, all, [&](int i, int c, int64_t e) {
    const int had = s_had[i];
    if ((int64_t)c * P < had) {
      if (s_own[i] && c == had / P) atomicSub(holders.refs + s_last[i], 1);  // it has a copy now
      else p.table_out[e] = fresh(p.table_in + (int64_t)s_src[i] * p.width + c);
    } else if ((int64_t)c * P >= (int64_t)had + s_add[i]) {
      p.table_out[e] = -1;
    }
  });
  for (int i = gt; i < n; i += all) {
    p.kv_out[i] = s_had[i] + s_add[i];
    if (!s_own[i]) *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
  }
  if (gt == 0) p.report[3] = n_free - need;
  if constexpr (kOne) {
    __syncthreads();
    for (int i = tid; i < p.n_pages; i += kPagesThreads) p.refs[i] = holders.refs[i];
  }
}

template <bool kOne>
__global__ void __launch_bounds__(kPagesThreads) pages_compact_kernel(const __grid_constant__ PagesParams p) {
  extern __shared__ int s_dyn[];
  __shared__ int s_warp[32], s_live[kMaxPagesCluster], s_hole[kMaxPagesCluster], s_mover[kMaxPagesCluster], s_bad;
  const Holders<kOne> holders{kOne ? s_dyn : p.refs};
  const int n_cta = kOne ? 1 : gridDim.x, rank = kOne ? 0 : blockIdx.x, tid = threadIdx.x;
  const int gt = rank * kPagesThreads + tid, all = n_cta * kPagesThreads;
  grid_go();
  grid_wait();
  if (tid == 0) s_bad = 0;
  for (int i = gt; i < p.n_pages; i += all) holders.refs[i] = 0;
  if (gt < 4) p.report[gt] = 0;
  sync_all<kOne>();
  int* const bad = kOne ? &s_bad : p.report + 2;
  for (int i = gt; i < p.n_seqs; i += all)
    if (pages_of(fresh(p.kv_in + i), p) < 0) atomicAdd(bad, 1);
  for_entries(p.n_seqs, p.width, gt, all, [&](int i, int c, int64_t e) {
    const int page = fresh(p.table_in + e);  // (asked for before the length is known)
    if (c >= pages_of(fresh(p.kv_in + i), p)) return;
    if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(holders.refs + page, 1);
    else atomicAdd(bad, 1);
  });
  sync_all<kOne>();
  const int chunk = (p.n_pages + n_cta - 1) / n_cta;
  const int first = min(p.n_pages, rank * chunk), end = min(p.n_pages, first + chunk);
  auto live = [&](int page) { return holders.get(page) > 0; };
  int n_live = count_pages(first, end, s_warp, live);
  if constexpr (!kOne) {
    if (tid == 0) tell_cluster(s_live, rank, n_cta, n_live);
    cluster_sync();
    n_live = 0;
    for (int r = 0; r < n_cta; ++r) n_live += s_live[r];
  }
  if ((kOne ? s_bad : __ldcg(p.report + 2)) > 0) {  // nothing is moved
    for_entries(p.n_seqs, p.width, gt, all, [&](int, int, int64_t e) { p.table_out[e] = fresh(p.table_in + e); });
    for (int i = gt; i < p.max_pairs; i += all) *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
    if (gt == 0) {
      p.report[0] = n_live;
      if (kOne) p.report[2] = s_bad;
      p.report[3] = p.n_pages - n_live;
    }
    if constexpr (kOne)
      for (int i = tid; i < p.n_pages; i += kPagesThreads) p.refs[i] = holders.refs[i];
    return;
  }
  // The holes are the free pages below n_live, the movers the live pages from there on: as many of the ones as of the others, and
  // no page is both, so the copies need no order.
  const int hole_end = min(end, max(first, n_live)), mover_first = max(first, min(end, n_live));
  auto hole = [&](int page) { return !live(page); };
  int n_moves = count_pages(first, hole_end, s_warp, hole), hole0 = 0, mover0 = 0;
  if constexpr (!kOne) {
    const int movers_here = count_pages(mover_first, end, s_warp, live);
    if (tid == 0) {
      tell_cluster(s_hole, rank, n_cta, n_moves);
      tell_cluster(s_mover, rank, n_cta, movers_here);
    }
    cluster_sync();
    n_moves = 0;
    for (int r = 0; r < n_cta; ++r) {
      if (r < rank) {
        hole0 += s_hole[r];
        mover0 += s_mover[r];
      }
      n_moves += s_hole[r];
    }
  }
  rank_pages(first, hole_end, hole0, s_warp, hole, [&](int page, int r) { p.pairs[2 * r + 1] = page; });
  rank_pages(mover_first, end, mover0, s_warp, live, [&](int page, int r) { p.pairs[2 * r] = page; });
  for (int i = n_moves + gt; i < p.max_pairs; i += all) *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
  sync_all<kOne>();
  // the holders go with the page; until the table is rewritten refs says where: -(target + 1)
  for (int r = gt; r < n_moves; r += all) {
    const int2 e = __ldcg(reinterpret_cast<const int2*>(p.pairs + 2 * r));
    holders.refs[e.y] = holders.get(e.x);
    holders.refs[e.x] = -e.y - 1;
  }
  sync_all<kOne>();
  for_entries(p.n_seqs, p.width, gt, all, [&](int i, int c, int64_t e) {
    int page = fresh(p.table_in + e);
    if (c >= pages_of(fresh(p.kv_in + i), p)) page = -1;
    else if (page >= n_live) page = -holders.get(page) - 1;
    p.table_out[e] = page;
  });
  if (gt == 0) {
    p.report[0] = n_live;
    p.report[1] = n_moves;
    p.report[3] = p.n_pages - n_live;
  }
  sync_all<kOne>();
  if constexpr (kOne) {
    for (int i = tid; i < p.n_pages; i += kPagesThreads) p.refs[i] = i < n_live ? holders.refs[i] : 0;
  } else {
    for (int i = max(first, n_live) + tid; i < end; i += kPagesThreads) p.refs[i] = 0;
  }
}

// Every CTA lists the valid pairs, 2048 at a time, and takes its share of their pages piece by piece: most of the list may be empty
// (fork: a pair a sequence; compaction: half the pool).
constexpr int kCopyThreads = 512, kCopyWindow = 2048, kCopyLoads = 8, kCopyPiece = kCopyThreads * 16 * kCopyLoads;

__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const __grid_constant__ PagesCopyParams p) {
  __shared__ int2 s_pair[kCopyWindow];
  __shared__ int s_warp[kCopyThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int pieces = (int)((p.page_bytes + kCopyPiece - 1) / kCopyPiece);
  grid_go();
  grid_wait();
  for (int w0 = 0; w0 < p.n_pairs; w0 += kCopyWindow) {
    const int n_w = min(kCopyWindow, p.n_pairs - w0);
    int n_there = 0;  // in the order of the list, so that all CTAs number the pieces alike
    for (int j0 = 0; j0 < n_w; j0 += kCopyThreads) {
      const int j = j0 + tid;
      int2 e = make_int2(-1, -1);
      if (j < n_w) e = make_int2(fresh(p.pairs + 2 * (int64_t)(w0 + j)), fresh(p.pairs + 2 * (int64_t)(w0 + j) + 1));
      const bool none = e.x == -1 || e.y == -1;
      const bool fine = (unsigned)e.x < (unsigned)p.n_pages && (unsigned)e.y < (unsigned)p.n_pages;
      if (!none && !fine && blockIdx.x == 0) paged_report(p.status, kBadPair, w0 + j, (unsigned)e.x < (unsigned)p.n_pages ? e.y : e.x);
      const bool there = !none && fine && e.x != e.y;
      const uint32_t m = __ballot_sync(0xffffffffu, there);
      __syncthreads();
      if (lane == 0) s_warp[warp] = __popc(m);
      __syncthreads();
      const int of = lane < kCopyThreads / 32 ? s_warp[lane] : 0;
      const int before = __reduce_add_sync(0xffffffffu, lane < warp ? of : 0);
      if (there) s_pair[n_there + before + __popc(m & ((1u << lane) - 1u))] = e;
      n_there += __reduce_add_sync(0xffffffffu, of);
    }
    __syncthreads();
    const int64_t items = (int64_t)n_there * p.n_pools * pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
      const int which = (int)(item / ((int64_t)p.n_pools * pieces));
      const int rest = (int)(item - (int64_t)which * p.n_pools * pieces), pool = rest / pieces;
      const int64_t off = (int64_t)(rest - pool * pieces) * kCopyPiece + tid * 16;
      const int2 e = s_pair[which];
      const char* src = static_cast<const char*>(p.pool[pool]) + e.x * p.page_stride[pool];
      char* dst = static_cast<char*>(p.pool[pool]) + e.y * p.page_stride[pool];
      uint4 v[kCopyLoads];
#pragma unroll
      for (int i = 0; i < kCopyLoads; ++i)
        if (off + i * kCopyThreads * 16 < p.page_bytes) v[i] = __ldcs(reinterpret_cast<const uint4*>(src + off + i * kCopyThreads * 16));
#pragma unroll
      for (int i = 0; i < kCopyLoads; ++i)
        if (off + i * kCopyThreads * 16 < p.page_bytes) __stcs(reinterpret_cast<uint4*>(dst + off + i * kCopyThreads * 16), v[i]);
    }
  }
}

}  // namespace

cudaError_t launch_pages_copy(const PagesCopyParams& p, cudaStream_t stream) {
  const int64_t pieces = (int64_t)p.n_pairs * p.n_pools * ((p.page_bytes + kCopyPiece - 1) / kCopyPiece);
  return launch_dependent(pages_copy_kernel, dim3((unsigned)std::min<int64_t>(pieces, 148 * 2)), kCopyThreads, 0, 1, true, stream, p);
}

// One CTA where the holders fit next to its tables and it has few entries to go through; a cluster otherwise.
static bool one_cta(const PagesParams& p, size_t smem) { return smem + (size_t)p.n_pages * 4 <= 160 * 1024 && (int64_t)p.n_seqs * p.width <= 32768; }
static cudaError_t launch_pages(void (*kernel)(PagesParams), const PagesParams& p, size_t smem, int n_cta, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess && n_cta > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3(n_cta), kPagesThreads, smem, n_cta, true, stream, p);
}
cudaError_t launch_pages_fork(const PagesParams& p, cudaStream_t stream) {
  if (p.n_seqs > kMaxForkSeqs) return cudaErrorInvalidValue;
  const size_t smem = (size_t)p.n_seqs * 24;
  if (one_cta(p, smem)) return launch_pages(pages_fork_kernel<true>, p, smem + (size_t)p.n_pages * 4, 1, stream);
  return launch_pages(pages_fork_kernel<false>, p, smem, kMaxPagesCluster, stream);
}
cudaError_t launch_pages_compact(const PagesParams& p, cudaStream_t stream) {
  if (one_cta(p, 0)) return launch_pages(pages_compact_kernel<true>, p, (size_t)p.n_pages * 4, 1, stream);
  return launch_pages(pages_compact_kernel<false>, p, 0, kMaxPagesCluster, stream);
}

}  // namespace cascade
