// Page tables of a paged cache on the device: a step of the tables (fork, free, room for new rows), compaction, and the copies of
// pages that both ask for.  Nothing is decided on the host, so a decode loop that forks its sequences stays a graph.
//
// Fork and compaction are chains of small steps over the tables and the pages (count the holders of every page, rank the free
// ones, hand them out), each of which needs all of the one before: latency, not bytes.  One cluster of CTAs does the whole chain
// in one launch, with the cluster's hardware barrier between the steps and the few totals that the CTAs exchange in distributed
// shared memory.  A page is free when no sequence holds it, so the holders are counted anew every time and no list of free pages
// has to be kept.  No list is written either: whoever ranks a free page looks up who takes the page of that rank.
// Copying is bound by HBM: twice the bytes of the pages.
#include "paged.cuh"

namespace cascade {

namespace {

constexpr int kPagesThreads = 1024, kMaxPagesCluster = 16;
constexpr int kMaxForkSeqs = 8192;  // whose places fit in shared memory

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

// Entries of row `row` of the table that are pages of it; a bad length has none.
__device__ __forceinline__ int pages_of(int rows, const PagesParams& p) {
  return rows < 0 || rows > (int64_t)p.width * p.page_size ? -1 : (rows + p.page_size - 1) / p.page_size;
}

__global__ void __launch_bounds__(kPagesThreads) pages_fork_kernel(const __grid_constant__ PagesParams p) {
  extern __shared__ int s_dyn[];
  __shared__ int s_warp[32], s_all[kMaxPagesCluster], s_bad, s_long, s_carry;
  const int n = p.n_seqs, P = p.page_size;
  int* s_at = s_dyn;          // pages that the sequences before take
  int* s_last = s_dyn + n;    // page that the sequence goes on writing, -1: none
  int* s_had = s_dyn + 2 * n;  // rows it has
  const int n_cta = gridDim.x, rank = blockIdx.x, tid = threadIdx.x;
  const int gt = rank * kPagesThreads + tid, all = n_cta * kPagesThreads;
  grid_go();
  grid_wait();
  if (tid == 0) s_bad = s_long = s_carry = 0;
  __syncthreads();
  for (int i = gt; i < p.n_pages; i += all) p.refs[i] = 0;
  if (gt < 4) p.report[gt] = 0;
  for (int i = tid; i < n; i += kPagesThreads) {
    const int src = __ldg(p.source + i), add = __ldg(p.add + i);
    int had = 0, last = -1;
    if (src < -1 || src >= n || add < 0) {
      atomicAdd(&s_bad, 1);
    } else if (src >= 0) {
      had = __ldg(p.kv_in + src);
      if (pages_of(had, p) < 0) {
        had = 0;
        atomicAdd(&s_bad, 1);
      } else if (add > 0 && had % P > 0) {
        last = __ldg(p.table_in + (int64_t)src * p.width + had / P);
      }
    }
    if ((int64_t)had + max(add, 0) > (int64_t)p.width * P) atomicAdd(&s_long, 1);
    s_had[i] = had;
    s_last[i] = last;
  }
  cluster_sync();
  // holders of every page
  for (int64_t e = gt; e < (int64_t)n * p.width; e += all) {
    const int i = (int)(e / p.width), c = (int)(e - (int64_t)i * p.width);
    if ((int64_t)c * P < s_had[i]) {
      const int page = __ldg(p.table_in + (int64_t)__ldg(p.source + i) * p.width + c);
      if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(p.refs + page, 1);
      else atomicAdd(p.report + 2, 1);
    }
  }
  cluster_sync();
  // A sequence that goes on writing a page that others hold, too, gets a copy of its own: except the first of them where all
  // would write it (they leave, it stays alone with it).  A reader among them sees the rows that it has and no more, but may write
  // there itself one day.
  for (int i = gt; i < n; i += all) {
    const int last = s_last[i];
    bool copied = false;
    if ((unsigned)last < (unsigned)p.n_pages) {
      const int holders = __ldcg(p.refs + last);
      if (holders > 1) {
        int writers = 0, first = n;
        for (int j = n - 1; j >= 0; --j)
          if (s_last[j] == last) {
            ++writers;
            first = j;
          }
        copied = !(writers == holders && first == i);
      }
    }
    *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(copied ? last : -1, -1);
  }
  cluster_sync();
  // pages that every sequence takes, and how many those before it take
  auto takes = [&](int i) {
    const int64_t rows = (int64_t)s_had[i] + max(0, __ldg(p.add + i));
    return (int)((rows + P - 1) / P) - (s_had[i] + P - 1) / P + (__ldcg(p.pairs + 2 * i) >= 0 ? 1 : 0);
  };
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
  auto is_free = [&](int page) { return __ldcg(p.refs + page) == 0; };
  const int n_free_here = count_pages(first, end, s_warp, is_free);
  if (tid == 0) tell_cluster(s_all, rank, n_cta, n_free_here);
  cluster_sync();
  int n_free = 0, rank0 = 0;
  for (int r = 0; r < n_cta; ++r) {
    if (r < rank) rank0 += s_all[r];
    n_free += s_all[r];
  }
  const int bad_pages = __ldcg(p.report + 2);
  if (s_bad + s_long + bad_pages > 0 || need > n_free) {  // nothing is done (the same decision in every CTA)
    cluster_sync();
    for (int i = gt; i < p.n_pages; i += all) p.refs[i] = 0;
    for (int i = gt; i < n; i += all) {
      *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
      p.kv_out[i] = __ldg(p.kv_in + i);
    }
    cluster_sync();
    for (int64_t e = gt; e < (int64_t)n * p.width; e += all) {
      const int i = (int)(e / p.width), page = __ldg(p.table_in + e);
      p.table_out[e] = page;
      if ((int)(e - (int64_t)i * p.width) < pages_of(__ldg(p.kv_in + i), p) && (unsigned)page < (unsigned)p.n_pages)
        atomicAdd(p.refs + page, 1);
    }
    cluster_sync();
    const int left = count_pages(first, end, s_warp, is_free);
    if (tid == 0) atomicAdd(p.report + 3, left);
    if (gt == 0) {
      p.report[0] = max(0, need - n_free);
      p.report[1] = s_long;
      p.report[2] = bad_pages + s_bad;
    }
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
    const int off = r - s_at[lo], old = (s_had[lo] + P - 1) / P;
    const bool copied = __ldcg(p.pairs + 2 * lo) >= 0;
    if (copied && off == 0) p.pairs[2 * lo + 1] = page;
    p.table_out[(int64_t)lo * p.width + old + off - (copied ? 1 : 0)] = page;
    p.refs[page] = 1;
  });
  for (int64_t e = gt; e < (int64_t)n * p.width; e += all) {
    const int i = (int)(e / p.width), c = (int)(e - (int64_t)i * p.width), had = s_had[i];
    if ((int64_t)c * P < had) {
      if (s_last[i] >= 0 && c == had / P && __ldcg(p.pairs + 2 * i) >= 0) atomicSub(p.refs + s_last[i], 1);  // it has a copy now
      else p.table_out[e] = __ldg(p.table_in + (int64_t)__ldg(p.source + i) * p.width + c);
    } else if ((int64_t)c * P >= (int64_t)had + __ldg(p.add + i)) {
      p.table_out[e] = -1;
    }
  }
  for (int i = gt; i < n; i += all) p.kv_out[i] = s_had[i] + __ldg(p.add + i);
  if (gt == 0) p.report[3] = n_free - need;
}

__global__ void __launch_bounds__(kPagesThreads) pages_compact_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int s_warp[32], s_live[kMaxPagesCluster], s_hole[kMaxPagesCluster], s_mover[kMaxPagesCluster];
  const int n_cta = gridDim.x, rank = blockIdx.x, tid = threadIdx.x;
  const int gt = rank * kPagesThreads + tid, all = n_cta * kPagesThreads;
  const int64_t entries = (int64_t)p.n_seqs * p.width;
  grid_go();
  grid_wait();
  for (int i = gt; i < p.n_pages; i += all) p.refs[i] = 0;
  if (gt < 4) p.report[gt] = 0;
  cluster_sync();
  auto kept = [&](int64_t e) {
    const int i = (int)(e / p.width);
    return (int)(e - (int64_t)i * p.width) < pages_of(__ldg(p.kv_in + i), p);
  };
  for (int i = gt; i < p.n_seqs; i += all)
    if (pages_of(__ldg(p.kv_in + i), p) < 0) atomicAdd(p.report + 2, 1);
  for (int64_t e = gt; e < entries; e += all) {
    if (!kept(e)) continue;
    const int page = __ldg(p.table_in + e);
    if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(p.refs + page, 1);
    else atomicAdd(p.report + 2, 1);
  }
  cluster_sync();
  const int chunk = (p.n_pages + n_cta - 1) / n_cta;
  const int first = min(p.n_pages, rank * chunk), end = min(p.n_pages, first + chunk);
  auto live = [&](int page) { return __ldcg(p.refs + page) > 0; };
  const int live_here = count_pages(first, end, s_warp, live);
  if (tid == 0) tell_cluster(s_live, rank, n_cta, live_here);
  cluster_sync();
  int n_live = 0;
  for (int r = 0; r < n_cta; ++r) n_live += s_live[r];
  if (__ldcg(p.report + 2) > 0) {  // nothing is moved
    for (int64_t e = gt; e < entries; e += all) p.table_out[e] = __ldg(p.table_in + e);
    for (int i = gt; i < p.max_pairs; i += all) *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
    if (gt == 0) {
      p.report[0] = n_live;
      p.report[3] = p.n_pages - n_live;
    }
    return;
  }
  // The holes are the free pages below n_live, the movers the live pages from there on: as many of the ones as of the others, and
  // no page is both, so the copies need no order.
  const int hole_end = min(end, max(first, n_live)), mover_first = max(first, min(end, n_live));
  auto hole = [&](int page) { return !live(page); };
  const int holes_here = count_pages(first, hole_end, s_warp, hole), movers_here = count_pages(mover_first, end, s_warp, live);
  if (tid == 0) {
    tell_cluster(s_hole, rank, n_cta, holes_here);
    tell_cluster(s_mover, rank, n_cta, movers_here);
  }
  cluster_sync();
  int hole0 = 0, mover0 = 0, n_moves = 0;
  for (int r = 0; r < n_cta; ++r) {
    if (r < rank) {
      hole0 += s_hole[r];
      mover0 += s_mover[r];
    }
    n_moves += s_hole[r];
  }
  rank_pages(first, hole_end, hole0, s_warp, hole, [&](int page, int r) { p.pairs[2 * r + 1] = page; });
  rank_pages(mover_first, end, mover0, s_warp, live, [&](int page, int r) { p.pairs[2 * r] = page; });
  for (int i = n_moves + gt; i < p.max_pairs; i += all) *reinterpret_cast<int2*>(p.pairs + 2 * i) = make_int2(-1, -1);
  cluster_sync();
  // the holders go with the page; until the table is rewritten refs says where: -(target + 1)
  rank_pages(mover_first, end, mover0, s_warp, live, [&](int page, int r) {
    const int to = __ldcg(p.pairs + 2 * r + 1);
    p.refs[to] = __ldcg(p.refs + page);
    p.refs[page] = -to - 1;
  });
  cluster_sync();
  for (int64_t e = gt; e < entries; e += all) {
    int page = -1;
    if (kept(e)) {
      page = __ldg(p.table_in + e);
      if (page >= n_live) page = -__ldcg(p.refs + page) - 1;
    }
    p.table_out[e] = page;
  }
  cluster_sync();
  for (int i = max(first, n_live) + tid; i < end; i += kPagesThreads) p.refs[i] = 0;
  if (gt == 0) {
    p.report[0] = n_live;
    p.report[1] = n_moves;
    p.report[3] = p.n_pages - n_live;
  }
}

// Every CTA lists the valid pairs, 2048 at a time, and takes its share of their pages piece by piece: most of the list may be empty
// (fork: a pair a sequence; compaction: half the pool).
constexpr int kCopyThreads = 512, kCopyWindow = 2048, kCopyLoads = 4, kCopyPiece = kCopyThreads * 16 * kCopyLoads;

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
      if (j < n_w) e = make_int2(__ldg(p.pairs + 2 * (int64_t)(w0 + j)), __ldg(p.pairs + 2 * (int64_t)(w0 + j) + 1));
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
  return launch_dependent(pages_copy_kernel, dim3((unsigned)std::min<int64_t>(pieces, 148 * 4)), kCopyThreads, 0, 1, true, stream, p);
}

static cudaError_t launch_pages(void (*kernel)(PagesParams), const PagesParams& p, size_t smem, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess && smem) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3(kMaxPagesCluster), kPagesThreads, smem, kMaxPagesCluster, true, stream, p);
}
cudaError_t launch_pages_fork(const PagesParams& p, cudaStream_t stream) {
  if (p.n_seqs > kMaxForkSeqs) return cudaErrorInvalidValue;
  return launch_pages(pages_fork_kernel, p, (size_t)p.n_seqs * 12, stream);
}
cudaError_t launch_pages_compact(const PagesParams& p, cudaStream_t stream) { return launch_pages(pages_compact_kernel, p, 0, stream); }

}  // namespace cascade
