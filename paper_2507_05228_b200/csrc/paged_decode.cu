// Single tokens and drafts over a paged cache (cascade_attn_paged for sequences of few rows): every K/V row is read once, so
// the bound is HBM for large batches and latency for small ones.
//
// The columns of warp-level mma.m16n8k16 products are (row, head) pairs: the rows of a sequence times the heads of a KV head (as many
// as divide its group, 16 at most), 8 to 32 of them.  A warp walks blocks of 16 keys, which lie in one page.
//   Up to 8 columns the fragments come straight from global memory, as in decode.cu, which says why.
//   More leave no registers for rows on their way.  Every warp then has a ring of 24 KiB in shared memory, filled by TMA a block at a
//   time (two requests of 16 rows each), and reads fragments by ldmatrix.  It waits for its own copies only; no warp waits for another.
//   us, 32 / 8 heads of 128, 16 sequences over 3000 to 9000 rows (bytes: 61): 2 rows each 74, 4 80, 6 83, 8 84; before, from registers 83
//   and 109, and from 5 rows on in tiles of 256 that are nearly empty 131.  4 sequences of 6 rows 52 -> 30.
// The weights go into the second product as two bf16 parts, the upper 16 bits and the rest, so that they keep 16 bits of mantissa: the
// loads are the limit, and with one part the rounding of few rows of weights was most of the error (2500 rows, 32 heads: 2.4e-3 of
// the output, 1.7e-3 with two, which is its own rounding).  From 17 columns on the products are a limit too: one part, rounded to
// nearest, as in the tile kernel with heads of 128 (us, two parts | one: 16 sequences of 6 rows 80 | 82, of 8 89 | 83, 4 of 6 27 | 24; 16 of 6
// with heads of 64 56 | 52).
//
// fp32 the same way with m16n8k8 products of operands cut into two tf32 parts (tf32.cuh); weights go from the lanes of their keys to
// those of their columns by shuffles, and every block's products with the values are summed by themselves and added in fp32.
//
// How the keys are shared out (rules and times at cluster_size).  Lengths differ between sequences, and only the device knows them.
//   Few (sequence, KV head) items over short caches, or one sequence: a cluster of CTAs has one and adds up in distributed shared
//   memory; one launch.
//   Few otherwise: every item gets a CTA, and the other CTAs of the chip go to the items by their length; what the CTAs of an item
//   leave is added up by a second, small kernel.
//   Many over caches that cannot be long: a CTA an item, no joining.
//   Many: the 16-key blocks of all items, one after another, are cut into as many equal ranges as CTAs are resident; an item that a
//   range covers whole is finished there, one that is cut leaves partials for the second kernel.
// Who has what follows from the lengths, which every CTA adds up for itself.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "decode_common.cuh"
#include "paged.cuh"
#include "tcgen05.cuh"
#include "tf32.cuh"

namespace cascade {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32, kJoinThreads = 128;
constexpr int kRangeWarps = 4, kRangeThreads = kRangeWarps * 32;  // of a CTA that walks ranges
constexpr int kMaxGroups = 2048;  // groups of 32 sequences
constexpr int kClusterMost = 16;
constexpr int kMostInRegisters = 8, kMostColumns = 32;

// Where a CTA's range starts: the item that holds its first block, and that block's place in the item.
struct RangeStart {
  int32_t b, item, before, blocks;  // blocks: of the item
  int64_t total;                    // of all items
};

struct DecodeArgs {
  int32_t Gi, items;  // heads of an item, items of a sequence
  int32_t n_cta;      // CTAs of the grid (ranges), or of a cluster
  RangeStart* starts;  // [n_cta], ranges
  int4* joins;         // [n_cta], shares: of the item whose first part is the CTA's, see paged_decode_join_shares_kernel
  float* partials;     // [n_cta][2][columns][D + 2]: of an item that starts before the range, and of one that ends behind it
};

// 16-key blocks of sequence b: none if its rows are not this kernel's.
__device__ __forceinline__ int blocks_of(const PagedDev& g, int b) {
  const int n = paged_rows(g, b).y;
  if (n < g.least || n > g.most) return 0;
  return (paged_len(g, b) + 15) / 16;
}
__device__ __forceinline__ int ranges_of(int64_t total, int n_cta) {  // a block for every warp at least
  return (int)max((int64_t)1, min((int64_t)n_cta, (total + kRangeWarps - 1) / kRangeWarps));
}

// Query fragments: B operand of a k-step, lane (column, j); fp32: the upper parts of both values, then the rests
template <typename T, int D>
struct Fragments;
template <int D>
struct Fragments<__nv_bfloat16, D> {
  uint2 step[D / 16][32];
};
template <int D>
struct Fragments<float, D> {
  uint4 step[D / 8][32];
};

// More than kMostInRegisters columns leave no registers for the rows of the cache: they come to shared memory by TMA then, every warp
// a ring of its own blocks.
template <typename T, int NT>
constexpr bool kStaged = sizeof(T) == 2 && NT > kMostInRegisters / 8;
template <int D>
constexpr int kStages = 384 / D;  // blocks of a warp's ring, 24 KiB
template <int D>
constexpr int kPartBytes = 16 * D * 2;  // keys or values of a block: boxes of 16 rows and 64 columns, 128-byte swizzle

template <typename T, int D, int NT, int W, bool kStaged>
struct Shared {
  float o[W][8 * NT][D + 4];
  float m[W][8 * NT], l[W][8 * NT];
  Fragments<T, D> q[NT];
  __device__ __forceinline__ float* out(int warp, int col) { return o[warp][col]; }
  __device__ __forceinline__ const float* out(int warp, int col) const { return o[warp][col]; }
};
template <typename T, int D, int NT, int W>
struct Shared<T, D, NT, W, true> {
  uint8_t ring[W][kStages<D>][2][kPartBytes<D>];  // and a warp's outputs, once it has walked all its blocks
  float m[W][8 * NT], l[W][8 * NT];
  Fragments<T, D> q[NT];
  uint64_t full[W][kStages<D>];
  int words[2 + W];  // WaitCtx
  static_assert(8 * NT * (D + 4) * 4 <= kStages<D> * 2 * kPartBytes<D>, "a warp's outputs lie in its ring");
  __device__ __forceinline__ float* out(int warp, int col) { return reinterpret_cast<float*>(ring[warp][0][0]) + col * (D + 4); }
  __device__ __forceinline__ const float* out(int warp, int col) const { return reinterpret_cast<const float*>(ring[warp][0][0]) + col * (D + 4); }
};
template <typename T, int D, int NT, int W>
using SharedOf = Shared<T, D, NT, W, kStaged<T, NT>>;
// CTAs of kRangeWarps that an SM takes
template <typename T, int D, int NT>
constexpr int kHalfCtas = sizeof(T) == 2 && D == 64 && !kStaged<T, NT> ? 4 : 2;
template <typename T, int D, int NT, int W>
constexpr int kSmemBytes = (int)sizeof(SharedOf<T, D, NT, W>) + (kStaged<T, NT> ? 1024 : 0);  // the ring starts at a multiple of 1024

struct alignas(64) PageMaps {
  CUtensorMap k, v;  // [page][head][64-column half][row of the page][64 columns]
};
struct NoMaps {};
template <typename T, int NT>
using MapsOf = std::conditional_t<kStaged<T, NT>, PageMaps, NoMaps>;

template <typename T, int D, int NT, int W>
__device__ __forceinline__ SharedOf<T, D, NT, W>& shared_of(uint8_t* smem) {
  if constexpr (kStaged<T, NT>) smem += (0u - tc::smem_u32(smem)) & 1023u;
  return *reinterpret_cast<SharedOf<T, D, NT, W>*>(smem);
}
// (every warp its own barriers; the words are there after the next __syncthreads)
template <typename T, int D, int NT, int W>
__device__ __forceinline__ void set_up(SharedOf<T, D, NT, W>& sh, int warp, int lane) {
  if constexpr (kStaged<T, NT>) {
    if (warp == 0 && lane < 2 + W) sh.words[lane] = 0;
    if (lane == 0)
      for (int i = 0; i < kStages<D>; ++i) tc::mbar_init(tc::smem_u32(&sh.full[warp][i]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
}
// A bounded wait has given up, here or in an earlier call: nothing is written.
template <typename T, int NT>
__device__ __forceinline__ bool gave_up(const AttnParams& p) {
  if constexpr (kStaged<T, NT>) return *reinterpret_cast<volatile const int32_t*>(p.paged.status) != 0;
  return false;
}

template <int D, int NT>
struct State {
  // o[t][e][2 r + h]: column 8 t + 2 j + h, output column x D / 8 + 2 e + r (staged: 16 e + 8 r + x)
  float o[NT][D / 16][4];
  float m[NT][2], l[NT][2];    // log2 units; l: this thread's share
};

// One sequence's rows and pages as a warp sees them
template <typename T, int D, int NT>
struct Walk {
  const AttnParams& p;
  const T *kp, *vp;  // this lane's columns of the KV head
  int b, g, len, lane;  // g: KV head
  float cs;
  int lim[NT][2];  // keys that this lane's columns see

  __device__ __forceinline__ int page_of(int block) const {  // block below those of the sequence
    return paged_page(p.paged, b, block * 16 / p.paged.page_size);
  }
  // the same asked for before it is known whether there is such a block; checked later
  static __device__ __forceinline__ int early_page(const PagedDev& g, int b, int block) {
    const int i = block * 16 / g.page_size;
    return i < g.max_pages ? fresh(g.table + (int64_t)b * g.table_stride + i) : 0;
  }
  // the weights of a block: sc[t][i] = the logit of key x (i < 2) or x + 8 and column 8 t + 2 j + i % 2 becomes its weight.  Returns
  // whether any lane's share has to be rescaled by alpha.
  __device__ __forceinline__ bool weigh(State<D, NT>& st, float (&sc)[NT][4], float (&alpha)[NT][2], int k0) const {
    const int x = lane >> 2;
    bool rescale = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float t0 = k0 + x < lim[nt][h] ? sc[nt][h] * cs : -INFINITY, t1 = k0 + x + 8 < lim[nt][h] ? sc[nt][2 + h] * cs : -INFINITY;
        float mx = fmaxf(t0, t1);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float m_new = fmaxf(st.m[nt][h], mx), m_use = m_new == -INFINITY ? 0.f : m_new;
        alpha[nt][h] = ex2f(st.m[nt][h] - m_use);  // 0 until something is seen
        sc[nt][h] = ex2f(t0 - m_use);
        sc[nt][2 + h] = ex2f(t1 - m_use);
        st.l[nt][h] = st.l[nt][h] * alpha[nt][h] + (sc[nt][h] + sc[nt][2 + h]);
        st.m[nt][h] = m_new;
        rescale = rescale || alpha[nt][h] != 1.f;
      }
    return rescale;
  }

  // bf16 weights of keys x and x + 8, transposed: upper 16 bits and the rest; or, of one part, rounded
  static constexpr int kParts = NT > 2 ? 1 : 2;
  static __device__ __forceinline__ void weights(const float (&w)[NT][4], uint32_t (&pa)[NT][kParts], uint32_t (&pb)[NT][kParts]) {
    auto rest = [](float y) { return y - __uint_as_float(__float_as_uint(y) & 0xffff0000u); };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if constexpr (kParts == 1) {
        pa[nt][0] = transpose8(pack2_bf16(w[nt][0], w[nt][1]));
        pb[nt][0] = transpose8(pack2_bf16(w[nt][2], w[nt][3]));
        continue;
      }
      pa[nt][0] = transpose8(__byte_perm(__float_as_uint(w[nt][0]), __float_as_uint(w[nt][1]), 0x7632));
      pb[nt][0] = transpose8(__byte_perm(__float_as_uint(w[nt][2]), __float_as_uint(w[nt][3]), 0x7632));
      pa[nt][kParts - 1] = transpose8(pack2_bf16(rest(w[nt][0]), rest(w[nt][1])));
      pb[nt][kParts - 1] = transpose8(pack2_bf16(rest(w[nt][2]), rest(w[nt][3])));
    }
  }
  static __device__ __forceinline__ void scale_all(State<D, NT>& st, const float (&alpha)[NT][2]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < D / 16; ++e)
#pragma unroll
        for (int c = 0; c < 4; ++c) st.o[nt][e][c] *= alpha[nt][c & 1];
  }

  // bf16: registers of a block's rows, and what is done with them
  struct RowsBf16 {
    uint32_t ka[D / 8], kb[D / 8], v[4][D / 16];
    __device__ __forceinline__ void load_k(const T* r0, const T* r1) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        load32(r0 + 64 * c, ka + 8 * c);
        load32(r1 + 64 * c, kb + 8 * c);
      }
    }
    static __device__ __forceinline__ int v_row(int i, int j) { return 2 * j + (i & 1) + (i >> 1) * 8; }
    __device__ __forceinline__ void load_v(int i, const T* row) {
      if constexpr (D == 128) load32(row, v[i]);
      else load16(row, v[i]);
    }
    __device__ __forceinline__ void logits(float (&sc)[NT][4], const Fragments<T, D> (&q)[NT], int lane) const {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint2 f = q[nt].step[i][lane];
          mma_16816(sc[nt], ka[2 * i], kb[2 * i], ka[2 * i + 1], kb[2 * i + 1], f.x, f.y);
        }
    }
    __device__ __forceinline__ void add(State<D, NT>& st, const float (&w)[NT][4], const float (&alpha)[NT][2], bool rescale, int) const {
      uint32_t pa[NT][kParts], pb[NT][kParts];
      weights(w, pa, pb);
      if (__any_sync(0xffffffffu, rescale)) scale_all(st, alpha);
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        const uint32_t a0 = __byte_perm(v[0][e], v[1][e], 0x5410), a1 = __byte_perm(v[0][e], v[1][e], 0x7632);
        const uint32_t a2 = __byte_perm(v[2][e], v[3][e], 0x5410), a3 = __byte_perm(v[2][e], v[3][e], 0x7632);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int i = 0; i < kParts; ++i) mma_16816(st.o[nt][e], a0, a1, a2, a3, pa[nt][i], pb[nt][i]);
        }
      }
    }
  };
  // fp32: lane (x, j) has columns 32 c + 8 j .. + 7 of key rows x and x + 8, and columns x D / 8 .. of value rows j, j + 4, j + 8, j + 12
  struct RowsF32 {
    uint32_t ka[D / 4], kb[D / 4], v[4][D / 8];
    __device__ __forceinline__ void load_k(const T* r0, const T* r1) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        load32(r0 + 32 * c, ka + 8 * c);
        load32(r1 + 32 * c, kb + 8 * c);
      }
    }
    static __device__ __forceinline__ int v_row(int i, int j) { return j + 4 * i; }
    __device__ __forceinline__ void load_v(int i, const T* row) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c) load32(row + 8 * c, v[i] + 8 * c);
    }
    __device__ __forceinline__ void logits(float (&sc)[NT][4], const Fragments<T, D> (&q)[NT], int lane) const {
      float low[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) low[nt][i] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        uint32_t hi[4], lo[4];
        cut(__uint_as_float(ka[2 * i]), hi[0], lo[0]);
        cut(__uint_as_float(kb[2 * i]), hi[1], lo[1]);
        cut(__uint_as_float(ka[2 * i + 1]), hi[2], lo[2]);
        cut(__uint_as_float(kb[2 * i + 1]), hi[3], lo[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 f = q[nt].step[i][lane];
          mma_tf32(low[nt], lo, f.x, f.y);
          mma_tf32(sc[nt], hi, f.x, f.y);
          mma_tf32(low[nt], hi, f.z, f.w);
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[nt][i] += low[nt][i];
    }
    __device__ __forceinline__ void add(State<D, NT>& st, const float (&w)[NT][4], const float (&alpha)[NT][2], bool, int lane) const {
      const int x = lane >> 2, j = lane & 3;
      uint32_t w_hi[NT][4], w_lo[NT][4];  // of keys j + 4 i and column x
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int from = (j + 4 * (i & 1)) * 4 + (x >> 1);  // the lane of that key and column
          const float even = __shfl_sync(0xffffffffu, w[nt][2 * (i >> 1)], from), odd = __shfl_sync(0xffffffffu, w[nt][2 * (i >> 1) + 1], from);
          cut_rounded(x & 1 ? odd : even, w_hi[nt][i], w_lo[nt][i]);
        }
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        float sum[NT][4], low[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[nt][c] = low[nt][c] = 0.f;
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // keys j, j + 4; j + 8, j + 12
          uint32_t hi[4], lo[4];
          cut(__uint_as_float(v[2 * half][2 * e]), hi[0], lo[0]);
          cut(__uint_as_float(v[2 * half][2 * e + 1]), hi[1], lo[1]);
          cut(__uint_as_float(v[2 * half + 1][2 * e]), hi[2], lo[2]);
          cut(__uint_as_float(v[2 * half + 1][2 * e + 1]), hi[3], lo[3]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_tf32(low[nt], lo, w_hi[nt][2 * half], w_hi[nt][2 * half + 1]);
            mma_tf32(sum[nt], hi, w_hi[nt][2 * half], w_hi[nt][2 * half + 1]);
            mma_tf32(low[nt], hi, w_lo[nt][2 * half], w_lo[nt][2 * half + 1]);
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) st.o[nt][e][c] = fmaf(st.o[nt][e][c], alpha[nt][c & 1], sum[nt][c] + low[nt][c]);
      }
    }
  };
  using Rows = std::conditional_t<sizeof(T) == 2, RowsBf16, RowsF32>;

  // bf16 rows in shared memory, fragments by ldmatrix: key (or value row) and 16-byte chunk of lane l's address, and what of it is fixed
  static __device__ __forceinline__ uint32_t k_at(int lane) {
    const int key = (lane & 7) + ((lane >> 3) & 1) * 8;
    return key * 128 + (((lane >> 4) ^ (key & 7)) << 4);
  }
  static __device__ __forceinline__ uint32_t v_at(int lane) {
    const int key = (lane & 7) + (lane >> 4) * 8;
    return key * 128 + ((((lane >> 3) & 1) ^ (key & 7)) << 4);
  }
  static __device__ __forceinline__ uint32_t chunk_at(uint32_t at, int step) {  // of 16 columns
    return (at ^ ((step & 3) << 5)) + (step >> 2) * 2048;
  }
  // (given up: copies in flight still write to shared memory; about a second at most)
  static __device__ __forceinline__ void landed(uint32_t bar, uint32_t parity) {
    const uint64_t t0 = tc::global_timer_ns();
    while (!tc::mbar_try_wait(bar, parity) && tc::global_timer_ns() - t0 < 1000000000ull) {
    }
  }
  // The same walk over rows that TMA brings.  `used`: blocks that the warp's ring has had.
  template <int W, typename Ready>
  __device__ __forceinline__ void run_staged(State<D, NT>& st, SharedOf<T, D, NT, W>& sh, const PageMaps& maps, uint32_t& used, int warp,
                                             int first, int stride, int count, Ready ready, const int* early = nullptr) const {
    constexpr int S = kStages<D>;
    const tc::WaitCtx<false, W> wc{tc::smem_u32(sh.words), p.paged.status};
    int pages = lane >= count ? 0 : early ? paged_checked(p.paged, b, *early) : page_of(first + lane * stride), pages_next = 0;
    auto page_at = [&](int t) {  // (asked in order)
      if ((t & 31) == 0 && t > 0) pages = pages_next;
      if ((t & 31) == 16) pages_next = (t & ~31) + 32 + lane < count ? page_of(first + ((t & ~31) + 32 + lane) * stride) : 0;
      return __shfl_sync(0xffffffffu, pages, t & 31);
    };
    auto request = [&](int t, int page) {
      if (lane != 0) return;
      const uint32_t u = (used + t) % S, bar = tc::smem_u32(&sh.full[warp][u]), to = tc::smem_u32(sh.ring[warp][u][0]);
      const int slot = (first + t * stride) * 16 % p.paged.page_size;
      tc::mbar_expect_tx(bar, 2 * kPartBytes<D>);
      auto load = [&](uint32_t dst, const CUtensorMap* map) {
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4, %5}], [%6];" ::"r"(dst),
            "l"(map), "r"(0), "r"(slot), "r"(g), "r"(page), "r"(bar)
            : "memory");
      };
      load(to, &maps.k);
      load(to + kPartBytes<D>, &maps.v);
    };
    if (lane == 0) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // behind what the ring was used for before
#pragma unroll
    for (int a = 0; a < S; ++a)
      if (a < count) request(a, page_at(a));
    ready();
#pragma unroll 1
    for (int t = 0; t < count; ++t) {
      const uint32_t u = (used + t) % S;
      if (!__all_sync(0xffffffffu, tc::wait_bar(wc, tc::smem_u32(&sh.full[warp][u]), ((used + t) / S) & 1, 13, t))) {
        if (lane == 0)
          for (int i = t; i < min(count, t + S); ++i) landed(tc::smem_u32(&sh.full[warp][(used + i) % S]), ((used + i) / S) & 1);
        break;
      }
      const int k0 = (first + t * stride) * 16;
      const uint32_t keys = tc::smem_u32(sh.ring[warp][u][0]), values = keys + kPartBytes<D>;
      float sc[NT][4], alpha[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[nt][i] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t f[4];
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3])
                     : "r"(keys + chunk_at(k_at(lane), i))
                     : "memory");
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint2 q = sh.q[nt].step[i][lane];
          mma_16816(sc[nt], f[0], f[1], f[2], f[3], q.x, q.y);
        }
      }
      if (k0 + 16 > len) {  // rows behind the last one may hold anything: their weights are 0, and 0 times them has to be
        for (int i = lane; i < (16 - (len - k0)) * (D / 8); i += 32) {
          const int row = len - k0 + i / (D / 8), c = i % (D / 8);
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(values + (c >> 3) * 2048 + row * 128 + ((c & 7) << 4)), "r"(0) : "memory");
        }
        __syncwarp();
      }
      const bool rescale = weigh(st, sc, alpha, k0);
      uint32_t pa[NT][kParts], pb[NT][kParts];
      weights(sc, pa, pb);
      if (__any_sync(0xffffffffu, rescale)) scale_all(st, alpha);
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        uint32_t f[4];
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3])
                     : "r"(values + chunk_at(v_at(lane), e))
                     : "memory");
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int i = 0; i < kParts; ++i) mma_16816(st.o[nt][e], f[0], f[1], f[2], f[3], pa[nt][i], pb[nt][i]);
        }
      }
      const int page = t + S < count ? page_at(t + S) : 0;
      __syncwarp();
      if (t + S < count) request(t + S, page);
    }
    used += max(count, 0);
    __syncwarp();  // the ring may be written
  }

  // how many of the blocks first, first + stride, .. lie below `last`, which is at most those of the sequence
  __device__ __forceinline__ int count(int first, int stride, int last) const {
    if (p.paged.visible) last = min(last, (len + 15) / 16);
    return first < last ? (last - first + stride - 1) / stride : 0;
  }
  // blocks first, first + stride, .. (count of them)
  template <int kAhead, int W, typename Ready>
  __device__ __forceinline__ void run(State<D, NT>& st, SharedOf<T, D, NT, W>& sh, const MapsOf<T, NT>& maps, uint32_t& used, int warp, int first,
                                      int stride, int count, Ready ready, const int* early = nullptr) const {
    if constexpr (kStaged<T, NT>) run_staged<W>(st, sh, maps, used, warp, first, stride, count, ready, early);
    else run_registers<kAhead>(st, sh.q, first, stride, count, ready, early);
  }
  template <int kAhead, typename Ready>
  __device__ __forceinline__ void run_registers(State<D, NT>& st, const Fragments<T, D> (&q)[NT], int first, int stride, int count, Ready ready,
                                                const int* early = nullptr) const {
    if (count <= 0) {
      ready();
      return;
    }
    const int x = lane >> 2, j = lane & 3;
    Rows rows[kAhead];
    // pages of the next 32 blocks, a lane each, and of the 32 after them
    int pages = lane >= count ? 0 : early ? paged_checked(p.paged, b, *early) : page_of(first + lane * stride), pages_next = 0;
    auto page_at = [&](int t) {  // (asked in order)
      if ((t & 31) == 0 && t > 0) pages = pages_next;
      if ((t & 31) == 16) pages_next = (t & ~31) + 32 + lane < count ? page_of(first + ((t & ~31) + 32 + lane) * stride) : 0;
      return __shfl_sync(0xffffffffu, pages, t & 31);
    };
    auto request = [&](Rows& to, int t, int page, bool keys) {
      const int k0 = (first + t * stride) * 16, n = len - k0, slot = k0 % p.paged.page_size;
      if (keys) {
        const T* r = kp + (int64_t)page * p.ks.batch + (int64_t)slot * p.ks.token;
        to.load_k(r + min(x, n - 1) * p.ks.token, r + min(x + 8, n - 1) * p.ks.token);
      } else {
        const T* r = vp + (int64_t)page * p.vs.batch + (int64_t)slot * p.vs.token;
#pragma unroll
        for (int i = 0; i < 4; ++i) to.load_v(i, r + min(Rows::v_row(i, j), n - 1) * p.vs.token);
      }
    };
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
      if (a < count) {
        const int page = page_at(a);
        request(rows[a], a, page, true);
        request(rows[a], a, page, false);
      }
    ready();
    auto block = [&](int t, Rows& r) {
      const bool more = t + kAhead < count;
      float sc[NT][4], alpha[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[nt][i] = 0.f;
      r.logits(sc, q, lane);
      int next = 0;
      if (more) {
        next = page_at(t + kAhead);
        request(r, t + kAhead, next, true);
      }
      const bool rescale = weigh(st, sc, alpha, (first + t * stride) * 16);
      r.add(st, sc, alpha, rescale, lane);
      if (more) request(r, t + kAhead, next, false);
    };
#pragma unroll 1
    for (int t = 0; t < count; t += kAhead) {
      block(t, rows[0]);
      if constexpr (kAhead == 2)
        if (t + 1 < count) block(t + 1, rows[1]);
    }
  }
};

template <typename T, int D, int NT, int W>
__device__ __forceinline__ void publish(SharedOf<T, D, NT, W>& sh, const State<D, NT>& st, int warp, int lane) {
  const int x = lane >> 2, j = lane & 3;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float l = st.l[nt][h];
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
      const int col = 8 * nt + 2 * j + h;
      if (x == 0) {
        sh.m[warp][col] = st.m[nt][h];
        sh.l[warp][col] = l;
      }
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        float* o = sh.out(warp, col);
        if constexpr (kStaged<T, NT>) {
          o[16 * e + x] = st.o[nt][e][h];
          o[16 * e + 8 + x] = st.o[nt][e][2 + h];
        } else {
          *reinterpret_cast<float2*>(o + x * (D / 8) + 2 * e) = make_float2(st.o[nt][e][h], st.o[nt][e][2 + h]);
        }
      }
    }
}
// Output columns c .. c + 3 of column `col`: maximum, sum of weights and weighted sums over the warps
__device__ __forceinline__ void add4(float4& acc, float f, const float4& v) {
  acc = make_float4(fmaf(f, v.x, acc.x), fmaf(f, v.y, acc.y), fmaf(f, v.z, acc.z), fmaf(f, v.w, acc.w));
}
template <typename T, int D, int NT, int W>
__device__ __forceinline__ void combine_warps(const SharedOf<T, D, NT, W>& sh, int col, int c, float& n, float& w, float4& acc) {
  n = -INFINITY;
#pragma unroll
  for (int i = 0; i < W; ++i) n = fmaxf(n, sh.m[i][col]);
  const float n_use = n == -INFINITY ? 0.f : n;
  w = 0.f;
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float f = ex2f(sh.m[i][col] - n_use);
    w = fmaf(f, sh.l[i][col], w);
    add4(acc, f, *reinterpret_cast<const float4*>(sh.out(i, col) + c));
  }
}
// The same over the partials of an item: part(k) for k < n_parts, each [columns][D], then the maxima, then the sums
template <int D, int NT, typename Part>
__device__ __forceinline__ void combine_parts(int n_parts, Part part, int col, int i, float& n, float& w, float4& acc) {
  n = -INFINITY;
#pragma unroll 4
  for (int k = 0; k < n_parts; ++k) n = fmaxf(n, __ldcg(part(k) + 8 * NT * D + col));
  const float n_use = n == -INFINITY ? 0.f : n;
  w = 0.f;
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < n_parts; ++k) {
    const float* q = part(k);
    const float f = ex2f(__ldcg(q + 8 * NT * D + col) - n_use);
    w = fmaf(f, __ldcg(q + 8 * NT * (D + 1) + col), w);
    add4(acc, f, __ldcg(reinterpret_cast<const float4*>(q + i)));
  }
}
template <int D, int NT>
__device__ __forceinline__ void store_part(float* part, int col, int c, float n, float w, const float4& acc) {
  *reinterpret_cast<float4*>(part + col * D + c) = acc;
  if (c == 0) {
    part[8 * NT * D + col] = n;
    part[8 * NT * (D + 1) + col] = w;
  }
}

// Output columns c .. c + 3 of (row, head) of column `col`: n and w in log2 units
template <typename T>
__device__ __forceinline__ void write_out(const AttnParams& p, const DecodeArgs& a, int row0, int item, int col, int c, float n, float w,
                                          const float4& acc) {
  const int r = col / a.Gi, row = row0 + r, head = item * a.Gi + col - r * a.Gi;
  T* o = static_cast<T*>(p.o_out) + (int64_t)row * p.os.token + (int64_t)head * p.os.head + c;
  const bool none = w == 0.f;  // nothing is seen; a sum that is not a number shows in the row
  const float4 v = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x / w, acc.y / w, acc.z / w, acc.w / w);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(o) = make_uint2(pack2_bf16(v.x, v.y), pack2_bf16(v.z, v.w));
  else *reinterpret_cast<float4*>(o) = v;
  if (c == 0 && p.lse_out) p.lse_out[(int64_t)row * p.H + head] = none ? -INFINITY : n * 0.6931471805599453f + logf(w);
}

// The query fragments of item `item` of a sequence of `n` rows from row0 on, by warps 0 .. NT - 1.  Where latency is all (clusters) they
// are put into shared memory after the first rows of the cache have been asked for (with the early look-ups 7.7 -> 7.4 us for one token
// over 2500 rows); elsewhere before, because the registers cost the walk more (64 tokens over up to 16384 rows 383 -> 412 us).
template <typename T, int D, int NT>
struct Queries {
  static constexpr int kLoads = D * (int)sizeof(T) / 64;
  uint4 x[kLoads];
  // bf16: columns 64 (c / 2) + 16 j + 8 (c % 2) ..; fp32: 32 (c / 2) + 8 j + 4 (c % 2) ..: two steps each
  __device__ __forceinline__ void load(const AttnParams& p, const DecodeArgs& a, int row0, int n, int item, int warp, int lane) {
    if (warp >= NT) return;
    const int col = 8 * warp + (lane >> 2), j = lane & 3, r = col / a.Gi;
    const T* q = static_cast<const T*>(p.q) + (int64_t)(row0 + r) * p.qs.token + (int64_t)(item * a.Gi + col - r * a.Gi) * p.qs.head;
#pragma unroll
    for (int c = 0; c < kLoads; ++c) {
      const int at = sizeof(T) == 2 ? 64 * (c >> 1) + 16 * j + 8 * (c & 1) : 32 * (c >> 1) + 8 * j + 4 * (c & 1);
      x[c] = r < n ? fresh(reinterpret_cast<const uint4*>(q + at)) : make_uint4(0u, 0u, 0u, 0u);
    }
  }
  template <typename Sh>
  __device__ __forceinline__ void store(Sh& sh, int warp, int lane) const {
    if (warp >= NT) return;
#pragma unroll
    for (int c = 0; c < kLoads; ++c) {
      if constexpr (kStaged<T, NT>) {  // columns as they are: 16 i + 2 j' and + 8 are what lane (x, j') has of step i
        uint32_t* step = reinterpret_cast<uint32_t*>(sh.q[warp].step[4 * (c >> 1) + (lane & 3)]) + (lane >> 2) * 8 + (c & 1);
        step[0] = x[c].x;
        step[2] = x[c].y;
        step[4] = x[c].z;
        step[6] = x[c].w;
      } else if constexpr (sizeof(T) == 2) {
        sh.q[warp].step[2 * c][lane] = make_uint2(x[c].x, x[c].y);
        sh.q[warp].step[2 * c + 1][lane] = make_uint2(x[c].z, x[c].w);
      } else {
        uint4 f0, f1;
        cut_query(__uint_as_float(x[c].x), f0.x, f0.z);
        cut_query(__uint_as_float(x[c].y), f0.y, f0.w);
        cut_query(__uint_as_float(x[c].z), f1.x, f1.z);
        cut_query(__uint_as_float(x[c].w), f1.y, f1.w);
        sh.q[warp].step[2 * c][lane] = f0;
        sh.q[warp].step[2 * c + 1][lane] = f1;
      }
    }
  }
};

// (With given prefixes the walk ends at the longest of its rows': what lies behind it may hold anything.  All lanes of a warp.)
template <typename T, int D, int NT>
__device__ __forceinline__ Walk<T, D, NT> make_walk(const AttnParams& p, const DecodeArgs& a, int b, int row0, int n, int len, int item, int lane) {
  const int x = lane >> 2, j = lane & 3, g = item * a.Gi / p.G;
  Walk<T, D, NT> w{p, static_cast<const T*>(p.k) + (int64_t)g * p.ks.head + (sizeof(T) == 2 ? 16 : 8) * j,
                   static_cast<const T*>(p.v) + (int64_t)g * p.vs.head + x * (D / 8), b, g, len, lane, p.scale * 1.4426950408889634f, {}};
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (8 * nt + 2 * j + h) / a.Gi;
      w.lim[nt][h] = r < n ? paged_seen(p.paged, p.plan.causal, n, len, r, row0 + r) : 0;
    }
  if (p.paged.visible) {
    w.len = 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) w.len = max(w.len, max(w.lim[nt][0], w.lim[nt][1]));
    w.len = __reduce_max_sync(0xffffffffu, w.len);
  }
  return w;
}
template <int D, int NT>
__device__ __forceinline__ void clear(State<D, NT>& st) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < D / 16; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.o[nt][e][i] = 0.f;
    st.m[nt][0] = st.m[nt][1] = -INFINITY;
    st.l[nt][0] = st.l[nt][1] = 0.f;
  }
}

// Behind the tile kernel of the same call (not alone) nothing has to wait for that kernel: it has waited for all that came before, and
// started this one after.  The two share no output, so this one takes the SMs that the last tiles leave idle (16 sequences of 1 to
// 701 rows over 40 to 3001, heads of 64: with the tiles of the longest caches first 113 us -> 99); only what comes next has to wait for both.
__device__ __forceinline__ void begin(const AttnParams& p) {
  grid_go();
  if (p.alone) grid_wait();
}
__device__ __forceinline__ void end(const AttnParams& p) {
  if (!p.alone) grid_wait();
}

// ---- an item per cluster
template <typename T, int D, int NT, int kAhead>
__global__ void __launch_bounds__(kThreads, 1)
    paged_decode_cluster_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ DecodeArgs a,
                               const __grid_constant__ MapsOf<T, NT> maps) {
  extern __shared__ __align__(16) uint8_t smem[];
  SharedOf<T, D, NT, kWarps>& sh = shared_of<T, D, NT, kWarps>(smem);
  __shared__ __align__(16) float s_o[8 * NT * D + 4 * kClusterMost];
  __shared__ float s_n[kClusterMost][8 * NT], s_w[kClusterMost][8 * NT];  // from each CTA of the cluster
  const int rank = blockIdx.x, n_cta = a.n_cta, item = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  set_up<T, D, NT, kWarps>(sh, warp, lane);
  uint32_t used = 0;
  begin(p);
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // everyone has started: its shared memory may be written
  // everything that may be needed is asked for at once
  const int first = rank * kWarps + warp, stride = n_cta * kWarps;
  const int early = Walk<T, D, NT>::early_page(p.paged, b, first + lane * stride);
  const int len = paged_len(p.paged, b);
  const int2 rows = paged_rows(p.paged, b);
  const bool mine = rows.y >= p.paged.least && rows.y <= p.paged.most;
  if (rows.y > p.paged.most && p.alone && tid == 0) paged_report(p.paged.status, kBadRows, b, rows.y);
  if (!mine) {  // (uniform for the cluster)
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    end(p);
    return;
  }
  const int blocks = (len + 15) / 16, cols = rows.y * a.Gi;
  Queries<T, D, NT> queries;
  queries.load(p, a, rows.x, rows.y, item, warp, lane);
  const Walk<T, D, NT> walk = make_walk<T, D, NT>(p, a, b, rows.x, rows.y, len, item, lane);
  State<D, NT> st;
  clear(st);
  walk.template run<kAhead, kWarps>(st, sh, maps, used, warp, first, stride, walk.count(first, stride, blocks), [&]() {
    queries.store(sh, warp, lane);
    __syncthreads();
  }, &early);
  publish<T, D, NT, kWarps>(sh, st, warp, lane);
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  // CTA r finishes outputs r * per_cta ..; every CTA sends it its share of them
  const int outputs = cols * D, per_cta = ((outputs + n_cta - 1) / n_cta + 3) & ~3;
  auto there = [&](const float* local, int to) {
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(to));
    return addr;
  };
  for (int i = 4 * tid; i < outputs; i += 4 * kThreads) {
    float n, w;
    float4 acc;
    combine_warps<T, D, NT, kWarps>(sh, i / D, i % D, n, w, acc);
    const int to = i / per_cta;
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(there(&s_o[rank * per_cta + i - to * per_cta], to)), "f"(acc.x),
                 "f"(acc.y), "f"(acc.z), "f"(acc.w)
                 : "memory");
    for (int c = i % D; c < min(i % D + 4, n_cta); ++c) {
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there(&s_n[rank][i / D], c)), "f"(n) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there(&s_w[rank][i / D], c)), "f"(w) : "memory");
    }
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  const int here = gave_up<T, NT>(p) ? 0 : min(per_cta, outputs - rank * per_cta);
  for (int o = 4 * tid; o < here; o += 4 * kThreads) {
    const int col = (rank * per_cta + o) / D, c = (rank * per_cta + o) % D;
    float n = -INFINITY, w = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r = 0; r < n_cta; ++r) n = fmaxf(n, s_n[r][col]);
    const float n_use = n == -INFINITY ? 0.f : n;
#pragma unroll 4
    for (int r = 0; r < n_cta; ++r) {
      const float f = ex2f(s_n[r][col] - n_use);
      w = fmaf(f, s_w[r][col], w);
      add4(acc, f, *reinterpret_cast<const float4*>(&s_o[r * per_cta + o]));
    }
    write_out<T>(p, a, rows.x, item, col, c, n, w, acc);
  }
  end(p);
}

// ---- an item per CTA
template <typename T, int D, int NT, int kAhead>
__global__ void __launch_bounds__(kRangeThreads, kHalfCtas<T, D, NT>)
    paged_decode_items_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ DecodeArgs a,
                               const __grid_constant__ MapsOf<T, NT> maps) {
  extern __shared__ __align__(16) uint8_t smem[];
  SharedOf<T, D, NT, kRangeWarps>& sh = shared_of<T, D, NT, kRangeWarps>(smem);
  const int item = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  set_up<T, D, NT, kRangeWarps>(sh, warp, lane);
  uint32_t used = 0;
  begin(p);
  const int early = Walk<T, D, NT>::early_page(p.paged, b, warp + lane * kRangeWarps);
  const int len = paged_len(p.paged, b);
  const int2 rows = paged_rows(p.paged, b);
  if (rows.y > p.paged.most && p.alone && tid == 0) paged_report(p.paged.status, kBadRows, b, rows.y);
  if (rows.y >= p.paged.least && rows.y <= p.paged.most) {
    Queries<T, D, NT> queries;
    queries.load(p, a, rows.x, rows.y, item, warp, lane);
    const Walk<T, D, NT> walk = make_walk<T, D, NT>(p, a, b, rows.x, rows.y, len, item, lane);
    State<D, NT> st;
    clear(st);
    walk.template run<kAhead, kRangeWarps>(st, sh, maps, used, warp, warp, kRangeWarps, walk.count(warp, kRangeWarps, (len + 15) / 16), [&]() {
      queries.store(sh, warp, lane);
      __syncthreads();
    }, &early);
    publish<T, D, NT, kRangeWarps>(sh, st, warp, lane);
    __syncthreads();
    const int outputs = gave_up<T, NT>(p) ? 0 : rows.y * a.Gi * D;
    for (int i = 4 * tid; i < outputs; i += 4 * kRangeThreads) {
      float n, w;
      float4 acc;
      combine_warps<T, D, NT, kRangeWarps>(sh, i / D, i % D, n, w, acc);
      write_out<T>(p, a, rows.x, item, i / D, i % D, n, w, acc);
    }
  }
  end(p);
}

// Zeros for the rows over an empty cache, by one warp of CTA `cta`
template <typename T, int D>
__device__ __forceinline__ void clear_empty(const AttnParams& p, int cta, int n_cta, int lane) {
  for (int b = cta + n_cta * lane; b < p.paged.batch; b += 32 * n_cta) {
    const int2 rows = paged_rows(p.paged, b);
    if (rows.y < p.paged.least || rows.y > p.paged.most || paged_len(p.paged, b) > 0) continue;
    for (int64_t e = 0; e < (int64_t)rows.y * p.H; ++e) {
      const int64_t row = rows.x + e / p.H, head = e % p.H;
      uint4* o = reinterpret_cast<uint4*>(static_cast<T*>(p.o_out) + row * p.os.token + head * p.os.head);
      for (int c = 0; c < D * (int)sizeof(T) / 16; ++c) o[c] = make_uint4(0u, 0u, 0u, 0u);
      if (p.lse_out) p.lse_out[row * p.H + head] = -INFINITY;
    }
  }
}

// ---- a share of one item per CTA
// Every item that has blocks gets a CTA, and what is left of them goes to the items by their length.
constexpr int kSets = 2;  // of 32 sequences: as many as there can be items (shares)
struct Share {
  int b, item, row0, rows, len;  // b -1: none
  int part, parts;
};
__device__ __forceinline__ Share share_of(const AttnParams& p, const DecodeArgs& a, int cta, int lane) {
  const PagedDev& g = p.paged;
  int row0[kSets], rows[kSets], len[kSets], total = 0, filled = 0;
#pragma unroll
  for (int s = 0; s < kSets; ++s) {
    row0[s] = rows[s] = len[s] = 0;
    const int b = 32 * s + lane;
    if (b < g.batch) {
      const int2 r = paged_rows(g, b);
      row0[s] = r.x;
      rows[s] = r.y;
      len[s] = paged_len(g, b);
      if (r.y > g.most && p.alone && cta == 0) paged_report(g.status, kBadRows, b, r.y);
      if (r.y < g.least || r.y > g.most) rows[s] = len[s] = 0;
    }
    total += (len[s] + 15) / 16;
    filled += len[s] > 0;
  }
  total = __reduce_add_sync(0xffffffffu, total);
  filled = __reduce_add_sync(0xffffffffu, filled) * a.items;
  const int spare = max(0, a.n_cta - filled);
  Share r = {-1, 0, 0, 0, 0, 0, 1};
  int before = 0;
#pragma unroll
  for (int s = 0; s < kSets; ++s) {
    const int nb = (len[s] + 15) / 16;
    const int n = nb ? min((nb + kWarps - 1) / kWarps, 1 + (int)((int64_t)nb * spare / ((int64_t)total * a.items))) : 0;
    int incl = n * a.items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += t;
    }
    const int off = cta - (before + incl - n * a.items);
    const uint32_t mine = __ballot_sync(0xffffffffu, off >= 0 && off < n * a.items);
    if (mine) {
      const int who = __ffs(mine) - 1, at = __shfl_sync(0xffffffffu, off, who);
      r.b = 32 * s + who;
      r.row0 = __shfl_sync(0xffffffffu, row0[s], who);
      r.rows = __shfl_sync(0xffffffffu, rows[s], who);
      r.len = __shfl_sync(0xffffffffu, len[s], who);
      r.parts = __shfl_sync(0xffffffffu, n, who);
      r.part = at / a.items;  // the KV heads of the same keys side by side
      r.item = at - r.part * a.items;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return r;
}

template <typename T, int D, int NT, int kAhead>
__global__ void __launch_bounds__(kThreads, 1)
    paged_decode_shares_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ DecodeArgs a,
                               const __grid_constant__ MapsOf<T, NT> maps) {
  extern __shared__ __align__(16) uint8_t smem[];
  SharedOf<T, D, NT, kWarps>& sh = shared_of<T, D, NT, kWarps>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
  set_up<T, D, NT, kWarps>(sh, warp, lane);
  uint32_t used = 0;
  begin(p);
  if (warp == kWarps - 1) clear_empty<T, D>(p, cta, a.n_cta, lane);
  const Share r = share_of(p, a, cta, lane);
  if (tid == 0) a.joins[cta] = make_int4(r.b < 0 || r.part > 0 || r.parts == 1 ? 0 : r.parts, r.row0, r.rows, r.item);
  if (r.b < 0) {
    end(p);
    return;
  }
  Queries<T, D, NT> queries;
  queries.load(p, a, r.row0, r.rows, r.item, warp, lane);
  queries.store(sh, warp, lane);
  const Walk<T, D, NT> walk = make_walk<T, D, NT>(p, a, r.b, r.row0, r.rows, r.len, r.item, lane);
  State<D, NT> st;
  clear(st);
  const int64_t blocks = (r.len + 15) / 16;
  const int last = (int)(blocks * (r.part + 1) / r.parts), first = (int)(blocks * r.part / r.parts) + warp;
  walk.template run<kAhead, kWarps>(st, sh, maps, used, warp, first, kWarps, walk.count(first, kWarps, last), []() { __syncthreads(); });
  publish<T, D, NT, kWarps>(sh, st, warp, lane);
  __syncthreads();
  float* part = a.partials + (int64_t)cta * (8 * NT * (D + 2));
  const bool keep = !gave_up<T, NT>(p);
  for (int i = 4 * tid; i < r.rows * a.Gi * D; i += 4 * kThreads) {
    const int col = i / D, c = i % D;
    float n, w;
    float4 acc;
    combine_warps<T, D, NT, kWarps>(sh, col, c, n, w, acc);
    if (r.parts > 1) store_part<D, NT>(part, col, c, n, w, acc);
    else if (keep) write_out<T>(p, a, r.row0, r.item, col, c, n, w, acc);
  }
  end(p);
}

// CTA (i, y) adds up a share of the columns of the item of which CTA i had the first part.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(kJoinThreads) paged_decode_join_shares_kernel(const __grid_constant__ AttnParams p,
                                                                const __grid_constant__ DecodeArgs a) {
  grid_go();
  grid_wait();
  const int4 j = __ldcg(a.joins + blockIdx.x);  // parts (0: none), first row, rows, item
  const int i = 4 * (blockIdx.y * kJoinThreads + threadIdx.x);
  if (i >= j.z * a.Gi * D || j.x == 0 || gave_up<T, NT>(p)) return;
  float n, w;
  float4 acc;
  auto part = [&](int k) { return a.partials + (int64_t)(blockIdx.x + k * a.items) * (8 * NT * (D + 2)); };
  combine_parts<D, NT>(j.x, part, i / D, i, n, w, acc);
  write_out<T>(p, a, j.y, j.w, i / D, i % D, n, w, acc);
}

// ---- ranges of equal length
// Two CTAs of four warps an SM (four with heads of 64), so that one streams while the other starts an item or leaves one.  us, one CTA of
// eight warps -> these, 32 / 8 heads of 128, single tokens: 24 sequences of 250 to 2500 rows 46 -> 37, 64 of them 93 -> 80, 64 of 1000 to
// 16384 376 -> 368; drafts of 2 to 6 rows, 64 of 250 to 2500 100 -> 94; 64 / 8 heads, 24 of 2 to 4 rows 60 -> 50.  (A thread had one output
// at a time when the shares are added up, here and in the joining kernels; with four side by side the last was 94.)
template <typename T, int D, int NT, int kAhead>
__global__ void __launch_bounds__(kRangeThreads, kHalfCtas<T, D, NT>)
    paged_decode_ranges_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ DecodeArgs a,
                               const __grid_constant__ MapsOf<T, NT> maps) {
  extern __shared__ __align__(16) uint8_t smem[];
  SharedOf<T, D, NT, kRangeWarps>& sh = shared_of<T, D, NT, kRangeWarps>(smem);
  int* s_group = reinterpret_cast<int*>(&sh);  // blocks (of one item) of the groups of 32 sequences before; rows and outputs come here later
  static_assert((kMaxGroups + 1) * 4 <= kRangeWarps * 8 * NT * (D + 4) * 4, "");
  __shared__ RangeStart s_start;
  const PagedDev& g = p.paged;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
  set_up<T, D, NT, kRangeWarps>(sh, warp, lane);
  uint32_t used = 0;
  begin(p);
  if (warp == kRangeWarps - 1) clear_empty<T, D>(p, cta, a.n_cta, lane);
  const int groups = (g.batch + 31) / 32;
  for (int i = warp; i < groups; i += kRangeWarps) {
    const int b = i * 32 + lane, n = b < g.batch ? blocks_of(g, b) : 0;
    const int sum = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) s_group[i] = sum;
    if (cta == 0 && b < g.batch) {
      const int rows = paged_rows(g, b).y;
      if (rows > g.most && p.alone) paged_report(g.status, kBadRows, b, rows);  // nobody else takes it
    }
  }
  __syncthreads();
  if (warp == 0) {
    int before = 0;
    for (int i0 = 0; i0 < groups; i0 += 32) {
      const int i = i0 + lane, n = i < groups ? s_group[i] : 0;
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
      }
      if (i < groups) s_group[i] = before + incl - n;
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) s_group[groups] = before;
    const int64_t total = (int64_t)before * a.items;
    const int n_ranges = ranges_of(total, a.n_cta);
    RangeStart r = {-1, 0, 0, 0, total};
    if (cta < n_ranges && total > 0) {
      const int64_t u = total * cta / n_ranges;
      const int at = (int)(u / a.items);  // some block of the sequence (sequences have items times their blocks)
      int lo = 0, hi = groups - 1;
      __syncwarp();
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_group[mid] <= at) lo = mid;
        else hi = mid - 1;
      }
      const int b = lo * 32 + lane, n = b < g.batch ? blocks_of(g, b) : 0;
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, (int64_t)(s_group[lo] + incl) * a.items > u);
      const int who = __ffs(past) - 1;  // the group holds block `at`
      const int nb = __shfl_sync(0xffffffffu, n, who), start = s_group[lo] + __shfl_sync(0xffffffffu, incl, who) - nb;
      const int64_t off = u - (int64_t)start * a.items;
      r.b = lo * 32 + who;
      r.item = (int)(off / nb);
      r.before = (int)(off - (int64_t)r.item * nb);
      r.blocks = nb;
    }
    if (lane == 0) {
      s_start = r;
      a.starts[cta] = r;
    }
  }
  __syncthreads();
  const RangeStart r = s_start;
  if (r.b < 0) {
    end(p);
    return;
  }
  const int n_ranges = ranges_of(r.total, a.n_cta);
  int64_t left = r.total * (cta + 1) / n_ranges - r.total * cta / n_ranges;
  int b = r.b, item = r.item, s0 = r.before, blocks = r.blocks;
  while (left > 0) {
    const int s1 = (int)min((int64_t)blocks, s0 + left);
    const int2 rows = paged_rows(g, b);
    const int len = paged_len(g, b), cols = rows.y * a.Gi;
    Queries<T, D, NT> queries;
    queries.load(p, a, rows.x, rows.y, item, warp, lane);
    queries.store(sh, warp, lane);
    const Walk<T, D, NT> walk = make_walk<T, D, NT>(p, a, b, rows.x, rows.y, len, item, lane);
    State<D, NT> st;
    clear(st);
    const int first = s0 + warp;
    walk.template run<kAhead, kRangeWarps>(st, sh, maps, used, warp, first, kRangeWarps, walk.count(first, kRangeWarps, s1), []() { __syncthreads(); });
    publish<T, D, NT, kRangeWarps>(sh, st, warp, lane);
    __syncthreads();
    const bool whole = s0 == 0 && s1 == blocks;
    float* part = a.partials + (int64_t)(cta * 2 + (s0 > 0 ? 0 : 1)) * (8 * NT * (D + 2));
    const bool keep = !gave_up<T, NT>(p);
    for (int i = 4 * tid; i < cols * D; i += 4 * kRangeThreads) {
      const int col = i / D, c = i % D;
      float n, w;
      float4 acc;
      combine_warps<T, D, NT, kRangeWarps>(sh, col, c, n, w, acc);
      if (!whole) store_part<D, NT>(part, col, c, n, w, acc);
      else if (keep) write_out<T>(p, a, rows.x, item, col, c, n, w, acc);
    }
    left -= s1 - s0;
    s0 = 0;
    if (left == 0) break;
    if (++item == a.items) {  // the next sequence that has blocks; there may be many idle places before it
      item = 0;
      for (++b; b < g.batch; b += 32) {
        const int n = b + lane < g.batch ? blocks_of(g, b + lane) : 0;
        const uint32_t some = __ballot_sync(0xffffffffu, n > 0);
        if (some) {
          const int who = __ffs(some) - 1;
          blocks = __shfl_sync(0xffffffffu, n, who);
          b += who;
          break;
        }
      }
      if (b >= g.batch) break;
    }
    __syncthreads();  // the shares and queries have been read
    if constexpr (kStaged<T, NT>)
      if (sh.words[1]) break;  // (of this CTA's waits, so the same for all of it)
  }
  end(p);
}

// CTA (i, y) adds up a share of the columns of the item that is cut for the first time where range i + 1 starts.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(kJoinThreads) paged_decode_join_kernel(const __grid_constant__ AttnParams p,
                                                                const __grid_constant__ DecodeArgs a) {
  grid_go();
  grid_wait();
  const int at = blockIdx.x + 1;
  const RangeStart r = a.starts[at];
  if (r.b < 0 || r.before == 0 || gave_up<T, NT>(p)) return;
  const int n_ranges = ranges_of(r.total, a.n_cta);
  auto start = [&](int i) { return r.total * i / n_ranges; };
  const int64_t u0 = start(at) - r.before, u1 = u0 + r.blocks;  // the item
  if (start(at - 1) > u0) return;  // cut before
  int last = at;  // the last range that has a part of it
  while (last + 1 < n_ranges && start(last + 1) < u1) ++last;
  const int2 rows = paged_rows(p.paged, r.b);
  const int cols = rows.y * a.Gi;
  const int i = 4 * (blockIdx.y * kJoinThreads + threadIdx.x);
  if (i >= cols * D) return;
  float n, w;
  float4 acc;
  auto part = [&](int k) { return a.partials + (int64_t)((at - 1 + k) * 2 + (k == 0 ? 1 : 0)) * (8 * NT * (D + 2)); };
  combine_parts<D, NT>(last - at + 2, part, i / D, i, n, w, acc);
  write_out<T>(p, a, rows.x, r.item, i / D, i % D, n, w, acc);
}

template <typename F>
cudaError_t with_shape(cascade_dtype_t dtype, int d, int columns, F f) {
  auto with_columns = [&](auto t, auto dim) {
    if constexpr (sizeof(t) == 2) {
      if (columns > 24) return f(t, dim, std::integral_constant<int, 4>());
      if (columns > 16) return f(t, dim, std::integral_constant<int, 3>());
    }
    return columns <= 8 ? f(t, dim, std::integral_constant<int, 1>()) : f(t, dim, std::integral_constant<int, 2>());
  };
  auto with_dim = [&](auto t) {
    return d == 128 ? with_columns(t, std::integral_constant<int, 128>()) : with_columns(t, std::integral_constant<int, 64>());
  };
  return dtype == CASCADE_BF16 ? with_dim(__nv_bfloat16()) : with_dim(float());
}

// CTAs that are resident at a time
int ranges_cta(cascade_dtype_t dtype, int d, int columns) { return d == 128 || dtype == CASCADE_F32 || columns > kMostInRegisters ? 296 : 592; }
int columns_most(cascade_dtype_t dtype) { return dtype == CASCADE_BF16 ? kMostColumns : 16; }
// Clusters only where all of them are resident at once with a CTA per SM (of 16, 10, 8, 4, 2 CTAs 7, 11, 15, 33, 74 are), and, with more
// than one sequence, only over short caches: it is not known here how long they are, and one long sequence would be left to its clusters.
// us, caches new to L2, 32 / 8 heads of 128 (clusters | shares, 6 us of them the events'): 4 sequences of 2500 rows 20 | 24, of 8000
// 35 | 39, 6 of 1000 to 8000 52 | 40, of 30000 163 | 132, 16 of 300 17 | 20.
int cluster_size(const AttnParams& p, int64_t items) {  // 0: shares or ranges
  const int64_t blocks = ((int64_t)p.paged.max_pages * p.paged.page_size + 15) / 16;
  int n = 0;
  for (const auto& fit : {std::pair<int, int>{148, 1}, {74, 2}, {33, 4}, {15, 8}, {11, 10}, {7, 16}})
    if (items <= fit.first) n = fit.second;
  if (n == 0) return 0;
  n = (int)std::min<int64_t>(n, (blocks + kWarps - 1) / kWarps);
  return p.paged.batch == 1 || blocks <= 10 * kWarps * n ? n : 0;
}
// And a CTA of four warps an item, one after another, where no sequence can be long: what is resident then evens out over the chip, and
// nothing has to be joined.  us, the same heads, single tokens (these | ranges): 24 sequences of 40 to 160 rows 6.4 | 13, 40 of 200 to 1000
// 29 | 32, 100 of them 54 | 64, 40 of 900 to 1000 44 | 39, 40 of 400 to 2000 54 | 47; drafts of 2 to 4 rows, 64 of 40 to 160 14 | 27, of 200
// to 1000 41 | 52; fp32, 100 of 100 to 500 63 | 74, of 900 to 1000 148 | 148, 40 of them 93 | 69.
bool one_each(const AttnParams& p, cascade_dtype_t dtype, int64_t items) {
  return items > 148 && p.paged.batch <= 65535 && (int64_t)p.paged.max_pages * p.paged.page_size <= (dtype == CASCADE_F32 ? 512 : 1024);
}
// Shares where items are few: whole CTAs are a coarse measure of many items' lengths, and ranges cut few items into many parts.  us, single
// tokens, the same heads (shares | ranges): 4 sequences of 1000 to 8000 rows 23 | 30, of 4000 to 30000 69 | 71, 6: 31 | 34 and 94 | 84, 8:
// 44 | 39 and 139 | 103; 16 / 4 heads of 64, 9 of 1000 to 8000 18 | 28, 16 30 | 28; drafts of 2 to 6 rows, 6: 32 | 41 and 86 | 92, 8: 44 | 46
// and 130 | 113, 9: 51 | 50 and 158 | 132.
bool shares(int64_t items, int columns) { return items <= (columns > 16 ? 64 : 40); }

bool encode_blocks(CUtensorMap* map, const void* base, const Strides& st, const AttnParams& p) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const PagedDev& g = p.paged;
  const cuuint64_t dims[5] = {64, (cuuint64_t)g.page_size, (cuuint64_t)p.d / 64, (cuuint64_t)p.Hkv, (cuuint64_t)g.n_pages};
  auto stride = [&](int64_t elems, int64_t extent) { return (cuuint64_t)(extent > 1 ? elems * 2 : p.d * 2); };
  const cuuint64_t strides[4] = {stride(st.token, g.page_size), 128, stride(st.head, p.Hkv), stride(st.batch, g.n_pages)};
  const cuuint32_t box[5] = {64, 16, (cuuint32_t)p.d / 64, 1, 1}, one[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

// Heads of an item of `rows` rows: the largest divisor of the group that fits the columns.
int paged_decode_heads(const AttnParams& p, cascade_dtype_t dtype, int rows) {
  for (int n = std::min(16, p.G); n > 1; --n)
    if (p.G % n == 0 && rows * n <= columns_most(dtype)) return n;
  return 1;
}
int paged_decode_rows(const AttnParams& p, cascade_dtype_t dtype) { return columns_most(dtype) / paged_decode_heads(p, dtype, 1); }

// More columns than that in two items or more, where the items are few: the rows of the cache are read by each (from L2 by all but one),
// and the products are as slow as they are.  us, 64 / 8 heads of 128 over 3000 to 9000 rows (split | tiles): 2 sequences of 8 rows
// 35 | 46, 4 of 6 55 | 51, 4 of 8 65 | 48; 8 / 1 heads, 16 of 2 to 6 rows 28 | 44.
bool paged_decode_splits(const AttnParams& p, cascade_dtype_t dtype, int rows) {
  return dtype == CASCADE_BF16 && rows <= 8 && (int64_t)p.paged.batch * (p.H / paged_decode_heads(p, dtype, rows)) <= 37;
}

size_t paged_decode_ws_bytes(const AttnParams& p, cascade_dtype_t dtype, int rows) {
  const int heads = paged_decode_heads(p, dtype, rows);
  const int64_t items = (int64_t)p.paged.batch * (p.H / heads);
  const int columns = (rows * heads + 7) / 8 * 8, n = ranges_cta(dtype, p.d, columns);
  if (one_each(p, dtype, items) || cluster_size(p, items) > 0) return 0;
  if (shares(items, columns)) return (size_t)n * (columns * (p.d + 2) * 4 + sizeof(int4));
  return (size_t)n * (2 * columns * (p.d + 2) * 4 + sizeof(RangeStart));
}

cudaError_t launch_paged_decode(const AttnParams& p, cascade_dtype_t dtype, int rows, void* workspace, cudaStream_t stream) {
  DecodeArgs a = {};
  a.Gi = paged_decode_heads(p, dtype, rows);
  a.items = p.H / a.Gi;
  const int64_t items = (int64_t)p.paged.batch * a.items;
  const int columns = rows * a.Gi, cluster = cluster_size(p, items);
  TimedLaunch timed(stream);
  return with_shape(dtype, p.d, columns, [&](auto t, auto d, auto nt) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, NT = decltype(nt)::value;
    constexpr int smem = kSmemBytes<T, D, NT, kWarps>;
    MapsOf<T, NT> maps;
    if constexpr (kStaged<T, NT>) {
      if (!encode_blocks(&maps.k, p.k, p.ks, p) || !encode_blocks(&maps.v, p.v, p.vs, p)) {
        set_error("cascade_attn_paged: could not build the TMA descriptors of the pages");
        return cudaErrorInvalidValue;
      }
    }
    // Blocks ahead: as many as an SM has registers for.  bf16, heads of 128: two, and eight warps an SM (one ahead and twice the warps keep as
    // many loads in flight, but the walk spills: 64 sequences of up to 16384 rows 466 us, 385 this way).
    constexpr int kAhead = sizeof(T) == 4 && D == 128 ? 1 : 2;
    constexpr int kAheadHalf = sizeof(T) == 2 ? (D == 128 && NT == 1 ? 2 : 1) : (D == 64 && NT == 1 ? 2 : 1);
    constexpr int smem_half = kSmemBytes<T, D, NT, kRangeWarps>;
    const int join_y = (rows * a.Gi * D / 4 + kJoinThreads - 1) / kJoinThreads;
    if (one_each(p, dtype, items)) {
      auto kernel = paged_decode_items_kernel<T, D, NT, kAheadHalf>;
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_half);
      if (e != cudaSuccess) return e;
      return launch_dependent(kernel, dim3(a.items, p.paged.batch), kRangeThreads, smem_half, 1, true, stream, p, a, maps);
    }
    if (cluster > 0) {
      auto kernel = paged_decode_cluster_kernel<T, D, NT, kAhead>;
      cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e == cudaSuccess && cluster > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      a.n_cta = cluster;
      return launch_dependent(kernel, dim3(cluster, a.items, p.paged.batch), kThreads, smem, cluster, true, stream, p, a, maps);
    }
    if (shares(items, columns)) {
      a.n_cta = 148;
      a.joins = static_cast<int4*>(workspace);
      a.partials = reinterpret_cast<float*>(a.joins + a.n_cta);
      auto kernel = paged_decode_shares_kernel<T, D, NT, kAhead>;
      cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e != cudaSuccess) return e;
      e = launch_dependent(kernel, dim3(a.n_cta), kThreads, smem, 1, true, stream, p, a, maps);
      if (e != cudaSuccess) return e;
      return launch_dependent(paged_decode_join_shares_kernel<T, D, NT>, dim3(a.n_cta, join_y), kJoinThreads, 0, 1, true, stream,
                              p, a);
    }
    a.n_cta = ranges_cta(dtype, p.d, columns);
    a.starts = static_cast<RangeStart*>(workspace);
    a.partials = reinterpret_cast<float*>(a.starts + a.n_cta);
    auto kernel = paged_decode_ranges_kernel<T, D, NT, kAheadHalf>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_half);
    if (e != cudaSuccess) return e;
    e = launch_dependent(kernel, dim3(a.n_cta), kRangeThreads, smem_half, 1, true, stream, p, a, maps);
    if (e != cudaSuccess) return e;
    return launch_dependent(paged_decode_join_kernel<T, D, NT>, dim3(a.n_cta - 1, join_y), kJoinThreads, 0, 1, true, stream, p, a);
  });
}

}  // namespace cascade
