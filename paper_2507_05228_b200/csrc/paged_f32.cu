// fp32 attention over a paged cache (cascade_attn_paged, sequences of more rows than paged_decode.cu takes): warp-level tensor-core
// products m16n8k8 on operands taken apart into two tf32 parts (tf32.cuh).
// (On the packed fp32 ALUs 8 sequences of 17 to 128 rows over 60 to 512 keys, 12 heads of 64, took 44 us, so 29.)
//
// The tensor core adds with truncation, so its sums are kept short: the logits over head_dim, the outputs over 32 keys, the small
// products by themselves; what is carried from tile to tile is added in fp32.  (With the small products in the same sums the error of
// the output was 7.8e-7, so it is 3.1e-7; the same in fp32 on the ALUs 4.1e-7.)
//
// A warp owns 16 rows (or 32, MT = 2: one cut of a key or value for two products each), (token, head) pairs with the heads of a KV
// head side by side.  The contraction index of a product may be any permutation as long as both operands use the same one, and so
// may the output columns; with (g, t) = (lane / 4, lane % 4):
//   q k^T  a lane's four columns 16 c + 4 t .. + 3 of a row are the indices t and t + 4 of two products: one 16-byte load
//   p v    the logits of keys 2 t and 2 t + 1, which a lane holds, are the indices t and t + 4 of the weights, so nothing is moved;
//          values are columns 4 g + 32 j .. + 3 of rows 2 t and 2 t + 1: one 16-byte load for four products
// The pitches (D + 16 for keys, D + 4 for values) make all of these loads free of bank conflicts.
//
// RW warps share a tile of 32 keys, KW groups of them take the tiles in turn and add up in shared memory at the end: 64 rows a CTA
// where sequences have them, 16 otherwise (16 in the example above: 40 us).  Where CTAs are few, key_parts of them share the keys and
// leave partials, which paged_combine_kernel adds up.
// What bounds it: half the time of the CTA with the longest keys is its products (12288 of 8 cycles, four at a time), a fifth the
// chain of look-ups and first loads.  Long chunks take 13.2 cycles a product where the units take 8.3 (512 rows over 4000, 32 / 8 heads of
// 128, 729 us; 327 at 96 TFLOP/s, a third of the rate of tf32).
#include <algorithm>

#include "paged.cuh"
#include "tf32.cuh"

namespace cascade {

namespace {

__device__ __forceinline__ void stage16(float* dst, const float* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr int kTile = 32, NK = kTile / 8;  // keys of a tile, products side by side

template <int D, int MT, int RW, int KW>
struct F32Cfg {
  static constexpr int kWarps = RW * KW, kRows = 16 * MT * RW;
  static constexpr int kQPitch = D + 16, kKPitch = D + 16, kVPitch = D + 4;
  static constexpr int kQ = kRows * kQPitch, kStage = kTile * (kKPitch + kVPitch), kGroup = 2 * kStage;
  static constexpr int kStats = KW * kRows * 2;
  static constexpr size_t kBytes = sizeof(float) * (kQ + KW * kGroup + kStats);
  static_assert(kBytes <= 232448, "exceeds the 227 KiB a CTA may use");
  static_assert(kGroup >= kRows * D, "a group's output is staged in its tiles");
};

template <int D, int MT, int RW, int KW>
__global__ void __launch_bounds__(32 * RW * KW)
paged_f32_kernel(const __grid_constant__ AttnParams p, int lg, int tile_major) {
  using C = F32Cfg<D, MT, RW, KW>;
  extern __shared__ __align__(16) float smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = warp / RW, gtid = tid % (RW * 32);
  const int wrow = warp % RW * 16 * MT, g = lane >> 2, t = lane & 3;
  grid_go();
  grid_wait();
  // tiles on the slowest axis, the longest first, unless there are too many for it
  const int2 tile = paged_tile(p.paged, tile_major ? blockIdx.z : blockIdx.x, C::kRows >> lg, lane);
  if (tile.x < 0) return;
  const int b = tile.x, key_part = tile_major ? blockIdx.y : blockIdx.z, h0 = (tile_major ? blockIdx.x : blockIdx.y) << lg, kv_head = h0 / p.G;
  const int2 rows = paged_rows(p.paged, b);
  const int len = paged_len(p.paged, b), tok0 = tile.y * (C::kRows >> lg), n_rows = min(C::kRows >> lg, rows.y - tok0) << lg;
  auto token_of = [&](int r) { return tok0 + (r >> lg); };
  auto seen_by = [&](int r) { return paged_seen(p.paged, p.plan.causal, rows.y, len, token_of(r), rows.x + token_of(r)); };
  float* sQ = smem;
  float* tiles = smem + C::kQ + group * C::kGroup;
  const float* q = static_cast<const float*>(p.q);
  for (int i = tid; i < C::kRows * (D / 4); i += 32 * C::kWarps) {
    const int r = i / (D / 4), c = i % (D / 4) * 4;
    const float* src = q + (r < n_rows ? (int64_t)(rows.x + token_of(r)) * p.qs.token + (int64_t)(h0 + (r & ((1 << lg) - 1))) * p.qs.head : 0);
    stage16(sQ + r * C::kQPitch + c, src + c, r < n_rows);
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
  int most = seen_by(n_rows - 1), least = seen_by(0);
  if (p.paged.visible) {  // in any order
    for (int r = 0; r < n_rows; r += 1 << lg) {
      const int n = seen_by(r);
      most = max(most, n);
      least = min(least, n);
    }
  }
  int sees[2 * MT];  // of rows wrow + g + 8 i
  float m[2 * MT], l[2 * MT];  // raw logits; l: this thread's share
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    sees[i] = seen_by(min(wrow + g + 8 * i, n_rows - 1));
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
  // this CTA's part of the tiles, and this group's
  const int all_tiles = (most + kTile - 1) / kTile;
  const int t_first = (int)((int64_t)all_tiles * key_part / p.key_parts), t_end = (int)((int64_t)all_tiles * (key_part + 1) / p.key_parts);
  const float* kb = static_cast<const float*>(p.k) + (int64_t)kv_head * p.ks.head;
  const float* vb = static_cast<const float*>(p.v) + (int64_t)kv_head * p.vs.head;
  constexpr int kPerRow = D / 4, kRowsAtOnce = RW * 32 / kPerRow, kLoads = kTile / kRowsAtOnce;
  static_assert(RW * 32 % kPerRow == 0 && kTile % kRowsAtOnce == 0, "whole rows at a time");
  const int lr = gtid / kPerRow, lc = gtid % kPerRow * 4;
  // pages and rows of the 16-key parts of a tile
  struct Place {
    int page[kTile / 16], slot[kTile / 16];
  };
  auto place_of = [&](int tl) {
    Place w;
#pragma unroll
    for (int i = 0; i < kTile / 16; ++i) {
      const int key = tl * kTile + 16 * i, index = key / p.paged.page_size;
      w.page[i] = tl < t_end && key < most ? paged_page(p.paged, b, index) : 0;
      w.slot[i] = key - index * p.paged.page_size;
    }
    return w;
  };
  auto stage = [&](int tl, const Place& w, int buf) {
    float* sK = tiles + buf * C::kStage;
    float* sV = sK + kTile * C::kKPitch;
    if (tl < t_end) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = i * kRowsAtOnce + lr, half = r >> 4;
        const bool there = tl * kTile + r < most;  // (rows behind the last one that is seen may hold anything)
        const int64_t row = there ? w.slot[half] + (r & 15) : 0, page = w.page[half];
        stage16(sK + r * C::kKPitch + lc, kb + page * p.ks.batch + row * p.ks.token + lc, there);
        stage16(sV + r * C::kVPitch + lc, vb + page * p.vs.batch + row * p.vs.token + lc, there);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto group_sync = [&]() {
    if constexpr (RW == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(RW * 32) : "memory");
  };
  Place next = place_of(t_first + group);
  stage(t_first + group, next, 0);
  next = place_of(t_first + group + KW);
  asm volatile("cp.async.wait_group 1;" ::: "memory");  // the queries
  __syncthreads();
  const float cs = p.scale * 1.4426950408889634f;
  auto load_q = [&](int mt, int c, uint32_t (&hi)[2][4], uint32_t (&lo)[2][4]) {  // columns 16 c ..: two products
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(sQ + (wrow + 16 * mt + g + 8 * i) * C::kQPitch + 16 * c + 4 * t);
      cut_query(x.x, hi[0][i], lo[0][i]);
      cut_query(x.y, hi[0][2 + i], lo[0][2 + i]);
      cut_query(x.z, hi[1][i], lo[1][i]);
      cut_query(x.w, hi[1][2 + i], lo[1][2 + i]);
    }
  };
  float o[MT][D / 8][4];  // o[mt][4 j + q][2 i + h]: row wrow + 16 mt + g + 8 i, column 8 t + 4 h + q + 32 j
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[mt][n][i] = 0.f;
  int buf = 0;
  for (int tl = t_first + group; tl < t_end; tl += KW, buf ^= 1) {
    stage(tl + KW, next, buf ^ 1);
    next = place_of(tl + 2 * KW);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    group_sync();
    if (RW > 1 && wrow >= n_rows) {  // (the rows of a tile that is not full)
      group_sync();
      continue;
    }
    const float* sK = tiles + buf * C::kStage;
    const float* sV = sK + kTile * C::kKPitch;
    float s[MT][NK][4];  // s[mt][n][2 i + h]: key 8 n + 2 t + h
    {
      float low[MT][NK][4];  // the products of parts by themselves
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[mt][n][i] = low[mt][n][i] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        uint32_t hi[MT][2][4], lo[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) load_q(mt, c, hi[mt], lo[mt]);
#pragma unroll
        for (int n = 0; n < NK; ++n) {
          const float4 x = *reinterpret_cast<const float4*>(sK + (8 * n + g) * C::kKPitch + 16 * c + 4 * t);
          uint32_t kh[4], kl[4];
          cut(x.x, kh[0], kl[0]);
          cut(x.y, kh[1], kl[1]);
          cut(x.z, kh[2], kl[2]);
          cut(x.w, kh[3], kl[3]);
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              mma_tf32(low[mt][n], lo[mt][i], kh[2 * i], kh[2 * i + 1]);
              mma_tf32(s[mt][n], hi[mt][i], kh[2 * i], kh[2 * i + 1]);
              mma_tf32(low[mt][n], hi[mt][i], kl[2 * i], kl[2 * i + 1]);
            }
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[mt][n][i] += low[mt][n][i];
    }
    if (tl * kTile + kTile > least) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (tl * kTile + 8 * n + 2 * t + (i & 1) >= sees[2 * mt + (i >> 1)]) s[mt][n][i] = -INFINITY;
    }
    float alpha[2 * MT];
    uint32_t p_hi[MT][NK][4], p_lo[MT][NK][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float(&x)[NK][4] = s[mt];
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < NK; ++n) mx = fmaxf(mx, fmaxf(x[n][2 * i], x[n][2 * i + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        float& m_i = m[2 * mt + i];
        const float m_new = fmaxf(m_i, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
        alpha[2 * mt + i] = ex2((m_i - m_use) * cs);
        m_i = m_new;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            x[n][2 * i + h] = ex2((x[n][2 * i + h] - m_use) * cs);
            sum += x[n][2 * i + h];
          }
        l[2 * mt + i] = l[2 * mt + i] * alpha[2 * mt + i] + sum;
      }
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        cut_rounded(s[mt][n][0], p_hi[mt][n][0], p_lo[mt][n][0]);
        cut_rounded(s[mt][n][2], p_hi[mt][n][1], p_lo[mt][n][1]);
        cut_rounded(s[mt][n][1], p_hi[mt][n][2], p_lo[mt][n][2]);
        cut_rounded(s[mt][n][3], p_hi[mt][n][3], p_lo[mt][n][3]);
      }
    }
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      float sum[MT][4][4], low[MT][4][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[mt][c][i] = low[mt][c][i] = 0.f;
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        const float4 v0 = *reinterpret_cast<const float4*>(sV + (8 * n + 2 * t) * C::kVPitch + 4 * g + 32 * j);
        const float4 v1 = *reinterpret_cast<const float4*>(sV + (8 * n + 2 * t + 1) * C::kVPitch + 4 * g + 32 * j);
        const float x0[4] = {v0.x, v0.y, v0.z, v0.w}, x1[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t h0b, l0b, h1b, l1b;
          cut(x0[c], h0b, l0b);
          cut(x1[c], h1b, l1b);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            mma_tf32(low[mt][c], p_lo[mt][n], h0b, h1b);
            mma_tf32(sum[mt][c], p_hi[mt][n], h0b, h1b);
            mma_tf32(low[mt][c], p_hi[mt][n], l0b, l1b);
          }
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            o[mt][4 * j + c][i] = fmaf(o[mt][4 * j + c][i], alpha[2 * mt + (i >> 1)], sum[mt][c][i] + low[mt][c][i]);
    }
    group_sync();  // the tile has been read
  }
  // finished rows, or this part's share of them
  auto put = [&](int row, int col, float4 x, float m_raw, float w) {
    if (row >= n_rows) return;
    const bool none = w == 0.f;  // nothing is seen; a sum that is not a number shows in the row
    const float inv = none ? 0.f : 1.f / w;
    x.x *= inv;
    x.y *= inv;
    x.z *= inv;
    x.w *= inv;
    const int64_t tok = rows.x + token_of(row), head = h0 + (row & ((1 << lg) - 1));
    if (p.key_parts > 1) {
      const int64_t stat = ((int64_t)key_part * p.paged.n_rows + tok) * p.H + head;
      *reinterpret_cast<float4*>(static_cast<float*>(p.o_part) + stat * D + col) = x;
      if (col == 0) {
        p.m_part[stat] = none ? -INFINITY : m_raw * p.scale;
        p.l_part[stat] = w;
      }
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(p.o_out) + tok * p.os.token + head * p.os.head + col) = x;
      if (col == 0 && p.lse_out) p.lse_out[tok * p.H + head] = none ? -INFINITY : m_raw * p.scale + logf(w);
    }
  };
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  {
    float* stats = smem + C::kQ + KW * C::kGroup;  // [group][row][m, l]
    group_sync();
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
      const int row = wrow + g + 8 * i;
      if (t == 0) {
        stats[(group * C::kRows + row) * 2] = m[i];
        stats[(group * C::kRows + row) * 2 + 1] = l[i];
      }
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = 2 * (i & 1) + h;
          *reinterpret_cast<float4*>(tiles + row * D + 8 * t + 4 * h + 32 * j) =
              make_float4(o[i >> 1][4 * j][at], o[i >> 1][4 * j + 1][at], o[i >> 1][4 * j + 2][at], o[i >> 1][4 * j + 3][at]);
        }
    }
    __syncthreads();
    for (int e = tid; e < n_rows * (D / 4); e += 32 * C::kWarps) {
      const int row = e / (D / 4), col = e % (D / 4) * 4;
      float n = -INFINITY;
#pragma unroll
      for (int k = 0; k < KW; ++k) n = fmaxf(n, stats[(k * C::kRows + row) * 2]);
      const float n_use = n == -INFINITY ? 0.f : n;
      float w = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float f = ex2((stats[(k * C::kRows + row) * 2] - n_use) * cs);
        const float4 u = *reinterpret_cast<const float4*>(smem + C::kQ + k * C::kGroup + row * D + col);
        w = fmaf(f, stats[(k * C::kRows + row) * 2 + 1], w);
        x.x = fmaf(f, u.x, x.x);
        x.y = fmaf(f, u.y, x.y);
        x.z = fmaf(f, u.z, x.z);
        x.w = fmaf(f, u.w, x.w);
      }
      put(row, col, x, n, w);
    }
  }
}

// o = sum over the parts of exp(m - n) l u / w for the rows that belong to a sequence; thread = four columns of a (row, head).
template <int D>
__global__ void __launch_bounds__(256) paged_combine_kernel(const __grid_constant__ AttnParams p) {
  grid_go();
  grid_wait();
  const int64_t item = (int64_t)blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4);
  const int col = threadIdx.x % (D / 4) * 4;
  const int64_t all = (int64_t)p.paged.n_rows * p.H, row = item / p.H;
  if (item >= all || row < fresh(p.paged.row_start) || row >= fresh(p.paged.row_start + p.paged.batch)) return;
  float n = -INFINITY, w = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0; k < p.key_parts; ++k) n = fmaxf(n, fresh(p.m_part + k * all + item));
  for (int k = 0; k < p.key_parts; ++k) {
    const float l = fresh(p.l_part + k * all + item);
    const float f = l == 0.f ? 0.f : l * expf(fresh(p.m_part + k * all + item) - n);
    const float4 u = fresh(reinterpret_cast<const float4*>(static_cast<const float*>(p.o_part) + (k * all + item) * D + col));
    w += f;
    o.x = fmaf(f, u.x, o.x);
    o.y = fmaf(f, u.y, o.y);
    o.z = fmaf(f, u.z, o.z);
    o.w = fmaf(f, u.w, o.w);
  }
  const float inv = w == 0.f ? 0.f : 1.f / w;
  const int head = (int)(item - row * p.H);
  *reinterpret_cast<float4*>(static_cast<float*>(p.o_out) + row * p.os.token + head * p.os.head + col) =
      make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (col == 0 && p.lse_out) p.lse_out[item] = w == 0.f ? -INFINITY : n + logf(w);
}

constexpr int64_t kSms = 148;

int heads_log2(int G) {  // heads of a tile: as many of the G as a power of two divides, at most 8
  int lg = 0;
  while (lg < 3 && G % (2 << lg) == 0) ++lg;
  return lg;
}
// Tiles of `height` (token, head) rows: every sequence that has rows can end in one that is not full.
int64_t tiles_bound(const AttnParams& p, int height) {
  const int per = height >> heads_log2(p.G);
  return p.paged.batch == 1 ? (p.paged.n_rows + per - 1) / per : p.paged.n_rows / per + std::min(p.paged.batch, p.paged.n_rows);
}
// Sixty-four rows a CTA where a sequence has half of them on average
bool wide(const AttnParams& p) { return (p.paged.n_rows / p.paged.batch) << heads_log2(p.G) >= 32; }

template <int D, int MT, int RW, int KW>
cudaError_t launch_one(const AttnParams& p, cudaStream_t stream) {
  using C = F32Cfg<D, MT, RW, KW>;
  auto kernel = paged_f32_kernel<D, MT, RW, KW>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kBytes);
  if (e != cudaSuccess) return e;
  const int lg = heads_log2(p.G);
  const unsigned heads = (unsigned)(p.H >> lg), parts = (unsigned)p.key_parts, tiles = (unsigned)tiles_bound(p, C::kRows);
  const int tile_major = tiles <= 65535;
  return launch_dependent(kernel, tile_major ? dim3(heads, parts, tiles) : dim3(tiles, heads, parts), 32 * C::kWarps, C::kBytes, 1, true, stream, p, lg,
                          tile_major);
}
template <int D>
cudaError_t launch_d(const AttnParams& p, cudaStream_t stream) {
  cudaError_t e = wide(p) ? (D == 64 ? launch_one<64, 2, 2, 4>(p, stream) : launch_one<128, 1, 4, 2>(p, stream))
                          : launch_one<D, 1, 1, D == 64 ? 4 : 3>(p, stream);
  if (e != cudaSuccess || p.key_parts == 1) return e;
  const int64_t items = (int64_t)p.paged.n_rows * p.H, per = 256 / (D / 4);
  return launch_dependent(paged_combine_kernel<D>, dim3((unsigned)((items + per - 1) / per)), 256, 0, 1, true, stream, p);
}

}  // namespace

// Keys of a tile are shared by as many CTAs, at least 256 keys of what the table can hold each, as make the rounds of a CTA per SM and the keys
// of a CTA, with 256 for its start and its end, come out shortest.  (us, as many CTAs as fit in one round | so: 299 rows over 3725, 16 / 8
// heads of 128, 80 tiles: 358 | 247; 512 over 4000, 12 heads of 64, 96 tiles: 183 | 130.  The 256, us, two CTAs per SM and 512 keys | one and
// 256: 3 drafts of 2 to 6 rows over 646 to 672, 32 / 8 heads of 128, 37 | 25; 28 over 4000, 12 heads of 128, 64 | 44.)
int paged_f32_parts(const AttnParams& p) {
  const int64_t ctas = tiles_bound(p, wide(p) ? 64 : 16) * (p.H >> heads_log2(p.G)), keys = (int64_t)p.paged.max_pages * p.paged.page_size;
  auto time = [&](int64_t parts) { return (ctas * parts + kSms - 1) / kSms * (keys / parts + 256); };
  int64_t best = 1;
  for (int64_t parts = 2; parts <= std::min<int64_t>(keys / 256, 64); ++parts)
    if (time(parts) < time(best)) best = parts;
  return time(best) * 10 < time(1) * 9 ? (int)best : 1;  // (joining the parts has to pay)
}
size_t paged_f32_ws_bytes(const AttnParams& p) {
  const int64_t parts = paged_f32_parts(p);
  return parts == 1 ? 0 : (size_t)(parts * p.paged.n_rows * p.H * (p.d + 2) * 4);
}
cudaError_t launch_paged_f32(AttnParams p, void* workspace, cudaStream_t stream) {
  p.key_parts = paged_f32_parts(p);
  if (p.key_parts > 1) {
    const int64_t items = (int64_t)p.key_parts * p.paged.n_rows * p.H;
    p.o_part = workspace;
    p.m_part = static_cast<float*>(workspace) + items * p.d;
    p.l_part = p.m_part + items;
  }
  TimedLaunch timed(stream);
  return p.d == 128 ? launch_d<128>(p, stream) : launch_d<64>(p, stream);
}

}  // namespace cascade
