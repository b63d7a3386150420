// Rotary positions of rows that stand anywhere (the Pre-Pass algorithm's q <- rotary_pos_emb(q, p^{R_i}) with a row of the table
// per row of the tensor), and the append of a chunk's rows to a paged cache, which turns them on the way ("Caching" in the appendix
// on cost optimizations: a node stores the rows of its shard).
//   y = R(angle) x on the pairs (i, i + r/2), or (2i, 2i + 1) if interleaved, of the first r columns; the others pass through.
// Computed in fp32, rounded once to the I/O type.
//
// Bound by HBM (a row is read and written once) or, for single tokens, by the launch.  A thread owns two 16-byte pieces of a head
// vector that hold whole pairs (half layout: one of each half; otherwise neighbours) and does the same piece of up to kHeads heads,
// so that the table, which is as long as two pieces in bf16 terms, is read once for them.  A warp is of one row: what it has to
// find out about the row (its sequence, page and position) is found out by the warp together.
#include "paged.cuh"

namespace cascade {

namespace {

template <typename T>
struct RowVec;
template <>
struct RowVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct RowVec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

constexpr int kHeads = 4;  // heads of a thread

// The sequence whose rows hold row r: the last one that starts at or before it (32 at a time, by the whole warp); -1 if r is behind
// the last sequence or before the first.
__device__ __forceinline__ int sequence_of(const PagedDev& g, int r, int lane) {
  int lo = 0, n = g.batch;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const bool starts = lane * step < n && fresh(g.row_start + at) <= r;
    const uint32_t m = __ballot_sync(0xffffffffu, starts);
    if (m == 0) return -1;
    const int last = 31 - __clz(m);
    const int end = min(lo + n, lo + (last + 1) * step);
    lo += last * step;
    n = end - lo;
  }
  return lo;
}

template <typename T, bool kAppend>
__global__ void __launch_bounds__(256) rope_rows_kernel(const __grid_constant__ RopeRowsParams p, int warps_per_row, int head_groups) {
  constexpr int N = RowVec<T>::N;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int row = (int)(w / warps_per_row);
  if (row >= p.n_rows) return;
  const int units = p.d / (2 * N);
  const int item = (int)(w - (int64_t)row * warps_per_row) * 32 + lane;
  grid_go();
  grid_wait();
  const int u = item % units, hg = item / units;
  // this thread's pieces: columns c0 .. and c1 .., and its pairs
  const int half = p.rot / 2;
  const bool turned = p.rope && u * 2 * N < p.rot;
  const int c0 = turned && !p.interleaved ? u * N : u * 2 * N, c1 = turned && !p.interleaved ? half + u * N : c0 + N;
  // The rows are asked for before it is known where they go: what has to be looked up for that (sequence, length, page, position) is
  // a chain of loads as long as their own (3153 rows of 48 heads 15.6 us behind it, so 13.9).
  const T* src[kHeads];
  uint4 a[kHeads], b[kHeads];
  const int heads = p.H + (kAppend ? 2 * p.Hkv : 0);
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = hg + i * head_groups;  // q heads, then those of k, then those of v
    src[i] = nullptr;
    if (hg >= head_groups || h >= heads) continue;
    if (!kAppend || h < p.H) src[i] = static_cast<const T*>(p.q) + (int64_t)row * p.qs.token + (int64_t)h * p.qs.head;
    else if (h < p.H + p.Hkv) src[i] = static_cast<const T*>(p.k) + (int64_t)row * p.ks.token + (int64_t)(h - p.H) * p.ks.head;
    else src[i] = static_cast<const T*>(p.v) + (int64_t)row * p.vs.token + (int64_t)(h - p.H - p.Hkv) * p.vs.head;
    a[i] = *reinterpret_cast<const uint4*>(src[i] + c0);
    b[i] = *reinterpret_cast<const uint4*>(src[i] + c1);
  }
  int64_t k_to = 0, v_to = 0;
  int position;
  if constexpr (kAppend) {
    const int s = sequence_of(p.paged, row, lane);
    if (s < 0) return;
    const int2 rows = paged_rows(p.paged, s);
    if (row < rows.x || row >= rows.x + rows.y) return;  // behind the last sequence
    const int len = fresh(p.paged.kv_len + s), y = len - rows.y + row - rows.x;  // its row of the cache
    const bool bad = len < 0 || len > (int64_t)p.paged.max_pages * p.paged.page_size;
    if (bad || y < 0) {  // (a length cut to what the table holds would put the row over an older one)
      if (lane == 0) paged_report(p.paged.status, kBadLength, s, bad ? len : y);
      return;
    }
    const int index = y / p.paged.page_size, slot = y - index * p.paged.page_size;
    const int id = fresh(p.paged.table + (int64_t)s * p.paged.table_stride + index);
    if ((unsigned)id >= (unsigned)p.paged.n_pages) {  // nothing is written
      if (lane == 0) paged_report(p.paged.status, kBadPage, s, id);
      return;
    }
    k_to = id * p.kos.batch + slot * p.kos.token;
    v_to = id * p.vos.batch + slot * p.vos.token;
    position = p.positions ? fresh(p.positions + row) : y;
  } else {
    position = fresh(p.positions + row);
    if (position < 0) return;  // a padded row stays as it is
  }
  if (p.rope && (unsigned)position >= (unsigned)p.n_positions) {
    if (lane == 0) paged_report(p.paged.status, kBadPosition, row, position);
    return;
  }
  float4 cs[N / 2];  // (cos, sin) of N pairs
  if (turned) {
    const float4* t = reinterpret_cast<const float4*>(p.rope + (int64_t)position * half + u * N);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) cs[e] = fresh(t + e);
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (!src[i]) continue;
    const int h = hg + i * head_groups;
    T* dst;
    if (!kAppend || h < p.H) dst = static_cast<T*>(p.q_out) + (int64_t)row * p.qos.token + (int64_t)h * p.qos.head;
    else if (h < p.H + p.Hkv) dst = static_cast<T*>(p.k_out) + k_to + (int64_t)(h - p.H) * p.kos.head;
    else dst = static_cast<T*>(p.v_out) + v_to + (int64_t)(h - p.H - p.Hkv) * p.vos.head;
    if (turned && (!kAppend || h < p.H + p.Hkv)) {
      float x[N], y[N], u0[N], u1[N];
      RowVec<T>::unpack(a[i], x);
      RowVec<T>::unpack(b[i], y);
      if (!p.interleaved) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float c = e & 1 ? cs[e / 2].z : cs[e / 2].x, s = e & 1 ? cs[e / 2].w : cs[e / 2].y;
          u0[e] = x[e] * c - y[e] * s;
          u1[e] = y[e] * c + x[e] * s;
        }
      } else {  // pairs (0, 1), (2, 3), .. of the 2 N columns x | y
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float c = e & 1 ? cs[e / 2].z : cs[e / 2].x, s = e & 1 ? cs[e / 2].w : cs[e / 2].y;
          const float re = e < N / 2 ? x[2 * e % N] : y[2 * e % N], im = e < N / 2 ? x[(2 * e + 1) % N] : y[(2 * e + 1) % N];
          const float re2 = re * c - im * s, im2 = im * c + re * s;
          if (e < N / 2) {
            u0[2 * e % N] = re2;
            u0[(2 * e + 1) % N] = im2;
          } else {
            u1[2 * e % N] = re2;
            u1[(2 * e + 1) % N] = im2;
          }
        }
      }
      a[i] = RowVec<T>::pack(u0);
      b[i] = RowVec<T>::pack(u1);
    }
    *reinterpret_cast<uint4*>(dst + c0) = a[i];
    *reinterpret_cast<uint4*>(dst + c1) = b[i];
  }
}

}  // namespace

cudaError_t launch_rope_rows(const RopeRowsParams& p, cascade_dtype_t dtype, cudaStream_t stream) {
  const bool append = p.k != nullptr;
  const int heads = p.H + (append ? 2 * p.Hkv : 0), units = p.d / (dtype == CASCADE_BF16 ? 16 : 8);
  const int head_groups = (heads + kHeads - 1) / kHeads, warps_per_row = (head_groups * units + 31) / 32;
  const int64_t warps = (int64_t)p.n_rows * warps_per_row;
  auto kernel = dtype == CASCADE_BF16 ? (append ? rope_rows_kernel<__nv_bfloat16, true> : rope_rows_kernel<__nv_bfloat16, false>)
                                      : (append ? rope_rows_kernel<float, true> : rope_rows_kernel<float, false>);
  return launch_dependent(kernel, dim3((unsigned)((warps + 7) / 8)), 256, 0, 1, true, stream, p, warps_per_row, head_groups);
}

namespace {

// Positional table with scaled angles.  theta_i = base^(-2i / r); in 64 bits throughout, rounded once.
//   1 linear   theta / factor (position interpolation, Chen et al. 2023)
//   2 base     base factor^(r / (r - 2)) in the place of base
//   3 bands    by the turns original theta / 2 pi of the original context: `high` and more kept, `low` and fewer divided by factor,
//              mixed linearly in the turns in between
//   4 ramp     by the dimension: those up to the one that turns `high` times in the original context kept, those from the one that
//              turns `low` times on divided by factor, mixed linearly in i in between (YaRN, Peng et al. 2023)
// cos and sin are multiplied by `attention`.
// The angles of one position come with the launch (their powers were a third of the time on the device).  A thread has one dimension
// and kRun positions: the first and the step go through sincos, the others are products, (cos, sin)(t + 1) = (cos, sin)(t) (cos,
// sin)(1) as complex numbers, off by a few 2^-53 each.  (32768 positions of 64 pairs: 61 us with a power and a sincos for each, now 6.2.)
constexpr int kRun = 16, kMaxPairs = 128;
struct RopeAngles {
  double theta[kMaxPairs];
  double attention;
  int32_t first, count, half;  // pairs first .. first + count - 1 of half
};
__global__ void __launch_bounds__(256) rope_table_scaled_kernel(int32_t n_positions, const __grid_constant__ RopeAngles a, float2* __restrict__ table) {
  const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t0 = idx / a.count * kRun;
  if (t0 >= n_positions) return;
  const int i = (int)(idx % a.count);
  double sn, cn, sn1, cn1;
  sincos((double)t0 * a.theta[i], &sn, &cn);
  sincos(a.theta[i], &sn1, &cn1);
  sn *= a.attention;
  cn *= a.attention;
  const int n = (int)min((int64_t)kRun, n_positions - t0);
  float2* to = table + t0 * a.half + a.first + i;
  for (int j = 0; j < n; ++j) {
    to[(int64_t)j * a.half] = make_float2((float)cn, (float)sn);
    const double c = cn * cn1 - sn * sn1;
    sn = sn * cn1 + cn * sn1;
    cn = c;
  }
}

}  // namespace

cudaError_t launch_rope_table_scaled(int32_t n_positions, int32_t rot, const RopeScaling& s, float2* table, cudaStream_t stream) {
  const double two_pi = 6.283185307179586476925, base = s.kind == 2 ? s.base * std::pow(s.factor, (double)rot / (rot - 2)) : s.base;
  auto turning = [&](double turns) { return rot * std::log(s.original / (two_pi * turns)) / (2 * std::log(base)); };
  const double first = s.kind == 4 ? std::max(0.0, std::floor(turning(s.high))) : 0;
  const double last = s.kind == 4 ? std::min(rot - 1.0, std::ceil(turning(s.low))) : 0;
  RopeAngles a;
  a.attention = s.attention;
  a.half = rot / 2;
  for (a.first = 0; a.first < a.half; a.first += kMaxPairs) {
    a.count = std::min(kMaxPairs, a.half - a.first);
    for (int j = 0; j < a.count; ++j) {
      const int i = a.first + j;
      double theta = std::pow(base, -(double)i / a.half), keep = 1;
      if (s.kind == 1) keep = 0;
      if (s.kind == 3) keep = std::min(1.0, std::max(0.0, (s.original * theta / two_pi - s.low) / (s.high - s.low)));
      if (s.kind == 4) keep = 1 - std::min(1.0, std::max(0.0, (i - first) / std::max(last - first, 0.001)));
      a.theta[j] = theta * keep + theta / s.factor * (1 - keep);
    }
    const int64_t n = ((int64_t)n_positions + kRun - 1) / kRun * a.count;
    rope_table_scaled_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(n_positions, a, table);
    count_launch();
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace cascade
