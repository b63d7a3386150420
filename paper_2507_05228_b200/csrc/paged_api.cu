// C ABI entry points of the paged calls: argument checks and kernel dispatch.
#include <string.h>

#include <atomic>

#include "paged.cuh"

namespace cascade {

namespace {

__device__ int32_t g_paged_status[kPagedStatusWords];

cascade_status_t fail(cascade_status_t code, const char* fn, const char* what) {
  set_error("%s: %s", fn, what);
  return code;
}
cascade_status_t launched(cudaError_t e, const char* fn) {
  if (e == cudaSuccess) return CASCADE_OK;
  set_error("%s: launch: %s", fn, cudaGetErrorString(e));
  return CASCADE_ERR_CUDA;
}
size_t elt_size(cascade_dtype_t t) { return t == CASCADE_BF16 ? 2 : 4; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
bool rows_aligned(const cascade_strides_t& s, size_t es) { return s.token * (int64_t)es % 16 == 0 && s.head * (int64_t)es % 16 == 0; }
bool pages_aligned(const cascade_strides_t& s, size_t es) { return rows_aligned(s, es) && s.batch * (int64_t)es % 16 == 0; }
Strides in(const cascade_strides_t& s) { return {s.batch, s.token, s.head}; }

cascade_status_t check_types(const char* fn, cascade_dtype_t dtype, int32_t d) {
  if (dtype != CASCADE_F32 && dtype != CASCADE_BF16) return fail(CASCADE_ERR_UNSUPPORTED, fn, "unknown dtype");
  if (d != 64 && d != 128) {
    set_error("%s: head_dim %d unsupported (64 or 128)", fn, d);
    return CASCADE_ERR_UNSUPPORTED;
  }
  return CASCADE_OK;
}
cascade_status_t check_rope(const char* fn, const float* table, int32_t n_positions, int32_t rot, int32_t d) {
  if (rot < 16 || rot % 16 != 0 || rot > d) {
    set_error("%s: rot_dim %d unsupported (a multiple of 16, at most head_dim)", fn, rot);
    return CASCADE_ERR_UNSUPPORTED;
  }
  if (n_positions < 1 || !aligned16(table)) return fail(CASCADE_ERR_INVALID_ARG, fn, "the table must have rows and be 16-byte aligned");
  return CASCADE_OK;
}
// (H 0: heads are not looked at)
cascade_status_t check_sizes(const char* fn, int32_t H, int32_t Hkv, int32_t page_size, int32_t max_pages) {
  if (H % Hkv != 0) {
    set_error("%s: n_heads %d is not a multiple of n_kv_heads %d", fn, H, Hkv);
    return CASCADE_ERR_UNSUPPORTED;
  }
  if (page_size < 16 || page_size % 16 != 0) {
    set_error("%s: page_size %d unsupported (a multiple of 16)", fn, page_size);
    return CASCADE_ERR_UNSUPPORTED;
  }
  if ((int64_t)max_pages * page_size > 1 << 30) return fail(CASCADE_ERR_UNSUPPORTED, fn, "a sequence of more than 2^30 rows");
  return CASCADE_OK;
}
cascade_status_t check_pages(const char* fn, int32_t batch, int32_t n_rows, int32_t H, int32_t Hkv, int32_t n_pages, int32_t page_size,
                             const int32_t* table, int64_t table_stride, int32_t max_pages, const int32_t* row_start, const int32_t* kv_len) {
  if (!table || !row_start || !kv_len) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  if (batch < 1 || n_rows < 1 || H < 1 || Hkv < 1 || n_pages < 1 || max_pages < 1 || table_stride < max_pages)
    return fail(CASCADE_ERR_INVALID_ARG, fn, "batch, rows, heads and pages must be positive, the table's rows at least max_pages apart");
  const cascade_status_t s = check_sizes(fn, 0, Hkv, page_size, max_pages);
  if (s != CASCADE_OK) return s;
  if (batch > 65535 || H > 65535 || Hkv > 65535) return fail(CASCADE_ERR_UNSUPPORTED, fn, "batch and heads may not exceed 65535");
  if (!aligned4(table) || !aligned4(row_start) || !aligned4(kv_len)) return fail(CASCADE_ERR_INVALID_ARG, fn, "int32 arrays must be 4-byte aligned");
  return CASCADE_OK;
}
// Blocks of 16 rows of all sequences are counted in 32 bits (a page may stand in the table any number of times, so memory is no bound).
cascade_status_t check_blocks(const char* fn, int32_t batch, int32_t page_size, int32_t max_pages) {
  if ((int64_t)batch * ((int64_t)max_pages * page_size / 16) > INT_MAX) return fail(CASCADE_ERR_UNSUPPORTED, fn, "tables with room for 2^35 rows or more");
  return CASCADE_OK;
}
PagedDev pages_dev(int32_t batch, int32_t n_rows, int32_t n_pages, int32_t page_size, const int32_t* table, int64_t table_stride,
                   int32_t max_pages, const int32_t* row_start, const int32_t* kv_len, const int32_t* visible) {
  PagedDev g;
  memset(&g, 0, sizeof(g));
  g.table = table;
  g.table_stride = table_stride;
  g.row_start = row_start;
  g.kv_len = kv_len;
  g.visible = visible;
  g.status = paged_status_words();
  g.batch = batch;
  g.n_rows = n_rows;
  g.n_pages = n_pages;
  g.max_pages = max_pages;
  g.page_size = page_size;
  g.least = 1;
  g.most = INT32_MAX;
  return g;
}
cascade_status_t no_status(const char* fn) { return fail(CASCADE_ERR_CUDA, fn, "the device's status words cannot be reached"); }

}  // namespace

int32_t* paged_status_words() {
  static std::atomic<int32_t*> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  int32_t* p = known[dev].load(std::memory_order_relaxed);
  if (!p) {
    void* at = nullptr;
    if (cudaGetSymbolAddress(&at, g_paged_status) != cudaSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    p = static_cast<int32_t*>(at);
    known[dev].store(p, std::memory_order_relaxed);
  }
  return p;
}

}  // namespace cascade

using namespace cascade;

extern "C" {

cascade_status_t cascade_paged_status(int32_t* out_code) {
  const char* fn = "cascade_paged_status";
  if (!out_code) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  int32_t* dev = paged_status_words();
  if (!dev) return no_status(fn);
  int32_t words[kPagedStatusWords];
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(words, dev, sizeof(words), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (words[0] != 0 || words[kBadIndexWord] != 0)) e = cudaMemset(dev, 0, sizeof(words));
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    set_error("%s: %s", fn, cudaGetErrorString(e));
    return CASCADE_ERR_CUDA;
  }
  *out_code = words[0] ? words[0] : words[kBadIndexWord];
  if (words[0] != 0) {
    set_error("%s: device status word = %d: a bounded wait inside a kernel gave up (block %d,%d,%d tile %d)", fn, words[0], words[1],
              words[2], words[3], words[4]);
    return CASCADE_ERR_TIMEOUT;
  }
  if (words[kBadIndexWord] != 0) {
    const char* what = "?";
    switch (words[kBadIndexWord]) {
      case kBadRowStart: what = "row_start falls or leaves the rows, sequence"; break;
      case kBadLength: what = "kv_len does not fit its pages or its new rows, sequence"; break;
      case kBadPage: what = "a page id outside the pool, sequence"; break;
      case kBadPosition: what = "a position outside the rotary table, row"; break;
      case kBadPair: what = "a page pair outside the pool, pair"; break;
      case kBadRows: what = "a sequence with more rows than max_rows, sequence"; break;
    }
    set_error("%s: code %d: %s %d, value %d", fn, words[kBadIndexWord], what, words[kBadIndexWord + 1], words[kBadIndexWord + 2]);
    return CASCADE_ERR_BAD_MAP;
  }
  return CASCADE_OK;
}

cascade_status_t cascade_rope_table_scaled(int32_t n_positions, int32_t rot_dim, double base, int32_t kind, double factor,
                                           double original_positions, double low, double high, double attention, float* table, void* stream) {
  const char* fn = "cascade_rope_table_scaled";
  if (!table || n_positions < 1 || rot_dim < 2 || rot_dim % 2 != 0 || !(base > 1.0) || !std::isfinite(base))
    return fail(CASCADE_ERR_INVALID_ARG, fn, "need a table pointer, n_positions >= 1, an even rot_dim >= 2 and base > 1");
  if (!aligned16(table)) return fail(CASCADE_ERR_INVALID_ARG, fn, "the table must be 16-byte aligned");
  if (kind < CASCADE_ROPE_NONE || kind > CASCADE_ROPE_RAMP) return fail(CASCADE_ERR_INVALID_ARG, fn, "unknown kind");
  if (kind != CASCADE_ROPE_NONE && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(CASCADE_ERR_INVALID_ARG, fn, "factor must be 1 or more");
  if (kind == CASCADE_ROPE_BASE && rot_dim < 4) return fail(CASCADE_ERR_INVALID_ARG, fn, "a scaled base needs rot_dim above 2");
  if (kind >= CASCADE_ROPE_BANDS && !(original_positions > 0 && low > 0 && high > low && std::isfinite(original_positions) && std::isfinite(high)))
    return fail(CASCADE_ERR_INVALID_ARG, fn, "need original_positions > 0 and 0 < low < high");
  if (!(attention >= 0) || !std::isfinite(attention)) return fail(CASCADE_ERR_INVALID_ARG, fn, "attention must not be negative");
  RopeScaling s;
  s.kind = kind;
  s.base = base;
  s.factor = kind == CASCADE_ROPE_NONE ? 1.0 : factor;
  s.original = original_positions;
  s.low = low;
  s.high = high;
  s.attention = attention > 0 ? attention : kind == CASCADE_ROPE_RAMP ? 0.1 * std::log(factor) + 1 : 1.0;
  return launched(launch_rope_table_scaled(n_positions, rot_dim, s, reinterpret_cast<float2*>(table), (cudaStream_t)stream), fn);
}

cascade_status_t cascade_rope_rows(cascade_dtype_t dtype, int32_t n_rows, int32_t n_heads, int32_t head_dim, int32_t rot_dim,
                                   int32_t interleaved, const void* x, cascade_strides_t x_strides, const int32_t* positions,
                                   const float* rope_table, int32_t n_positions, void* y, cascade_strides_t y_strides, void* stream) {
  const char* fn = "cascade_rope_rows";
  if (!x || !y || !positions || !rope_table) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  cascade_status_t s = check_types(fn, dtype, head_dim);
  if (s == CASCADE_OK) s = check_rope(fn, rope_table, n_positions, rot_dim, head_dim);
  if (s != CASCADE_OK) return s;
  if (n_rows < 1 || n_heads < 1) return fail(CASCADE_ERR_INVALID_ARG, fn, "rows and heads must be positive");
  if (n_heads > 65535) return fail(CASCADE_ERR_UNSUPPORTED, fn, "heads may not exceed 65535");
  const size_t es = elt_size(dtype);
  if (!aligned16(x) || !aligned16(y) || !rows_aligned(x_strides, es) || !rows_aligned(y_strides, es) || !aligned4(positions))
    return fail(CASCADE_ERR_INVALID_ARG, fn, "pointers and row strides must be 16-byte aligned");
  RopeRowsParams p;
  memset(&p, 0, sizeof(p));
  p.q = x;
  p.q_out = y;
  p.qs = in(x_strides);
  p.qos = in(y_strides);
  p.rope = reinterpret_cast<const float2*>(rope_table);
  p.positions = positions;
  p.paged.status = paged_status_words();
  p.n_rows = n_rows;
  p.H = n_heads;
  p.d = head_dim;
  p.rot = rot_dim;
  p.interleaved = interleaved != 0;
  p.n_positions = n_positions;
  if (!p.paged.status) return no_status(fn);
  return launched(launch_rope_rows(p, dtype, (cudaStream_t)stream), fn);
}

cascade_status_t cascade_paged_append(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t head_dim, const void* q, cascade_strides_t q_strides, void* q_out,
                                      cascade_strides_t q_out_strides, const void* k, cascade_strides_t k_strides, const void* v,
                                      cascade_strides_t v_strides, const int32_t* positions, const float* rope_table,
                                      int32_t n_positions, int32_t rot_dim, int32_t interleaved, void* k_pages,
                                      cascade_strides_t k_page_strides, void* v_pages, cascade_strides_t v_page_strides,
                                      int32_t n_pages, int32_t page_size, const int32_t* page_table, int64_t table_stride,
                                      int32_t max_pages, const int32_t* row_start, const int32_t* kv_len, void* stream) {
  const char* fn = "cascade_paged_append";
  if (!k || !v || !k_pages || !v_pages || (q == nullptr) != (q_out == nullptr)) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  cascade_status_t s = check_types(fn, dtype, head_dim);
  if (s == CASCADE_OK)
    s = check_pages(fn, batch, n_rows, q ? n_heads : 1, n_kv_heads, n_pages, page_size, page_table, table_stride, max_pages, row_start, kv_len);
  if (s == CASCADE_OK && rope_table) s = check_rope(fn, rope_table, n_positions, rot_dim, head_dim);
  if (s != CASCADE_OK) return s;
  const size_t es = elt_size(dtype);
  if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(v) || !aligned16(k_pages) || !aligned16(v_pages) ||
      (q && (!rows_aligned(q_strides, es) || !rows_aligned(q_out_strides, es))) || !rows_aligned(k_strides, es) ||
      !rows_aligned(v_strides, es) || !pages_aligned(k_page_strides, es) || !pages_aligned(v_page_strides, es) || !aligned4(positions))
    return fail(CASCADE_ERR_INVALID_ARG, fn, "pointers and row strides must be 16-byte aligned");
  RopeRowsParams p;
  memset(&p, 0, sizeof(p));
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_out = q_out;
  p.k_out = k_pages;
  p.v_out = v_pages;
  p.qs = in(q_strides);
  p.qos = in(q_out_strides);
  p.ks = in(k_strides);
  p.vs = in(v_strides);
  p.kos = in(k_page_strides);
  p.vos = in(v_page_strides);
  p.rope = reinterpret_cast<const float2*>(rope_table);
  p.positions = positions;
  p.paged = pages_dev(batch, n_rows, n_pages, page_size, page_table, table_stride, max_pages, row_start, kv_len, nullptr);
  p.n_rows = n_rows;
  p.H = q ? n_heads : 0;
  p.Hkv = n_kv_heads;
  p.d = head_dim;
  p.rot = rope_table ? rot_dim : 0;
  p.interleaved = interleaved != 0;
  p.n_positions = n_positions;
  if (!p.paged.status) return no_status(fn);
  return launched(launch_rope_rows(p, dtype, (cudaStream_t)stream), fn);
}

}  // extern "C"

namespace cascade {
namespace {

// What the choice of kernels and the scratch go by
AttnParams paged_shape(int32_t batch, int32_t n_rows, int32_t max_rows, int32_t H, int32_t Hkv, int32_t d, int32_t page_size, int32_t max_pages) {
  AttnParams p;
  memset(&p, 0, sizeof(p));
  p.batch = batch;
  p.H = H;
  p.Hkv = Hkv;
  p.G = H / Hkv;
  p.d = d;
  p.rule_kv_heads = Hkv;
  p.fused = 1;
  p.key_parts = 1;
  p.paged.batch = batch;
  p.paged.n_rows = n_rows;
  p.paged.page_size = page_size;
  p.paged.max_pages = max_pages;
  p.paged.least = 1;
  p.paged.most = max_rows;
  return p;
}
// Which kernels take the sequences of a call: those of at most `rows` rows the decode kernel (0: none), the others a kernel on tiles.
struct PagedRoute {
  int rows;
  bool tiles;
};
PagedRoute paged_route(const AttnParams& p, cascade_dtype_t dtype, int32_t max_rows) {
  const int few = paged_decode_rows(p, dtype), rows = std::min(max_rows, p.paged.n_rows);
  if (rows <= few || paged_decode_splits(p, dtype, rows)) return {rows, false};
  // One sequence has max_rows rows, unless they are padded.  In fp32 the kernel on tiles takes all: what adds up the parts of its keys
  // writes every row.
  return {p.paged.batch == 1 || dtype == CASCADE_F32 ? 0 : few, true};
}
size_t paged_ws_bytes(const AttnParams& p, cascade_dtype_t dtype, int32_t max_rows) {
  const PagedRoute r = paged_route(p, dtype, max_rows);
  return r.rows > 0 ? paged_decode_ws_bytes(p, dtype, r.rows) : dtype == CASCADE_F32 ? paged_f32_ws_bytes(p) : 0;
}

}  // namespace
}  // namespace cascade

extern "C" {

cascade_status_t cascade_attn_paged_workspace_bytes(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t max_rows, int32_t n_heads,
                                                    int32_t n_kv_heads, int32_t head_dim, int32_t page_size, int32_t max_pages,
                                                    size_t* out_bytes) {
  const char* fn = "cascade_attn_paged_workspace_bytes";
  if (!out_bytes) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  cascade_status_t s = check_types(fn, dtype, head_dim);
  if (s != CASCADE_OK) return s;
  if (batch < 1 || n_rows < 1 || max_rows < 1 || n_heads < 1 || n_kv_heads < 1 || max_pages < 1)
    return fail(CASCADE_ERR_INVALID_ARG, fn, "sizes must be positive");
  s = check_sizes(fn, n_heads, n_kv_heads, page_size, max_pages);
  if (s == CASCADE_OK) s = check_blocks(fn, batch, page_size, max_pages);
  if (s != CASCADE_OK) return s;
  *out_bytes = paged_ws_bytes(paged_shape(batch, n_rows, max_rows, n_heads, n_kv_heads, head_dim, page_size, max_pages), dtype, max_rows);
  return CASCADE_OK;
}

cascade_status_t cascade_attn_paged(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t max_rows, int32_t n_heads,
                                    int32_t n_kv_heads, int32_t head_dim, float scale, int32_t causal, const void* q,
                                    cascade_strides_t q_strides, const void* k_pages, cascade_strides_t k_page_strides,
                                    const void* v_pages, cascade_strides_t v_page_strides, int32_t n_pages, int32_t page_size,
                                    const int32_t* page_table, int64_t table_stride, int32_t max_pages, const int32_t* row_start,
                                    const int32_t* kv_len, const int32_t* visible, void* o_out, cascade_strides_t o_strides,
                                    float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "cascade_attn_paged";
  if (!q || !k_pages || !v_pages || !o_out) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  cascade_status_t s = check_types(fn, dtype, head_dim);
  if (s == CASCADE_OK)
    s = check_pages(fn, batch, n_rows, n_heads, n_kv_heads, n_pages, page_size, page_table, table_stride, max_pages, row_start, kv_len);
  if (s != CASCADE_OK) return s;
  if (max_rows < 1) return fail(CASCADE_ERR_INVALID_ARG, fn, "max_rows must be positive");
  s = check_sizes(fn, n_heads, n_kv_heads, page_size, max_pages);
  if (s == CASCADE_OK) s = check_blocks(fn, batch, page_size, max_pages);
  if (s != CASCADE_OK) return s;
  if (!(scale > 0.f) || !std::isfinite(scale)) return fail(CASCADE_ERR_INVALID_ARG, fn, "scale must be positive and finite");
  const size_t es = elt_size(dtype);
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(o_out) || !rows_aligned(q_strides, es) ||
      !rows_aligned(o_strides, es) || !pages_aligned(k_page_strides, es) || !pages_aligned(v_page_strides, es) || !aligned4(visible) ||
      !aligned4(lse_out))
    return fail(CASCADE_ERR_INVALID_ARG, fn, "pointers and row strides must be 16-byte aligned");
  AttnParams p = paged_shape(batch, n_rows, max_rows, n_heads, n_kv_heads, head_dim, page_size, max_pages);
  const size_t need = paged_ws_bytes(p, dtype, max_rows);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) {
    set_error("%s: workspace of %zu bytes (256-byte aligned) required, got %zu", fn, need, workspace ? workspace_bytes : (size_t)0);
    return CASCADE_ERR_WORKSPACE;
  }
  p.plan.causal = causal != 0;
  p.paged = pages_dev(batch, n_rows, n_pages, page_size, page_table, table_stride, max_pages, row_start, kv_len, visible);
  if (!p.paged.status) return no_status(fn);
  p.plan.status = p.paged.status;
  p.q = q;
  p.k = k_pages;
  p.v = v_pages;
  p.qs = {0, q_strides.token, q_strides.head};
  p.ks = in(k_page_strides);
  p.vs = in(v_page_strides);
  p.scale = scale;
  p.o_out = o_out;
  p.os = {0, o_strides.token, o_strides.head};
  p.lse_out = lse_out;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == CASCADE_BF16 && !paged_tc_takes(p))
    return fail(CASCADE_ERR_UNSUPPORTED, fn, "bf16 pages whose strides are not positive and below 2^38 elements");
  const PagedRoute r = paged_route(p, dtype, max_rows);
  cudaError_t e = cudaSuccess;
  if (r.tiles) {
    AttnParams many = p;
    many.paged.least = r.rows + 1;
    e = dtype == CASCADE_BF16 ? launch_paged_tc(many, max_rows, st) : launch_paged_f32(many, workspace, st);
  }
  if (e == cudaSuccess && r.rows > 0) {
    p.paged.most = r.rows;
    p.alone = !r.tiles;
    e = launch_paged_decode(p, dtype, r.rows, workspace, st);
  }
  return launched(e, fn);
}

static cascade_status_t check_tables(const char* fn, int32_t n_seqs, int32_t width, int32_t n_pages, int32_t page_size, const void* a,
                                     const void* b, const void* c, const void* d, const void* e, const void* f) {
  if (!a || !b || !c || !d || !e || !f) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  if (n_seqs < 1 || width < 1 || n_pages < 1 || page_size < 1) return fail(CASCADE_ERR_INVALID_ARG, fn, "sizes must be positive");
  if ((int64_t)width * page_size > 1 << 30) return fail(CASCADE_ERR_UNSUPPORTED, fn, "a sequence of more than 2^30 rows");
  // pages are walked, and what the sequences ask for is added up, in 32 bits
  if (n_pages > 1 << 30) return fail(CASCADE_ERR_UNSUPPORTED, fn, "more than 2^30 pages");
  if ((int64_t)n_seqs * width > INT_MAX) return fail(CASCADE_ERR_UNSUPPORTED, fn, "a table of 2^31 entries or more");
  if (a == b) return fail(CASCADE_ERR_INVALID_ARG, fn, "the new table may not be the old one");
  return CASCADE_OK;
}

cascade_status_t cascade_pages_fork(int32_t n_seqs, int32_t width, int32_t n_pages, int32_t page_size, const int32_t* table_in,
                                    const int32_t* kv_len_in, const int32_t* source, const int32_t* add, int32_t* table_out,
                                    int32_t* kv_len_out, int32_t* refs, int32_t* copies, int32_t* report, void* stream) {
  const char* fn = "cascade_pages_fork";
  cascade_status_t s = check_tables(fn, n_seqs, width, n_pages, page_size, table_in, table_out, kv_len_in, refs, copies, report);
  if (s != CASCADE_OK) return s;
  if (!source || !add || !kv_len_out) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  if (kv_len_out == kv_len_in) return fail(CASCADE_ERR_INVALID_ARG, fn, "the new lengths may not be the old ones");
  if (((uintptr_t)copies & 7) != 0) return fail(CASCADE_ERR_INVALID_ARG, fn, "copies must be 8-byte aligned");
  if (n_seqs > 8192) return fail(CASCADE_ERR_UNSUPPORTED, fn, "more than 8192 sequences");
  PagesParams p;
  memset(&p, 0, sizeof(p));
  p.table_in = table_in;
  p.kv_in = kv_len_in;
  p.source = source;
  p.add = add;
  p.table_out = table_out;
  p.kv_out = kv_len_out;
  p.refs = refs;
  p.pairs = copies;
  p.report = report;
  p.n_seqs = n_seqs;
  p.width = width;
  p.n_pages = n_pages;
  p.page_size = page_size;
  return launched(launch_pages_fork(p, (cudaStream_t)stream), fn);
}

cascade_status_t cascade_pages_compact(int32_t n_seqs, int32_t width, int32_t n_pages, int32_t page_size, const int32_t* table_in,
                                       const int32_t* kv_len, int32_t* table_out, int32_t* refs, int32_t* moves, int32_t* report,
                                       void* stream) {
  const char* fn = "cascade_pages_compact";
  const void* moves_or = n_pages < 2 ? static_cast<const void*>(refs) : moves;  // (a pool of one page has no moves)
  cascade_status_t s = check_tables(fn, n_seqs, width, n_pages, page_size, table_in, table_out, kv_len, refs, moves_or, report);
  if (s != CASCADE_OK) return s;
  if (((uintptr_t)moves & 7) != 0) return fail(CASCADE_ERR_INVALID_ARG, fn, "moves must be 8-byte aligned");
  PagesParams p;
  memset(&p, 0, sizeof(p));
  p.table_in = table_in;
  p.kv_in = kv_len;
  p.table_out = table_out;
  p.refs = refs;
  p.pairs = moves;
  p.max_pairs = n_pages / 2;
  p.report = report;
  p.n_seqs = n_seqs;
  p.width = width;
  p.n_pages = n_pages;
  p.page_size = page_size;
  return launched(launch_pages_compact(p, (cudaStream_t)stream), fn);
}

cascade_status_t cascade_pages_copy(int32_t n_pools, void* const* pools, const int64_t* page_strides, int64_t page_bytes, int32_t n_pages,
                                    const int32_t* pairs, int32_t n_pairs, void* stream) {
  const char* fn = "cascade_pages_copy";
  if (!pools || !page_strides || (n_pairs > 0 && !pairs)) return fail(CASCADE_ERR_INVALID_ARG, fn, "null pointer");
  if (n_pools < 1 || n_pages < 1 || n_pairs < 0 || page_bytes < 16 || page_bytes % 16 != 0 || page_bytes > (int64_t)1 << 40)
    return fail(CASCADE_ERR_INVALID_ARG, fn, "sizes must be positive and page_bytes a multiple of 16");
  if (n_pairs > 1 << 30) return fail(CASCADE_ERR_UNSUPPORTED, fn, "more than 2^30 pairs");
  if (n_pools > kMaxPools) {
    set_error("%s: %d pools, at most %d", fn, n_pools, kMaxPools);
    return CASCADE_ERR_UNSUPPORTED;
  }
  PagesCopyParams p;
  memset(&p, 0, sizeof(p));
  for (int i = 0; i < n_pools; ++i) {
    if (!pools[i] || !aligned16(pools[i]) || page_strides[i] < page_bytes || page_strides[i] % 16 != 0)
      return fail(CASCADE_ERR_INVALID_ARG, fn, "pools must be 16-byte aligned, their pages at least page_bytes apart");
    p.pool[i] = pools[i];
    p.page_stride[i] = page_strides[i];
  }
  if (n_pairs == 0) return CASCADE_OK;
  p.page_bytes = page_bytes;
  p.pairs = pairs;
  p.status = paged_status_words();
  p.n_pools = n_pools;
  p.n_pairs = n_pairs;
  p.n_pages = n_pages;
  if (!p.status) return no_status(fn);
  return launched(launch_pages_copy(p, (cudaStream_t)stream), fn);
}

}  // extern "C"
