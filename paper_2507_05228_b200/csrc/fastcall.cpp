// The per-layer calls of the Python binding as one native call each: unpacks the tensors (pointers, sizes, strides), makes
// what the caller left out (output, statistics, workspace), reads the current stream and calls the C ABI.
// The same steps through ctypes and tensor methods took 17 to 29 us of host time per call, more than the kernels of a
// decode step or a short prompt; here it is 1 to 2 us plus the launches.  No arithmetic and no CUDA call of its own.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <vector>

#include "cascade.h"

namespace {

struct Api {
  decltype(&cascade_last_error) last_error;
  decltype(&cascade_workspace_bytes) workspace_bytes;
  decltype(&cascade_attn_sharded) attn_sharded;
  decltype(&cascade_attn_sharded_rope) attn_sharded_rope;
  decltype(&cascade_attn_partials) attn_partials;
  decltype(&cascade_merge) merge;
  decltype(&cascade_decode_step_rope) decode_step_rope;
  decltype(&cascade_attn_decode_static) decode_static;
  decltype(&cascade_plan_advance) plan_advance;
  decltype(&cascade_rope_table_scaled) rope_table_scaled;
  decltype(&cascade_rope_rows) rope_rows;
  decltype(&cascade_paged_append) paged_append;
  decltype(&cascade_attn_paged) attn_paged;
  decltype(&cascade_attn_paged_workspace_bytes) attn_paged_workspace_bytes;
  decltype(&cascade_pages_fork) pages_fork;
  decltype(&cascade_pages_compact) pages_compact;
  decltype(&cascade_pages_copy) pages_copy;
};
Api api;
PyObject* cascade_error = nullptr;  // CascadeError(status, message)

struct PyFailure {};  // a Python exception is set

void raise_status(int status, const char* message) {
  PyObject* e = PyObject_CallFunction(cascade_error, "is", status, message);
  if (e) {
    PyErr_SetObject(cascade_error, e);
    Py_DECREF(e);
  }
  throw PyFailure();
}
void check(cascade_status_t status) {
  if (status != CASCADE_OK) raise_status(status, api.last_error());
}
[[noreturn]] void raise(PyObject* type, const char* message) {
  PyErr_SetString(type, message);
  throw PyFailure();
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "a tensor is expected");
  return THPVariable_Unpack(o);
}
cascade_strides_t strides(const at::Tensor& t) {
  if (t.dim() != 4 || t.stride(3) != 1)
    raise(PyExc_AssertionError, "expected [batch, tokens, heads, head_dim] with contiguous head_dim");
  return {t.stride(0), t.stride(1), t.stride(2)};
}
cascade_dtype_t dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return CASCADE_F32;
  if (t.scalar_type() != at::kBFloat16)
    raise_status(CASCADE_ERR_UNSUPPORTED, ("dtype " + std::string(c10::toString(t.scalar_type())) + " unsupported").c_str());
  return CASCADE_BF16;
}
int32_t size(const at::Tensor& t, int dim) { return (int32_t)t.size(dim); }
void need_dims(const at::Tensor& t, int n) {
  if (t.dim() != n) raise(PyExc_ValueError, "wrong number of tensor dimensions");
}
void* stream() {  // of the current device, as torch.cuda.current_stream()
  static const bool any = c10::cuda::device_count() > 0;
  return any ? c10::cuda::getCurrentCUDAStream().stream() : nullptr;
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyFailure();
  return v;
}
template <typename T>
T* address(PyObject* o) {
  if (o == Py_None) return nullptr;
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw PyFailure();
  return static_cast<T*>(p);
}
float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyFailure();
  return (float)v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PyFailure();
  return v != 0;
}

at::Tensor output_or(PyObject* out, const at::Tensor& like, at::IntArrayRef shape) {
  return out == Py_None ? at::empty(shape, like.options()) : tensor(out);
}
at::Tensor lse_for(bool want, const at::Tensor& q) {
  if (!want) return at::Tensor();
  return at::empty({q.size(0), q.size(1), q.size(2)}, q.options().dtype(at::kFloat));
}
float* data_or_null(const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; }

// Bytes of a workspace: no more than lie in its memory (a view may show the same ones many times).
size_t bytes_of(const at::Tensor& t) {
  const size_t es = t.element_size(), all = t.storage().nbytes(), before = (size_t)t.storage_offset() * es;
  return std::min((size_t)t.numel() * es, all > before ? all - before : 0);
}
struct Scratch {
  at::Tensor own;
  void* ptr = nullptr;
  size_t bytes = 0;
};
Scratch scratch(const cascade_plan_t* plan, int call, cascade_dtype_t code, const at::Tensor& q, int n_kv_heads,
                PyObject* given) {
  Scratch s;
  size_t need = 0;
  check(api.workspace_bytes(plan, call, code, size(q, 0), size(q, 2), n_kv_heads, size(q, 3), &need));
  if (need == 0) return s;
  s.own = given == Py_None ? at::empty({(int64_t)need}, q.options().dtype(at::kByte)) : tensor(given);
  s.ptr = s.own.data_ptr();
  s.bytes = bytes_of(s.own);
  return s;
}

PyObject* wrap(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject* pair(PyObject* given_out, const at::Tensor& o, const at::Tensor& lse) {
  PyObject* r = PyTuple_New(2);
  if (!r) throw PyFailure();
  if (given_out != Py_None) {
    Py_INCREF(given_out);
    PyTuple_SET_ITEM(r, 0, given_out);
  } else {
    PyTuple_SET_ITEM(r, 0, wrap(o));
  }
  PyTuple_SET_ITEM(r, 1, wrap(lse));
  return r;
}

// The C calls run without the interpreter lock.  `f` must not throw, which would leave the lock behind: sizes and data pointers
// are taken before (a tensor without storage, as torch.func.vmap hands out, throws when asked for its pointer).
template <typename F>
cascade_status_t unlocked(F&& f) {
  cascade_status_t status;
  Py_BEGIN_ALLOW_THREADS
  status = f();
  Py_END_ALLOW_THREADS
  return status;
}

template <int N, PyObject* (*F)(PyObject* const*)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments are expected, got %zd", N, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const PyFailure&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (plan, q, k, v, scale, rope_table or None, out or None, want_lse, workspace or None) -> (o, lse or None)
PyObject* attn_sharded(PyObject* const* a) {
  const auto* plan = address<const cascade_plan_t>(a[0]);
  const at::Tensor &q = tensor(a[1]), &k = tensor(a[2]), &v = tensor(a[3]);
  need_dims(q, 4);
  const cascade_strides_t qs = strides(q), ks = strides(k), vs = strides(v);
  const cascade_dtype_t code = dtype_code(q);
  const float scale = number(a[4]);
  const int32_t B = size(q, 0), H = size(q, 2), Hkv = size(k, 2), d = size(q, 3);
  const at::Tensor o = output_or(a[6], q, q.sizes());
  const cascade_strides_t os = strides(o);
  const at::Tensor lse = lse_for(truth(a[7]), q);
  const Scratch ws = scratch(plan, CASCADE_CALL_SHARDED, code, q, Hkv, a[8]);
  void *st = stream(), *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = o.data_ptr();
  float* lp = data_or_null(lse);
  if (a[5] == Py_None) {
    check(unlocked([&] {
      return api.attn_sharded(plan, code, B, H, Hkv, d, scale, qp, qs, kp, ks, vp, vs, op, os, lp, ws.ptr, ws.bytes, st);
    }));
  } else {
    const at::Tensor& table = tensor(a[5]);
    if (table.scalar_type() != at::kFloat || !table.is_contiguous() || table.dim() != 3 || table.size(1) != d / 2 ||
        table.size(2) != 2)
      raise(PyExc_AssertionError, "the positional table is fp32 [positions, head_dim / 2, 2], contiguous");
    const auto* tp = static_cast<const float*>(table.data_ptr());
    const int32_t n_positions = size(table, 0);
    check(unlocked([&] {
      return api.attn_sharded_rope(plan, code, B, H, Hkv, d, scale, qp, qs, kp, ks, vp, vs, tp, n_positions, op, os, lp,
                                   ws.ptr, ws.bytes, st);
    }));
  }
  return pair(a[6], o, lse);
}

// (plan, n_kv_shards, q, k, v, scale, out or None, workspace or None) -> (o_part, m_part, l_part)
PyObject* attn_partials(PyObject* const* a) {
  const auto* plan = address<const cascade_plan_t>(a[0]);
  const int64_t P = integer(a[1]);
  const at::Tensor &q = tensor(a[2]), &k = tensor(a[3]), &v = tensor(a[4]);
  need_dims(q, 4);
  const cascade_strides_t qs = strides(q), ks = strides(k), vs = strides(v);
  const cascade_dtype_t code = dtype_code(q);
  const float scale = number(a[5]);
  at::Tensor o, m, l;
  if (a[6] == Py_None) {
    const int64_t B = q.size(0), n = q.size(1), H = q.size(2);
    o = at::empty({B, P, n, H, q.size(3)}, q.options());
    m = at::empty({B, P, n, H}, q.options().dtype(at::kFloat));
    l = at::empty_like(m);
  } else {
    PyObject* seq = PySequence_Fast(a[6], "out: (o_part, m_part, l_part) is expected");
    if (!seq) throw PyFailure();
    if (PySequence_Fast_GET_SIZE(seq) != 3) {
      Py_DECREF(seq);
      raise(PyExc_ValueError, "out: (o_part, m_part, l_part) is expected");
    }
    PyObject** item = PySequence_Fast_ITEMS(seq);
    const bool fine = THPVariable_Check(item[0]) && THPVariable_Check(item[1]) && THPVariable_Check(item[2]);
    if (fine) {
      o = THPVariable_Unpack(item[0]);
      m = THPVariable_Unpack(item[1]);
      l = THPVariable_Unpack(item[2]);
    }
    Py_DECREF(seq);
    if (!fine) raise(PyExc_TypeError, "out: three tensors are expected");
  }
  const int32_t B = size(q, 0), H = size(q, 2), Hkv = size(k, 2), d = size(q, 3);
  const Scratch ws = scratch(plan, CASCADE_CALL_PARTIALS, code, q, Hkv, a[7]);
  void *st = stream(), *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = o.data_ptr();
  float *mp = static_cast<float*>(m.data_ptr()), *lp = static_cast<float*>(l.data_ptr());
  check(unlocked([&] {
    return api.attn_partials(plan, code, B, H, Hkv, d, scale, qp, qs, kp, ks, vp, vs, op, mp, lp, ws.ptr, ws.bytes, st);
  }));
  PyObject* r = PyTuple_New(3);
  if (!r) throw PyFailure();
  PyTuple_SET_ITEM(r, 0, wrap(o));
  PyTuple_SET_ITEM(r, 1, wrap(m));
  PyTuple_SET_ITEM(r, 2, wrap(l));
  return r;
}

// (o_part, m_part, l_part, row_scatter address, batch stride, out or None, want_lse) -> (o, lse or None)
PyObject* merge(PyObject* const* a) {
  const at::Tensor &parts = tensor(a[0]), &m = tensor(a[1]), &l = tensor(a[2]);
  need_dims(parts, 5);
  const cascade_dtype_t code = dtype_code(parts);
  const int64_t B = parts.size(0), n = parts.size(2), H = parts.size(3), d = parts.size(4);
  const int32_t n_parts = size(parts, 1);
  const auto* rows = address<const int32_t>(a[3]);
  const int64_t row_stride = integer(a[4]);
  const at::Tensor o = output_or(a[5], parts, {B, n, H, d});
  const cascade_strides_t os = strides(o);
  at::Tensor lse;
  if (truth(a[6])) lse = at::empty({B, n, H}, parts.options().dtype(at::kFloat));
  void *st = stream(), *pp = parts.data_ptr(), *op = o.data_ptr();
  const auto *mp = static_cast<const float*>(m.data_ptr()), *lp = static_cast<const float*>(l.data_ptr());
  float* lse_p = data_or_null(lse);
  check(unlocked([&] {
    return api.merge(code, (int32_t)B, n_parts, (int32_t)n, (int32_t)H, (int32_t)d, pp, mp, lp, rows, row_stride, op, os,
                     lse_p, st);
  }));
  return pair(a[5], o, lse);
}

// (plan, q_new, k_new, v_new, k_cache, v_cache, position, scale, rope_table, out or None, want_lse, workspace or None)
PyObject* decode_step_rope(PyObject* const* a) {
  auto* plan = address<cascade_plan_t>(a[0]);
  const at::Tensor &q = tensor(a[1]), &kn = tensor(a[2]), &vn = tensor(a[3]), &kc = tensor(a[4]), &vc = tensor(a[5]);
  const at::Tensor& table = tensor(a[8]);
  need_dims(q, 4);
  const cascade_strides_t qs = strides(q), kns = strides(kn), vns = strides(vn), kcs = strides(kc), vcs = strides(vc);
  const int32_t position = (int32_t)integer(a[6]);
  const float scale = number(a[7]);
  const at::Tensor o = a[9] == Py_None ? at::empty_like(q) : tensor(a[9]);
  const cascade_strides_t os = strides(o);
  const at::Tensor lse = lse_for(truth(a[10]), q);
  const int32_t B = size(q, 0), H = size(q, 2), Hkv = size(kn, 2), n_positions = size(table, 0);
  const Scratch ws = scratch(plan, CASCADE_CALL_DECODE_STEP_ROPE, CASCADE_BF16, q, Hkv, a[11]);
  void *st = stream(), *qp = q.data_ptr(), *knp = kn.data_ptr(), *vnp = vn.data_ptr(), *kcp = kc.data_ptr(),
       *vcp = vc.data_ptr(), *op = o.data_ptr();
  const auto* tp = static_cast<const float*>(table.data_ptr());
  float* lp = data_or_null(lse);
  check(unlocked([&] {
    return api.decode_step_rope(plan, B, H, Hkv, scale, qp, qs, knp, kns, vnp, vns, kcp, kcs, vcp, vcs, position, tp,
                                n_positions, op, os, lp, ws.ptr, ws.bytes, st);
  }));
  return pair(a[9], o, lse);
}

// (plan, q, k, v, scale, out or None, want_lse) -> (o, lse or None)
PyObject* attn_decode_static(PyObject* const* a) {
  const auto* plan = address<const cascade_plan_t>(a[0]);
  const at::Tensor &q = tensor(a[1]), &k = tensor(a[2]), &v = tensor(a[3]);
  need_dims(q, 4);
  if (q.size(1) != 1 || q.size(3) != 128 || q.scalar_type() != at::kBFloat16)
    raise(PyExc_AssertionError, "one bf16 query row of head_dim 128 per sequence is expected");
  const cascade_strides_t qs = strides(q), ks = strides(k), vs = strides(v);
  const float scale = number(a[4]);
  const at::Tensor o = output_or(a[5], q, q.sizes());
  const cascade_strides_t os = strides(o);
  const at::Tensor lse = lse_for(truth(a[6]), q);
  const int32_t B = size(q, 0), H = size(q, 2), Hkv = size(k, 2);
  void *st = stream(), *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = o.data_ptr();
  float* lp = data_or_null(lse);
  check(unlocked([&] {
    return api.decode_static(plan, B, H, Hkv, scale, qp, qs, kp, ks, vp, vs, op, os, lp, st);
  }));
  return pair(a[5], o, lse);
}

// (plan, q_pos_offset)
PyObject* plan_advance(PyObject* const* a) {
  auto* plan = address<cascade_plan_t>(a[0]);
  const int32_t offset = (int32_t)integer(a[1]);
  void* st = stream();
  check(unlocked([&] { return api.plan_advance(plan, offset, st); }));
  Py_RETURN_NONE;
}

// ---------------------------------------------------------------------------------------------------- paged caches

// A tensor of the current device, whose stream the call goes to.
const at::Tensor& here(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda()) raise(PyExc_ValueError, "a tensor on the GPU is expected");
  if (t.get_device() != c10::cuda::current_device()) raise(PyExc_ValueError, "a tensor is on another device than the current one");
  return t;
}
cascade_strides_t row_strides(const at::Tensor& t) {  // [rows, heads, head_dim]
  if (t.dim() != 3 || t.stride(2) != 1) raise(PyExc_AssertionError, "expected [rows, heads, head_dim] with contiguous head_dim");
  return {0, t.stride(0), t.stride(1)};
}
cascade_strides_t page_strides(const at::Tensor& t) {
  if (t.dim() != 4 || t.stride(3) != 1)
    raise(PyExc_AssertionError, "expected pages [n_pages, page_size, kv_heads, head_dim] with contiguous head_dim");
  return {t.stride(0), t.stride(1), t.stride(2)};
}
void need(bool fine, const char* message) {
  if (!fine) raise(PyExc_ValueError, message);
}
const int32_t* ints(const at::Tensor& t, int64_t n, const char* message) {
  if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1)) raise(PyExc_ValueError, message);
  return static_cast<const int32_t*>(t.data_ptr());
}
const float* rope_table(const at::Tensor& t, int32_t& n_positions, int32_t& rot) {
  if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.dim() != 3 || t.size(2) != 2)
    raise(PyExc_AssertionError, "the positional table is fp32 [positions, rot_dim / 2, 2], contiguous");
  n_positions = size(t, 0);
  rot = 2 * size(t, 1);
  return static_cast<const float*>(t.data_ptr());
}
struct Pages {
  const at::Tensor &k, &v, &table;
  cascade_strides_t ks, vs;
  void *kp, *vp;
  const int32_t *tp, *starts, *len;
  int64_t table_stride;
  int32_t n_pages, page_size, Hkv, d, batch, max_pages;
  Pages(PyObject* k_, PyObject* v_, PyObject* table_, PyObject* starts_, PyObject* len_)
      : k(here(k_)), v(here(v_)), table(here(table_)), ks(page_strides(k)), vs(page_strides(v)) {
    need(k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type(), "k_pages and v_pages must be of one shape and type");
    need(table.scalar_type() == at::kInt && table.dim() == 2 && (table.size(1) <= 1 || table.stride(1) == 1),
         "the page table is int32 [sequences, pages] with contiguous rows");
    n_pages = size(k, 0);
    page_size = size(k, 1);
    Hkv = size(k, 2);
    d = size(k, 3);
    batch = size(table, 0);
    max_pages = size(table, 1);
    table_stride = batch > 1 ? table.stride(0) : max_pages;
    starts = ints(here(starts_), (int64_t)batch + 1, "row_start is int32 [sequences + 1]");
    len = ints(here(len_), batch, "kv_len is int32 [sequences]");
    kp = k.data_ptr();
    vp = v.data_ptr();
    tp = static_cast<const int32_t*>(table.data_ptr());
  }
};

double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyFailure();
  return v;
}
// (n_positions, rot_dim, base, kind, factor, original_positions, low, high, attention, table or None: on the current device) -> table
PyObject* rope_table_scaled(PyObject* const* a) {
  const long long n = integer(a[0]), rot = integer(a[1]);
  need(n > INT32_MIN && n <= INT32_MAX && rot > INT32_MIN && rot <= INT32_MAX, "n_positions and rot_dim are 32-bit numbers");
  const int32_t kind = (int32_t)integer(a[3]);
  const double base = real(a[2]), factor = real(a[4]), original = real(a[5]), low = real(a[6]), high = real(a[7]), attention = real(a[8]);
  const at::Tensor table = a[9] != Py_None ? here(a[9])
                                           : at::empty({std::max(n, 0LL), std::max(rot, 0LL) / 2, 2},
                                                       at::TensorOptions(at::kFloat).device(at::kCUDA, c10::cuda::current_device()));
  auto* tp = static_cast<float*>(table.data_ptr());
  void* st = stream();
  check(unlocked([&] { return api.rope_table_scaled((int32_t)n, (int32_t)rot, base, kind, factor, original, low, high, attention, tp, st); }));
  return wrap(table);
}

// (x, positions, rope_table, interleaved, out or None) -> out
PyObject* rope_rows(PyObject* const* a) {
  const at::Tensor &x = here(a[0]), &positions = here(a[1]), &table = here(a[2]);
  const cascade_strides_t xs = row_strides(x);
  const cascade_dtype_t code = dtype_code(x);
  const int32_t n = size(x, 0), H = size(x, 1), d = size(x, 2);
  const int32_t* pos = ints(positions, n, "positions is int32 [rows]");
  int32_t n_positions, rot;
  const float* tp = rope_table(table, n_positions, rot);
  const int32_t interleaved = truth(a[3]);
  const at::Tensor y = a[4] == Py_None ? at::empty_like(x) : here(a[4]);
  const cascade_strides_t ys = row_strides(y);
  need(y.sizes() == x.sizes() && y.scalar_type() == x.scalar_type(), "out must be of x's shape and type");
  if (n > 0) {
    void *st = stream(), *xp = x.data_ptr(), *yp = y.data_ptr();
    check(unlocked([&] { return api.rope_rows(code, n, H, d, rot, interleaved, xp, xs, pos, tp, n_positions, yp, ys, st); }));
  }
  return wrap(y);
}

// (k, v, k_pages, v_pages, page_table, row_start, kv_len, q or None, positions or None, rope_table or None, interleaved, q_out or None)
// -> q_out or None
PyObject* paged_append(PyObject* const* a) {
  const at::Tensor &k = here(a[0]), &v = here(a[1]);
  const Pages g(a[2], a[3], a[4], a[5], a[6]);
  const cascade_strides_t ks = row_strides(k), vs = row_strides(v);
  const cascade_dtype_t code = dtype_code(k);
  const int32_t n = size(k, 0);
  need(k.sizes() == v.sizes() && size(k, 1) == g.Hkv && size(k, 2) == g.d, "k and v must be [rows, kv_heads, head_dim] of the pages");
  need(v.scalar_type() == k.scalar_type() && g.k.scalar_type() == k.scalar_type(), "k, v and the pages must be of one type");
  at::Tensor q, q_out;
  cascade_strides_t qs = {0, 0, 0}, qos = {0, 0, 0};
  int32_t H = 0;
  if (a[7] != Py_None) {
    q = here(a[7]);
    qs = row_strides(q);
    H = size(q, 1);
    need(size(q, 0) == n && size(q, 2) == g.d && q.scalar_type() == k.scalar_type(), "q must be [rows, heads, head_dim] of k's type");
    q_out = a[11] == Py_None ? at::empty_like(q) : here(a[11]);
    qos = row_strides(q_out);
    need(q_out.sizes() == q.sizes() && q_out.scalar_type() == q.scalar_type(), "q_out must be of q's shape and type");
  }
  const int32_t* pos = a[8] == Py_None ? nullptr : ints(here(a[8]), n, "positions is int32 [rows]");
  int32_t n_positions = 0, rot = 0;
  const float* tp = a[9] == Py_None ? nullptr : rope_table(here(a[9]), n_positions, rot);
  const int32_t interleaved = truth(a[10]);
  if (n > 0) {
    void *st = stream(), *kp = k.data_ptr(), *vp = v.data_ptr(), *qp = q.defined() ? q.data_ptr() : nullptr,
         *qop = q.defined() ? q_out.data_ptr() : nullptr;
    check(unlocked([&] {
      return api.paged_append(code, g.batch, n, H, g.Hkv, g.d, qp, qs, qop, qos, kp, ks, vp, vs, pos, tp, n_positions, rot, interleaved,
                              g.kp, g.ks, g.vp, g.vs, g.n_pages, g.page_size, g.tp, g.table_stride, g.max_pages, g.starts, g.len, st);
    }));
  }
  return wrap(q_out);
}

// (q, k_pages, v_pages, page_table, row_start, kv_len, scale, causal, visible or None, max_rows or None, out or None, want_lse,
// workspace or None) -> (o, lse or None)
PyObject* attn_paged(PyObject* const* a) {
  const at::Tensor& q = here(a[0]);
  const Pages g(a[1], a[2], a[3], a[4], a[5]);
  const cascade_strides_t qs = row_strides(q);
  const cascade_dtype_t code = dtype_code(q);
  const int32_t n = size(q, 0), H = size(q, 1);
  need(size(q, 2) == g.d && g.k.scalar_type() == q.scalar_type(), "q and the pages must be of one head_dim and type");
  const float scale = number(a[6]);
  const int32_t causal = truth(a[7]);
  const int32_t* visible = a[8] == Py_None ? nullptr : ints(here(a[8]), n, "visible is int32 [rows]");
  const long long most = a[9] == Py_None ? std::max(n, 1) : integer(a[9]);
  need(most >= INT32_MIN && most <= INT32_MAX, "max_rows is a 32-bit number");
  const auto max_rows = (int32_t)most;
  const at::Tensor o = a[10] == Py_None ? at::empty_like(q) : here(a[10]);
  const cascade_strides_t os = row_strides(o);
  need(o.sizes() == q.sizes() && o.scalar_type() == q.scalar_type(), "out must be of q's shape and type");
  at::Tensor lse;
  if (truth(a[11])) lse = at::empty({n, H}, q.options().dtype(at::kFloat));
  if (n > 0) {
    size_t bytes = 0;
    check(api.attn_paged_workspace_bytes(code, g.batch, n, max_rows, H, g.Hkv, g.d, g.page_size, g.max_pages, &bytes));
    Scratch ws;
    if (bytes > 0) {
      ws.own = a[12] == Py_None ? at::empty({(int64_t)bytes}, q.options().dtype(at::kByte)) : here(a[12]);
      ws.ptr = ws.own.data_ptr();
      ws.bytes = bytes_of(ws.own);
    }
    void *st = stream(), *qp = q.data_ptr(), *op = o.data_ptr();
    float* lp = data_or_null(lse);
    check(unlocked([&] {
      return api.attn_paged(code, g.batch, n, max_rows, H, g.Hkv, g.d, scale, causal, qp, qs, g.kp, g.ks, g.vp, g.vs, g.n_pages, g.page_size,
                            g.tp, g.table_stride, g.max_pages, g.starts, g.len, visible, op, os, lp, ws.ptr, ws.bytes, st);
    }));
  }
  return pair(a[10], o, lse);
}

at::Tensor like_ints(const at::Tensor& t, at::IntArrayRef shape) { return at::empty(shape, t.options().dtype(at::kInt)); }
// `out`: a sequence of n tensors for the results, or None
std::vector<at::Tensor> results(PyObject* out, const at::Tensor& like, std::initializer_list<std::vector<int64_t>> shapes) {
  std::vector<at::Tensor> r;
  if (out == Py_None) {
    for (const auto& s : shapes) r.push_back(like_ints(like, s));
    return r;
  }
  need(PyTuple_Check(out) && PyTuple_GET_SIZE(out) == (Py_ssize_t)shapes.size(), "out: a tuple of the result tensors is expected");
  Py_ssize_t i = 0;
  for (const auto& s : shapes) {
    const at::Tensor& t = here(PyTuple_GET_ITEM(out, i++));
    need(t.scalar_type() == at::kInt && t.sizes() == at::IntArrayRef(s) && t.is_contiguous(), "out: contiguous int32 tensors of the results' shapes are expected");
    r.push_back(t);
  }
  return r;
}
PyObject* tuple_of(const std::vector<at::Tensor>& r) {
  PyObject* t = PyTuple_New((Py_ssize_t)r.size());
  if (!t) throw PyFailure();
  for (size_t i = 0; i < r.size(); ++i) PyTuple_SET_ITEM(t, (Py_ssize_t)i, wrap(r[i]));
  return t;
}
int32_t* ints_of(const at::Tensor& t) { return static_cast<int32_t*>(t.data_ptr()); }
const at::Tensor& whole_table(PyObject* o) {
  const at::Tensor& t = here(o);
  need(t.scalar_type() == at::kInt && t.dim() == 2 && t.is_contiguous(), "the page table is int32 [sequences, pages], contiguous");
  return t;
}

// (page_table, kv_len, source, add, n_pages, page_size, out or None) -> (page_table, kv_len, refs, copies, report)
PyObject* pages_fork(PyObject* const* a) {
  const at::Tensor& table = whole_table(a[0]);
  const int64_t n = table.size(0), width = table.size(1), n_pages = integer(a[4]), page_size = integer(a[5]);
  need(n_pages > 0 && n_pages <= INT32_MAX && page_size > 0 && page_size <= INT32_MAX, "n_pages and page_size must be positive");
  const int32_t* len = ints(here(a[1]), n, "kv_len is int32 [sequences]");
  const int32_t* source = ints(here(a[2]), n, "source is int32 [sequences]");
  const int32_t* add = ints(here(a[3]), n, "add is int32 [sequences]");
  const auto r = results(a[6], table, {{n, width}, {n}, {n_pages}, {n, 2}, {4}});
  void* st = stream();
  const int32_t* tp = ints_of(table);
  int32_t* rp[5];
  for (int i = 0; i < 5; ++i) rp[i] = ints_of(r[i]);
  check(unlocked([&] {
    return api.pages_fork((int32_t)n, (int32_t)width, (int32_t)n_pages, (int32_t)page_size, tp, len, source, add, rp[0], rp[1], rp[2], rp[3], rp[4], st);
  }));
  return tuple_of(r);
}

// (page_table, kv_len, n_pages, page_size, out or None) -> (page_table, refs, moves, report)
PyObject* pages_compact(PyObject* const* a) {
  const at::Tensor& table = whole_table(a[0]);
  const int64_t n = table.size(0), width = table.size(1), n_pages = integer(a[2]), page_size = integer(a[3]);
  need(n_pages > 0 && n_pages <= INT32_MAX && page_size > 0 && page_size <= INT32_MAX, "n_pages and page_size must be positive");
  const int32_t* len = ints(here(a[1]), n, "kv_len is int32 [sequences]");
  const auto r = results(a[4], table, {{n, width}, {n_pages}, {n_pages / 2, 2}, {4}});
  void* st = stream();
  const int32_t* tp = ints_of(table);
  int32_t* rp[4];
  for (int i = 0; i < 4; ++i) rp[i] = ints_of(r[i]);
  check(unlocked([&] {
    return api.pages_compact((int32_t)n, (int32_t)width, (int32_t)n_pages, (int32_t)page_size, tp, len, rp[0], rp[1], rp[2], rp[3], st);
  }));
  return tuple_of(r);
}

// (pools, pairs): pools = sequence of tensors [n_pages, ...] whose pages are dense
PyObject* pages_copy(PyObject* const* a) {
  constexpr Py_ssize_t kMost = 256;
  void* at[kMost];
  int64_t stride[kMost], bytes = 0, n_pages = 0;
  const at::Tensor& pairs = here(a[1]);
  need(pairs.scalar_type() == at::kInt && pairs.dim() == 2 && pairs.size(1) == 2 && pairs.is_contiguous(), "pairs is int32 [n, 2], contiguous");
  need(PyList_Check(a[0]) || PyTuple_Check(a[0]), "pools: a list of tensors is expected");
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
  if (n > kMost) raise_status(CASCADE_ERR_UNSUPPORTED, "cascade_pages_copy: more than 256 pools");
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor& t = here(PySequence_Fast_GET_ITEM(a[0], i));
    need(t.dim() >= 2 && t.size(0) > 0, "a pool is [n_pages, ...]");
    int64_t dense = 1;  // a page is dense if its strides are those of some order of its dimensions
    bool used[8] = {};
    need(t.dim() <= 8, "a pool has at most eight dimensions");
    for (int64_t left = 1; left < t.dim(); ++left) {
      int64_t next = -1;
      for (int64_t j = 1; j < t.dim(); ++j)
        if (!used[j] && (t.size(j) == 1 || t.stride(j) == dense)) {
          next = j;
          if (t.size(j) > 1) break;
        }
      need(next >= 0, "the pages of a pool must be dense");
      used[next] = true;
      dense *= t.size(next);
    }
    const int64_t es = (int64_t)t.element_size();
    need(i == 0 || (dense * es == bytes && t.size(0) == n_pages), "all pools must have as many pages, of one size");
    bytes = dense * es;
    n_pages = t.size(0);
    at[i] = t.data_ptr();
    stride[i] = n_pages > 1 ? t.stride(0) * es : bytes;
  }
  need(n_pages <= INT32_MAX && pairs.size(0) <= INT32_MAX, "too many pages or pairs");
  void* st = stream();
  const int32_t* pp = ints_of(pairs);
  const int32_t n_pairs = size(pairs, 0);
  check(unlocked([&] { return api.pages_copy((int32_t)n, at, stride, bytes, (int32_t)n_pages, pp, n_pairs, st); }));
  Py_RETURN_NONE;
}

// load(path of the CUDA library, CascadeError)
PyObject* load(PyObject*, PyObject* args) {
  const char* path = nullptr;
  PyObject* error = nullptr;
  if (!PyArg_ParseTuple(args, "sO", &path, &error)) return nullptr;
  void* h = dlopen(path, RTLD_NOW);
  if (!h) {
    PyErr_SetString(PyExc_ImportError, dlerror());
    return nullptr;
  }
  auto find = [&](auto& fn, const char* name) {
    fn = reinterpret_cast<std::remove_reference_t<decltype(fn)>>(dlsym(h, name));
    if (!fn && !PyErr_Occurred()) PyErr_Format(PyExc_ImportError, "%s has no %s", path, name);
  };
  find(api.last_error, "cascade_last_error");
  find(api.workspace_bytes, "cascade_workspace_bytes");
  find(api.attn_sharded, "cascade_attn_sharded");
  find(api.attn_sharded_rope, "cascade_attn_sharded_rope");
  find(api.attn_partials, "cascade_attn_partials");
  find(api.merge, "cascade_merge");
  find(api.decode_step_rope, "cascade_decode_step_rope");
  find(api.decode_static, "cascade_attn_decode_static");
  find(api.plan_advance, "cascade_plan_advance");
  find(api.rope_table_scaled, "cascade_rope_table_scaled");
  find(api.rope_rows, "cascade_rope_rows");
  find(api.paged_append, "cascade_paged_append");
  find(api.attn_paged, "cascade_attn_paged");
  find(api.attn_paged_workspace_bytes, "cascade_attn_paged_workspace_bytes");
  find(api.pages_fork, "cascade_pages_fork");
  find(api.pages_compact, "cascade_pages_compact");
  find(api.pages_copy, "cascade_pages_copy");
  if (PyErr_Occurred()) return nullptr;
  Py_INCREF(error);
  Py_XDECREF(cascade_error);
  cascade_error = error;
  Py_RETURN_NONE;
}

template <int N, PyObject* (*F)(PyObject* const*)>
constexpr PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<N, F>));
}

PyMethodDef methods[] = {
    {"load", load, METH_VARARGS, nullptr},
    {"attn_sharded", fast<9, attn_sharded>(), METH_FASTCALL, nullptr},
    {"attn_partials", fast<8, attn_partials>(), METH_FASTCALL, nullptr},
    {"merge", fast<7, merge>(), METH_FASTCALL, nullptr},
    {"decode_step_rope", fast<12, decode_step_rope>(), METH_FASTCALL, nullptr},
    {"attn_decode_static", fast<7, attn_decode_static>(), METH_FASTCALL, nullptr},
    {"plan_advance", fast<2, plan_advance>(), METH_FASTCALL, nullptr},
    {"rope_table_scaled", fast<10, rope_table_scaled>(), METH_FASTCALL, nullptr},
    {"rope_rows", fast<5, rope_rows>(), METH_FASTCALL, nullptr},
    {"paged_append", fast<12, paged_append>(), METH_FASTCALL, nullptr},
    {"attn_paged", fast<13, attn_paged>(), METH_FASTCALL, nullptr},
    {"pages_fork", fast<7, pages_fork>(), METH_FASTCALL, nullptr},
    {"pages_compact", fast<5, pages_compact>(), METH_FASTCALL, nullptr},
    {"pages_copy", fast<2, pages_copy>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__fastcall(void) { return PyModule_Create(&module); }
