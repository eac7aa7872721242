// Native marshalling for the calls a decode step or a small compression makes: from torch tensors to the C ABI's
// layouts and pointers without a Python object per field (a call of the ctypes route builds a dozen and takes 10 to
// 17 us, as long as the kernels of a short cache run; these take 2 to 4, the launch included).
//
// Each function takes the well-formed case only: tensors of the plain class on a GPU, outputs and workspace given,
// numbers in range.  It returns the library's status, or None for anything else - the caller then takes the
// ctypes route, which handles or refuses it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "ckv.h"

namespace {

struct Entry {
  decltype(&ckv_compress) compress;
  decltype(&ckv_append) append;
  decltype(&ckv_decode_attn) decode_attn;
  decltype(&ckv_paged_append) paged_append;
  decltype(&ckv_paged_decode_attn) paged_decode_attn;
} entry;

struct Tables {
  decltype(&ckv_paged_reserve) reserve;
  decltype(&ckv_paged_trim) trim;
  decltype(&ckv_paged_write_strided) write;
  decltype(&ckv_paged_bounds) bounds;
  decltype(&ckv_paged_select) select;
  decltype(&ckv_paged_sparse_decode_attn) sparse_attn;
} tables;

struct Pages {
  decltype(&ckv_paged_chunk_attn) chunk_attn;
  decltype(&ckv_paged_fork) fork;
  decltype(&ckv_paged_compact) compact;
  decltype(&ckv_paged_copy) copy;
} pages;

// a tensor argument: NULL for None; `ok` turns false for what this file does not take
const at::TensorBase* tensor(PyObject* x, bool& ok) {
  if (x == Py_None) return nullptr;
  if (!THPVariable_CheckExact(x)) { ok = false; return nullptr; }
  const at::TensorBase& t = THPVariable_Unpack(x);
  if (!t.is_cuda() || t.layout() != at::kStrided) { ok = false; return nullptr; }
  return &t;
}
const at::TensorBase* given(PyObject* x, bool& ok) {
  const at::TensorBase* t = tensor(x, ok);
  if (!t) ok = false;
  return t;
}
template <typename T = void>
T* ptr(const at::TensorBase* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

int32_t small_int(PyObject* x, bool& ok) {
  if (!PyLong_CheckExact(x)) { ok = false; return 0; }
  int over = 0;
  const long long v = PyLong_AsLongLongAndOverflow(x, &over);
  if (over || v < INT32_MIN || v > INT32_MAX) { ok = false; return 0; }
  return (int32_t)v;
}
float number(PyObject* x, bool& ok) {
  if (PyFloat_CheckExact(x)) return (float)PyFloat_AS_DOUBLE(x);
  return (float)small_int(x, ok);
}
void* stream(PyObject* x) { return PyLong_AsVoidPtr(x); }   // the caller's own number

int dtype_of(const at::TensorBase& t, bool& ok) {
  if (t.scalar_type() == at::kFloat) return CKV_F32;
  if (t.scalar_type() == at::kBFloat16) return CKV_BF16;
  ok = false;
  return 0;
}
int32_t fits(int64_t v, bool& ok) {
  if (v < 0 || v > INT32_MAX) ok = false;
  return (int32_t)v;
}

// what layout_of() makes of a cache tensor and its degrees
ckv_layout layout(const at::TensorBase& t, const at::TensorBase* deg, bool& ok) {
  ckv_layout l{};
  if (t.dim() != 4) { ok = false; return l; }
  const auto n = t.sizes(), s = t.strides();
  l.dtype = dtype_of(t, ok);
  if (s[3] != 1) ok = false;
  l.batch = fits(n[0], ok); l.heads = fits(n[1], ok); l.seq = fits(n[2], ok); l.dim = fits(n[3], ok);
  l.stride_b = s[0]; l.stride_h = s[1]; l.stride_s = s[2];
  if (deg) {
    if (deg->scalar_type() != at::kInt || deg->dim() != 3 || deg->size(0) != n[0] || deg->size(1) != n[1] ||
        deg->size(2) != n[2] || (n[2] > 1 && deg->stride(2) != 1))
      ok = false;
    else {
      const auto d = deg->strides();
      l.deg_stride = n[1] > 1 ? d[1] : n[0] > 1 ? d[0] : n[2];
      if (n[0] > 1 && n[1] > 1 && d[0] != n[1] * d[1]) ok = false;
    }
  }
  return l;
}
bool rows_of(const at::TensorBase& t, int64_t b, int64_t h, int64_t d, at::ScalarType type) {
  return t.dim() == 3 && t.size(0) == b && t.size(1) == h && t.size(2) == d && t.is_contiguous() && t.scalar_type() == type;
}
ckv_paged_layout paged(const at::TensorBase& pool, const at::TensorBase& table, bool& ok) {
  ckv_paged_layout l{};
  if (pool.dim() != 4 || !pool.is_contiguous() || table.dim() != 2 || table.scalar_type() != at::kInt || !table.is_contiguous()) {
    ok = false;
    return l;
  }
  l.batch = fits(table.size(0), ok); l.heads = fits(pool.size(1), ok); l.dim = fits(pool.size(3), ok);
  l.dtype = dtype_of(pool, ok); l.block_size = fits(pool.size(2), ok); l.max_blocks = fits(table.size(1), ok);
  l.n_blocks = fits(pool.size(0), ok);
  return l;
}

// Counts the arguments, runs `body` (ok may turn false at any point) and turns its status into a Python number.
template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F&& body) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  bool ok = true;
  int status = 0;
  try {
    status = body(ok);
  } catch (...) {              // (a tensor without storage and the like: the ctypes route reports it)
    ok = false;
  }
  if (PyErr_Occurred()) PyErr_Clear();
  if (!ok) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}
template <typename F>
int unlocked(F&& call) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return status;
}

// K, V, deg, chunk, retain_ratio, rounds, n_sink, n_recent, scope, flags, K_out, V_out, deg_out, assign, workspace, stream
PyObject* compress(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&](bool& ok) -> int {
    const auto *K = given(a[0], ok), *V = given(a[1], ok), *deg = tensor(a[2], ok);
    const auto *oK = given(a[10], ok), *oV = given(a[11], ok), *od = given(a[12], ok), *assign = tensor(a[13], ok);
    const auto* ws = given(a[14], ok);
    ckv_params p{};
    p.chunk = small_int(a[3], ok);
    p.retain_ratio = number(a[4], ok);
    p.n_sink = small_int(a[6], ok);
    p.n_recent = small_int(a[7], ok);
    p.scope = small_int(a[8], ok);
    p.flags = (uint32_t)small_int(a[9], ok);
    if (a[5] != Py_None) {
      if (!PyList_CheckExact(a[5])) ok = false;
      else {
        const Py_ssize_t m = PyList_GET_SIZE(a[5]);
        if (m < 1 || m > CKV_MAX_ROUNDS) ok = false;
        else for (Py_ssize_t j = 0; j < m; ++j) p.r[j] = number(PyList_GET_ITEM(a[5], j), ok);
        p.n_rounds = (int32_t)m;
      }
    }
    if (!ok) return 0;
    const ckv_layout in = layout(*K, deg, ok), out = layout(*oK, od, ok);
    (void)layout(*V, nullptr, ok);
    if (!ok || V->scalar_type() != K->scalar_type() || V->sizes() != K->sizes()) { ok = false; return 0; }
    void *k = ptr(K), *v = ptr(V), *ok_p = ptr(oK), *ov = ptr(oV), *w = ptr(ws);
    const int32_t* d = ptr<int32_t>(deg);
    int32_t *dout = ptr<int32_t>(od), *as = ptr<int32_t>(assign);
    const size_t nw = (size_t)ws->numel();
    void* s = stream(a[15]);
    return unlocked([&] { return entry.compress(k, v, d, &in, &p, ok_p, ov, dout, &out, as, w, nw, s); });
  });
}

// k_new, v_new, K, V, deg, lens, pos, stream
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&](bool& ok) -> int {
    const auto *kn = given(a[0], ok), *vn = given(a[1], ok), *K = given(a[2], ok), *V = given(a[3], ok);
    const auto *deg = tensor(a[4], ok), *lens = tensor(a[5], ok);
    const int32_t pos = small_int(a[6], ok);
    if (!ok) return 0;
    const ckv_layout l = layout(*K, deg, ok);
    (void)layout(*V, nullptr, ok);
    if (!ok || !rows_of(*kn, l.batch, l.heads, l.dim, K->scalar_type()) || !rows_of(*vn, l.batch, l.heads, l.dim, K->scalar_type()) ||
        V->sizes() != K->sizes() || V->strides() != K->strides()) {
      ok = false;
      return 0;
    }
    void *k1 = ptr(kn), *v1 = ptr(vn), *k = ptr(K), *v = ptr(V), *s = stream(a[7]);
    int32_t *d = ptr<int32_t>(deg), *ls = ptr<int32_t>(lens);
    return unlocked([&] { return entry.append(k1, v1, k, v, d, &l, ls, pos, s); });
  });
}

// q, K, V, lens, deg, scale, out, workspace, stream
PyObject* decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&](bool& ok) -> int {
    const auto *q = given(a[0], ok), *K = given(a[1], ok), *V = given(a[2], ok), *lens = tensor(a[3], ok), *deg = tensor(a[4], ok);
    const auto *out = given(a[6], ok), *ws = given(a[7], ok);
    const float scale = number(a[5], ok);
    if (!ok) return 0;
    const ckv_layout l = layout(*K, deg, ok);
    const int o_type = dtype_of(*out, ok);
    if (!ok || q->dim() != 3 || !q->is_contiguous() || q->scalar_type() != K->scalar_type()) { ok = false; return 0; }
    const int32_t heads = fits(q->size(1), ok);
    void *qp = ptr(q), *k = ptr(K), *v = ptr(V), *o = ptr(out), *w = ptr(ws), *s = stream(a[8]);
    const int32_t *d = ptr<int32_t>(deg), *ls = ptr<int32_t>(lens);
    const size_t nw = (size_t)ws->numel();
    return unlocked([&] { return entry.decode_attn(qp, heads, k, v, &l, ls, d, scale, o, o_type, w, nw, s); });
  });
}

// k_new, v_new, K_pool, V_pool, deg_pool, block_table, lens, stream
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&](bool& ok) -> int {
    const auto *kn = given(a[0], ok), *vn = given(a[1], ok), *K = given(a[2], ok), *V = given(a[3], ok);
    const auto *deg = tensor(a[4], ok), *table = given(a[5], ok), *lens = given(a[6], ok);
    if (!ok) return 0;
    const ckv_paged_layout l = paged(*K, *table, ok);
    if (!ok || !rows_of(*kn, l.batch, l.heads, l.dim, K->scalar_type()) || !rows_of(*vn, l.batch, l.heads, l.dim, K->scalar_type())) {
      ok = false;
      return 0;
    }
    void *k1 = ptr(kn), *v1 = ptr(vn), *k = ptr(K), *v = ptr(V), *s = stream(a[7]);
    int32_t *d = ptr<int32_t>(deg), *ls = ptr<int32_t>(lens);
    const int32_t* t = ptr<int32_t>(table);
    return unlocked([&] { return entry.paged_append(k1, v1, k, v, d, t, ls, &l, s); });
  });
}

// q, K_pool, V_pool, deg_pool, block_table, lens, max_len, scale, out, workspace, stream
PyObject* paged_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&](bool& ok) -> int {
    const auto *q = given(a[0], ok), *K = given(a[1], ok), *V = given(a[2], ok), *deg = tensor(a[3], ok);
    const auto *table = given(a[4], ok), *lens = given(a[5], ok), *out = given(a[8], ok), *ws = given(a[9], ok);
    const int32_t max_len = small_int(a[6], ok);
    const float scale = number(a[7], ok);
    if (!ok) return 0;
    const ckv_paged_layout l = paged(*K, *table, ok);
    const int o_type = dtype_of(*out, ok);
    if (!ok || q->dim() != 3 || !q->is_contiguous() || q->scalar_type() != K->scalar_type()) { ok = false; return 0; }
    const int32_t heads = fits(q->size(1), ok);
    void *qp = ptr(q), *k = ptr(K), *v = ptr(V), *o = ptr(out), *w = ptr(ws), *s = stream(a[10]);
    const int32_t *d = ptr<int32_t>(deg), *ls = ptr<int32_t>(lens), *t = ptr<int32_t>(table);
    const size_t nw = (size_t)ws->numel();
    return unlocked([&] { return entry.paged_decode_attn(qp, heads, k, v, d, t, ls, &l, max_len, scale, o, o_type, w, nw, s); });
  });
}

// Tensor arguments of the calls below: contiguous, and all of one call on the GPU `device`.
struct Here {
  int32_t device;
  bool& ok;
  const at::TensorBase* take(PyObject* x) const {       // None is NULL
    const at::TensorBase* t = tensor(x, ok);
    if (t && t->get_device() != device) ok = false;
    return t;
  }
  const at::TensorBase* need(PyObject* x) const {
    const at::TensorBase* t = take(x);
    if (!t) ok = false;
    return t;
  }
  // int32 of these sizes (-1: any)
  const at::TensorBase* ints(PyObject* x, std::initializer_list<int64_t> shape, bool none = false) const {
    const at::TensorBase* t = none ? take(x) : need(x);
    if (!t) return t;
    bool fine = t->scalar_type() == at::kInt && t->dim() == (int64_t)shape.size() && t->is_contiguous();
    int64_t i = 0;
    for (const int64_t n : shape) { fine = fine && (n < 0 || t->size(i) == n); ++i; }
    if (!fine) ok = false;
    return t;
  }
};
int32_t listed_blocks(const at::TensorBase* list, bool& ok) {       // of a free list
  const int64_t n = list ? list->numel() : 0;
  if (n < 6 || n % 2) { ok = false; return 0; }
  return fits((n - 4) / 2, ok);
}
// pools of one shape and their degrees: heads, dim, dtype, block_size and n_blocks of a layout
ckv_paged_layout pools(const Here& at, PyObject* K, PyObject* V, PyObject* deg) {
  ckv_paged_layout l{};
  const auto *k = at.need(K), *v = at.need(V);
  if (!at.ok || k->dim() != 4 || !k->is_contiguous() || !v->is_contiguous() || v->sizes() != k->sizes() || v->scalar_type() != k->scalar_type()) {
    at.ok = false;
    return l;
  }
  l.dtype = dtype_of(*k, at.ok);
  l.n_blocks = fits(k->size(0), at.ok); l.heads = fits(k->size(1), at.ok);
  l.block_size = fits(k->size(2), at.ok); l.dim = fits(k->size(3), at.ok);
  l.batch = l.max_blocks = 1;
  at.ints(deg, {k->size(0), k->size(1), k->size(2)}, true);
  return l;
}
bool bounds_fit(const at::TensorBase* bounds, const at::TensorBase* mass, at::ScalarType type, int64_t dim) {
  return mass->dim() == 2 && bounds->dim() == 4 && bounds->is_contiguous() && bounds->scalar_type() == type &&
         bounds->size(0) == mass->size(0) && bounds->size(1) == mass->size(1) && bounds->size(2) == 2 && bounds->size(3) == dim;
}
size_t bytes_of(const at::TensorBase* t) { return (size_t)t->numel() * t->element_size(); }

// block_table, lens, n_new, free_list, block_size, n_slots, slots, starts, granted, device, stream
PyObject* paged_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&](bool& ok) -> int {
    const Here at{small_int(a[9], ok), ok};
    const auto *table = at.ints(a[0], {-1, -1}), *list = at.ints(a[3], {-1});
    if (!ok) return 0;
    const int64_t b = table->size(0);
    const int32_t bs = small_int(a[4], ok), n_slots = small_int(a[5], ok), blocks = listed_blocks(list, ok), width = fits(table->size(1), ok);
    if (n_slots < 0) ok = false;
    const auto *lens = at.ints(a[1], {b}), *fresh = at.ints(a[2], {b});
    const auto *slots = at.ints(a[6], {n_slots}), *starts = at.ints(a[7], {b + 1}), *granted = at.ints(a[8], {b});
    const int32_t batch = fits(b, ok);
    if (!ok) return 0;
    int32_t *t = ptr<int32_t>(table), *l = ptr<int32_t>(lens), *nn = ptr<int32_t>(fresh), *f = ptr<int32_t>(list);
    int32_t *sl = ptr<int32_t>(slots), *s0 = ptr<int32_t>(starts), *g = ptr<int32_t>(granted);
    void* s = stream(a[10]);
    return unlocked([&] { return tables.reserve(t, l, nn, f, batch, width, blocks, bs, sl, n_slots, s0, g, s); });
  });
}

// block_table, lens, new_lens, free_list, block_size, device, stream
PyObject* paged_trim(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&](bool& ok) -> int {
    const Here at{small_int(a[5], ok), ok};
    const auto *table = at.ints(a[0], {-1, -1}), *list = at.ints(a[3], {-1});
    if (!ok) return 0;
    const int32_t bs = small_int(a[4], ok), blocks = listed_blocks(list, ok), batch = fits(table->size(0), ok), width = fits(table->size(1), ok);
    const auto *lens = at.ints(a[1], {batch}), *cut = at.ints(a[2], {batch});
    if (!ok) return 0;
    int32_t *t = ptr<int32_t>(table), *l = ptr<int32_t>(lens), *c = ptr<int32_t>(cut), *f = ptr<int32_t>(list);
    void* s = stream(a[6]);
    return unlocked([&] { return tables.trim(t, l, c, f, batch, width, blocks, bs, s); });
  });
}

// k, v, slots, K_pool, V_pool, deg_pool, device, stream
PyObject* paged_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&](bool& ok) -> int {
    const Here at{small_int(a[6], ok), ok};
    const auto *k = at.need(a[0]), *v = at.need(a[1]), *slots = at.ints(a[2], {-1});
    const ckv_paged_layout l = pools(at, a[3], a[4], a[5]);
    if (!ok) return 0;
    const int32_t rows = fits(slots->numel(), ok);
    const auto type = l.dtype == CKV_BF16 ? at::kBFloat16 : at::kFloat;
    for (const auto* t : {k, v})
      if (t->dim() != 3 || t->size(0) != rows || t->size(1) != l.heads || t->size(2) != l.dim || t->scalar_type() != type || t->stride(2) != 1)
        ok = false;
    if (!ok) return 0;
    // (of a single row or head, whatever stride the tensor has there)
    auto row = [&](const at::TensorBase* t) { return rows > 1 ? t->stride(0) : (int64_t)l.heads * l.dim; };
    auto head = [&](const at::TensorBase* t) { return l.heads > 1 ? t->stride(1) : (int64_t)l.dim; };
    const int64_t k_row = row(k), k_head = head(k), v_row = row(v), v_head = head(v);
    void *kp = ptr(k), *vp = ptr(v), *K = ptr(tensor(a[3], ok)), *V = ptr(tensor(a[4], ok)), *s = stream(a[7]);
    int32_t *sl = ptr<int32_t>(slots), *d = ptr<int32_t>(tensor(a[5], ok));
    return unlocked([&] { return tables.write(kp, k_row, k_head, vp, v_row, v_head, sl, rows, K, V, d, &l, s); });
  });
}

// K_pool, deg_pool, block_table, lens, since, max_new, bounds, mass, device, stream
PyObject* paged_bounds(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&](bool& ok) -> int {
    const Here at{small_int(a[8], ok), ok};
    ckv_paged_layout l = pools(at, a[0], a[0], a[1]);
    const auto* table = at.ints(a[2], {-1, -1});
    if (!ok) return 0;
    l.batch = fits(table->size(0), ok);
    l.max_blocks = fits(table->size(1), ok);
    const int32_t max_new = small_int(a[5], ok);
    const auto *lens = at.ints(a[3], {l.batch}), *since = at.ints(a[4], {l.batch}, true);
    const auto *bounds = at.need(a[6]), *mass = at.ints(a[7], {l.n_blocks, l.heads});
    if (!ok || !bounds_fit(bounds, mass, l.dtype == CKV_BF16 ? at::kBFloat16 : at::kFloat, l.dim)) { ok = false; return 0; }
    void *K = ptr(tensor(a[0], ok)), *bp = ptr(bounds), *s = stream(a[9]);
    int32_t *d = ptr<int32_t>(tensor(a[1], ok)), *t = ptr<int32_t>(table), *ls = ptr<int32_t>(lens), *si = ptr<int32_t>(since);
    int32_t* m = ptr<int32_t>(mass);
    return unlocked([&] { return tables.bounds(K, d, t, ls, si, &l, max_new, bp, m, s); });
  });
}

// q, bounds, mass, block_table, lens, max_len, n_select, block_size, n_sink, n_recent, scale, sel, sel_lens, workspace, device, stream
PyObject* paged_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&](bool& ok) -> int {
    const Here at{small_int(a[14], ok), ok};
    const auto *q = at.need(a[0]), *bounds = at.need(a[1]), *mass = at.ints(a[2], {-1, -1}), *table = at.ints(a[3], {-1, -1});
    const auto* ws = at.need(a[13]);
    const int32_t max_len = small_int(a[5], ok), n_select = small_int(a[6], ok), n_sink = small_int(a[8], ok), n_recent = small_int(a[9], ok);
    const float scale = number(a[10], ok);
    ckv_paged_layout l{};
    l.block_size = small_int(a[7], ok);
    if (!ok || n_select < 1 || q->dim() != 3 || !q->is_contiguous() || table->size(0) != q->size(0) ||
        !bounds_fit(bounds, mass, q->scalar_type(), q->size(2))) {
      ok = false;
      return 0;
    }
    l.batch = fits(q->size(0), ok); l.heads = fits(mass->size(1), ok); l.dim = fits(q->size(2), ok); l.dtype = dtype_of(*q, ok);
    l.max_blocks = fits(table->size(1), ok); l.n_blocks = fits(mass->size(0), ok);
    const int32_t heads = fits(q->size(1), ok);
    const auto *lens = at.ints(a[4], {l.batch}), *sel = at.ints(a[11], {l.batch, l.heads, n_select}), *sl = at.ints(a[12], {l.batch, l.heads});
    if (!ok) return 0;
    void *qp = ptr(q), *bp = ptr(bounds), *w = ptr(ws), *s = stream(a[15]);
    int32_t *m = ptr<int32_t>(mass), *t = ptr<int32_t>(table), *ls = ptr<int32_t>(lens), *se = ptr<int32_t>(sel), *sn = ptr<int32_t>(sl);
    const size_t nw = bytes_of(ws);
    return unlocked([&] { return tables.select(qp, heads, bp, m, t, ls, &l, max_len, n_select, n_sink, n_recent, scale, se, sn, w, nw, s); });
  });
}

// q, K_pool, V_pool, deg_pool, sel, sel_lens, scale, out, workspace, device, stream
PyObject* paged_sparse_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&](bool& ok) -> int {
    const Here at{small_int(a[9], ok), ok};
    const auto *q = at.need(a[0]), *out = at.need(a[7]), *ws = at.need(a[8]);
    ckv_paged_layout l = pools(at, a[1], a[2], a[3]);
    const float scale = number(a[6], ok);
    if (!ok || q->dim() != 3 || !q->is_contiguous() || q->size(2) != l.dim || q->scalar_type() != (l.dtype == CKV_BF16 ? at::kBFloat16 : at::kFloat) ||
        !out->is_contiguous() || out->sizes() != q->sizes()) {
      ok = false;
      return 0;
    }
    l.batch = fits(q->size(0), ok);
    const int32_t heads = fits(q->size(1), ok);
    const int o_type = dtype_of(*out, ok);
    const auto *sel = at.ints(a[4], {l.batch, l.heads, -1}), *sl = at.ints(a[5], {l.batch, l.heads});
    if (!ok) return 0;
    const int32_t n_select = fits(sel->size(2), ok);
    if (!ok || n_select < 1) { ok = false; return 0; }
    l.max_blocks = n_select;
    void *qp = ptr(q), *K = ptr(tensor(a[1], ok)), *V = ptr(tensor(a[2], ok)), *o = ptr(out), *w = ptr(ws), *s = stream(a[10]);
    int32_t *d = ptr<int32_t>(tensor(a[3], ok)), *se = ptr<int32_t>(sel), *sn = ptr<int32_t>(sl);
    const size_t nw = bytes_of(ws);
    return unlocked([&] { return tables.sparse_attn(qp, heads, K, V, d, se, sn, &l, n_select, scale, o, o_type, w, nw, s); });
  });
}

// q, K_pool, V_pool, deg_pool, block_table, lens, starts, max_len, scale, causal, out, workspace, device, stream
PyObject* paged_chunk_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&](bool& ok) -> int {
    const Here at{small_int(a[12], ok), ok};
    const auto *q = at.need(a[0]), *out = at.need(a[10]), *ws = at.need(a[11]);
    ckv_paged_layout l = pools(at, a[1], a[2], a[3]);
    const auto* table = at.ints(a[4], {-1, -1});
    const int32_t max_len = small_int(a[7], ok);
    const float scale = number(a[8], ok);
    if (!PyBool_Check(a[9])) ok = false;
    if (!ok || q->dim() != 3 || q->stride(2) != 1 || q->size(2) != l.dim || q->scalar_type() != (l.dtype == CKV_BF16 ? at::kBFloat16 : at::kFloat) ||
        !out->is_contiguous() || out->sizes() != q->sizes() || !ws->is_contiguous()) {
      ok = false;
      return 0;
    }
    l.batch = fits(table->size(0), ok);
    l.max_blocks = fits(table->size(1), ok);
    const auto *lens = at.ints(a[5], {l.batch}), *starts = at.ints(a[6], {(int64_t)l.batch + 1});
    const int32_t rows = fits(q->size(0), ok), heads = fits(q->size(1), ok);
    const int o_type = dtype_of(*out, ok);
    if (!ok) return 0;
    // (of a single row or head, whatever stride the tensor has there)
    const int64_t q_row = rows > 1 ? q->stride(0) : (int64_t)heads * l.dim, q_head = heads > 1 ? q->stride(1) : (int64_t)l.dim;
    const int32_t causal = a[9] == Py_True;
    void *qp = ptr(q), *K = ptr(tensor(a[1], ok)), *V = ptr(tensor(a[2], ok)), *o = ptr(out), *w = ptr(ws), *s = stream(a[13]);
    int32_t *d = ptr<int32_t>(tensor(a[3], ok)), *t = ptr<int32_t>(table), *ls = ptr<int32_t>(lens), *s0 = ptr<int32_t>(starts);
    const size_t nw = bytes_of(ws);
    return unlocked([&] {
      return pages.chunk_attn(qp, q_row, q_head, heads, s0, rows, K, V, d, t, ls, &l, max_len, scale, causal, o, o_type, w, nw, s);
    });
  });
}

// block_table, lens, source, free_list, block_size, n_moves, moves, granted, device, stream
PyObject* paged_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&](bool& ok) -> int {
    const Here at{small_int(a[8], ok), ok};
    const auto *table = at.ints(a[0], {-1, -1}), *list = at.ints(a[3], {-1});
    if (!ok) return 0;
    const int32_t bs = small_int(a[4], ok), n_moves = small_int(a[5], ok), blocks = listed_blocks(list, ok);
    const int32_t batch = fits(table->size(0), ok), width = fits(table->size(1), ok);
    if (n_moves < 0) ok = false;
    const auto *lens = at.ints(a[1], {batch}), *source = at.ints(a[2], {batch}), *moves = at.ints(a[6], {n_moves, 2}), *granted = at.ints(a[7], {batch});
    if (!ok) return 0;
    int32_t *t = ptr<int32_t>(table), *l = ptr<int32_t>(lens), *f = ptr<int32_t>(list), *sr = ptr<int32_t>(source), *m = ptr<int32_t>(moves);
    int32_t* g = ptr<int32_t>(granted);
    void* s = stream(a[9]);
    return unlocked([&] { return pages.fork(t, l, sr, f, batch, width, blocks, bs, m, n_moves, g, s); });
  });
}

// block_table, lens, free_list, block_size, n_moves, moves, extent, workspace, device, stream
PyObject* paged_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&](bool& ok) -> int {
    const Here at{small_int(a[8], ok), ok};
    const auto *table = at.ints(a[0], {-1, -1}), *list = at.ints(a[2], {-1}), *ws = at.need(a[7]);
    if (!ok || !ws->is_contiguous()) { ok = false; return 0; }
    const int32_t bs = small_int(a[3], ok), n_moves = small_int(a[4], ok), blocks = listed_blocks(list, ok);
    const int32_t batch = fits(table->size(0), ok), width = fits(table->size(1), ok);
    if (n_moves < 0) ok = false;
    const auto *lens = at.ints(a[1], {batch}), *moves = at.ints(a[5], {n_moves, 2}), *extent = at.ints(a[6], {1});
    if (!ok) return 0;
    int32_t *t = ptr<int32_t>(table), *l = ptr<int32_t>(lens), *f = ptr<int32_t>(list), *m = ptr<int32_t>(moves), *e = ptr<int32_t>(extent);
    void *w = ptr(ws), *s = stream(a[9]);
    const size_t nw = bytes_of(ws);
    return unlocked([&] { return pages.compact(t, l, f, batch, width, blocks, bs, m, n_moves, e, w, nw, s); });
  });
}

// moves, K_pool, V_pool, deg_pool, bounds, mass, device, stream
PyObject* paged_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&](bool& ok) -> int {
    const Here at{small_int(a[6], ok), ok};
    const auto *moves = at.ints(a[0], {-1, 2}), *bounds = at.take(a[4]), *mass = at.ints(a[5], {-1, -1}, true);
    const ckv_paged_layout l = pools(at, a[1], a[2], a[3]);
    if (!ok || !bounds != !mass || (bounds && (mass->size(0) != l.n_blocks || mass->size(1) != l.heads ||
                                               !bounds_fit(bounds, mass, l.dtype == CKV_BF16 ? at::kBFloat16 : at::kFloat, l.dim)))) {
      ok = false;
      return 0;
    }
    const int32_t n_moves = fits(moves->size(0), ok);
    if (!ok) return 0;
    void *K = ptr(tensor(a[1], ok)), *V = ptr(tensor(a[2], ok)), *b = ptr(bounds), *s = stream(a[7]);
    int32_t *mv = ptr<int32_t>(moves), *d = ptr<int32_t>(tensor(a[3], ok)), *ms = ptr<int32_t>(mass);
    return unlocked([&] { return pages.copy(mv, n_moves, K, V, d, b, ms, &l, s); });
  });
}

// the addresses of the library's entry points, in Entry's order
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "five addresses");
    return nullptr;
  }
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  entry.compress = reinterpret_cast<decltype(&ckv_compress)>(p[0]);
  entry.append = reinterpret_cast<decltype(&ckv_append)>(p[1]);
  entry.decode_attn = reinterpret_cast<decltype(&ckv_decode_attn)>(p[2]);
  entry.paged_append = reinterpret_cast<decltype(&ckv_paged_append)>(p[3]);
  entry.paged_decode_attn = reinterpret_cast<decltype(&ckv_paged_decode_attn)>(p[4]);
  Py_RETURN_NONE;
}

// the same for Tables
PyObject* bind_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "six addresses");
    return nullptr;
  }
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  tables.reserve = reinterpret_cast<decltype(&ckv_paged_reserve)>(p[0]);
  tables.trim = reinterpret_cast<decltype(&ckv_paged_trim)>(p[1]);
  tables.write = reinterpret_cast<decltype(&ckv_paged_write_strided)>(p[2]);
  tables.bounds = reinterpret_cast<decltype(&ckv_paged_bounds)>(p[3]);
  tables.select = reinterpret_cast<decltype(&ckv_paged_select)>(p[4]);
  tables.sparse_attn = reinterpret_cast<decltype(&ckv_paged_sparse_decode_attn)>(p[5]);
  Py_RETURN_NONE;
}

// the same for Pages
PyObject* bind_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "four addresses");
    return nullptr;
  }
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  pages.chunk_attn = reinterpret_cast<decltype(&ckv_paged_chunk_attn)>(p[0]);
  pages.fork = reinterpret_cast<decltype(&ckv_paged_fork)>(p[1]);
  pages.compact = reinterpret_cast<decltype(&ckv_paged_compact)>(p[2]);
  pages.copy = reinterpret_cast<decltype(&ckv_paged_copy)>(p[3]);
  Py_RETURN_NONE;
}

#define CKV_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CKV_METHOD(bind), CKV_METHOD(compress), CKV_METHOD(append), CKV_METHOD(decode_attn),
                         CKV_METHOD(paged_append), CKV_METHOD(paged_decode_attn), CKV_METHOD(bind_tables),
                         CKV_METHOD(paged_reserve), CKV_METHOD(paged_trim), CKV_METHOD(paged_write), CKV_METHOD(paged_bounds),
                         CKV_METHOD(paged_select), CKV_METHOD(paged_sparse_decode_attn), CKV_METHOD(bind_pages),
                         CKV_METHOD(paged_chunk_attn), CKV_METHOD(paged_fork), CKV_METHOD(paged_compact), CKV_METHOD(paged_copy), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ckv_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ckv_binding(void) { return PyModule_Create(&module); }
