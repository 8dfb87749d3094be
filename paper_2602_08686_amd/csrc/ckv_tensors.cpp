// What the binding hands to the paged cache's calls: tensors as the structs of the call describe them, or a ValueError, and their addresses. A kernel
// reads what an address says; a tensor of another type, shape or layout would be read past its end or in another order. In C++ because the
// checks then take no longer than asking each tensor for its address did (host time of a call of eight tensors, the library's part aside: 1.2 us
// without checks, 0.9 with these; asked one by one from Python, the same questions take some 3 us).
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "ckv.h"

namespace {

// A ctypes structure's memory; null for None.
template <class T>
class Struct {
 public:
  explicit Struct(PyObject *o) {
    if (o == Py_None) return;
    if (PyObject_GetBuffer(o, &view_, PyBUF_SIMPLE) != 0) throw std::invalid_argument("a structure of the library is needed");
    held_ = true;
    if (view_.len != (Py_ssize_t)sizeof(T)) throw std::invalid_argument("a structure of the library has another size");
  }
  ~Struct() {
    if (held_) PyBuffer_Release(&view_);
  }
  Struct(const Struct &) = delete;
  const T *get() const { return held_ ? static_cast<const T *>(view_.buf) : nullptr; }
  const T *operator->() const { return get(); }

 private:
  Py_buffer view_;
  bool held_ = false;
};

const char *type_name(at::ScalarType t) {
  return t == at::kInt ? "int32" : t == at::kLong ? "int64" : t == at::kFloat ? "float32" : "bfloat16";
}

class Tensors {
 public:
  explicit Tensors(PyObject *device) : device_(PyLong_AsLong(device)) {}

  // One of these sizes and this type; dense, or with the given strides of the axes in front of the last (an axis of one entry has any).
  void add(PyObject *o, const char *name, at::ScalarType type, std::initializer_list<int64_t> sizes, const int64_t *strides = nullptr) {
    const at::Tensor *t = tensor(o, name);
    if (t) {
      bool ok = t->scalar_type() == type && t->dim() == (int64_t)sizes.size();
      int i = 0;
      for (const int64_t size : sizes) ok = ok && t->size(i++) == size;
      if (!ok || !laid_out(*t, strides)) refuse(name, type, sizes, strides ? "with the strides that the call describes" : "contiguous");
    }
  }
  // Any strides, the last axis contiguous: the binding takes them from the tensor.
  void add_rows(PyObject *o, const char *name, at::ScalarType type, std::initializer_list<int64_t> sizes) {
    const at::Tensor *t = tensor(o, name);
    if (t) {
      bool ok = t->scalar_type() == type && t->dim() == (int64_t)sizes.size() && t->stride(-1) == 1;
      int i = 0;
      for (const int64_t size : sizes) ok = ok && t->size(i++) == size;
      if (!ok) refuse(name, type, sizes, "with a contiguous last axis");
    }
  }
  void add_table(PyObject *o, const ckv_params *p, const ckv_pages *g) {
    const at::Tensor *t = tensor(o, "table");
    if (t) {
      const bool all = t->dim() == 2;
      bool ok = t->scalar_type() == at::kInt && (all || t->dim() == 3) && t->size(0) == p->batch && t->size(-1) == g->max_pages;
      ok = ok && (t->size(-1) == 1 || t->stride(-1) == 1) && (t->size(0) == 1 || t->stride(0) == g->table_stride[0]);
      ok = ok && (all ? p->n_kv_heads == 1 || g->table_stride[1] == 0
                      : t->size(1) == p->n_kv_heads && (t->size(1) == 1 || t->stride(1) == g->table_stride[1]));
      if (!ok) refuse("table", at::kInt, {p->batch, p->n_kv_heads, g->max_pages}, "(or without the heads' axis) with the strides that the pages describe");
    }
  }
  // Of lists, as the call describes them.
  void add_list(PyObject *o, const char *name, const ckv_lists *l) {
    const at::Tensor *t = tensor(o, name);
    if (!t) return;
    const bool all = t->dim() == 2;
    bool ok = t->scalar_type() == at::kInt && (all || t->dim() == 3) && t->size(0) == l->batch && t->size(-1) == l->max_pages;
    ok = ok && (t->size(-1) == 1 || t->stride(-1) == 1) && (t->size(0) == 1 || t->stride(0) == l->table_stride[0]);
    ok = ok && (all ? l->n_kv_heads == 1 || l->table_stride[1] == 0
                    : t->size(1) == l->n_kv_heads && (t->size(1) == 1 || t->stride(1) == l->table_stride[1]));
    if (!ok) refuse(name, at::kInt, {l->batch, l->n_kv_heads, l->max_pages}, "(or without the heads' axis) with the strides that the lists describe");
  }
  // Numbers of rows that stay, one list for all heads of a sequence or one for each: any strides over the axes in front of the last.
  const at::Tensor &add_idx(PyObject *o, const ckv_params *p) {
    const at::Tensor *t = needed(o, "idx");
    bool ok = t->scalar_type() == at::kInt && (t->dim() == 2 || t->dim() == 3) && t->size(0) == p->batch && t->size(-1) > 0;
    ok = ok && t->size(-1) <= INT32_MAX && (t->size(-1) == 1 || t->stride(-1) == 1) && (t->dim() == 2 || t->size(1) == p->n_kv_heads);
    if (!ok) refuse("idx", at::kInt, {p->batch, p->n_kv_heads, t->dim() > 0 ? t->size(-1) : 0}, "(or without the heads' axis) with a contiguous last axis");
    return *t;
  }
  // Of a tensor's own sizes, as many axes as `dims`; added by add() with them. The library takes such a size as an int32.
  static const at::Tensor &sized(PyObject *o, const char *name, int64_t dims) {
    if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != dims)
      throw std::invalid_argument(std::string(name) + " has to be a tensor of " + std::to_string(dims) + " axes");
    const at::Tensor &t = THPVariable_Unpack(o);
    for (const int64_t size : t.sizes())
      if (size > INT32_MAX) throw std::invalid_argument(std::string(name) + " has to be a tensor of axes below 2^31");
    return t;
  }
  // Bytes, of any type.
  Py_ssize_t add_bytes(PyObject *o, const char *name) {
    const at::Tensor *t = tensor(o, name);
    if (!t) return 0;
    if (!t->is_contiguous()) throw std::invalid_argument(std::string(name) + " has to be contiguous");
    return (Py_ssize_t)t->nbytes();
  }

  // Their addresses, in the order of the additions, and `more` as an entry behind them if that is not negative.
  PyObject *addresses(Py_ssize_t more = -1) const {
    for (int i = 0; i < n_; ++i) {
      if (!tensors_[i]) continue;
      const int64_t at = tensors_[i]->is_cuda() ? (int64_t)tensors_[i]->get_device() : -1;
      if (at < 0 || (device_ >= 0 && at != device_))
        throw std::invalid_argument(std::string(names_[i]) + " has to be on the GPU of the call's stream");
    }
    PyObject *out = PyTuple_New(n_ + (more >= 0));
    if (!out) return nullptr;
    for (int i = 0; i < n_; ++i) {
      PyObject *x = tensors_[i] ? PyLong_FromVoidPtr(tensors_[i]->data_ptr()) : nullptr;
      if (!tensors_[i]) Py_INCREF(x = Py_None);
      PyTuple_SET_ITEM(out, i, x);
    }
    if (more >= 0) PyTuple_SET_ITEM(out, n_, PyLong_FromSsize_t(more));
    return out;
  }

 private:
  const at::Tensor *needed(PyObject *o, const char *name) {
    const at::Tensor *t = tensor(o, name);
    if (!t) throw std::invalid_argument(std::string(name) + " has to be a tensor");
    return t;
  }
  const at::Tensor *tensor(PyObject *o, const char *name) {
    const at::Tensor *t = nullptr;
    if (o != Py_None) {
      if (!THPVariable_Check(o)) throw std::invalid_argument(std::string(name) + " has to be a tensor or None");
      t = &THPVariable_Unpack(o);
      if (t->layout() != at::kStrided) throw std::invalid_argument(std::string(name) + " has to be a strided tensor");
    }
    names_[n_] = name;
    tensors_[n_++] = t;
    return t;
  }
  static bool laid_out(const at::Tensor &t, const int64_t *strides) {
    if (!strides) return t.is_contiguous();
    for (int64_t i = 0; i + 1 < t.dim(); ++i)
      if (t.size(i) > 1 && t.stride(i) != strides[i]) return false;
    return t.stride(-1) == 1;
  }
  [[noreturn]] static void refuse(const char *name, at::ScalarType type, std::initializer_list<int64_t> sizes, const char *how) {
    std::string text = std::string(name) + " has to be " + type_name(type) + " [";
    for (const int64_t size : sizes) text += std::to_string(size) + ",";
    text.back() = ']';
    throw std::invalid_argument(text + " " + how);
  }

  int64_t device_;
  int n_ = 0;
  const char *names_[16];
  const at::Tensor *tensors_[16];
};

at::ScalarType row_type(const ckv_params *p) {
  if (!p) throw std::invalid_argument("params are needed");
  if (p->dtype != CKV_F32 && p->dtype != CKV_BF16) throw std::invalid_argument("params name no type");
  return p->dtype == CKV_F32 ? at::kFloat : at::kBFloat16;
}

void add_transform(Tensors &t, const ckv_params *p, const ckv_rotation *r, PyObject *positions, PyObject *inv_freq, PyObject *q_weight, PyObject *k_weight) {
  const bool turned = r && r->rot_dim > 0, normed = r && r->norm;   // what is not read may be anything
  const at::ScalarType type = row_type(p);
  t.add(turned ? positions : Py_None, "positions", at::kInt, {p->batch, p->seq_len});
  t.add(turned ? inv_freq : Py_None, "inv_freq", at::kFloat, {turned ? r->rot_dim / 2 : 0});
  t.add(normed ? q_weight : Py_None, "q_weight", type, {p->head_dim});
  t.add(normed ? k_weight : Py_None, "k_weight", type, {p->head_dim});
}

void add_pools(Tensors &t, const ckv_params *p, const ckv_pages *g, PyObject *k_pages, PyObject *v_pages) {
  if (!g) throw std::invalid_argument("pages are needed");
  t.add(k_pages, "k_pages", row_type(p), {g->n_pages, p->n_kv_heads, g->page_rows, p->head_dim}, g->k_stride);
  t.add(v_pages, "v_pages", row_type(p), {g->n_pages, p->n_kv_heads, g->page_rows, p->head_dim}, g->v_stride);
}

// Calls `body`, exceptions turned into Python's.
template <class Body>
PyObject *checked(Py_ssize_t n, Py_ssize_t expected, Body body) {
  try {
    if (n != expected) throw std::invalid_argument("wrong number of arguments");
    return body();
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_ValueError, "a tensor that cannot be described");
  }
  return nullptr;
}

// (params, rotation, device, q, k, positions, inv_freq, q_weight, k_weight, count, q_out, k_out); device: index, -1 for any GPU
PyObject *norm_rotate(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 12, [&] {
    const Struct<ckv_params> p(a[0]);
    const Struct<ckv_rotation> r(a[1]);
    const at::ScalarType type = row_type(p.get());
    Tensors t(a[2]);
    t.add(a[3], "q", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim}, p->q_stride);
    t.add(a[4], "k", type, {p->batch, p->n_kv_heads, p->seq_len, p->head_dim}, p->k_stride);
    add_transform(t, p.get(), r.get(), a[5], a[6], a[7], a[8]);
    t.add(a[9], "count", at::kInt, {p->batch, p->n_kv_heads});
    t.add(a[10], "q_out", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim});
    t.add(a[11], "k_out", type, {p->batch, p->n_kv_heads, p->seq_len, p->head_dim});
    return t.addresses();
  });
}

// (params, rotation or None, pages, device, q, k, v, positions, inv_freq, q_weight, k_weight, table, length, count, k_pages, v_pages, q_out)
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 17, [&] {
    const Struct<ckv_params> p(a[0]);
    const Struct<ckv_rotation> r(a[1]);
    const Struct<ckv_pages> g(a[2]);
    const at::ScalarType type = row_type(p.get());
    Tensors t(a[3]);
    t.add(a[4], "q", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim}, p->q_stride);
    t.add(a[5], "k", type, {p->batch, p->n_kv_heads, p->seq_len, p->head_dim}, p->k_stride);
    t.add(a[6], "v", type, {p->batch, p->n_kv_heads, p->seq_len, p->head_dim}, p->v_stride);
    add_transform(t, p.get(), r.get(), a[7], a[8], a[9], a[10]);
    if (!g.get()) throw std::invalid_argument("pages are needed");
    t.add_table(a[11], p.get(), g.get());
    t.add(a[12], "length", at::kInt, {p->batch, p->n_kv_heads});
    t.add(a[13], "count", at::kInt, {p->batch, p->n_kv_heads});
    add_pools(t, p.get(), g.get(), a[14], a[15]);
    t.add(a[16], "q_out", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim});
    return t.addresses();
  });
}

// (params, pages, device, q, k_pages, v_pages, table, length, count, out, lse, workspace), and for trees sees in front of out; behind the
// addresses the workspace's bytes
template <bool TREE>
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 12 + TREE, [&] {
    const Struct<ckv_params> p(a[0]);
    const Struct<ckv_pages> g(a[1]);
    const at::ScalarType type = row_type(p.get());
    Tensors t(a[2]);
    t.add(a[3], "q", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim}, p->q_stride);
    add_pools(t, p.get(), g.get(), a[4], a[5]);
    t.add_table(a[6], p.get(), g.get());
    t.add(a[7], "length", at::kInt, {p->batch, p->n_kv_heads});
    t.add(a[8], "count", at::kInt, {p->batch, p->n_kv_heads});
    if (TREE) t.add(a[9], "sees", at::kLong, {p->batch, p->seq_len, ((int64_t)p->seq_len + 63) / 64});
    t.add_rows(a[9 + TREE], "out", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim});
    t.add(a[10 + TREE], "lse", at::kFloat, {p->batch, p->n_q_heads, p->seq_len});
    const Py_ssize_t bytes = t.add_bytes(a[11 + TREE], "workspace");
    return t.addresses(bytes);
  });
}

// The entries of `made` with `more` in front of entry `at`; both references are taken over.
PyObject *with(PyObject *made, Py_ssize_t at, std::initializer_list<PyObject *> more) {
  const Py_ssize_t n = made ? PyTuple_GET_SIZE(made) : 0;
  PyObject *out = made ? PyTuple_New(n + (Py_ssize_t)more.size()) : nullptr;
  Py_ssize_t to = 0;
  for (Py_ssize_t i = 0; i <= n; ++i) {
    if (i == at)
      for (PyObject *x : more) {
        if (out) PyTuple_SET_ITEM(out, to++, x);
        else Py_XDECREF(x);
      }
    if (out && i < n) {
      PyObject *x = PyTuple_GET_ITEM(made, i);
      Py_INCREF(x);
      PyTuple_SET_ITEM(out, to++, x);
    }
  }
  Py_XDECREF(made);
  return out;
}

// (device, parent, start, sees, positions); in front of the addresses batch and tokens
PyObject *tree_sees(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 5, [&] {
    const at::Tensor &parent = Tensors::sized(a[1], "parent", 2);
    const int64_t batch = parent.size(0), tokens = parent.size(1);
    Tensors t(a[0]);
    t.add(a[1], "parent", at::kInt, {batch, tokens});
    t.add(a[2], "start", at::kInt, {batch});
    t.add(a[3], "sees", at::kLong, {batch, tokens, (tokens + 63) / 64});
    t.add(a[4], "positions", at::kInt, {batch, tokens});
    PyObject *at = t.addresses();
    return with(at, 0, {PyLong_FromLongLong(batch), PyLong_FromLongLong(tokens)});
  });
}

// (params, pages, device, table, length, count, idx, kept, k_pages, v_pages, length_out); behind the address of idx its strides and length
PyObject *paged_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 11, [&] {
    const Struct<ckv_params> p(a[0]);
    const Struct<ckv_pages> g(a[1]);
    row_type(p.get());
    if (!g.get()) throw std::invalid_argument("pages are needed");
    Tensors t(a[2]);
    t.add_table(a[3], p.get(), g.get());
    t.add(a[4], "length", at::kInt, {p->batch, p->n_kv_heads});
    t.add(a[5], "count", at::kInt, {p->batch, p->n_kv_heads});
    const at::Tensor &idx = t.add_idx(a[6], p.get());
    t.add(a[7], "kept", at::kInt, {p->batch, p->n_kv_heads});
    add_pools(t, p.get(), g.get(), a[8], a[9]);
    t.add(a[10], "length_out", at::kInt, {p->batch, p->n_kv_heads});
    const int64_t strides[2] = {idx.stride(0), idx.dim() == 3 ? idx.stride(1) : 0};
    PyObject *at = t.addresses();
    return with(at, 4, {PyBytes_FromStringAndSize(reinterpret_cast<const char *>(strides), sizeof strides), PyLong_FromLongLong(idx.size(-1))});
  });
}

// (params, pages, device, copy, k_pages, v_pages); behind the address of copy the number of pairs
PyObject *pages_copy(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 6, [&] {
    const Struct<ckv_params> p(a[0]);
    const Struct<ckv_pages> g(a[1]);
    row_type(p.get());
    const int64_t pairs = Tensors::sized(a[3], "copy", 2).size(0);
    Tensors t(a[2]);
    t.add(a[3], "copy", at::kInt, {pairs, 2});
    add_pools(t, p.get(), g.get(), a[4], a[5]);
    PyObject *at = t.addresses();
    return with(at, 1, {PyLong_FromLongLong(pairs)});
  });
}

void add_counts(Tensors &t, const ckv_lists *l, PyObject *refs, PyObject *taken) {
  t.add(refs, "refs", at::kInt, {l->n_pages});
  t.add(taken, "taken", at::kInt, {((int64_t)l->n_pages + 31) / 32});
}

const ckv_lists *needed(const Struct<ckv_lists> &l) {
  if (!l.get()) throw std::invalid_argument("lists are needed");
  return l.get();
}

// (lists, device, table, parent, table_out, refs, taken, length, length_out)
PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 9, [&] {
    const Struct<ckv_lists> held(a[0]);
    const ckv_lists *l = needed(held);
    Tensors t(a[1]);
    t.add_list(a[2], "table", l);
    t.add(a[3], "parent", at::kInt, {l->batch});
    t.add_list(a[4], "table_out", l);
    add_counts(t, l, a[5], a[6]);
    t.add(a[7], "length", at::kInt, {l->batch, l->n_kv_heads});
    t.add(a[8], "length_out", at::kInt, {l->batch, l->n_kv_heads});
    return t.addresses();
  });
}

// (lists, device, table, first, end, refs, taken, copy, result); behind the address of copy the number of its pairs
PyObject *pages_reserve(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 9, [&] {
    const Struct<ckv_lists> held(a[0]);
    const ckv_lists *l = needed(held);
    const int64_t pairs = a[7] == Py_None ? 0 : Tensors::sized(a[7], "copy", 2).size(0);
    Tensors t(a[1]);
    t.add_list(a[2], "table", l);
    t.add(a[3], "first", at::kInt, {l->batch, l->n_kv_heads});
    t.add(a[4], "end", at::kInt, {l->batch, l->n_kv_heads});
    add_counts(t, l, a[5], a[6]);
    t.add(a[7], "copy", at::kInt, {pairs, 2});
    t.add(a[8], "result", at::kInt, {2});
    PyObject *at = t.addresses();
    return with(at, 6, {PyLong_FromLongLong(pairs)});
  });
}

// (lists, device, table, keep, refs, taken)
PyObject *pages_free(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 6, [&] {
    const Struct<ckv_lists> held(a[0]);
    const ckv_lists *l = needed(held);
    Tensors t(a[1]);
    t.add_list(a[2], "table", l);
    t.add(a[3], "keep", at::kInt, {l->batch, l->n_kv_heads});
    add_counts(t, l, a[4], a[5]);
    return t.addresses();
  });
}

template <class F>
PyMethodDef method(const char *name, F f) { return {name, (PyCFunction)(void (*)())f, METH_FASTCALL, nullptr}; }

PyMethodDef methods[] = {method("norm_rotate", norm_rotate),
                         method("paged_append", paged_append),
                         method("paged_attention", paged_attention<false>),
                         method("paged_tree_attention", paged_attention<true>),
                         method("tree_sees", tree_sees),
                         method("paged_compact", paged_compact),
                         method("pages_copy", pages_copy),
                         method("pages_fork", pages_fork),
                         method("pages_reserve", pages_reserve),
                         method("pages_free", pages_free),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "Tensors of the paged cache's calls, checked, and their addresses.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
