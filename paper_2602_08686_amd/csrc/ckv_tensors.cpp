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
  return t == at::kInt ? "int32" : t == at::kFloat ? "float32" : "bfloat16";
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

// (params, pages, device, q, k_pages, v_pages, table, length, count, out, lse, workspace); behind the addresses the workspace's bytes
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return checked(n, 12, [&] {
    const Struct<ckv_params> p(a[0]);
    const Struct<ckv_pages> g(a[1]);
    const at::ScalarType type = row_type(p.get());
    Tensors t(a[2]);
    t.add(a[3], "q", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim}, p->q_stride);
    add_pools(t, p.get(), g.get(), a[4], a[5]);
    t.add_table(a[6], p.get(), g.get());
    t.add(a[7], "length", at::kInt, {p->batch, p->n_kv_heads});
    t.add(a[8], "count", at::kInt, {p->batch, p->n_kv_heads});
    t.add_rows(a[9], "out", type, {p->batch, p->n_q_heads, p->seq_len, p->head_dim});
    t.add(a[10], "lse", at::kFloat, {p->batch, p->n_q_heads, p->seq_len});
    const Py_ssize_t bytes = t.add_bytes(a[11], "workspace");
    return t.addresses(bytes);
  });
}

PyMethodDef methods[] = {{"norm_rotate", (PyCFunction)(void (*)())norm_rotate, METH_FASTCALL, nullptr},
                         {"paged_append", (PyCFunction)(void (*)())paged_append, METH_FASTCALL, nullptr},
                         {"paged_attention", (PyCFunction)(void (*)())paged_attention, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "Tensors of the paged cache's calls, checked, and their addresses.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
