// gm_torch.cpp -- the operators over a paged cache on torch tensors, for ops.py: the
// checks of tensors and the C structs are made here, in a module that Python calls
// directly.  Through ctypes and Python the host side of a call took 8.4 us (attention)
// and 10.2 us (append with queries), longer than the kernels of a decode step run.
//
// Functions return a tensor, or the code of a gm_* call that refused; wrong tensors raise
// ValueError.  The device is current already, and the stream belongs to it.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>

#include <climits>
#include <initializer_list>
#include <sstream>
#include <string>
#include <vector>

#include "gm.h"

namespace {

struct Refused {};     // a Python error is set

[[noreturn]] void refuse(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor, not %s", name, Py_TYPE(o)->tp_name);
    throw Refused();
  }
  return THPVariable_Unpack(o);
}

std::string told(at::IntArrayRef sizes) {
  std::ostringstream s;
  s << "(";
  for (size_t i = 0; i < sizes.size(); ++i) s << (i ? ", " : "") << sizes[i];
  s << ")";
  return s.str();
}

// A contiguous array of `sizes`; NULL for None.
const void* array(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes,
                  const at::Tensor& k) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.sizes() != at::IntArrayRef(sizes) || !t.is_contiguous() || t.device() != k.device()) {
    std::ostringstream s;
    s << name << " must be a contiguous " << at::toString(type) << " tensor of shape " << told(sizes) << " on "
      << k.device().str();
    refuse(s.str());
  }
  return t.data_ptr();
}

int32_t small(int64_t x, const char* name) {
  if (x > INT_MAX) refuse(std::string(name) + " is too large");
  return static_cast<int32_t>(x);
}

// New tokens [*tokens, heads, head_dim] like `first`, in its first dimensions.
gm_tensor rows(const at::Tensor& t, const char* name, const at::Tensor& first, int64_t heads, int64_t head_dim,
               const at::Tensor& k) {
  const int64_t d = first.dim();
  bool ok = t.dim() == d && t.scalar_type() == k.scalar_type() && t.device() == k.device();
  for (int64_t i = 0; ok && i < d - 2; ++i) ok = t.size(i) == first.size(i);
  if (!ok || t.size(d - 2) != heads || t.size(d - 1) != head_dim) {
    std::vector<int64_t> want(first.sizes().begin(), first.sizes().end());
    want[d - 2] = heads;
    want[d - 1] = head_dim;
    std::ostringstream s;
    s << name << " must be " << at::toString(k.scalar_type()) << " of shape " << told(want) << " on " << k.device().str()
      << ", not " << at::toString(t.scalar_type()) << " of " << told(t.sizes()) << " on " << t.device().str();
    refuse(s.str());
  }
  if (t.stride(d - 1) != 1 && t.numel()) refuse(std::string("the channels of ") + name + " must be contiguous");
  return gm_tensor{t.data_ptr(), d == 4 ? t.stride(0) : 0, t.stride(d - 3), t.stride(d - 2)};
}

gm_paged_rows places(const at::Tensor& t, const char* name, PyObject* table_, PyObject* lengths, PyObject* offsets,
                     const at::Tensor& k) {
  const at::Tensor& table = tensor(table_, "table");
  if (table.dim() != 2 || table.scalar_type() != at::kInt || table.device() != k.device() ||
      (table.size(1) > 1 && table.stride(1) != 1))
    refuse("table must be an int32 tensor [batch, width] with contiguous rows on " + k.device().str());
  const int64_t B = table.size(0);
  if (offsets == Py_None) {
    if (t.dim() != 4 || t.size(0) != B)
      refuse(std::string(name) + " must be [batch, tokens, heads, head_dim] of the table's " + std::to_string(B) +
             " sequences without offsets, not " + told(t.sizes()));
  } else if (t.dim() != 3) {
    refuse(std::string(name) + " must be [tokens, heads, head_dim] with offsets");
  }
  if (lengths == Py_None) refuse("lengths is missing");
  gm_paged_rows r;
  r.B = small(B, "the batch");
  r.n = small(t.size(t.dim() - 3), "the number of tokens");
  r.width = small(table.size(1), "the table's width");
  r.table_stride = table.stride(0);
  r.table = static_cast<const int32_t*>(table.data_ptr());
  r.lengths = static_cast<const int32_t*>(array(lengths, "lengths", at::kInt, {B}, k));
  r.offsets = static_cast<const int32_t*>(array(offsets, "offsets", at::kInt, {B + 1}, k));
  return r;
}

const gm_paged_cache* cache_at(PyObject* address) {
  const gm_paged_cache* c = static_cast<const gm_paged_cache*>(PyLong_AsVoidPtr(address));
  if (PyErr_Occurred()) throw Refused();
  return c;
}
// The pools of a cache, (k, v) or k alone: the struct holds the addresses that they had when
// it was made, and calls are refused once they lie elsewhere (resized, or given other memory).
const at::Tensor& pool_of(PyObject* o, const gm_paged_cache* c) {
  const bool both = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2;
  const at::Tensor& k = tensor(both ? PyTuple_GET_ITEM(o, 0) : o, "the cache");
  if (k.data_ptr() != c->k || (both && tensor(PyTuple_GET_ITEM(o, 1), "the cache").data_ptr() != c->v))
    refuse("the cache's k or v is not where it was when the cache was made");
  return k;
}
hipStream_t stream_at(PyObject* handle) {
  void* s = PyLong_AsVoidPtr(handle);
  if (PyErr_Occurred()) throw Refused();
  return static_cast<hipStream_t>(s);
}
float number(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (PyErr_Occurred()) throw Refused();
  return static_cast<float>(x);
}

// `out`, or a new contiguous tensor like `like`.
at::Tensor output(PyObject* out, const char* name, const at::Tensor& like) {
  return out == Py_None ? at::empty(like.sizes(), like.options()) : tensor(out, name);
}
PyObject* returned(PyObject* out, const at::Tensor& t) {
  if (out == Py_None) return THPVariable_Wrap(t);
  Py_INCREF(out);
  return out;
}

template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Refused&) {
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    if (type) PyErr_SetString(type, e.what_without_backtrace());
    Py_XDECREF(type);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// (cache address, its pools, k, v, table, lengths, offsets, cos, sin, q, q_out, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 12) refuse("12 arguments are wanted");
    gm_paged_append_args g;
    g.cache = cache_at(a[0]);
    const at::Tensor &pool = pool_of(a[1], g.cache), &k = tensor(a[2], "k"), &v = tensor(a[3], "v");
    g.rows = places(k, "k", a[4], a[5], a[6], pool);
    const int64_t hd = g.cache->head_dim;
    g.k = rows(k, "k", k, g.cache->heads, hd, pool);
    g.v = rows(v, "v", k, g.cache->heads, hd, pool);
    g.rot = 0;
    g.cos = g.sin = nullptr;
    g.positions = 0;
    if (a[7] != Py_None) {
      const at::Tensor& cos = tensor(a[7], "cos");
      if (cos.dim() != 2) refuse("cos must be [positions, r / 2]");
      g.positions = cos.size(0);
      g.rot = small(2 * cos.size(1), "r");
      g.cos = static_cast<const float*>(array(a[7], "cos", at::kFloat, {cos.size(0), cos.size(1)}, pool));
      g.sin = static_cast<const float*>(array(a[8], "sin", at::kFloat, {cos.size(0), cos.size(1)}, pool));
    } else if (a[8] != Py_None) {
      refuse("sin needs cos");
    }
    g.n_q_heads = 0;
    g.q = g.q_out = gm_tensor{nullptr, 0, 0, 0};
    at::Tensor out;
    if (a[9] != Py_None) {
      const at::Tensor& q = tensor(a[9], "q");
      if (q.dim() != k.dim()) refuse("q must have as many dimensions as k");
      const int64_t heads = q.size(q.dim() - 2);
      g.n_q_heads = small(heads, "the number of heads");
      g.q = rows(q, "q", k, heads, hd, pool);
      out = output(a[10], "q_out", q);
      g.q_out = rows(out, "q_out", k, heads, hd, pool);
    } else if (a[10] != Py_None) {
      refuse("q_out needs q");
    }
    const hipStream_t stream = stream_at(a[11]);
    int rc;
    // (a launch may wait for room in the queue)
    Py_BEGIN_ALLOW_THREADS
    rc = gm_paged_append(&g, stream);
    Py_END_ALLOW_THREADS
    if (rc) return PyLong_FromLong(rc);
    if (a[9] == Py_None) Py_RETURN_NONE;
    return returned(a[10], out);
  });
}

// (cache address, its pools, q, table, lengths, offsets, window, softcap, slopes, scale, out, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 12) refuse("12 arguments are wanted");
    gm_paged_attention_args g;
    g.cache = cache_at(a[0]);
    const at::Tensor &pool = pool_of(a[1], g.cache), &q = tensor(a[2], "q");
    g.rows = places(q, "q", a[3], a[4], a[5], pool);
    const int64_t heads = q.size(q.dim() - 2);
    g.n_heads = small(heads, "the number of heads");
    g.q = rows(q, "q", q, heads, g.cache->head_dim, pool);
    const long window = PyLong_AsLong(a[6]);
    if (PyErr_Occurred()) throw Refused();
    g.window = window < 0 || window > INT_MAX ? -1 : static_cast<int32_t>(window);
    g.scores.softcap = number(a[7]);
    g.scores.slopes = static_cast<const float*>(array(a[8], "slopes", at::kFloat, {heads}, pool));
    g.scores.scale = number(a[9]);
    const at::Tensor out = output(a[10], "out", q);
    g.out = rows(out, "out", q, heads, g.cache->head_dim, pool);
    g.workspace_bytes = gm_paged_attention_workspace(g.cache, g.rows.B, g.rows.n, g.rows.width, g.n_heads, g.window,
                                                     g.rows.offsets != nullptr);
    at::Tensor work;
    g.workspace = nullptr;
    if (g.workspace_bytes) {
      work = at::empty({static_cast<int64_t>(g.workspace_bytes)}, q.options().dtype(at::kByte));
      g.workspace = work.data_ptr();
    }
    const hipStream_t stream = stream_at(a[11]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = gm_paged_attention(&g, stream);
    Py_END_ALLOW_THREADS
    return rc ? PyLong_FromLong(rc) : returned(a[10], out);
  });
}

PyMethodDef methods[] = {
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gm_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gm_torch() { return PyModule_Create(&module); }
