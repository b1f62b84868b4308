// Calls of the paged step's operators from Python without a detour: checks of tensors and the library's entry in one native call.
//
// A call of a few tokens is bound by its host work: 3.4 of 8 us were attribute reads in the interpreter (0.3 to 0.5 us a tensor), 0.8
// ctypes (four rows of heads: 8.3 us a call, 4.9 so; a turn of 64 sequences 15.1 and 8.3). Here only a sound call is
// recognised; for any other the answer is None, and the interpreter's checks say what is wrong with it or take what this file does
// not know (addresses, subclasses of tensors).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "dcl.h"

namespace {

struct {
  decltype(&dcl_pages_extend) extend;
  decltype(&dcl_pages_shrink) shrink;
  decltype(&dcl_heads_norm_rope) heads;
  decltype(&dcl_pages_write) write;
  decltype(&dcl_pages_read) read;
  decltype(&dcl_pages_attention) attention;
} entry;

// The arguments in their order; `sound` turns false at the first that is not as the call needs it.
struct Args {
  PyObject* const* arg;
  Py_ssize_t n, at = 0;
  int64_t dev = -1;
  bool sound = true;

  Args(PyObject* const* a, Py_ssize_t count, Py_ssize_t want) : arg(a), n(count) { sound = n == want; }
  PyObject* next() { return arg[at++]; }
  long long number(long long lo, long long hi) {
    PyObject* x = sound ? next() : nullptr;
    if (!x || !PyLong_Check(x)) return sound = false, 0;
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(x, &over);
    if (over || v < lo || v > hi) sound = false;
    return v;
  }
  int32_t i32() { return (int32_t)number(INT32_MIN, INT32_MAX); }
  int64_t size() { return number(0, INT64_MAX); }
  void* address() {  // of what is no tensor: never NULL but for the default stream
    PyObject* x = sound ? next() : nullptr;
    if (!x || !PyLong_Check(x)) return sound = false, nullptr;
    void* p = PyLong_AsVoidPtr(x);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      sound = false;
    }
    return p;
  }
  float f32() {
    PyObject* x = sound ? next() : nullptr;
    if (!x || !PyFloat_CheckExact(x)) return sound = false, 0.f;
    return (float)PyFloat_AS_DOUBLE(x);
  }
  // nullptr where it is None or no sound call
  const at::Tensor* tensor() {
    PyObject* x = sound ? next() : nullptr;
    if (!x || x == Py_None) return nullptr;
    if (!THPVariable_CheckExact(x)) return sound = false, nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != dev) return sound = false, nullptr;
    return &t;
  }
  void* flat(at::ScalarType type, int64_t numel) {
    const at::Tensor* t = tensor();
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->numel() < numel || !t->is_contiguous()) return sound = false, nullptr;
    return t->data_ptr();
  }
  static bool bits16(at::ScalarType t) { return t == at::kBFloat16 || t == at::kShort || t == at::kUInt16; }
  void* flat16(int64_t numel) {
    const at::Tensor* t = tensor();
    if (!t) return nullptr;
    if (!bits16(t->scalar_type()) || t->numel() < numel || !t->is_contiguous()) return sound = false, nullptr;
    return t->data_ptr();
  }
  void* space(int64_t* bytes) {  // the workspace, and how much of it there is to be
    const at::Tensor* t = tensor();
    *bytes = size();
    if (!t || !sound) return nullptr;
    if (t->numel() * (int64_t)t->element_size() < *bytes || !t->is_contiguous()) return sound = false, nullptr;
    return t->data_ptr();
  }
  // [>= T, heads, dim] of 16 bits, rows apart by any stride
  void* packed(int64_t T, int64_t heads, int64_t dim, int64_t* stride) {
    const at::Tensor* t = tensor();
    *stride = heads * dim;
    if (!t) return nullptr;
    if (t->dim() != 3 || t->size(0) < T || t->size(1) != heads || t->size(2) != dim || t->stride(2) != 1 ||
        (t->stride(1) != dim && heads != 1) || !bits16(t->scalar_type()))
      return sound = false, nullptr;
    if (T > 1) *stride = t->stride(0);
    return t->data_ptr();
  }
  int32_t* table(int64_t B, int32_t* width) {
    const at::Tensor* t = tensor();
    if (!t || t->dim() != 2 || t->size(1) > INT32_MAX || t->scalar_type() != at::kInt || t->numel() < B * t->size(1) || !t->is_contiguous())
      return sound = false, nullptr;
    *width = (int32_t)t->size(1);
    return static_cast<int32_t*>(t->data_ptr());
  }
  int32_t* ints(int64_t n) { return static_cast<int32_t*>(flat(at::kInt, n)); }
};

int64_t up(int64_t n) { return n < 0 ? 0 : n; }

// The body of a call: reads its arguments, and returns the library's status unless they are not sound.
template <class F>
PyObject* guarded(F&& body) {
  try {
    return body();
  } catch (...) {  // a tensor without memory of its own
    PyErr_Clear();
  }
  Py_RETURN_NONE;
}
#define CALL(status_of)           \
  do {                            \
    if (!a.sound) Py_RETURN_NONE; \
    dcl_status st;                \
    Py_BEGIN_ALLOW_THREADS        \
    st = status_of;               \
    Py_END_ALLOW_THREADS          \
    return PyLong_FromLong(st);   \
  } while (0)

// What all start with: the current device, its stream's handle; and the pool where there is one.
hipStream_t where(Args& a) {
  a.dev = a.number(0, 1 << 20);
  return static_cast<hipStream_t>(a.address());
}
const dcl_pages* pool_of(Args& a) {
  const dcl_pages* g = static_cast<const dcl_pages*>(a.address());
  if (!g) a.sound = false;
  return g;
}

PyObject* extend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 15);
    const hipStream_t s = where(a);
    const dcl_pages* g = pool_of(a);
    const int32_t B = a.i32(), T = a.i32();
    int32_t width = 0;
    int32_t *table = a.table(up(B), &width), *len = a.ints(up(B)), *count = a.ints(up(B));
    int32_t *list = a.ints(a.sound ? g->n_pages : 0), *n_free = a.ints(1), *cu = a.ints(up(B) + 1), *pos = a.ints(up(T));
    int64_t *slot = static_cast<int64_t*>(a.flat(at::kLong, up(T))), bytes;
    void* ws = a.space(&bytes);
    CALL(entry.extend(g, table, width, len, count, B, T, list, n_free, cu, pos, slot, ws, (size_t)bytes, s));
  });
}

PyObject* shrink(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 11);
    const hipStream_t s = where(a);
    const dcl_pages* g = pool_of(a);
    const int32_t B = a.i32();
    int32_t width = 0;
    int32_t *table = a.table(up(B), &width), *len = a.ints(up(B)), *keep = a.ints(up(B));
    int32_t *list = a.ints(a.sound ? g->n_pages : 0), *n_free = a.ints(1);
    int64_t bytes;
    void* ws = a.space(&bytes);
    CALL(entry.shrink(g, table, width, len, keep, B, list, n_free, ws, (size_t)bytes, s));
  });
}

PyObject* heads(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 16);
    const hipStream_t s = where(a);
    const int32_t T = a.i32(), H = a.i32(), Hkv = a.i32(), dim = a.i32(), rot = a.i32();
    const float eps = a.f32(), base = a.f32();
    if (H < 1 || Hkv < 1) a.sound = false;  // operands that are not there
    int64_t qs, qos, ks, kos;
    void *q = a.packed(T, H, dim, &qs), *q_out = a.packed(T, H, dim, &qos);
    void *k = a.packed(T, Hkv, dim, &ks), *k_out = a.packed(T, Hkv, dim, &kos);
    int32_t* pos = a.ints(T);
    float *gq = static_cast<float*>(a.flat(at::kFloat, dim)), *gk = static_cast<float*>(a.flat(at::kFloat, dim));
    CALL(entry.heads(q, qs, k, ks, pos, T, H, Hkv, dim, gq, gk, eps, base, rot, q_out, qos, k_out, kos, s));
  });
}

// What the calls over pages start with.
struct Batch {
  const dcl_pages* g;
  hipStream_t s;
  int32_t B, T, max_new, width = 0, *table, *len, *cu;
  explicit Batch(Args& a) {
    s = where(a);
    g = pool_of(a);
    B = a.i32(), T = a.i32(), max_new = a.i32();
    table = a.table(up(B), &width);
    len = a.ints(up(B)), cu = a.ints(up(B) + 1);
  }
};

PyObject* rows(PyObject* const* args, Py_ssize_t n, bool out) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 11);
    const Batch b(a);
    const int64_t h = a.sound ? b.g->n_kv_heads : 0, dim = a.sound ? b.g->head_dim : 0;
    int64_t ks, vs;
    void *k = a.packed(b.T, h, dim, &ks), *v = a.packed(b.T, h, dim, &vs);
    CALL(out ? entry.read(b.g, b.table, b.width, b.len, b.cu, b.B, b.T, b.max_new, k, ks, v, vs, b.s)
             : entry.write(b.g, b.table, b.width, b.len, b.cu, b.B, b.T, b.max_new, k, ks, v, vs, b.s));
  });
}
PyObject* write_rows(PyObject*, PyObject* const* args, Py_ssize_t n) { return rows(args, n, false); }
PyObject* read_rows(PyObject*, PyObject* const* args, Py_ssize_t n) { return rows(args, n, true); }

PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Args a(args, n, 17);
    const Batch b(a);
    const int32_t H = a.i32(), causal = a.i32();
    const float scale = a.f32();
    const int64_t dim = a.sound ? b.g->head_dim : 0, each = up(b.T) * H;
    int64_t qs, bytes;
    void *q = a.packed(b.T, H, dim, &qs), *out = a.flat16(each * dim);
    float* lse = static_cast<float*>(a.flat(at::kFloat, each));
    void* ws = a.space(&bytes);
    CALL(entry.attention(b.g, b.table, b.width, b.len, b.cu, b.B, b.T, b.max_new, q, qs, H, scale, causal, out, lse, ws, (size_t)bytes, b.s));
  });
}

// The library's entries, in the order of `entry`.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* p[6];
  if (n != 6) return PyErr_Format(PyExc_TypeError, "six addresses"), nullptr;
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : (PyErr_Format(PyExc_ValueError, "an address is 0"), nullptr);
  }
  entry = {reinterpret_cast<decltype(entry.extend)>(p[0]), reinterpret_cast<decltype(entry.shrink)>(p[1]),
           reinterpret_cast<decltype(entry.heads)>(p[2]), reinterpret_cast<decltype(entry.write)>(p[3]),
           reinterpret_cast<decltype(entry.read)>(p[4]), reinterpret_cast<decltype(entry.attention)>(p[5])};
  Py_RETURN_NONE;
}

PyMethodDef method(const char* name, PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}

}  // namespace

PyMODINIT_FUNC PyInit__operands() {
  static PyMethodDef methods[] = {
      method("bind", bind),
      method("pages_extend", extend),
      method("pages_shrink", shrink),
      method("heads_norm_rope", heads),
      method("pages_write", write_rows),
      method("pages_read", read_rows),
      method("pages_attention", attention),
      {nullptr, nullptr, 0, nullptr}};
  static PyModuleDef def = {PyModuleDef_HEAD_INIT, "_operands", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
  return PyModule_Create(&def);
}
