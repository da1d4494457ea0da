// What the binding asks of a tensor before a launch, each question in one call: a small operator takes a
// few microseconds on the GPU, and the same attributes read one by one from Python took as long again (0.7
// us per tensor).  Per call, back to back, with these questions instead: layer norm of 8 rows 4.3 us (6.7),
// rotary positions of 16 + 16 heads with their norm 6.8 (13), the projection of 8 tokens 10.5 (15.7).
// A tensor that is not as it should be is answered with None; the binding then finds out why.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "ress.h"

namespace {

// ress_dtype, or kBits: 16-bit integers, which hold the bits of bf16 from arrays without that type.
constexpr int kBits = 3, kOther = 4;

int code_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return 0;
    case at::kHalf: return 1;
    case at::kFloat: return 2;
    case at::kShort: case at::kUInt16: return kBits;
    default: return kOther;
  }
}

// The CUDA tensor that an object is, or null.
const at::Tensor* cuda_tensor(PyObject* o) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

PyObject* pointer(const at::Tensor& t) { return PyLong_FromVoidPtr(t.data_ptr()); }

PyObject* none() { Py_RETURN_NONE; }

// Integer arguments; false with an exception set.
template <int N>
bool integers(PyObject* const* args, long long (&out)[N]) {
  for (int i = 0; i < N; i++) {
    out[i] = PyLong_AsLongLong(args[i]);
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

// n contiguous elements of a type whose bit is set (None: null).
bool vector_at(PyObject* o, long long n, int types, const void*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = cuda_tensor(o);
  if (!t || t->numel() != n || !t->is_contiguous() || !(types >> code_of(*t) & 1)) return false;
  p = t->data_ptr();
  return true;
}

// [tokens, heads, head_dim] with contiguous channels (None: null); heads < 0: any number, which it becomes.
struct Heads {
  const void* p = nullptr;
  int64_t token = 0, head = 0;
};

bool heads_at(PyObject* o, long long tokens, long long& heads, long long head_dim, int code, Heads& h) {
  if (o == Py_None) return true;
  const at::Tensor* t = cuda_tensor(o);
  if (!t || t->dim() != 3 || t->size(0) != tokens || (heads >= 0 && t->size(1) != heads) || t->size(2) != head_dim ||
      code_of(*t) != code || t->stride(2) != 1)
    return false;
  heads = t->size(1);
  h = {t->data_ptr(), t->stride(0), t->stride(1)};
  return true;
}

// Two tensors or None (a tuple or list), or None for neither.
bool two(PyObject* o, PyObject*& a, PyObject*& b) {
  a = b = Py_None;
  if (o == Py_None) return true;
  if (!(PyTuple_Check(o) || PyList_Check(o)) || PySequence_Fast_GET_SIZE(o) != 2) return false;
  a = PySequence_Fast_GET_ITEM(o, 0);
  b = PySequence_Fast_GET_ITEM(o, 1);
  return true;
}

// vector(t, n, types): pointer of n contiguous elements of a type whose bit is set (t None: 0).
PyObject* vector(PyObject* const* args) {
  long long v[2];
  const void* p;
  if (!integers(args + 1, v)) return nullptr;
  return vector_at(args[0], v[0], static_cast<int>(v[1]), p) ? PyLong_FromVoidPtr(const_cast<void*>(p)) : none();
}

// rope_heads(y, x, dx, norm, grads, tokens, head_dim, ress_dtype): the bytes of a ress_rope_heads.
PyObject* rope_heads(PyObject* const* args) {
  long long v[3], n = -1;
  if (!integers(args + 5, v)) return nullptr;
  Heads y, x, dx;
  PyObject *w, *b, *dw, *db;
  ress_rope_heads r = {};
  const void *pdw, *pdb;
  for (int i = 0; i < 3; i++)
    if (!heads_at(args[i], v[0], n, v[1], static_cast<int>(v[2]), i == 0 ? y : i == 1 ? x : dx)) return none();
  if (n < 0 || n > INT32_MAX || !two(args[3], w, b) || !two(args[4], dw, db) || !vector_at(w, v[1], 7, r.norm.weight) ||
      !vector_at(b, v[1], 7, r.norm.bias) || !vector_at(dw, v[1], 4, pdw) || !vector_at(db, v[1], 4, pdb))
    return none();
  r.n_heads = static_cast<int32_t>(n);
  r.norm.enabled = args[3] != Py_None;
  const auto to = [](ress_heads& h, const Heads& t) {
    h.data = const_cast<void*>(t.p);
    h.token_stride = t.token;
    h.head_stride = t.head;
  };
  to(r.x, x), to(r.y, y), to(r.dx, dx);
  r.dweight = static_cast<float*>(const_cast<void*>(pdw));
  r.dbias = static_cast<float*>(const_cast<void*>(pdb));
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&r), sizeof r);
}

// shape(x): (rows, width, ress_dtype) of rows [..., width].
PyObject* shape(PyObject* const* args) {
  const at::Tensor* t = cuda_tensor(args[0]);
  if (!t || t->dim() < 1 || t->size(-1) < 1 || code_of(*t) >= kBits) return none();
  const long long width = t->size(-1);
  return Py_BuildValue("LLi", static_cast<long long>(t->numel()) / width, width, code_of(*t));
}

// rows(t, like): (pointer, elements between rows) of rows of like's shape.
PyObject* rows(PyObject* const* args) {
  const at::Tensor *t = cuda_tensor(args[0]), *like = cuda_tensor(args[1]);
  if (!t || !like || t->sizes() != like->sizes()) return none();
  if (t->is_contiguous()) return Py_BuildValue("NL", pointer(*t), static_cast<long long>(t->size(-1)));
  if (t->dim() != 2 || (t->stride(1) != 1 && t->size(1) != 1)) return none();
  return Py_BuildValue("NL", pointer(*t), static_cast<long long>(t->stride(0)));
}

// positions(t, tokens, axes): pointer of contiguous int32 [tokens, axes].
PyObject* positions(PyObject* const* args) {
  long long v[2];
  if (!integers(args + 1, v)) return nullptr;
  const at::Tensor* t = cuda_tensor(args[0]);
  return t && t->dim() == 2 && t->size(0) == v[0] && t->size(1) == v[1] && t->scalar_type() == at::kInt && t->is_contiguous()
             ? pointer(*t)
             : none();
}

// scratch(t): (pointer, bytes) of a workspace (t None: zeros).
PyObject* scratch(PyObject* const* args) {
  if (args[0] == Py_None) return Py_BuildValue("ii", 0, 0);
  const at::Tensor* t = cuda_tensor(args[0]);
  return t && t->is_contiguous() ? Py_BuildValue("NL", pointer(*t), static_cast<long long>(t->nbytes())) : none();
}

// code(*params): the one ress_dtype of those that are not None (float32 if none is given).
PyObject* code(PyObject* const* args, Py_ssize_t n) {
  int c = -1;
  for (Py_ssize_t i = 0; i < n; i++) {
    if (args[i] == Py_None) continue;
    if (!THPVariable_Check(args[i])) return none();
    const int ci = code_of(THPVariable_Unpack(args[i]));
    if (ci >= kBits || (c >= 0 && ci != c)) return none();
    c = ci;
  }
  return PyLong_FromLong(c < 0 ? 2 : c);
}

// Torch's C++ exceptions (a tensor without storage) end here.
template <typename F>
PyObject* guarded(F&& ask) {
  try {
    return ask();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
    return nullptr;
  }
}

// Python's entries: of a question with N arguments, and of code.
template <PyObject* (*ASK)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, n);
    return nullptr;
  }
  return guarded([&] { return ASK(args); });
}
PyObject* entry_code(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&] { return code(args, n); });
}

template <PyObject* (*ASK)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<ASK, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<vector, 3>("vector"), method<shape, 1>("shape"), method<rows, 2>("rows"),
                         method<rope_heads, 8>("rope_heads"), method<positions, 3>("positions"), method<scratch, 1>("scratch"),
                         {"code", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry_code)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
