// What the binding asks of a tensor before a launch, each question in one call: a small operator takes a
// few microseconds on the GPU, and the same attributes read one by one from Python took as long again (0.7
// us per tensor).  Per call, back to back, with these questions instead: layer norm of 8 rows 4.3 us (6.7),
// rotary positions of 16 + 16 heads with their norm 6.8 (13), the projection of 8 tokens 10.5 (15.7).
// A tensor that is not as it should be is answered with None; the binding then finds out why.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <type_traits>

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

// [tokens, heads, 64] of a type, channels next to each other, on a device (pages: the rows of one more, outer
// dimension, which is left to the caller).
bool tiles_at(const at::Tensor* t, int dims, int code, const at::Tensor& like, ress_heads& h) {
  if (!t || t->dim() != dims || t->size(dims - 1) != RESS_HEAD_DIM || t->stride(dims - 1) != 1 || code_of(*t) != code ||
      t->device() != like.device())
    return false;
  h.data = t->data_ptr();
  h.token_stride = t->stride(dims - 3);
  h.head_stride = t->stride(dims - 2);
  return true;
}

// Contiguous int32 (or float32) numbers on like's device; n < 0: any number, which it becomes (None: null).
template <typename T>
bool numbers_at(PyObject* o, long long& n, const at::Tensor& like, T*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = cuda_tensor(o);
  if (!t || t->scalar_type() != (std::is_same<std::remove_const_t<T>, float>::value ? at::kFloat : at::kInt) ||
      !t->is_contiguous() || t->device() != like.device() || (n >= 0 && t->numel() != n))
    return false;
  n = t->numel();
  p = static_cast<T*>(t->data_ptr());
  return true;
}

// attn_args(q, k, v, o, lse, q_start, k_start, prefix, slopes, causal, cap, paged): the bytes of a ress_attn_args.
PyObject* attn_args(PyObject* const* args) {
  long long v[1];
  if (!integers(args + 9, v)) return nullptr;
  const double cap = PyFloat_AsDouble(args[10]);
  if (cap == -1.0 && PyErr_Occurred()) return nullptr;
  const bool paged = args[11] == Py_True;
  const int kd = paged ? 4 : 3;
  const at::Tensor *q = cuda_tensor(args[0]), *k = cuda_tensor(args[1]), *w = cuda_tensor(args[2]), *o = cuda_tensor(args[3]);
  ress_attn_args a = {};
  if (!q || !k || !o || code_of(*q) > 1) return none();
  a.type = code_of(*q);
  if (!tiles_at(q, 3, a.type, *q, a.q) || !tiles_at(k, kd, a.type, *q, a.k) || !tiles_at(w, kd, a.type, *q, a.v) ||
      !tiles_at(o, 3, a.type, *q, a.o) || o->sizes() != q->sizes() || w->sizes() != k->sizes())
    return none();
  a.rows = q->size(0), a.keys = paged ? 0 : k->size(0);
  if (q->size(1) > INT32_MAX || k->size(kd - 2) > INT32_MAX) return none();
  a.q_heads = static_cast<int32_t>(q->size(1)), a.kv_heads = static_cast<int32_t>(k->size(kd - 2));
  long long n = -1, all = a.rows * a.q_heads, heads = a.q_heads;
  if (!numbers_at(args[5], n, *q, a.q_start) || !numbers_at(args[6], n, *q, a.k_start) ||
      (!paged && (args[5] == Py_None) != (args[6] == Py_None)) || n == 0 || n > INT32_MAX)
    return none();
  a.n_seqs = n < 0 ? 1 : static_cast<int32_t>(n - 1);
  long long seqs = a.n_seqs;
  if (!numbers_at(args[7], seqs, *q, a.prefix) || !numbers_at(args[8], heads, *q, a.slopes) ||
      !numbers_at(args[4], all, *q, a.lse))
    return none();
  a.causal = v[0] != 0;
  a.cap = static_cast<float>(cap);
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&a), sizeof a);
}

// attn_grads(d_o, dq, dk, dv, q, k): the bytes of a ress_attn_grads.
PyObject* attn_grads(PyObject* const* args) {
  const at::Tensor *q = cuda_tensor(args[4]), *k = cuda_tensor(args[5]);
  ress_attn_grads g = {};
  ress_heads* to[4] = {&g.d_o, &g.dq, &g.dk, &g.dv};
  if (!q || !k) return none();
  for (int i = 0; i < 4; i++) {
    const at::Tensor* t = cuda_tensor(args[i]);
    if (!tiles_at(t, 3, code_of(*q), *q, *to[i]) || t->sizes() != (i < 2 ? q : k)->sizes()) return none();
  }
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&g), sizeof g);
}

// pages(k_pages, v_pages, table, lens, n_seqs): the bytes of a ress_pages.
PyObject* pages(PyObject* const* args) {
  long long v[1];
  if (!integers(args + 4, v)) return nullptr;
  const at::Tensor *k = cuda_tensor(args[0]), *w = cuda_tensor(args[1]), *t = cuda_tensor(args[2]);
  ress_pages p = {};
  if (!k || !w || k->dim() != 4 || w->dim() != 4 || !t || t->dim() != 2 || t->size(0) != v[0] || t->scalar_type() != at::kInt ||
      (t->size(1) > 1 && t->stride(1) != 1) || t->device() != k->device() || t->size(1) > INT32_MAX || k->size(1) > INT32_MAX ||
      args[3] == Py_None || !numbers_at(args[3], v[0], *k, p.lens))
    return none();
  p.table = static_cast<const int32_t*>(t->data_ptr());
  p.table_stride = t->stride(0), p.table_cols = static_cast<int32_t>(t->size(1));
  p.page = static_cast<int32_t>(k->size(1)), p.n_pages = k->size(0);
  p.k_page_stride = k->stride(0), p.v_page_stride = w->stride(0);
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&p), sizeof p);
}

// tables(have, add, free, taken, table, page, lens, q_start, slots, pos, taken_out): the bytes of a ress_tables.
PyObject* tables(PyObject* const* args) {
  long long v[1];
  if (!integers(args + 5, v)) return nullptr;
  const at::Tensor* t = cuda_tensor(args[4]);
  ress_tables r = {};
  if (!t || t->dim() != 2 || t->scalar_type() != at::kInt || (t->size(1) > 1 && t->stride(1) != 1) || t->size(0) > INT32_MAX ||
      t->size(1) > INT32_MAX || v[0] < 1 || v[0] > INT32_MAX)
    return none();
  for (int i = 0; i < 11; i++)
    if (i != 5 && args[i] == Py_None) return none();
  long long seqs = t->size(0), starts = seqs + 1, one = 1, more = 1, any = -1, slots = -1;
  if (!numbers_at(args[0], seqs, *t, r.have) || !numbers_at(args[1], seqs, *t, r.add) || !numbers_at(args[2], any, *t, r.free) ||
      !numbers_at(args[3], one, *t, r.taken) || !numbers_at(args[6], seqs, *t, r.lens) ||
      !numbers_at(args[7], starts, *t, r.q_start) || !numbers_at(args[8], slots, *t, r.slots) ||
      !numbers_at(args[9], slots, *t, r.pos) || !numbers_at(args[10], more, *t, r.taken_out))
    return none();
  r.table = static_cast<int32_t*>(t->data_ptr());
  r.n_seqs = static_cast<int32_t>(seqs), r.page = static_cast<int32_t>(v[0]);
  r.table_cols = static_cast<int32_t>(t->size(1)), r.table_stride = t->stride(0);
  r.n_free = any, r.n_slots = slots;
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&r), sizeof r);
}

// cache_rows(k, v, slots, k_pages, v_pages): what ress_cache_write takes but the workspace, as a tuple with the bytes of
// the four ress_heads.
PyObject* cache_rows(PyObject* const* args) {
  const at::Tensor *k = cuda_tensor(args[0]), *w = cuda_tensor(args[1]), *kp = cuda_tensor(args[3]), *vp = cuda_tensor(args[4]);
  ress_heads h[4];
  const int32_t* slots;
  if (!k || !w || !kp || !vp || code_of(*k) > 1 || args[2] == Py_None) return none();
  const int code = code_of(*k);
  if (!tiles_at(k, 3, code, *k, h[0]) || !tiles_at(w, 3, code, *k, h[1]) || !tiles_at(kp, 4, code, *k, h[2]) ||
      !tiles_at(vp, 4, code, *k, h[3]) || w->sizes() != k->sizes() || vp->sizes() != kp->sizes() || kp->size(2) != k->size(1) ||
      k->size(1) > INT32_MAX || kp->size(1) > INT32_MAX)
    return none();
  long long tokens = k->size(0);
  if (!numbers_at(args[2], tokens, *k, slots)) return none();
  const auto bytes = [&](int i) { return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&h[i]), sizeof h[i]); };
  return Py_BuildValue("LiNNNNNLLiL", tokens, static_cast<int>(k->size(1)), bytes(0), bytes(1),
                       PyLong_FromVoidPtr(const_cast<int32_t*>(slots)), bytes(2), bytes(3),
                       static_cast<long long>(kp->stride(0)), static_cast<long long>(vp->stride(0)),
                       static_cast<int>(kp->size(1)), static_cast<long long>(kp->size(0)));
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
                         method<attn_args, 12>("attn_args"), method<attn_grads, 6>("attn_grads"), method<pages, 5>("pages"), method<tables, 11>("tables"),
                         method<cache_rows, 5>("cache_rows"),
                         {"code", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry_code)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
