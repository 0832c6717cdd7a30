// Argument marshalling of the Python binding, natively: tensors become device pointers, the parameter struct its
// address, the current torch stream the library's stream.  Nothing else happens here; every function
// forwards to the extern "C" entry point of its name and returns its status.
//
// A decode step launches one kernel of 5 to 8 us, and through ctypes a call cost 11 us of host time, five of them
// for fifteen attribute calls and argument conversions in the interpreter: an eager decode loop ran at the
// host's pace.  Measured per calidrop_decode call, host time: 11.2 -> 3.1 us; a
// token of eight layers, called layer by layer: 89 -> 59 us at 4 kv heads x 4333 rows, 89 -> 72 us at 32 x 2111.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/calidrop.h"

namespace {

#define CALIDROP_ENTRIES(X)                                                                                         \
  X(compress) X(calibrate) X(gather_evicted) X(recalibrate) X(accumulated_scores) X(select_from_scores)             \
  X(select_streaming) X(decode) X(decode_batched) X(decode_static)                                                  \
  X(paged_append) X(paged_prefill) X(paged_decode) X(paged_prefix_decode)
#define DECLARE(name) decltype(&calidrop_##name) f_##name = nullptr;
CALIDROP_ENTRIES(DECLARE)
#undef DECLARE
decltype(&calidrop_paged_workspace_bytes) f_paged_workspace_bytes = nullptr;

PyTypeObject* params_type = nullptr;   // the binding's ctypes structures (see open)
PyTypeObject* layer_type = nullptr;
PyTypeObject* paged_type = nullptr;

// The positional arguments of one call.  A conversion that fails sets a Python error, after which `ok` is
// false and the entry point is not called.
struct Args {
  PyObject* const* a;
  bool ok;
  Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : a(args), ok(n == want) {
    if (!ok) PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
  }
  // device pointer of a tensor, a raw address, or null for None
  void* ptr(int i) {
    PyObject* o = a[i];
    if (!ok || o == Py_None) return nullptr;
    if (PyLong_Check(o)) return address(o);
    if (THPVariable_CheckExact(o)) {
      // (torch throws for a tensor without memory of its own, sparse or wrapped: no exception may leave through
      // the interpreter's frames, and the tensor's own methods raise it properly)
      try {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_contiguous()) return t.data_ptr();
        not_contiguous();
        return nullptr;
      } catch (...) {
      }
    }
    // subclasses of torch.Tensor and anything else with its methods
    if (!method(o, "data_ptr")) return nullptr;
    PyObject* contiguous = call(o, "is_contiguous");
    if (!contiguous) return nullptr;
    const int c = PyObject_IsTrue(contiguous);
    Py_DECREF(contiguous);
    if (c < 0) ok = false;
    else if (c == 0) not_contiguous();
    if (!ok) return nullptr;
    PyObject* p = call(o, "data_ptr");
    if (!p) return nullptr;
    void* const r = address(p);
    Py_DECREF(p);
    return r;
  }
  size_t nbytes(int i) {
    PyObject* o = a[i];
    if (!ok) return 0;
    if (THPVariable_CheckExact(o)) {
      try {
        return THPVariable_Unpack(o).nbytes();
      } catch (...) {
      }
    }
    if (!method(o, "element_size")) return 0;
    size_t bytes = 1;
    for (const char* m : {"numel", "element_size"}) {
      PyObject* v = call(o, m);
      if (!v) return 0;
      bytes *= PyLong_AsSize_t(v);
      Py_DECREF(v);
      if (PyErr_Occurred()) { ok = false; return 0; }
    }
    return bytes;
  }
  void not_contiguous() {
    PyErr_SetString(PyExc_AssertionError, "tensors passed to the library must be contiguous");
    ok = false;
  }
  void* address(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) ok = false;
    return p;
  }
  bool method(PyObject* o, const char* name) {
    if (!PyObject_HasAttrString(o, name)) {
      PyErr_SetString(PyExc_TypeError, "a tensor, an address or None expected");
      ok = false;
    }
    return ok;
  }
  PyObject* call(PyObject* o, const char* name) {
    PyObject* r = PyObject_CallMethod(o, name, nullptr);
    if (!r) ok = false;
    return r;
  }
  int32_t i32(int i) {
    if (!ok) return 0;
    PyObject* o = PyLong_Check(a[i]) ? Py_NewRef(a[i]) : PyNumber_Long(a[i]);
    if (!o) { ok = false; return 0; }
    const long v = PyLong_AsLong(o);
    Py_DECREF(o);
    if (v == -1 && PyErr_Occurred()) ok = false;
    else if (v != (int32_t)v) { PyErr_SetString(PyExc_OverflowError, "argument out of the range of int32"); ok = false; }
    return (int32_t)v;
  }
  // address of a ctypes structure or array
  void* buf(int i) {
    Py_buffer v;
    if (PyObject_GetBuffer(a[i], &v, PyBUF_SIMPLE) != 0) { ok = false; return nullptr; }
    void* p = v.buf;
    PyBuffer_Release(&v);   // the caller holds the object for the length of the call
    return p;
  }
  Py_ssize_t len(int i) {
    if (!ok) return 0;
    const Py_ssize_t n = PyObject_Length(a[i]);
    if (n < 0) ok = false;
    return n;
  }
  // Structures are taken by their type, as ctypes would: a buffer of other bytes would be read as pointers and sizes.
  const calidrop_params* params(int i) {
    if (!ok) return nullptr;
    if (PyObject_TypeCheck(a[i], params_type)) return (const calidrop_params*)buf(i);
    PyErr_SetString(PyExc_TypeError, "a Params structure expected");
    ok = false;
    return nullptr;
  }
  const calidrop_paged_params* paged(int i) {
    if (!ok) return nullptr;
    if (PyObject_TypeCheck(a[i], paged_type)) return (const calidrop_paged_params*)buf(i);
    PyErr_SetString(PyExc_TypeError, "a PagedParams structure expected");
    ok = false;
    return nullptr;
  }
  // Device pointer of a tensor whose first dimension may have a stride of its own: `stride` elements (0: what its packed
  // form has), the others packed.  An address or None is taken as it is.
  void* rows(int i, int64_t stride) {
    PyObject* o = a[i];
    if (!ok || o == Py_None || !THPVariable_CheckExact(o)) return ptr(i);
    try {
      const at::Tensor& t = THPVariable_Unpack(o);
      int64_t want = 1;
      bool same = t.dim() > 0;
      for (int64_t d = t.dim() - 1; same && d >= 1; --d) {
        same = t.size(d) == 1 || t.stride(d) == want;
        want *= t.size(d);
      }
      same = same && (t.size(0) <= 1 || t.stride(0) == (stride ? stride : want));
      if (same) return t.data_ptr();
      PyErr_SetString(PyExc_AssertionError, "the tensor's strides are not those of the parameters");
      ok = false;
      return nullptr;
    } catch (...) {
    }
    return ptr(i);
  }
  // The tensor that an argument is, of a subclass or not; null: it is none, or None, or an address.
  const at::Tensor* tensor(int i) {
    PyObject* o = a[i];
    if (!ok || o == Py_None || PyLong_Check(o)) return nullptr;
    if (!THPVariable_CheckExact(o)) {
      const int is = THPVariableClass ? PyObject_IsInstance(o, THPVariableClass) : 0;
      if (is < 0) ok = false;
      if (is <= 0) return nullptr;
    }
    return &THPVariable_Unpack(o);
  }
  // No tensor of another device, and none of the host's: its address would mean nothing to the kernels.
  void on_this_device(Py_ssize_t n) {
    int device = -1;                     // the current one, asked for once
    for (Py_ssize_t i = 1; ok && i < n; ++i) {
      const at::Tensor* const x = tensor(i);
      if (!x) continue;
      try {
        const at::Tensor& t = *x;
        if (t.is_cuda() && device < 0) device = c10::cuda::current_device();
        if (t.is_cuda() && t.get_device() == device) continue;
        PyErr_SetString(PyExc_ValueError, "tensors on the current CUDA device expected");
      } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
      }
      ok = false;
    }
  }
  // Tensors hold elements of the type that the library reads there (what an address points at is the caller's word).
  void type(int i, const char* name, at::ScalarType want) {
    const at::Tensor* const x = tensor(i);
    if (!x || x->scalar_type() == want) return;
    PyErr_Format(PyExc_ValueError, "%s has elements of type %s, %s expected", name, c10::toString(x->scalar_type()), c10::toString(want));
    ok = false;
  }
  // ... and n rows of `row` elements.  A tensor whose dimensions behind the first make a row, `stride` elements apart (0: packed), has as
  // many as its first dimension says; of one in another shape that is packed the elements are counted (`shaped`: only of a single
  // row or a flat tensor, since the rows of a table would lie elsewhere).
  void size(int i, const char* name, int64_t n, int64_t row, int64_t stride = 0, bool shaped = false) {
    const at::Tensor* const x = tensor(i);
    if (!x) return;
    const int64_t dims = x->dim(), all = x->numel(), first = dims > 0 ? x->size(0) : 1;
    bool by_rows = dims > 0;
    if (by_rows) {
      int64_t behind = 1;
      for (int64_t d = 1; d < dims; ++d) behind *= x->size(d);
      by_rows = behind == row;
    }
    const bool counted = (stride == 0 || stride == row) && (!shaped || n <= 1 || dims <= 1);
    if (by_rows ? first >= n : counted && all >= n * row) return;
    PyErr_Format(PyExc_ValueError, "%s is too small or of another shape: %lld rows of %lld elements expected", name, (long long)n, (long long)row);
    ok = false;
  }
  // the first dimension of a tensor
  int32_t tokens(int i) {
    if (ok && THPVariable_CheckExact(a[i])) {
      try {
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (t.dim() > 0 && t.size(0) == (int32_t)t.size(0)) return (int32_t)t.size(0);
      } catch (...) {
      }
    }
    PyObject* s = ok ? PyObject_GetAttrString(a[i], "shape") : nullptr;
    PyObject* n = s ? PySequence_GetItem(s, 0) : nullptr;
    Py_XDECREF(s);
    const long v = n ? PyLong_AsLong(n) : -1;
    Py_XDECREF(n);
    if (!n || (v == -1 && PyErr_Occurred())) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "a tensor expected");
      ok = false;
      return 0;
    }
    if (v != (int32_t)v) { PyErr_SetString(PyExc_OverflowError, "more tokens than int32 counts"); ok = false; }
    return (int32_t)v;
  }
  const calidrop_decode_layer* layers(int i) {
    if (!ok) return nullptr;
    PyObject* element = PyObject_GetAttrString((PyObject*)Py_TYPE(a[i]), "_type_");   // of an array type
    if (!element) PyErr_Clear();
    const bool match = element && element == (PyObject*)layer_type && PyObject_CheckBuffer(a[i]);
    Py_XDECREF(element);
    if (match) return (const calidrop_decode_layer*)buf(i);
    PyErr_SetString(PyExc_TypeError, "an array of DecodeLayer structures expected");
    ok = false;
    return nullptr;
  }
  void* stream() {
    if (!ok) return nullptr;
    try {
      return (void*)c10::cuda::getCurrentCUDAStream().stream();
    } catch (const std::exception& e) {
      PyErr_SetString(PyExc_RuntimeError, e.what());
      ok = false;
      return nullptr;
    }
  }
};

// (the arguments are converted in any order: one that fails turns the later ones into nulls, and no call is made)
template <typename F, typename... A>
PyObject* forward(Args& x, F f, A... v) {
  if (!x.ok) return nullptr;
  void* const stream = x.stream();
  if (!x.ok) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS   // a launch may have to wait for room in the stream's queue
  rc = f(v..., stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

#define ENTRY(name, n_args, ...)                                                        \
  PyObject* py_##name(PyObject*, PyObject* const* args, Py_ssize_t n) {                 \
    Args x(args, n, n_args);                                                            \
    if (!x.ok) return nullptr;                                                          \
    return forward(x, f_##name, __VA_ARGS__);                                           \
  }

ENTRY(compress, 12, x.params(0), x.ptr(1), x.ptr(2), x.ptr(3), (const float*)x.ptr(4), (int32_t*)x.ptr(5), x.ptr(6),
      x.ptr(7), (float*)x.ptr(8), (float*)x.ptr(9), x.ptr(10), x.ptr(11), x.nbytes(11))
ENTRY(calibrate, 12, x.params(0), x.ptr(1), x.ptr(2), x.ptr(3), (const float*)x.ptr(4), (const int32_t*)x.ptr(5),
      x.ptr(6), x.ptr(7), (float*)x.ptr(8), (float*)x.ptr(9), x.ptr(10), x.ptr(11), x.nbytes(11))
ENTRY(gather_evicted, 8, x.params(0), x.ptr(1), x.ptr(2), (const int32_t*)x.ptr(3), (int32_t*)x.ptr(4), x.ptr(5),
      x.ptr(6), x.ptr(7), x.nbytes(7))
ENTRY(recalibrate, 10, x.params(0), x.ptr(1), x.ptr(2), x.ptr(3), x.i32(4), x.i32(5), (float*)x.ptr(6),
      (float*)x.ptr(7), x.ptr(8), x.ptr(9), x.nbytes(9))
ENTRY(accumulated_scores, 5, x.params(0), x.ptr(1), x.ptr(2), (float*)x.ptr(3), x.ptr(4), x.nbytes(4))
ENTRY(select_from_scores, 5, x.params(0), (const float*)x.ptr(1), x.i32(2), (int32_t*)x.ptr(3), x.ptr(4), x.nbytes(4))
ENTRY(select_streaming, 3, x.params(0), x.i32(1), (int32_t*)x.ptr(2))
ENTRY(decode, 14, x.params(0), x.ptr(1), x.ptr(2), x.ptr(3), x.ptr(4), x.ptr(5), x.i32(6), (const float*)x.ptr(7),
      (const float*)x.ptr(8), x.ptr(9), x.ptr(10), (float*)x.ptr(11), (uint8_t*)x.ptr(12), x.ptr(13), x.nbytes(13))
ENTRY(decode_batched, 4, x.params(0), (int32_t)x.len(1), x.layers(1), x.i32(2), x.ptr(3),
      x.nbytes(3))
ENTRY(decode_static, 13, x.params(0), x.ptr(1), x.ptr(2), x.ptr(3), x.ptr(4), x.ptr(5), x.i32(6), (const float*)x.ptr(7),
      (const float*)x.ptr(8), x.ptr(9), x.ptr(10), (float*)x.ptr(11), (uint8_t*)x.ptr(12))

// What the tensors of the entry points over a cache in pages have to be.  Parameters that the library refuses are left to it.
struct PagedCheck {
  Args& x;
  const calidrop_paged_params* p;
  int64_t n;                                           // tokens
  const at::ScalarType half;
  PagedCheck(Args& x, const calidrop_paged_params* p, int64_t n)
      : x(x), p(p), n(n), half(p->dtype == CALIDROP_FP16 ? at::kHalf : at::kBFloat16) {}
  void heads(int i, const char* name, int64_t count, int64_t stride = 0) {             // of the tokens
    x.type(i, name, half);
    x.size(i, name, n, count * p->D, stride);
  }
  void pages(int i, const char* name) {
    x.type(i, name, half);
    const at::Tensor* const t = x.tensor(i);
    if (t && t->dim() == 4 && (t->size(1) != p->Hkv || t->size(2) != p->page_size || t->size(3) != p->D)) {
      PyErr_Format(PyExc_ValueError, "%s: pages of [Hkv][page_size][D] elements expected", name);
      x.ok = false;
    }
    x.size(i, name, p->n_pages, (int64_t)p->Hkv * p->page_size * p->D, p->page_stride);
  }
  void ints(int i, const char* name, int64_t count) {
    x.type(i, name, at::kInt);
    x.size(i, name, count, 1);
  }
  void table(int i, const char* name, int64_t count, int64_t row) {
    x.type(i, name, at::kInt);
    x.size(i, name, count, row, 0, true);
  }
  void floats(int i, const char* name, int64_t count, int64_t row, bool shaped) {
    x.type(i, name, at::kFloat);
    x.size(i, name, count, row, 0, shaped);
  }
};

void check_paged_append(PagedCheck c) {
  const calidrop_paged_params* p = c.p;
  c.heads(1, "q", p->Hq, p->q_stride); c.heads(2, "k", p->Hkv, p->k_stride); c.heads(3, "v", p->Hkv, p->v_stride);
  c.ints(4, "positions", c.n);
  if (p->rot_dim) c.floats(5, "cos_sin", p->max_pos, p->rot_dim, true);
  c.pages(6, "K_pages"); c.pages(7, "V_pages");
  c.table(8, "block_table", p->B, p->max_pages); c.ints(9, "q_start", (int64_t)p->B + 1); c.ints(10, "kv_len", p->B);
  if (c.x.a[1] != Py_None) c.heads(11, "q_out", p->Hq);
}
void check_paged_prefill(PagedCheck c) {
  const calidrop_paged_params* p = c.p;
  c.heads(1, "q", p->Hq, p->q_stride); c.pages(2, "K_pages"); c.pages(3, "V_pages");
  c.table(4, "block_table", p->B, p->max_pages); c.ints(5, "q_start", (int64_t)p->B + 1); c.ints(6, "kv_len", p->B);
  c.heads(7, "out", p->Hq); c.floats(8, "lse", c.n, p->Hq, false);
}
void check_paged_decode(PagedCheck c) {
  const calidrop_paged_params* p = c.p;
  c.heads(1, "q", p->Hq, p->q_stride); c.pages(2, "K_pages"); c.pages(3, "V_pages");
  c.table(4, "block_table", p->B, p->max_pages); c.ints(5, "kv_len", p->B);
  c.heads(6, "out", p->Hq); c.floats(7, "lse", c.n, p->Hq, false);
}
void check_paged_prefix_decode(PagedCheck c) {
  const calidrop_paged_params* p = c.p;
  c.heads(1, "q", p->Hq, p->q_stride); c.pages(2, "K_pages"); c.pages(3, "V_pages");
  c.ints(4, "group_start", (int64_t)p->n_groups + 1); c.table(5, "prefix_table", p->n_groups, p->max_prefix_pages);
  c.ints(6, "prefix_len", p->n_groups);
  c.table(7, "block_table", p->B, p->max_pages); c.ints(8, "kv_len", p->B);
  c.heads(9, "out", p->Hq); c.floats(10, "lse", c.n, p->Hq, false);
}

#define PAGED_ENTRY(name, n_args, n_tokens, ...)                                                  \
  PyObject* py_##name(PyObject*, PyObject* const* args, Py_ssize_t n) {                 \
    Args x(args, n, n_args);                                                            \
    const calidrop_paged_params* p = x.paged(0);                                        \
    const int32_t count = x.ok ? n_tokens : 0;                                          \
    if (x.ok && f_paged_workspace_bytes(p, 0)) check_##name(PagedCheck(x, p, count));   \
    x.on_this_device(n);                                                                \
    if (!x.ok) return nullptr;                                                          \
    return forward(x, f_##name, p, __VA_ARGS__);                                        \
  }
PAGED_ENTRY(paged_append, 13, x.tokens(2), count, x.rows(1, p->q_stride), x.rows(2, p->k_stride), x.rows(3, p->v_stride),
            (const int32_t*)x.ptr(4), (const float*)x.ptr(5), x.rows(6, p->page_stride), x.rows(7, p->page_stride),
            (const int32_t*)x.ptr(8), (const int32_t*)x.ptr(9), (const int32_t*)x.ptr(10), x.ptr(11), x.ptr(12), x.nbytes(12))
PAGED_ENTRY(paged_prefill, 10, x.tokens(1), count, x.rows(1, p->q_stride), x.rows(2, p->page_stride), x.rows(3, p->page_stride),
            (const int32_t*)x.ptr(4), (const int32_t*)x.ptr(5), (const int32_t*)x.ptr(6), x.ptr(7), (float*)x.ptr(8), x.ptr(9),
            x.nbytes(9))
PAGED_ENTRY(paged_decode, 9, p->B, x.rows(1, p->q_stride), x.rows(2, p->page_stride), x.rows(3, p->page_stride),
            (const int32_t*)x.ptr(4), (const int32_t*)x.ptr(5), x.ptr(6), (float*)x.ptr(7), x.ptr(8), x.nbytes(8))
PAGED_ENTRY(paged_prefix_decode, 12, p->B, x.rows(1, p->q_stride), x.rows(2, p->page_stride), x.rows(3, p->page_stride),
            (const int32_t*)x.ptr(4), (const int32_t*)x.ptr(5), (const int32_t*)x.ptr(6), (const int32_t*)x.ptr(7),
            (const int32_t*)x.ptr(8), x.ptr(9), (float*)x.ptr(10), x.ptr(11), x.nbytes(11))

// open(path, Params, DecodeLayer, PagedParams): the shared library whose entry points the functions forward to, and the ctypes
// structures of its arguments
PyObject* py_open(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4 || !PyType_Check(args[1]) || !PyType_Check(args[2]) || !PyType_Check(args[3]))
    return PyErr_Format(PyExc_TypeError, "a path and three structure types expected");
  const size_t sizes[4] = {0, sizeof(calidrop_params), sizeof(calidrop_decode_layer), sizeof(calidrop_paged_params)};
  const char* s = PyUnicode_AsUTF8(args[0]);
  if (!s) return nullptr;
  for (int i = 1; i < 4; ++i) {
    PyObject* o = PyObject_CallNoArgs(args[i]);
    Py_buffer v;
    if (!o) return nullptr;
    const bool buffer = PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) == 0;
    Py_DECREF(o);
    if (!buffer) return nullptr;
    const bool same = v.len == (Py_ssize_t)sizes[i];
    PyBuffer_Release(&v);
    if (!same) return PyErr_Format(PyExc_TypeError, "the structure's size is not the library's");
  }
  void* h = dlopen(s, RTLD_NOW | RTLD_LOCAL);
  if (!h) return PyErr_Format(PyExc_ImportError, "%s", dlerror());
#define RESOLVE(name)                                                                               \
  f_##name = (decltype(f_##name))dlsym(h, "calidrop_" #name);                                        \
  if (!f_##name) return PyErr_Format(PyExc_ImportError, "%s does not export calidrop_" #name, s);
  CALIDROP_ENTRIES(RESOLVE)
  RESOLVE(paged_workspace_bytes)
#undef RESOLVE
  params_type = (PyTypeObject*)Py_NewRef(args[1]);
  layer_type = (PyTypeObject*)Py_NewRef(args[2]);
  paged_type = (PyTypeObject*)Py_NewRef(args[3]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"open", (PyCFunction)(void (*)(void))py_open, METH_FASTCALL, nullptr},
#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr},
    CALIDROP_ENTRIES(METHOD)
#undef METHOD
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
