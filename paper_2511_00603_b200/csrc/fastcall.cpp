// Python side of epara_collect without ctypes.  A serving loop asks once per request, so that a step of forty small requests
// spends as long in the foreign-function call (0.8 us an answer) as in everything else it does on the host; here an answer is
// 0.4 us, the library's own work included.  (Two small MLPs, 8 + 32 requests: 72 us a step through ctypes, 52 like this.)
// The calls of the 8-bit decoder layer, whose sixteen and more arguments ctypes takes 1.5 us to convert, half as long as the launch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>

#include "../../include/epara.h"

namespace {

struct Collect {
  int (*fn)(void* ctx, uint64_t ticket, void* out);
  int (*ready)(void* ctx, uint64_t ticket, void* out);   // the same for answers that are there already
  int pending;           // its answer for the others
  PyObject* out_type;    // the ctypes structure that an answer is returned in
  PyObject* general;     // the same method through ctypes, for calls of any other form
  PyObject* handle;      // name of the attribute that holds the context's address as an int
};

void free_collect(PyObject* capsule) {
  Collect* c = static_cast<Collect*>(PyCapsule_GetPointer(capsule, nullptr));
  if (!c) return;
  Py_XDECREF(c->out_type);
  Py_XDECREF(c->general);
  Py_XDECREF(c->handle);
  PyMem_Free(c);
}

// (status, Output) = self.epara_collect(ticket)
PyObject* collect(PyObject* capsule, PyObject* const* args, Py_ssize_t n, PyObject* names) {
  Collect* c = static_cast<Collect*>(PyCapsule_GetPointer(capsule, nullptr));
  if (!c) return nullptr;
  if (n != 2 || names || !PyLong_CheckExact(args[1])) return PyObject_Vectorcall(c->general, args, n, names);
  PyObject* h = PyObject_GetAttr(args[0], c->handle);
  if (!h) return nullptr;
  const uint64_t ctx = PyLong_AsUnsignedLongLong(h);
  Py_DECREF(h);
  if (ctx == (uint64_t)-1 && PyErr_Occurred()) return nullptr;
  const uint64_t ticket = PyLong_AsUnsignedLongLongMask(args[1]);
  if (ticket == (uint64_t)-1 && PyErr_Occurred()) return nullptr;
  PyObject* out = PyObject_CallNoArgs(c->out_type);
  if (!out) return nullptr;
  Py_buffer view;
  if (PyObject_GetBuffer(out, &view, PyBUF_WRITABLE) < 0) { Py_DECREF(out); return nullptr; }
  // An answer that is there already is a look into a table.  For the others, usually a step's first, the library asks the CUDA driver
  // whether the step is through, and the driver's own lock can be held by another thread's launches: without the interpreter lock
  // then, as ctypes does it.  (Letting it go for every answer: two small MLPs 38.3 -> 40.7 us a step.)
  int status = c->ready(reinterpret_cast<void*>(static_cast<uintptr_t>(ctx)), ticket, view.buf);
  if (status == c->pending) {
    Py_BEGIN_ALLOW_THREADS
    status = c->fn(reinterpret_cast<void*>(static_cast<uintptr_t>(ctx)), ticket, view.buf);
    Py_END_ALLOW_THREADS
  }
  PyBuffer_Release(&view);
  PyObject* s = PyLong_FromLong(status);
  PyObject* r = s ? PyTuple_New(2) : nullptr;
  if (!r) { Py_XDECREF(s); Py_DECREF(out); return nullptr; }
  PyTuple_SET_ITEM(r, 0, s);
  PyTuple_SET_ITEM(r, 1, out);
  return r;
}

PyMethodDef collect_def = {"epara_collect", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(collect)), METH_FASTCALL | METH_KEYWORDS,
                           "(status, Output) of a ticket"};

// collect_method(addresses of epara_collect and epara_collect_ready, EPARA_PENDING, Output, general, name of the handle's attribute)
// -> method for the context class
PyObject* collect_method(PyObject*, PyObject* args) {
  unsigned long long fn, ready;
  int pending;
  PyObject *out_type, *general, *handle;
  if (!PyArg_ParseTuple(args, "KKiOOU", &fn, &ready, &pending, &out_type, &general, &handle)) return nullptr;
  Collect* c = static_cast<Collect*>(PyMem_Malloc(sizeof(Collect)));
  if (!c) return PyErr_NoMemory();
  c->fn = reinterpret_cast<int (*)(void*, uint64_t, void*)>(static_cast<uintptr_t>(fn));
  c->ready = reinterpret_cast<int (*)(void*, uint64_t, void*)>(static_cast<uintptr_t>(ready));
  c->pending = pending;
  c->out_type = Py_NewRef(out_type);
  c->general = Py_NewRef(general);
  c->handle = Py_NewRef(handle);
  PyObject* capsule = PyCapsule_New(c, nullptr, free_collect);
  if (!capsule) { Py_DECREF(out_type); Py_DECREF(general); Py_DECREF(handle); PyMem_Free(c); return nullptr; }
  PyObject* f = PyCFunction_New(&collect_def, capsule);
  Py_DECREF(capsule);
  if (!f) return nullptr;
  PyObject* m = PyInstanceMethod_New(f);          // (a builtin does not bind to the instance by itself)
  Py_DECREF(f);
  return m;
}

// Arguments of a call: whole numbers, None for a null pointer, numbers.  `bad` is set by the first one that is neither.
struct Args {
  PyObject* const* a;
  bool bad;
  long long whole(int i) {
    const long long v = PyLong_AsLongLong(a[i]);
    bad |= v == -1 && PyErr_Occurred();
    return v;
  }
  int integer(int i) {
    const long long v = whole(i);
    if (!bad && v != (int)v) {
      PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
      bad = true;
    }
    return (int)v;
  }
  template <class T>
  T* ptr(int i) {
    if (a[i] == Py_None) return nullptr;
    const unsigned long long v = PyLong_AsUnsignedLongLong(a[i]);
    bad |= v == (unsigned long long)-1 && PyErr_Occurred();
    return reinterpret_cast<T*>(static_cast<uintptr_t>(v));
  }
  float number(int i) {
    const double v = PyFloat_AsDouble(a[i]);
    bad |= v == -1.0 && PyErr_Occurred();
    return (float)v;
  }
};
template <class F>
PyObject* answer(const Args& x, F call) {
  if (x.bad) return nullptr;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}
bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, not %zd", want, n);
  return n == want;
}

decltype(&epara_rms_norm_i8) rms_norm_i8_fn;
decltype(&epara_gemm_i8) gemm_i8_fn;
decltype(&epara_kv8_append) kv8_append_fn;
decltype(&epara_kv8_attention) kv8_attention_fn;

// The arguments of the C functions, in their order (gemm: device, stream, the problem's fields, status).
PyObject* rms_norm_i8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count_is(n, 16)) return nullptr;
  Args x = {args, false};
  const int device = x.integer(0), x_type = x.integer(3), rows = x.integer(14), d = x.integer(15);
  void *stream = x.ptr<void>(1), *in = x.ptr<void>(2), *gain = x.ptr<void>(9);
  float *resid = x.ptr<float>(5), *resid_out = x.ptr<float>(7), *scales = x.ptr<float>(13), eps = x.number(10);
  const long long x_stride = x.whole(4), resid_stride = x.whole(6), out_stride = x.whole(8), q_stride = x.whole(12);
  signed char* q = x.ptr<signed char>(11);
  return answer(x, [&] { return rms_norm_i8_fn(device, stream, in, x_type, x_stride, resid, resid_stride, resid_out, out_stride, gain, eps, q, q_stride, scales, rows, d); });
}
PyObject* gemm_i8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count_is(n, 16)) return nullptr;
  Args x = {args, false};
  const int device = x.integer(0);
  void* stream = x.ptr<void>(1);
  epara_gemm_i8_problem p;
  p.A = x.ptr<signed char>(2); p.W = x.ptr<signed char>(3); p.a_scale = x.ptr<float>(4); p.w_scale = x.ptr<float>(5); p.C = x.ptr<void>(6); p.bias = x.ptr<void>(7);
  p.M = x.integer(8); p.N = x.integer(9); p.K = x.integer(10); p.lda = x.integer(11); p.ldw = x.integer(12); p.ldc = x.integer(13); p.epilogue = x.integer(14);
  int* status = x.ptr<int>(15);
  return answer(x, [&] { return gemm_i8_fn(device, stream, &p, status); });
}
PyObject* kv8_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count_is(n, 20)) return nullptr;
  Args x = {args, false};
  const int device = x.integer(0), k_stride = x.integer(3), v_stride = x.integer(5), table_stride = x.integer(12), B = x.integer(13), T = x.integer(14), Hkv = x.integer(15),
            hd = x.integer(16), max_q = x.integer(17), max_len = x.integer(18);
  void *stream = x.ptr<void>(1), *k = x.ptr<void>(2), *v = x.ptr<void>(4), *layer = x.ptr<void>(6);
  float* scales = x.ptr<float>(7);
  const long long pages = x.whole(8);
  int32_t *q_rows = x.ptr<int32_t>(9), *lens = x.ptr<int32_t>(10), *tables = x.ptr<int32_t>(11);
  int* status = x.ptr<int>(19);
  return answer(x, [&] { return kv8_append_fn(device, stream, k, k_stride, v, v_stride, layer, scales, pages, q_rows, lens, tables, table_stride, B, T, Hkv, hd, max_q, max_len, status); });
}
PyObject* kv8_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!count_is(n, 22)) return nullptr;
  Args x = {args, false};
  const int device = x.integer(0), q_stride = x.integer(3), table_stride = x.integer(10), B = x.integer(12), T = x.integer(13), Hq = x.integer(14), Hkv = x.integer(15),
            hd = x.integer(16), max_q = x.integer(17), max_len = x.integer(18);
  void *stream = x.ptr<void>(1), *q = x.ptr<void>(2), *layer = x.ptr<void>(4), *out = x.ptr<void>(11), *scratch = x.ptr<void>(19);
  float* scales = x.ptr<float>(5);
  const long long pages = x.whole(6), scratch_bytes = x.whole(20);
  int32_t *q_rows = x.ptr<int32_t>(7), *lens = x.ptr<int32_t>(8), *tables = x.ptr<int32_t>(9);
  int* status = x.ptr<int>(21);
  return answer(x, [&] { return kv8_attention_fn(device, stream, q, q_stride, layer, scales, pages, q_rows, lens, tables, table_stride, out, B, T, Hq, Hkv, hd, max_q, max_len, scratch, (size_t)scratch_bytes, status); });
}
#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL
PyMethodDef layer8_defs[] = {{"epara_rms_norm_i8", FAST(rms_norm_i8), "status"}, {"epara_gemm_i8", FAST(gemm_i8), "status"}, {"epara_kv8_append", FAST(kv8_append), "status"},
                             {"epara_kv8_attention", FAST(kv8_attention), "status"}};

// layer8_calls(addresses of epara_rms_norm_i8, epara_gemm_i8, epara_kv8_append, epara_kv8_attention) -> the four calls
PyObject* layer8_calls(PyObject*, PyObject* args) {
  unsigned long long a[4];
  if (!PyArg_ParseTuple(args, "KKKK", &a[0], &a[1], &a[2], &a[3])) return nullptr;
  rms_norm_i8_fn = reinterpret_cast<decltype(rms_norm_i8_fn)>(static_cast<uintptr_t>(a[0]));
  gemm_i8_fn = reinterpret_cast<decltype(gemm_i8_fn)>(static_cast<uintptr_t>(a[1]));
  kv8_append_fn = reinterpret_cast<decltype(kv8_append_fn)>(static_cast<uintptr_t>(a[2]));
  kv8_attention_fn = reinterpret_cast<decltype(kv8_attention_fn)>(static_cast<uintptr_t>(a[3]));
  PyObject* r = PyTuple_New(4);
  for (int i = 0; r && i < 4; ++i) {
    PyObject* f = PyCFunction_New(&layer8_defs[i], nullptr);
    if (!f) { Py_DECREF(r); return nullptr; }
    PyTuple_SET_ITEM(r, i, f);
  }
  return r;
}

PyMethodDef methods[] = {{"layer8_calls", layer8_calls, METH_VARARGS, "the calls of the 8-bit decoder layer"},
                         {"collect_method", collect_method, METH_VARARGS, "epara_collect as a method of the context class"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) { return PyModule_Create(&module); }
