// CPython extension `_call`: turns the tensors of a block call into pointers and calls the C ABI.  Host code only.
//
// A small block's kernels take a few microseconds each, so a call's own cost on the host is what such a block waits
// for.  Marshalling fourteen tensors through ctypes (a Python function per tensor, a stream object per call) took
// 5-7 us a call; here it takes well under one.
//
//   call(address, desc, groups, tensors..., ws, stream) -> status
//   call_rows(address, desc, kinds, tensors..., ws, stream) -> status     (8-bit rows, gated product: desc is a convbn_qdesc)
//   call_norm(address, desc, kinds, tensors..., ws, stream) -> status     (group norm: desc is a convbn_norm_desc)
//
// `address` is the entry point's address, `desc` a convbn_desc (any object with the buffer protocol), groups None
// means that the entry point takes none; a tensor is None, a device tensor or an int (a raw address); ws is None or a
// device tensor, passed on as pointer and size (NO_WS: the entry point takes none); stream is None (the current
// stream) or a raw handle.  Tensors are dense.  call_rows checks each against the descriptor, by one letter of `kinds`:
//   x z h y  rows of desc's type, [M, K] ldx apart, [M, N] ldz, [M, 2 K] ldx, [M, K] ldz;   W  a dense weight [N, K]
//   c d e    codes of M, N, 2 M rows of K channels;   s n t m  fp32 vectors of M, N, 2 M, 2 N
//   f g      scale bytes of M, N rows of K channels in 8-bit floating point;   V  dense [2 N, K] of desc's type;   l  dense fp32 [M, 2 N]
// call_norm:
//   x y      rows of desc's type, [M P, C], ldx or ldy apart;   v  fp32 vectors of C;   s  dense fp32 [M, groups, 4]
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>

#include "../../include/convbn.h"

static_assert(sizeof(convbn_desc) != sizeof(convbn_qdesc) && sizeof(convbn_norm_desc) != sizeof(convbn_qdesc) &&
                  sizeof(convbn_norm_desc) != sizeof(convbn_desc), "the calls tell the descriptors apart by their size");

namespace {

constexpr int kMaxPtr = 16;

PyObject* g_no_ws = nullptr;   // the NO_WS marker

// Torch throws where a tensor has no memory of its own or there is no device; the interpreter's C frames let no C++
// exception through, so it becomes a Python error.
template <typename F>
bool guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return false;
}

// Address of a tensor argument; false (with a Python error set) where it is neither None, an int nor a device tensor, dense unless it
// has been looked at already.
bool pointer_of(PyObject* o, void** out, bool dense = true) {
  if (o == Py_None) { *out = nullptr; return true; }
  if (THPVariable_Check(o)) return guarded([&] {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || (dense && !t.is_contiguous())) {
      PyErr_SetString(PyExc_AssertionError, "device, dense tensors only");
      return false;
    }
    *out = t.data_ptr();
    return true;
  });
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
  }
  PyErr_Format(PyExc_TypeError, "expected a tensor, an address or None, got %s", Py_TYPE(o)->tp_name);
  return false;
}

// What a letter of `kinds` stands for: rows of `width` elements ld apart, or a dense fp32 vector of `rows`.
struct Spec {
  int64_t rows = 0, width = 1, ld = 0;
  bool bytes = false, vector = false;
};
int64_t times(int64_t a, int64_t b) { return (int64_t)((uint64_t)a * (uint64_t)b); }   // (the library refuses what overflows)
Spec spec_of(char kind, const convbn_qdesc* d) {
  const int64_t M = d->M, K = d->K, N = d->N, Kp = (K + 15) / 16 * 16, Sp = (K + 511) / 512 * 4;
  switch (kind) {
    case 'x': return {M, K, d->ldx};
    case 'z': return {M, N, d->ldz};
    case 'h': return {M, 2 * K, d->ldx};
    case 'y': return {M, K, d->ldz};
    case 'W': return {N, K};
    case 'V': return {2 * N, K};
    case 'l': return {times(M, 2 * N), 1, 0, false, true};
    case 'c': return {M, Kp, 0, true};
    case 'd': return {N, Kp, 0, true};
    case 'e': return {2 * M, Kp, 0, true};
    case 'f': return {M, Sp, 0, true};
    case 'g': return {N, Sp, 0, true};
    case 's': return {M, 1, 0, false, true};
    case 'n': return {N, 1, 0, false, true};
    case 't': return {2 * M, 1, 0, false, true};
    case 'm': return {2 * N, 1, 0, false, true};
  }
  return {M};
}
Spec spec_of(char kind, const convbn_norm_desc* d) {
  switch (kind) {
    case 'x': return {times(d->M, d->P), d->C, d->ldx};
    case 'y': return {times(d->M, d->P), d->C, d->ldy};
    case 'v': return {d->C, 1, 0, false, true};
  }
  return {times(d->M, 4 * (int64_t)d->groups), 1, 0, false, true};
}

// Whether a tensor is what an entry point reads or writes in its place; false with a Python error set.
bool fits(PyObject* o, Spec s, int32_t dtype, int at) {
  if (!THPVariable_Check(o)) return true;   // (None and addresses: the library's own checks)
  return guarded([&] {
    const at::Tensor& t = THPVariable_Unpack(o);
    const int64_t rows = s.rows, width = s.width, ld = s.ld ? s.ld : s.width;
    bool ok;
    if (s.vector) ok = t.scalar_type() == at::kFloat && t.numel() == rows && t.is_contiguous();
    else
      ok = (s.bytes ? t.element_size() == 1 : t.scalar_type() == (dtype == CONVBN_BF16 ? at::kBFloat16 : at::kFloat)) && t.dim() == 2 &&
           t.size(0) == rows && t.size(1) == width && (rows <= 1 || t.stride(0) == ld) && (width <= 1 || t.stride(1) == 1 || rows == 0);
    if (!ok)
      PyErr_Format(PyExc_ValueError, "tensor %d: expected %s%s [%lld, %lld], rows %lld elements apart", at,
                   s.vector ? "float32 vector" : s.bytes ? "bytes" : dtype == CONVBN_BF16 ? "bfloat16" : "float32", s.vector ? ", as" : "",
                   (long long)rows, (long long)width, (long long)ld);
    return ok;
  });
}

bool stream_of(PyObject* o, void** out) {
  if (o == Py_None) return guarded([&] {
    *out = c10::hip::getCurrentHIPStream().stream();
    return true;
  });
  *out = PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}

template <typename... A>
int invoke(void* f, A... a) { return reinterpret_cast<int (*)(A...)>(f)(a...); }

// desc [, groups], n pointers [, ws, bytes], stream
#define P4 p[0], p[1], p[2], p[3]
#define P8 P4, p[4], p[5], p[6], p[7]
#define P12 P8, p[8], p[9], p[10], p[11]
template <typename... T>
int dispatch(void* f, int n, void* const* p, bool* known, const void* d, T... tail) {
  switch (n) {
    case 3: return invoke(f, d, p[0], p[1], p[2], tail...);
    case 4: return invoke(f, d, P4, tail...);
    case 5:   // (always with a workspace)
      if constexpr (sizeof...(tail) == 3) return invoke(f, d, P4, p[4], tail...);
      break;
    case 6: return invoke(f, d, P4, p[4], p[5], tail...);
    case 7: return invoke(f, d, P4, p[4], p[5], p[6], tail...);
    case 8: return invoke(f, d, P8, tail...);
    case 9: return invoke(f, d, P8, p[8], tail...);
    case 11: return invoke(f, d, P8, p[8], p[9], p[10], tail...);
    case 13: return invoke(f, d, P12, p[12], tail...);
  }
  *known = false;
  return 0;
}
template <typename... T>
int dispatch_groups(void* f, int n, void* const* p, bool* known, const void* d, int groups, T... tail) {
  switch (n) {
    case 9: return invoke(f, d, groups, P8, p[8], tail...);
    case 13: return invoke(f, d, groups, P12, p[12], tail...);
  }
  *known = false;
  return 0;
}

// The descriptor's bytes for the length of a call.
struct DescView {
  Py_buffer b;
  bool held = false;
  bool get(PyObject* o, size_t size, const char* name) {
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
    held = true;
    if (b.len == (Py_ssize_t)size) return true;
    PyErr_Format(PyExc_TypeError, "expected a %s", name);
    return false;
  }
  ~DescView() { if (held) PyBuffer_Release(&b); }
};

// args: `n` tensors (kinds: which of them have been looked at), ws, stream
PyObject* call_with(void* f, const DescView& d, const char* kinds, bool has_groups, int groups, PyObject* const* args, Py_ssize_t n) {
  void* p[kMaxPtr];
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!pointer_of(args[i], &p[i], !kinds)) return nullptr;
  PyObject* ws_o = args[n];
  const bool has_ws = ws_o != g_no_ws;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (has_ws) {
    if (!pointer_of(ws_o, &ws)) return nullptr;
    if (THPVariable_Check(ws_o) && !guarded([&] { ws_bytes = THPVariable_Unpack(ws_o).nbytes(); return true; })) return nullptr;
  }
  void* stream = nullptr;
  if (!stream_of(args[n + 1], &stream)) return nullptr;
  bool known = true;
  int st = 0;
  Py_BEGIN_ALLOW_THREADS
  if (has_groups) st = dispatch_groups(f, (int)n, p, &known, d.b.buf, groups, ws, ws_bytes, stream);
  else if (has_ws) st = dispatch(f, (int)n, p, &known, d.b.buf, ws, ws_bytes, stream);
  else st = dispatch(f, (int)n, p, &known, d.b.buf, stream);
  Py_END_ALLOW_THREADS
  if (!known) {
    PyErr_SetString(PyExc_TypeError, "no entry point takes this number of tensors");
    return nullptr;
  }
  return PyLong_FromLong(st);
}

PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  const Py_ssize_t n = nargs - 5;   // tensors
  if (n < 1 || n > kMaxPtr) {
    PyErr_SetString(PyExc_TypeError, "call(address, desc, groups, tensors..., ws, stream)");
    return nullptr;
  }
  void* f = PyLong_AsVoidPtr(args[0]);
  const bool has_groups = args[2] != Py_None;
  const long groups = has_groups ? PyLong_AsLong(args[2]) : 0;
  if (PyErr_Occurred()) return nullptr;
  DescView d;
  if (!d.get(args[1], sizeof(convbn_desc), "convbn_desc")) return nullptr;
  return call_with(f, d, nullptr, has_groups, (int)groups, args + 3, n);
}

template <class D> PyObject* call_kinds(PyObject* const* args, Py_ssize_t nargs, const char* desc, const char* usage) {
  const Py_ssize_t n = nargs - 5;
  if (n < 1 || n > kMaxPtr) {
    PyErr_SetString(PyExc_TypeError, usage);
    return nullptr;
  }
  void* f = PyLong_AsVoidPtr(args[0]);
  if (PyErr_Occurred()) return nullptr;
  DescView d;
  if (!d.get(args[1], sizeof(D), desc)) return nullptr;
  Py_ssize_t length = 0;
  const char* kinds = PyUnicode_AsUTF8AndSize(args[2], &length);
  if (!kinds) return nullptr;
  if (length != n) {
    PyErr_SetString(PyExc_TypeError, "one kind for each tensor");
    return nullptr;
  }
  const D* at = static_cast<const D*>(d.b.buf);
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!fits(args[3 + i], spec_of(kinds[i], at), at->dtype, (int)i)) return nullptr;
  return call_with(f, d, kinds, false, 0, args + 3, n);
}
PyObject* call_rows(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return call_kinds<convbn_qdesc>(args, nargs, "convbn_qdesc", "call_rows(address, desc, kinds, tensors..., ws, stream)");
}
PyObject* call_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return call_kinds<convbn_norm_desc>(args, nargs, "convbn_norm_desc", "call_norm(address, desc, kinds, tensors..., ws, stream)");
}

// pointer(tensor) -> address or None, stream(None or handle) -> handle: for the entry points that take no descriptor.
PyObject* pointer(PyObject*, PyObject* o) {
  void* p = nullptr;
  if (!pointer_of(o, &p)) return nullptr;
  if (!p) Py_RETURN_NONE;
  return PyLong_FromVoidPtr(p);
}
PyObject* stream(PyObject*, PyObject* o) {
  void* p = nullptr;
  if (!stream_of(o, &p)) return nullptr;
  return PyLong_FromVoidPtr(p);
}

PyMethodDef methods[] = {
    {"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL, nullptr},
    {"call_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call_rows)), METH_FASTCALL, nullptr},
    {"call_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call_norm)), METH_FASTCALL, nullptr},
    {"pointer", pointer, METH_O, nullptr},
    {"stream", stream, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() {
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  g_no_ws = PyUnicode_FromString("NO_WS");
  if (!g_no_ws) return nullptr;
  Py_INCREF(g_no_ws);
  if (PyModule_AddObject(m, "NO_WS", g_no_ws) != 0) return nullptr;
  return m;
}
