// Argument blocks of the Python binding: tensors checked and written out as the structures the library takes.
//
// pack(codes, names, device, d, n, max_q, *args) -> bytes.  One argument a code, written one behind the other:
//   P  a whole number (an address), 8 bytes         i  a whole number, 4 bytes         d  a float, 8 bytes
//   C  address of the descriptor of a Cache or QCache (its pointers set from its tensors) and, 8 bytes, whether it is a QCache
//   H  kvc_heads of a bf16 tensor [rows, heads, d]  p  kvc_probs of a float32 tensor [rows, entries]
//   r  address of an int32 tensor of the probabilities' rows, f  of a float32 one
//   n  address of an int32 tensor of n entries, u  of a float32 one
//   K  address of an int32 tensor [n, max_q or more] and, 8 bytes, its row length
//   F  address of a float32 tensor, A  of any tensor
// H, p, n, F and A take None too (zeros).  Lists are contiguous, and every tensor lives on `device`.  Wrong ones raise KvcError
// with the name of the argument.  Done in Python the same costs a call of four tensors 5 us, more than its kernel takes.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "../../include/kvc.h"

namespace {

PyObject *g_error, *g_bf16, *g_f32, *g_i32;                       // KvcError and the types, from setup()
PyObject *s_made, *s_k, *s_v, *s_scale_k, *s_scale_v, *s_page_table;
PyObject *s_shape, *s_stride, *s_dtype, *s_data_ptr, *s_get_device, *s_is_contiguous;

bool refuse(int code, PyObject* names, Py_ssize_t i, const char* why) {
  PyErr_Clear();
  const char* name = i < PyTuple_GET_SIZE(names) ? PyUnicode_AsUTF8(PyTuple_GET_ITEM(names, i)) : "argument";
  PyObject* what = PyUnicode_FromFormat("%s%s%s", name ? name : "argument", *why ? ": " : "", why);
  PyObject* e = what ? PyObject_CallFunction(g_error, "iO", code, what) : nullptr;
  Py_XDECREF(what);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return false;
}

// numbers of a tuple of exactly n; false (without an error set) where it is no such thing
bool numbers(PyObject* t, int64_t* v, Py_ssize_t n) {
  if (!t || !PyTuple_Check(t) || PyTuple_GET_SIZE(t) != n) return false;
  for (Py_ssize_t i = 0; i < n; ++i) {
    v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    if (v[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}
bool sizes(PyObject* t, int64_t* shape, int64_t* stride, Py_ssize_t n) {
  PyObject* a = PyObject_GetAttr(t, s_shape);
  bool ok = numbers(a, shape, n);
  Py_XDECREF(a);
  if (!ok) return false;
  a = PyObject_CallMethodNoArgs(t, s_stride);
  ok = numbers(a, stride, n);
  Py_XDECREF(a);
  return ok;
}
bool is_type(PyObject* t, PyObject* type) {
  PyObject* a = PyObject_GetAttr(t, s_dtype);
  const bool ok = a == type;
  Py_XDECREF(a);
  return ok;
}
bool number_of(PyObject* t, PyObject* method, int64_t* v) {
  PyObject* a = PyObject_CallMethodNoArgs(t, method);
  if (!a) return false;
  *v = PyLong_AsLongLong(a);
  Py_DECREF(a);
  return !(*v == -1 && PyErr_Occurred());
}
bool contiguous(PyObject* t) {
  PyObject* a = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  const bool ok = a == Py_True;
  Py_XDECREF(a);
  return ok;
}

// Sets one pointer of a descriptor from the object's tensor; false with an error set.
bool set_pointer(PyObject* c, PyObject* name, void* to, bool may_be_none) {
  PyObject* t = PyObject_GetAttr(c, name);
  if (!t) return false;
  int64_t at = 0;
  const bool ok = (may_be_none && t == Py_None) || number_of(t, s_data_ptr, &at);
  if (ok && t != Py_None) memcpy(to, &at, 8);
  Py_DECREF(t);
  return ok;
}
// `made`: (address of the descriptor, device, its rows, its kvc_qcache or None), kept in the object by the binding
bool describe(PyObject* c, int64_t device, PyObject* names, Py_ssize_t name, int64_t* out) {
  PyObject* made = PyObject_GetAttr(c, s_made);
  if (!made || !PyTuple_Check(made) || PyTuple_GET_SIZE(made) != 4) {
    Py_XDECREF(made);
    return refuse(KVC_E_INVALID_ARG, names, name, "a Cache or QCache expected");
  }
  const int64_t at = PyLong_AsLongLong(PyTuple_GET_ITEM(made, 0)), where = PyLong_AsLongLong(PyTuple_GET_ITEM(made, 1));
  const bool q8 = PyTuple_GET_ITEM(made, 3) != Py_None;
  Py_DECREF(made);                                                // the object holds it
  if (PyErr_Occurred()) return false;
  if (where != device) return refuse(KVC_E_INVALID_ARG, names, name, "tensors on the current CUDA device expected");
  kvc_qcache* q = reinterpret_cast<kvc_qcache*>(at);
  kvc_cache* rows = q8 ? &q->codes : reinterpret_cast<kvc_cache*>(at);
  if (!set_pointer(c, s_k, &rows->k, false) || !set_pointer(c, s_v, &rows->v, false) || !set_pointer(c, s_page_table, &rows->page_table, true)) return false;
  if (q8 && (!set_pointer(c, s_scale_k, &q->scale_k, false) || !set_pointer(c, s_scale_v, &q->scale_v, false))) return false;
  out[0] = at;
  out[1] = q8;
  return true;
}

PyObject* pack(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  constexpr Py_ssize_t kHead = 6;
  if (nargs < kHead) return PyErr_Format(PyExc_TypeError, "pack(codes, names, device, d, n, max_q, ...)");
  Py_ssize_t n = 0;
  const char* codes = PyUnicode_AsUTF8AndSize(args[0], &n);
  if (!codes || !PyTuple_Check(args[1])) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_TypeError, "names: a tuple");
  if (nargs != kHead + n || n > 64) return PyErr_Format(PyExc_TypeError, "an argument a code, 64 at most");
  PyObject* names = args[1];
  const int64_t device = PyLong_AsLongLong(args[2]), d = PyLong_AsLongLong(args[3]), requests = PyLong_AsLongLong(args[4]), max_q = PyLong_AsLongLong(args[5]);
  if (PyErr_Occurred()) return nullptr;
  int64_t rows = -1;                                              // of the probabilities
  unsigned char block[64 * sizeof(kvc_heads)];
  size_t at = 0;
  Py_ssize_t tensor = 0;                                          // among the tensors: its name
  auto put = [&](const void* p, size_t bytes) {
    memcpy(block + at, p, bytes);
    at += bytes;
  };
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* x = args[kHead + i];
    const char code = codes[i];
    if (code == 'P' || code == 'i') {
      const long long v = PyLong_AsLongLong(x);
      if (v == -1 && PyErr_Occurred()) return nullptr;
      if (code == 'P') {
        put(&v, 8);
      } else {
        const int32_t w = (int32_t)v;
        if (w != v) return PyErr_Format(PyExc_OverflowError, "%lld is no 32-bit number", v);
        put(&w, 4);
      }
      continue;
    }
    if (code == 'd') {
      const double v = PyFloat_AsDouble(x);
      if (v == -1.0 && PyErr_Occurred()) return nullptr;
      put(&v, 8);
      continue;
    }
    const Py_ssize_t name = tensor++;
    if (code == 'C') {
      int64_t made[2];
      if (!describe(x, device, names, name, made)) return nullptr;
      put(made, 16);
      continue;
    }
    kvc_heads h;
    kvc_probs p;
    memset(&h, 0, sizeof(h));
    memset(&p, 0, sizeof(p));
    int64_t address = 0, length = 0;
    if (x != Py_None || code == 'K' || code == 'r' || code == 'f' || code == 'u') {
      int64_t shape[3], stride[3], where = 0;
      if (code == 'H') {
        if (!sizes(x, shape, stride, 3) || !is_type(x, g_bf16)) return refuse(KVC_E_INVALID_ARG, names, name, "bf16 [rows, heads, d] expected"), nullptr;
        if (shape[2] != d) return refuse(KVC_E_SHAPE, names, name, ""), nullptr;
        if (stride[2] != 1 || (shape[0] > 1 && stride[0] == 0) || (shape[1] > 1 && stride[1] == 0))
          return refuse(KVC_E_UNSUPPORTED, names, name, "contiguous channels and no broadcast rows expected"), nullptr;
        if (shape[0] > INT32_MAX || shape[1] > INT32_MAX) return refuse(KVC_E_UNSUPPORTED, names, name, "too many rows"), nullptr;
        h.n_rows = (int32_t)shape[0];
        h.n_heads = (int32_t)shape[1];
        h.s_row = shape[0] > 1 ? stride[0] : 0;
        h.s_head = shape[1] > 1 ? stride[1] : 0;
      } else if (code == 'p') {
        if (!sizes(x, shape, stride, 2) || !is_type(x, g_f32)) return refuse(KVC_E_INVALID_ARG, names, name, "float32 [rows, n] expected"), nullptr;
        if ((shape[1] > 1 && stride[1] != 1) || (shape[0] > 1 && stride[0] < shape[1]))
          return refuse(KVC_E_UNSUPPORTED, names, name, "contiguous entries and no broadcast rows expected"), nullptr;
        if (shape[0] > INT32_MAX || shape[1] > INT32_MAX) return refuse(KVC_E_UNSUPPORTED, names, name, "too many rows"), nullptr;
        p.n_rows = (int32_t)shape[0];
        p.n = (int32_t)shape[1];
        p.s_row = shape[0] > 1 ? stride[0] : 0;
        if (rows < 0) rows = shape[0];
      } else if (code == 'K') {
        if (!sizes(x, shape, stride, 2) || !is_type(x, g_i32) || !contiguous(x)) return refuse(KVC_E_INVALID_ARG, names, name, "contiguous int32 [requests, max_q or more] expected"), nullptr;
        if (shape[0] != requests || shape[1] < max_q || shape[1] > INT32_MAX) return refuse(KVC_E_SHAPE, names, name, "[requests, max_q or more] expected"), nullptr;
      } else if (code == 'n' || code == 'u' || code == 'r' || code == 'f') {
        const bool whole = code == 'n' || code == 'r';
        if (!is_type(x, whole ? g_i32 : g_f32) || !contiguous(x)) return refuse(KVC_E_INVALID_ARG, names, name, whole ? "contiguous int32 expected" : "contiguous float32 expected"), nullptr;
        PyObject* a = PyObject_GetAttr(x, s_shape);
        const bool one = numbers(a, shape, 1);
        Py_XDECREF(a);
        if (!one || shape[0] != (code == 'n' || code == 'u' ? requests : rows)) return refuse(KVC_E_SHAPE, names, name, code == 'n' || code == 'u' ? "[requests] expected" : "[rows] expected"), nullptr;
      } else if ((code == 'F' && !is_type(x, g_f32)) || !contiguous(x)) {
        return refuse(KVC_E_INVALID_ARG, names, name, code == 'F' ? "contiguous float32 expected" : "a contiguous tensor expected"), nullptr;
      }
      if (code == 'K') length = shape[1];
      if (!number_of(x, s_data_ptr, &address) || !number_of(x, s_get_device, &where)) return refuse(KVC_E_INVALID_ARG, names, name, "a tensor expected"), nullptr;
      if (where != device) return refuse(KVC_E_INVALID_ARG, names, name, "tensors on the current CUDA device expected"), nullptr;
    }
    if (code == 'H') {
      h.data = reinterpret_cast<void*>(address);
      put(&h, sizeof(h));
    } else if (code == 'p') {
      p.p = reinterpret_cast<const float*>(address);
      put(&p, sizeof(p));
    } else {
      put(&address, 8);
      if (code == 'K') put(&length, 8);
    }
  }
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(block), (Py_ssize_t)at);
}

PyObject* setup(PyObject*, PyObject* args) {
  PyObject *e, *b, *f, *i;
  if (!PyArg_ParseTuple(args, "OOOO", &e, &b, &f, &i)) return nullptr;
  PyObject** const to[] = {&g_error, &g_bf16, &g_f32, &g_i32};
  PyObject* const from[] = {e, b, f, i};
  for (int k = 0; k < 4; ++k) {
    Py_INCREF(from[k]);
    Py_XSETREF(*to[k], from[k]);
  }
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"pack", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(pack)), METH_FASTCALL, "an argument block"},
                         {"setup", setup, METH_VARARGS, "KvcError, torch.bfloat16, torch.float32, torch.int32"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  struct {
    PyObject** to;
    const char* name;
  } const names[] = {{&s_shape, "shape"}, {&s_made, "_made"}, {&s_k, "k"}, {&s_v, "v"}, {&s_scale_k, "scale_k"}, {&s_scale_v, "scale_v"}, {&s_page_table, "page_table"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_data_ptr, "data_ptr"}, {&s_get_device, "get_device"}, {&s_is_contiguous, "is_contiguous"}};
  for (const auto& x : names)
    if (!(*x.to = PyUnicode_InternFromString(x.name))) return nullptr;
  return PyModule_Create(&module);
}
