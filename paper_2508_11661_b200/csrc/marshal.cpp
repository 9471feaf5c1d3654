// Fast paths of the Python binding.  A call on a paged cache takes up to a dozen tensors, and checking each of them in Python
// (0.5 us) and handing them over by ctypes (2 us a call) costs more than the small calls themselves take on the GPU.  Here are the
// checks of an argument that is as it should be (0.09 us, rows 0.15 us; anything else is left to the Python form, which says what
// is wrong), and the call itself.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>

#include <tuple>
#include <utility>

#include "samkv.h"

namespace {

PyObject* g_device_ptr = nullptr;    // the Python forms
PyObject* g_rows = nullptr;

// A tensor of this type and shape (a tuple of int) on this CUDA device (-1: in host memory).
const at::Tensor* as_wanted(PyObject* t, PyObject* dtype, PyObject* shape, PyObject* device) {
  if (!THPVariable_Check(t) || !THPDtype_Check(dtype) || !PyTuple_Check(shape) || !PyLong_Check(device)) return nullptr;
  const at::Tensor& x = THPVariable_Unpack(t);
  if (!x.defined() || x.layout() != at::kStrided || x.get_device() != PyLong_AsLong(device)) return nullptr;
  if (x.scalar_type() != reinterpret_cast<THPDtype*>(dtype)->scalar_type || x.dim() != PyTuple_GET_SIZE(shape)) return nullptr;
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(shape); ++i)
    if (x.size(i) != PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i))) return nullptr;
  return &x;
}

// What both take: (t, what, dtype, shape, device).
bool five(Py_ssize_t n) {
  if (n != 5) PyErr_SetString(PyExc_TypeError, "expected (tensor, what, dtype, shape, device)");
  return n == 5;
}

// Asking a tensor may throw (one without storage, inside a function transform, has no address); an exception that leaves a C
// function would end the process, so it counts as "not as it should be", and the Python form raises its own.

// Address of a contiguous tensor, None for None.
PyObject* device_ptr(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!five(n)) return nullptr;
  if (a[0] == Py_None) Py_RETURN_NONE;
  try {
    const at::Tensor* x = as_wanted(a[0], a[2], a[3], a[4]);
    if (x != nullptr && x->is_contiguous()) return PyLong_FromVoidPtr(x->data_ptr());
  } catch (...) {
  }
  PyErr_Clear();
  return PyObject_Vectorcall(g_device_ptr, a, 5, nullptr);
}

// (address, token stride, head stride) of a tensor of three dimensions whose last one is contiguous.
PyObject* rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!five(n)) return nullptr;
  try {
    const at::Tensor* x = as_wanted(a[0], a[2], a[3], a[4]);
    if (x != nullptr && x->dim() == 3 && x->stride(2) == 1) {
      void* data = x->data_ptr();
      return Py_BuildValue("(NLL)", PyLong_FromVoidPtr(data), (long long)x->stride(0), (long long)x->stride(1));
    }
  } catch (...) {
  }
  PyErr_Clear();
  return PyObject_Vectorcall(g_rows, a, 5, nullptr);
}

// otherwise(device_ptr, rows): the Python forms.
PyObject* otherwise(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "otherwise: expected two functions");
    return nullptr;
  }
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(g_device_ptr, a[0]);
  Py_XSETREF(g_rows, a[1]);
  Py_RETURN_NONE;
}

// A Python value as a parameter of type T; take() says what is wrong by a Python exception.
bool not_a(const char* what) {
  PyErr_Format(PyExc_TypeError, "call: expected %s", what);
  return false;
}
template <typename T>
struct Arg;
// Integers: int, bool and what has __index__ (numpy's), but no float.
template <typename T>
struct Integer {
  T v = 0;
  T get() const { return v; }
  bool take(PyObject* x) {
    if (!PyIndex_Check(x)) return not_a("an integer");
    PyObject* whole = PyNumber_Index(x);
    if (whole == nullptr) return false;
    const long long wide = PyLong_AsLongLong(whole);
    Py_DECREF(whole);
    if (wide == -1 && PyErr_Occurred()) return false;
    v = static_cast<T>(wide);
    if (v == wide) return true;
    PyErr_SetString(PyExc_OverflowError, "call: an integer has more than 32 bits");
    return false;
  }
};
template <>
struct Arg<int32_t> : Integer<int32_t> {};
template <>
struct Arg<int64_t> : Integer<int64_t> {};
template <>
struct Arg<float> {
  float v = 0.f;
  float get() const { return v; }
  bool take(PyObject* x) {
    if (!PyFloat_Check(x)) return not_a("a float");
    v = static_cast<float>(PyFloat_AS_DOUBLE(x));
    return true;
  }
};
// Memory of the device, streams and handles: their address, None for null.
template <typename T>
struct Arg<T*> {
  void* v = nullptr;
  T* get() const { return static_cast<T*>(v); }
  bool take(PyObject* x) {
    if (x == Py_None) return true;
    if (!PyLong_Check(x)) return not_a("an address");
    v = PyLong_AsVoidPtr(x);
    return v != nullptr || !PyErr_Occurred();
  }
};
// Packed tensors: what `rows` makes.
template <>
struct Arg<const samkv_rows_t*> {
  samkv_rows_t v = {};
  bool given = false;
  const samkv_rows_t* get() const { return given ? &v : nullptr; }
  bool take(PyObject* x) {
    if (x == Py_None) return true;
    if (!PyTuple_Check(x) || PyTuple_GET_SIZE(x) != 3) return not_a("a packed tensor");
    Arg<void*> data;
    Arg<int64_t> token, head;
    if (!data.take(PyTuple_GET_ITEM(x, 0)) || !token.take(PyTuple_GET_ITEM(x, 1)) || !head.take(PyTuple_GET_ITEM(x, 2))) return false;
    v.data = data.v;
    v.token_stride = token.v;
    v.head_stride = head.v;
    given = true;
    return true;
  }
};
// Descriptions: ctypes structures of the same size, by their memory.
template <typename S>
struct Description {
  Py_buffer b = {};
  Description() = default;
  Description(const Description&) = delete;
  ~Description() { PyBuffer_Release(&b); }     // (nothing to do where there is none)
  const S* get() const { return static_cast<const S*>(b.buf); }
  bool take(PyObject* x) {
    if (x == Py_None) return true;
    if (PyObject_GetBuffer(x, &b, PyBUF_SIMPLE) != 0) return false;
    return b.len == sizeof(S) || not_a("another description");
  }
};
template <>
struct Arg<const samkv_packed_t*> : Description<samkv_packed_t> {};
template <>
struct Arg<const samkv_pages_t*> : Description<samkv_pages_t> {};
template <>
struct Arg<const samkv_rope_t*> : Description<samkv_rope_t> {};
template <>
struct Arg<const samkv_rope_axes_t*> : Description<samkv_rope_axes_t> {};
template <>
struct Arg<const samkv_scores_t*> : Description<samkv_scores_t> {};

// name(address, arguments ...): the status of the library function at that address, whose type is that of the header's
// declaration, so that every argument has its place and its type.
template <typename F>
struct Call;
template <typename... T>
struct Call<samkv_status_t (*)(T...)> {
  template <size_t... I>
  static PyObject* with(samkv_status_t (*f)(T...), PyObject* const* a, std::index_sequence<I...>) {
    std::tuple<Arg<T>...> args;
    if (!(std::get<I>(args).take(a[I]) && ...)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = f(std::get<I>(args).get()...);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
  }
  static PyObject* call(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 1 + (Py_ssize_t)sizeof...(T) || !PyLong_Check(a[0]))
      return not_a("an address and the library function's arguments"), nullptr;
    void* f = PyLong_AsVoidPtr(a[0]);
    if (f == nullptr) return PyErr_Occurred() || not_a("an address"), nullptr;
    return with(reinterpret_cast<samkv_status_t (*)(T...)>(f), a + 1, std::index_sequence_for<T...>{});
  }
};

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef kMethods[] = {{"device_ptr", fast(device_ptr), METH_FASTCALL, nullptr},
                          {"rows", fast(rows), METH_FASTCALL, nullptr},
                          {"otherwise", fast(otherwise), METH_FASTCALL, nullptr},
#define SAMKV_CALL(name) {#name, fast(Call<decltype(&name)>::call), METH_FASTCALL, nullptr}
                          SAMKV_CALL(samkv_prefill),
                          SAMKV_CALL(samkv_append),
                          SAMKV_CALL(samkv_paged_attn),
                          SAMKV_CALL(samkv_page_tables),
                          SAMKV_CALL(samkv_release_pages),
                          SAMKV_CALL(samkv_append_axes),
                          SAMKV_CALL(samkv_prefill_scores),
                          SAMKV_CALL(samkv_paged_attn_scores),
#undef SAMKV_CALL
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&kModule);
  // (whose tensors this code knows)
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", SAMKV_TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
