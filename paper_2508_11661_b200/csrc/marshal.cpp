// Fast paths of the Python binding.  A call on a paged cache takes up to a dozen tensors, and checking each of them in Python
// (0.5 us) and handing them over by ctypes (2 us a call) costs more than the small calls themselves take on the GPU.  Here are the
// checks of an argument that is as it should be (0.09 us, rows 0.15 us; anything else is left to the Python form, which says what
// is wrong), and the call itself.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>

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

// Arguments of a call that are not numbers: descriptions (ctypes structures, by their memory) and packed tensors (tuples made by
// `rows`).
struct Rows {
  void* data;
  int64_t token_stride, head_stride;
};
constexpr int kMostArgs = 16;
struct Args {
  long value[kMostArgs] = {};
  Rows rows[kMostArgs];
  Py_buffer buffers[kMostArgs];
  int n_buffers = 0;
  float scale = 0.f;           // the one argument of the library's packed calls that is no integer
  int n = 0;
  ~Args() {
    for (int i = 0; i < n_buffers; ++i) PyBuffer_Release(&buffers[i]);
  }
  bool add(PyObject* x) {
    if (PyFloat_Check(x)) {
      scale = static_cast<float>(PyFloat_AS_DOUBLE(x));
      return true;
    }
    if (n == kMostArgs) {
      PyErr_SetString(PyExc_TypeError, "call: too many arguments");
      return false;
    }
    long& v = value[n];
    if (x == Py_None) {
      v = 0;
    } else if (PyLong_Check(x)) {
      v = static_cast<long>(PyLong_AsUnsignedLongLongMask(x));
      if (PyErr_Occurred()) return false;
    } else if (PyIndex_Check(x)) {           // numpy's integers, which are buffers as well
      PyObject* whole = PyNumber_Index(x);
      if (whole == nullptr) return false;
      v = static_cast<long>(PyLong_AsUnsignedLongLongMask(whole));
      Py_DECREF(whole);
      if (PyErr_Occurred()) return false;
    } else if (PyTuple_Check(x)) {
      Rows& r = rows[n];
      long long ts, hs;
      PyObject* p;
      if (!PyArg_ParseTuple(x, "OLL", &p, &ts, &hs)) return false;
      r.data = PyLong_AsVoidPtr(p);
      r.token_stride = ts;
      r.head_stride = hs;
      if (PyErr_Occurred()) return false;
      v = reinterpret_cast<long>(&r);
    } else {
      if (PyObject_GetBuffer(x, &buffers[n_buffers], PyBUF_SIMPLE) != 0) return false;
      v = reinterpret_cast<long>(buffers[n_buffers++].buf);
    }
    ++n;
    return true;
  }
};

// call(address, arguments ...): the status of a library function whose arguments are integers, pointers and at most one float.
// Integers and floats travel in registers of their own on x86-64, integers behind the sixth on the stack in their order, and
// arguments that a function does not look at do no harm, so that one function type serves all of them.
PyObject* call(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n < 1 || !PyLong_Check(a[0])) {
    PyErr_SetString(PyExc_TypeError, "call: expected an address and arguments");
    return nullptr;
  }
  Args args;
  for (Py_ssize_t i = 1; i < n; ++i)
    if (!args.add(a[i])) return nullptr;
  using Fn = int (*)(float, long, long, long, long, long, long, long, long, long, long, long, long, long, long, long, long);
  const Fn f = reinterpret_cast<Fn>(PyLong_AsVoidPtr(a[0]));
  const long* v = args.value;
  int status;
  Py_BEGIN_ALLOW_THREADS;
  status = f(args.scale, v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15]);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(status);
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef kMethods[] = {{"device_ptr", fast(device_ptr), METH_FASTCALL, nullptr},
                          {"rows", fast(rows), METH_FASTCALL, nullptr},
                          {"call", fast(call), METH_FASTCALL, nullptr},
                          {"otherwise", fast(otherwise), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&kModule); }
