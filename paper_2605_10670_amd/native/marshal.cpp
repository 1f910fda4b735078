// Argument marshalling of the per-step calls (binding.py): one Python call checks the tensors, takes
// their addresses and calls the library's C entry point, without the interpreter in between.
//
// What bounds a small step that is called eagerly is the host: a launch costs about 2.5 us, and ctypes with
// the checks written in Python added 1.2 to 2.2 us to each call.  Measured (a step of four calls, 128 fp32
// tokens, top-2, host time without waiting; layout / dispatch / expert stand-in / combine): 3.8 / 4.1 / 4.5 /
// 4.7 us that way, 3.4 / 3.6 / 3.9 / 4.1 this way, the step 17.9 and 16.3.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

namespace {

PyObject *name_contiguous, *name_data_ptr, *name_cuda_stream, *name_nbytes;

// Device address of a tensor (must be contiguous), an int, or None.
bool pointer_of(PyObject* o, uint64_t* out) {
  if (o == Py_None) {
    *out = 0;
    return true;
  }
  if (!PyLong_Check(o)) {
    PyObject* whole = PyObject_CallMethodNoArgs(o, name_contiguous);
    if (whole == nullptr) return false;
    const int yes = PyObject_IsTrue(whole);
    Py_DECREF(whole);
    if (yes < 0) return false;
    if (yes == 0) {
      PyErr_SetString(PyExc_ValueError, "tensor must be contiguous");
      return false;
    }
    PyObject* address = PyObject_CallMethodNoArgs(o, name_data_ptr);
    if (address == nullptr) return false;
    *out = PyLong_AsUnsignedLongLongMask(address);
    Py_DECREF(address);
  } else {
    *out = PyLong_AsUnsignedLongLongMask(o);
  }
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

// A stream's raw handle, or None for the default stream.
bool stream_of(PyObject* o, uint64_t* out) {
  if (o == Py_None || PyLong_Check(o)) return pointer_of(o, out);
  PyObject* handle = PyObject_GetAttr(o, name_cuda_stream);
  if (handle == nullptr) return false;
  *out = PyLong_AsUnsignedLongLongMask(handle);
  Py_DECREF(handle);
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

// call(entry point's address, "kinds of its arguments", arguments...) -> its return code.  Kinds: p a device
// address (tensor, int or None), i an int32, h a handle as an int, s the stream.  Every argument is of the
// integer class, so it travels in a 64-bit register or stack slot whatever its width.
// call_sized(address, kinds, needs, count, arguments...): the same for entry points of up to ten arguments that read and write
// tensors of known sizes.  needs: for every p in turn the bytes that it has to hold for each of `count`, or as a negative
// number for all; what is not a tensor is not looked at.  -(kTooSmall + i) where the i-th argument holds fewer, and
// nothing is called.  (Host time of a call with the norm's seven tensors: 3.0 us checked in Python, 2.2 here.)
constexpr int kMost = 9, kMostSized = 10, kTooSmall = 1000;
PyObject* call_any(PyObject* const* args, Py_ssize_t nargs, int most, PyObject* needs, PyObject* count) {
  Py_ssize_t n = 0;
  const char* kinds = nargs >= 2 ? PyUnicode_AsUTF8AndSize(args[1], &n) : nullptr;
  const int skip = needs != nullptr ? 4 : 2;
  if (kinds == nullptr || n != nargs - skip || n < 1 || n > most) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "call(address, kinds, arguments...)");
    return nullptr;
  }
  const uint64_t entry = PyLong_AsUnsignedLongLong(args[0]);
  if (entry == (uint64_t)-1 && PyErr_Occurred()) return nullptr;
  int64_t rows = 0;
  if (needs != nullptr) {
    if (!PyTuple_Check(needs)) {
      PyErr_SetString(PyExc_TypeError, "needs must be a tuple");
      return nullptr;
    }
    rows = PyLong_AsLongLong(count);
    if (rows == -1 && PyErr_Occurred()) return nullptr;
  }
  uint64_t a[kMostSized] = {};
  Py_ssize_t pointers = 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* o = args[i + skip];
    bool ok = true;
    switch (kinds[i]) {
      case 'p':
        ok = pointer_of(o, &a[i]);
        if (ok && needs != nullptr) {
          if (pointers >= PyTuple_GET_SIZE(needs)) {
            PyErr_SetString(PyExc_TypeError, "needs must say one size for every pointer");
            return nullptr;
          }
          const int64_t need = PyLong_AsLongLong(PyTuple_GET_ITEM(needs, pointers++));
          if (need == -1 && PyErr_Occurred()) return nullptr;
          if (o != Py_None && !PyLong_Check(o)) {
            PyObject* held = PyObject_GetAttr(o, name_nbytes);
            if (held == nullptr) return nullptr;
            const int64_t bytes = PyLong_AsLongLong(held);
            Py_DECREF(held);
            if (bytes == -1 && PyErr_Occurred()) return nullptr;
            if (bytes < (need < 0 ? -need : need * rows)) return PyLong_FromLong(-(long)(kTooSmall + i));
          }
        }
        break;
      case 's': ok = stream_of(o, &a[i]); break;
      default: {
        PyObject* number = PyNumber_Index(o);
        if (number == nullptr) return nullptr;
        a[i] = PyLong_AsUnsignedLongLongMask(number);
        Py_DECREF(number);
        ok = !(a[i] == (uint64_t)-1 && PyErr_Occurred());
      }
    }
    if (!ok) return nullptr;
  }
  int code;
  typedef uint64_t U;
  typedef int (*Entry)(U, U, U, U, U, U, U, U, U);
  typedef int (*LongEntry)(U, U, U, U, U, U, U, U, U, U);
  Py_BEGIN_ALLOW_THREADS  // (arguments past the entry point's own are not looked at)
  if (n <= kMost)
    code = reinterpret_cast<Entry>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]);
  else
    code = reinterpret_cast<LongEntry>(entry)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(code);
}

PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return call_any(args, nargs, kMost, nullptr, nullptr);
}

PyObject* call_sized(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs < 4) {
    PyErr_SetString(PyExc_TypeError, "call_sized(address, kinds, needs, count, arguments...)");
    return nullptr;
  }
  return call_any(args, nargs, kMostSized, args[2], args[3]);
}

PyMethodDef methods[] = {{"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL,
                          "call(address, kinds, arguments...) -> return code"},
                         {"call_sized", (PyCFunction)(void (*)(void))call_sized, METH_FASTCALL,
                          "call_sized(address, kinds, needs, count, arguments...) -> return code"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  name_contiguous = PyUnicode_InternFromString("is_contiguous");
  name_data_ptr = PyUnicode_InternFromString("data_ptr");
  name_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  name_nbytes = PyUnicode_InternFromString("nbytes");
  if (!name_contiguous || !name_data_ptr || !name_cuda_stream || !name_nbytes) return nullptr;
  return PyModule_Create(&module);
}
