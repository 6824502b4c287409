// _mccall: calls a function of libmooncake_hip.so with the arguments of a Python wrapper (binding.py), laid out here instead of
// through ctypes.  Small calls are bound by the host: an attention call of the tiny fp32 request was 7.3 us of it, now 4.9, 4 of
// them in the library.  Marshalling only; the library itself is loaded by binding.py, which hands the address over.
//
//   call(address, kinds, *arguments) -> status        one letter of `kinds` per argument:
//     p  device (or pinned) tensor: its data_ptr(); None: a null pointer
//     s  a ctypes structure: its address; None: a null pointer
//     i  an integer (32 or 64 bits; the function takes the bits it has parameters for, as with ctypes)
//     I  a list of n integers as int32[n], or an integer address
//     Q  a list of n integers as int64[n], or an integer address
//
// and three looks at tensors before a call, made here because a dozen of them through Python are a sixth of a small call (one new
// token a row, rotation and append, launch included: 8.9 us of the host, so 7.6):
//
//   misfit(device, dtype, tensor, least, tensor, least, ...) -> the first that is not a dense tensor of dtype on the device with
//                                                              at least so many elements, or -1
//   row_stride(device, dtype, tensor, tokens, heads, dim) -> elements from token to token of [tokens, heads, dim] or
//                                                              [tokens, heads * dim] whose heads are dense, -1 if it is none
//   head_strides(device, dtype, tensor, tokens, heads, dim) -> elements from token to token and from head to head of [tokens, heads, dim]
//                                                              whose rows are dense, None if it is none
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include <vector>

#if !defined(__x86_64__)
#error "Function below rests on the x86-64 System V calling convention"
#endif

namespace {

constexpr int kMaxArgs = 20;
// every parameter is an integer or a pointer, so one signature does: registers and stack words the callee has no parameter for
// are not looked at (x86-64 calling convention, the caller clears the stack)
typedef int (*Function)(uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t,
                        uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t);

PyObject* g_data_ptr = nullptr;                            // "data_ptr", and the others' names
PyObject *g_dtype = nullptr, *g_get_device = nullptr, *g_is_contiguous = nullptr, *g_numel = nullptr, *g_shape = nullptr, *g_stride = nullptr;

// low 64 bits of an integer; false with an exception set for what is none
bool bits_of(PyObject* o, uint64_t* out) {
  if (!PyLong_Check(o)) {
    PyObject* index = PyNumber_Index(o);
    if (index == nullptr) return false;
    *out = PyLong_AsUnsignedLongLongMask(index);
    Py_DECREF(index);
  } else {
    *out = PyLong_AsUnsignedLongLongMask(o);
  }
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

template <typename Int>
bool lay_out(PyObject* list, std::vector<uint64_t>& room) {
  const Py_ssize_t n = PyList_GET_SIZE(list);
  room.resize((size_t)n * sizeof(Int) / 8 + 1);
  Int* to = reinterpret_cast<Int*>(room.data());
  for (Py_ssize_t i = 0; i < n && i < PyList_GET_SIZE(list); ++i) {
    PyObject* item = PyList_GET_ITEM(list, i);
    uint64_t v;
    if (PyLong_Check(item)) {
      if (!bits_of(item, &v)) return false;
    } else {                                               // as int() takes it: numpy integers, floats
      Py_INCREF(item);
      PyObject* whole = PyNumber_Long(item);
      Py_DECREF(item);
      if (whole == nullptr) return false;
      const bool fine = bits_of(whole, &v);
      Py_DECREF(whole);
      if (!fine) return false;
    }
    to[i] = (Int)v;
  }
  return true;
}

PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args < 2 || !PyUnicode_Check(args[1])) {
    PyErr_SetString(PyExc_TypeError, "call(address, kinds, *arguments)");
    return nullptr;
  }
  Py_ssize_t n = 0;
  const char* kinds = PyUnicode_AsUTF8AndSize(args[1], &n);
  uint64_t address = 0;
  if (kinds == nullptr || !bits_of(args[0], &address)) return nullptr;
  if (n != n_args - 2 || n > kMaxArgs || address == 0) {
    PyErr_SetString(PyExc_TypeError, "one letter of kinds per argument, at most 20");
    return nullptr;
  }
  uint64_t a[kMaxArgs] = {0};
  std::vector<uint64_t> lists[2];
  int n_lists = 0;
  try {
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* o = args[i + 2];
      if (kinds[i] == 'p') {
        if (o == Py_None) continue;
        PyObject* ptr = PyObject_CallMethodNoArgs(o, g_data_ptr);
        if (ptr == nullptr) return nullptr;
        const bool fine = bits_of(ptr, &a[i]);
        Py_DECREF(ptr);
        if (!fine) return nullptr;
      } else if (kinds[i] == 's') {
        if (o == Py_None) continue;
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return nullptr;
        a[i] = reinterpret_cast<uint64_t>(view.buf);       // (the caller holds the object, which owns the memory)
        PyBuffer_Release(&view);
      } else if ((kinds[i] == 'I' || kinds[i] == 'Q') && PyList_CheckExact(o)) {
        if (n_lists == 2) {
          PyErr_SetString(PyExc_TypeError, "at most two lists");
          return nullptr;
        }
        std::vector<uint64_t>& room = lists[n_lists++];
        if (!(kinds[i] == 'I' ? lay_out<int32_t>(o, room) : lay_out<int64_t>(o, room))) return nullptr;
        a[i] = reinterpret_cast<uint64_t>(room.data());
      } else if (!bits_of(o, &a[i])) {
        return nullptr;
      }
    }
  } catch (const std::exception&) {                        // no memory for a list
    return PyErr_NoMemory();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = reinterpret_cast<Function>(address)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12],
                                               a[13], a[14], a[15], a[16], a[17], a[18], a[19]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// An integer that a method of o returns; false with an exception set.
bool ask(PyObject* o, PyObject* name, long long* out) {
  PyObject* got = PyObject_CallMethodNoArgs(o, name);
  if (got == nullptr) return false;
  *out = got == Py_True ? 1 : got == Py_False ? 0 : PyLong_AsLongLong(got);
  Py_DECREF(got);
  return !(*out == -1 && PyErr_Occurred());
}
// 1: of this type on this device, 0: not, -1: an exception
int lies(PyObject* o, long long device, PyObject* dtype) {
  PyObject* type = PyObject_GetAttr(o, g_dtype);
  if (type == nullptr) return -1;
  const bool same = type == dtype;
  Py_DECREF(type);
  long long at;
  if (!same) return 0;
  return !ask(o, g_get_device, &at) ? -1 : at == device;
}

PyObject* misfit(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 2 || n % 2 != 0) {
    PyErr_SetString(PyExc_TypeError, "misfit(device, dtype, tensor, least, ...)");
    return nullptr;
  }
  const long long device = PyLong_AsLongLong(args[0]);
  if (device == -1 && PyErr_Occurred()) return nullptr;
  for (Py_ssize_t i = 2; i < n; i += 2) {
    const long long least = PyLong_AsLongLong(args[i + 1]);
    if (least == -1 && PyErr_Occurred()) return nullptr;
    const int there = lies(args[i], device, args[1]);
    if (there < 0) return nullptr;
    long long dense = 0, size = 0;
    if (there == 1 && (!ask(args[i], g_is_contiguous, &dense) || !ask(args[i], g_numel, &size))) return nullptr;
    if (there == 0 || !dense || size < least) return PyLong_FromSsize_t(i / 2 - 1);
  }
  return PyLong_FromLong(-1);
}

// the integers of a tuple of at most 3; their number, or -1 for anything else
int integers(PyObject* t, long long (&out)[3]) {
  if (t == nullptr || !PyTuple_Check(t) || PyTuple_GET_SIZE(t) > 3) return -1;
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(t); ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    if (out[i] == -1 && PyErr_Occurred()) return -1;
  }
  return (int)PyTuple_GET_SIZE(t);
}

PyObject* row_stride(PyObject*, PyObject* const* args, Py_ssize_t n) {
  long long device, tokens, heads, dim;
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "row_stride(device, dtype, tensor, tokens, heads, dim)");
    return nullptr;
  }
  device = PyLong_AsLongLong(args[0]), tokens = PyLong_AsLongLong(args[3]), heads = PyLong_AsLongLong(args[4]), dim = PyLong_AsLongLong(args[5]);
  if (PyErr_Occurred()) return nullptr;
  const int there = lies(args[2], device, args[1]);
  if (there < 0) return nullptr;
  if (there == 0) return PyLong_FromLong(-1);
  PyObject* shape = PyObject_GetAttr(args[2], g_shape);
  PyObject* stride = shape == nullptr ? nullptr : PyObject_CallMethodNoArgs(args[2], g_stride);
  long long size[3] = {0, 0, 0}, step[3] = {0, 0, 0};
  const int dims = integers(shape, size), steps = integers(stride, step);
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  if (PyErr_Occurred()) return nullptr;
  const bool fits = dims == steps && dims >= 2 && size[0] == tokens &&
                    (dims == 2 ? size[1] == heads * dim && step[1] == 1
                               : size[1] == heads && size[2] == dim && step[2] == 1 && (step[1] == dim || heads == 1));
  return PyLong_FromLongLong(!fits ? -1 : tokens > 1 ? step[0] : heads * dim);
}

PyObject* head_strides(PyObject*, PyObject* const* args, Py_ssize_t n) {
  long long device, tokens, heads, dim;
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "head_strides(device, dtype, tensor, tokens, heads, dim)");
    return nullptr;
  }
  device = PyLong_AsLongLong(args[0]), tokens = PyLong_AsLongLong(args[3]), heads = PyLong_AsLongLong(args[4]), dim = PyLong_AsLongLong(args[5]);
  if (PyErr_Occurred()) return nullptr;
  const int there = lies(args[2], device, args[1]);
  if (there < 0) return nullptr;
  if (there == 0) Py_RETURN_NONE;
  PyObject* shape = PyObject_GetAttr(args[2], g_shape);
  PyObject* stride = shape == nullptr ? nullptr : PyObject_CallMethodNoArgs(args[2], g_stride);
  long long size[3] = {0, 0, 0}, step[3] = {0, 0, 0};
  const int dims = integers(shape, size), steps = integers(stride, step);
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  if (PyErr_Occurred()) return nullptr;
  if (dims != 3 || steps != 3 || size[0] != tokens || size[1] != heads || size[2] != dim || step[2] != 1) Py_RETURN_NONE;
  return Py_BuildValue("LL", tokens > 1 ? step[0] : heads * dim, heads > 1 ? step[1] : dim);
}

PyMethodDef g_methods[] = {{"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, "call(address, kinds, *arguments) -> status"},
                           {"misfit", (PyCFunction)(void (*)(void))misfit, METH_FASTCALL, "misfit(device, dtype, tensor, least, ...) -> index or -1"},
                           {"row_stride", (PyCFunction)(void (*)(void))row_stride, METH_FASTCALL, "row_stride(device, dtype, tensor, tokens, heads, dim) -> stride or -1"},
                           {"head_strides", (PyCFunction)(void (*)(void))head_strides, METH_FASTCALL, "head_strides(device, dtype, tensor, tokens, heads, dim) -> strides or None"},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_mccall", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mccall(void) {
  PyObject** const names[] = {&g_data_ptr, &g_dtype, &g_get_device, &g_is_contiguous, &g_numel, &g_shape, &g_stride};
  const char* const texts[] = {"data_ptr", "dtype", "get_device", "is_contiguous", "numel", "shape", "stride"};
  for (int i = 0; i < 7; ++i)
    if ((*names[i] = PyUnicode_InternFromString(texts[i])) == nullptr) return nullptr;
  return PyModule_Create(&g_module);
}
