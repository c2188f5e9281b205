// Python's way to entry points whose calls are mostly the host's time: the arguments are converted here, by the types that the header declares, where
// ctypes takes 1 to 2 us of a call of 5 for them.  A pointer argument takes an address, None, or anything with data_ptr().  The library is not
// linked: bind() is given the addresses.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <cstring>
#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/mllm_stage.h"

namespace {

PyObject* data_ptr_name;

template <typename T>
bool convert(PyObject* o, T* out) {
  if constexpr (std::is_pointer_v<T>) {
    void* p = nullptr;
    if (o != Py_None) {
      PyObject* address = PyLong_Check(o) ? Py_NewRef(o) : PyObject_CallMethodNoArgs(o, data_ptr_name);
      if (!address) return false;
      p = PyLong_AsVoidPtr(address);
      Py_DECREF(address);
      if (!p && PyErr_Occurred()) return false;
    }
    *out = static_cast<T>(p);
  } else if constexpr (std::is_floating_point_v<T>) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) return false;
    *out = static_cast<T>(v);
  } else if constexpr (std::is_unsigned_v<T>) {
    PyObject* whole = PyNumber_Index(o);
    if (!whole) return false;
    const unsigned long long v = PyLong_AsUnsignedLongLong(whole);
    Py_DECREF(whole);
    if (v == static_cast<unsigned long long>(-1) && PyErr_Occurred()) return false;
    *out = static_cast<T>(v);
  } else {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < std::numeric_limits<T>::min() || v > std::numeric_limits<T>::max()) {
      PyErr_Format(PyExc_OverflowError, "%lld does not fit the argument", v);
      return false;
    }
    *out = static_cast<T>(v);
  }
  return true;
}

template <typename F, int ID>
struct Entry;
template <typename... A, int ID>
struct Entry<mllm_status_t (*)(A...), ID> {
  static inline mllm_status_t (*target)(A...) = nullptr;
  template <size_t... I>
  static PyObject* run(PyObject* const* args, std::index_sequence<I...>) {
    std::tuple<A...> v{};
    if (!(convert(args[I], &std::get<I>(v)) && ...)) return nullptr;
    mllm_status_t status;
    Py_BEGIN_ALLOW_THREADS
    status = target(std::get<I>(v)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
  }
  static PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (!target) {
      PyErr_SetString(PyExc_RuntimeError, "the library is not loaded");
      return nullptr;
    }
    if (n != static_cast<Py_ssize_t>(sizeof...(A))) {
      PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, static_cast<Py_ssize_t>(sizeof...(A)));
      return nullptr;
    }
    return run(args, std::index_sequence_for<A...>{});
  }
};

#define ENTRIES(X)                                                                                                                         \
  X(mllm_op_grid_positions) X(mllm_op_rope_freq_table) X(mllm_op_rope_axes) X(mllm_op_residual_norm_fwd) X(mllm_op_residual_norm_bwd)      \
  X(mllm_op_keep8) X(mllm_op_keep8_load) X(mllm_op_act_fwd_keep8) X(mllm_op_act_bwd_keep8) X(mllm_op_linear_bwd_keep8)
enum Ids {
#define X(name) ID_##name,
  ENTRIES(X)
#undef X
};
#define ENTRY(name) Entry<decltype(&name), ID_##name>

PyObject* bind(PyObject*, PyObject* args) {
  const char* name;
  PyObject* address;
  if (!PyArg_ParseTuple(args, "sO", &name, &address)) return nullptr;
  void* p = PyLong_AsVoidPtr(address);
  if (!p) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address");
    return nullptr;
  }
#define X(entry)                                                            \
  if (std::strcmp(name, #entry) == 0) {                                     \
    ENTRY(entry)::target = reinterpret_cast<decltype(&entry)>(p);           \
    Py_RETURN_NONE;                                                         \
  }
  ENTRIES(X)
#undef X
  PyErr_Format(PyExc_KeyError, "%s", name);
  return nullptr;
}

PyMethodDef methods[] = {
#define X(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&ENTRY(name)::call)), METH_FASTCALL, nullptr},
    ENTRIES(X)
#undef X
    {"bind", bind, METH_VARARGS, "bind(name, address): the library's entry point of that name."},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
  data_ptr_name = PyUnicode_InternFromString("data_ptr");
  return data_ptr_name ? PyModule_Create(&module) : nullptr;
}
