// Argument marshalling for the Python binding: one CPython entry per C ABI function that takes device tensors.  A Python
// call hands over tensors or None for pointers, integers for sizes and modes, for a stream its handle or Ellipsis (the
// current stream of the current device), and for an optimizer step the address of the struct; each is converted to the
// type of the C parameter in that place, and nothing else is taken for it: an integer is no tensor, and a tensor no
// integer.  Doing this through ctypes and attribute look-ups cost 6 to 10 us a call, as much as the launches of a small
// layer.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/efqat.h"

namespace {

struct BadArgument {};

[[noreturn]] void refuse(PyObject* type, const char* what, PyObject* got) {
  PyErr_Format(type, "%s expected, got %.100s", what, Py_TYPE(got)->tp_name);
  throw BadArgument();
}

long long integer(PyObject* o, const char* what) {
  // other integer types (numpy's) by their __index__; a tensor's would wait for the GPU
  if (!PyLong_Check(o) && (!PyIndex_Check(o) || THPVariable_Check(o))) refuse(PyExc_TypeError, what, o);
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw BadArgument();
  return v;
}

void* tensor_address(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "tensor", o);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) {
    PyErr_SetString(PyExc_ValueError, "tensor must live on the GPU");
    throw BadArgument();
  }
  if (!t.is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "tensor must be contiguous");
    throw BadArgument();
  }
  return t.data_ptr();
}

// rows that may lie apart: the elements of a row are neighbours (its row stride is an argument of its own)
void* rows_address(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "tensor", o);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) {
    PyErr_SetString(PyExc_ValueError, "tensor must live on the GPU");
    throw BadArgument();
  }
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) {
    PyErr_SetString(PyExc_ValueError, "tensor must be two-dimensional with contiguous rows");
    throw BadArgument();
  }
  return t.data_ptr();
}

// STREAM: the parameter is a stream (every entry ends in `void* stream` or `void* stream, void* side_stream`).
// ROWS: the pointer is followed by the stride of its rows
template <class T, bool STREAM, bool ROWS>
T from_python(PyObject* o) {
  if constexpr (STREAM) {
    if (o == Py_None) return nullptr;
    if (o == Py_Ellipsis) return (T)c10::hip::getCurrentHIPStream().stream();
    return (T)(uintptr_t)integer(o, "stream handle");
  } else if constexpr (std::is_same_v<T, const efqat_opt_step*>) {
    return o == Py_None ? nullptr : (T)(uintptr_t)integer(o, "address of an efqat_opt_step");
  } else if constexpr (std::is_pointer_v<T>) {
    return (T)(ROWS ? rows_address(o) : tensor_address(o));
  } else if constexpr (std::is_floating_point_v<T>) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw BadArgument();
    return (T)v;
  } else {
    return (T)integer(o, "integer");
  }
}

template <class... A>
constexpr bool is_stream(size_t i) {
  constexpr bool is_void[] = {std::is_same_v<A, void*>...};
  constexpr size_t n = sizeof...(A);
  static_assert(is_void[n - 1], "an entry ends in a stream");
  return i == n - 1 || (i == n - 2 && is_void[i]);
}

// row-strided tensors: an untyped pointer whose next parameter is a 64-bit stride, in entries that have such (APART)
template <bool APART, class... A>
constexpr bool is_rows(size_t i) {
  constexpr bool is_void[] = {std::is_same_v<A, void*> || std::is_same_v<A, const void*>...};
  constexpr bool is_long[] = {std::is_same_v<A, int64_t>...};
  return APART && is_void[i] && i + 1 < sizeof...(A) && is_long[i + 1];
}

template <bool APART, class... A, size_t... I>
PyObject* call(int (*fn)(A...), PyObject* const* args, std::index_sequence<I...>) {
  try {
    std::tuple<A...> a{from_python<A, is_stream<A...>(I), is_rows<APART, A...>(I)>(args[I])...};     // braces: in order, so that the first bad argument is reported
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = std::apply(fn, a);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const BadArgument&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

template <bool APART, class... A>
PyObject* call_n(int (*fn)(A...), PyObject* const* args, Py_ssize_t n) {
  if (n != (Py_ssize_t)sizeof...(A)) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, (Py_ssize_t)sizeof...(A));
    return nullptr;
  }
  return call<APART>(fn, args, std::index_sequence_for<A...>{});
}

template <auto FN, bool APART>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) { return call_n<APART>(FN, args, n); }

// a workspace query
template <class... A, size_t... I>
PyObject* ask(size_t (*fn)(A...), PyObject* const* args, std::index_sequence<I...>) {
  try {
    std::tuple<A...> a{(A)integer(args[I], "integer")...};
    return PyLong_FromSize_t(std::apply(fn, a));
  } catch (const BadArgument&) {
    return nullptr;
  }
}
template <class... A>
PyObject* ask_n(size_t (*fn)(A...), PyObject* const* args, Py_ssize_t n) {
  if (n != (Py_ssize_t)sizeof...(A)) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, (Py_ssize_t)sizeof...(A));
    return nullptr;
  }
  return ask(fn, args, std::index_sequence_for<A...>{});
}
template <auto FN>
PyObject* query(PyObject*, PyObject* const* args, Py_ssize_t n) { return ask_n(FN, args, n); }

// New tensors on the device of the first argument, by three integers each: type (0: the first argument's, 1: fp32, 2: int8, 3: int32,
// 4: bytes), rows, columns (-1: one dimension).  torch.empty of Python takes 1.8 us a tensor, this 0.5.
PyObject* empty(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    if (n < 4 || n % 3 != 1 || !THPVariable_Check(args[0])) {
      PyErr_SetString(PyExc_TypeError, "a tensor and three integers for each new one expected");
      return nullptr;
    }
    const at::Tensor& like = THPVariable_Unpack(args[0]);
    static const at::ScalarType types[] = {at::kFloat, at::kFloat, at::kChar, at::kInt, at::kByte};
    PyObject* out = PyTuple_New(n / 3);
    if (!out) return nullptr;
    for (Py_ssize_t i = 0; i < n / 3; ++i) {
      try {
        const long long type = integer(args[1 + 3 * i], "integer"), rows = integer(args[2 + 3 * i], "integer"), cols = integer(args[3 + 3 * i], "integer");
        if (type < 0 || type > 4) refuse(PyExc_ValueError, "type number", args[1 + 3 * i]);
        const int64_t shape[2] = {rows, cols};
        const auto opt = like.options().dtype(type == 0 ? like.scalar_type() : types[type]);
        PyTuple_SET_ITEM(out, i, THPVariable_Wrap(at::empty(at::IntArrayRef(shape, cols < 0 ? 1 : 2), opt)));
      } catch (...) {
        Py_DECREF(out);
        throw;
      }
    }
    return out;
  } catch (const BadArgument&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define EFQAT_QUERY(name) {#name, (PyCFunction)(void (*)(void))query<efqat_##name>, METH_FASTCALL, nullptr}
#define EFQAT_ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<efqat_##name, false>, METH_FASTCALL, nullptr}
#define EFQAT_ENTRY_ROWS(name) {#name, (PyCFunction)(void (*)(void))entry<efqat_##name, true>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    EFQAT_ENTRY(fakequant_fwd),  EFQAT_ENTRY(channel_select), EFQAT_ENTRY(channel_select_static),
    EFQAT_ENTRY(weight_quant_select), EFQAT_ENTRY(network_select), EFQAT_ENTRY(layer_select),
    EFQAT_ENTRY(bias_grad),      EFQAT_ENTRY(linear_bwd_ex),  EFQAT_ENTRY(linear_bwd_weight_operand),
    EFQAT_ENTRY(conv_bwd_ex),    EFQAT_ENTRY(linear_fwd),
    EFQAT_ENTRY_ROWS(ckpt8_save), EFQAT_ENTRY_ROWS(ckpt8_load), EFQAT_ENTRY_ROWS(act_fwd), EFQAT_ENTRY_ROWS(act_bwd),
    EFQAT_ENTRY_ROWS(layer_norm_fwd), EFQAT_ENTRY_ROWS(layer_norm_bwd), EFQAT_ENTRY_ROWS(linear_xent_fwd),
    EFQAT_ENTRY_ROWS(linear_xent_bwd),
    EFQAT_QUERY(layer_norm_bwd_workspace_bytes), EFQAT_QUERY(linear_xent_fwd_workspace_bytes),
    EFQAT_QUERY(linear_xent_bwd_workspace_bytes), {"empty", (PyCFunction)(void (*)(void))empty, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_efqat_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__efqat_torch() { return PyModule_Create(&module_def); }
