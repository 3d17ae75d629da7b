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

// as a C type: what it does not hold is refused, not cut to its lowest bits
template <class T>
T integer_as(PyObject* o, const char* what) {
  static_assert(std::is_integral_v<T>);
  const long long v = integer(o, what);
  if ((v < 0 && std::is_unsigned_v<T>) || (long long)(T)v != v) {
    PyErr_Format(PyExc_OverflowError, "%s: out of range", what);
    throw BadArgument();
  }
  return (T)v;
}

// what has no truth (an array of several elements) is an error of the call
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw BadArgument();
  return v != 0;
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
  } else {
    return integer_as<T>(o, "integer");
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
    std::tuple<A...> a{integer_as<A>(args[I], "integer")...};
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

// ---- Entries that take the tensors of a call and nothing that follows from them: sizes, row strides and types are read here, what is
// not handed over is made here, and whatever a kernel takes by its address alone is checked here.  They return a tuple of tensors, or
// the error code of the call as an integer.  A call of the smallest size is mostly this work (in Python it took 4 us of 7).
[[noreturn]] void refuse_value(const char* format, const char* what) {
  PyErr_Format(PyExc_ValueError, format, what);
  throw BadArgument();
}
const at::Tensor& gpu_tensor(PyObject* o) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "tensor", o);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse_value("tensor must live on the GPU", "");
  return t;
}
// activations: rows that may lie apart
struct Rows {
  void* p;
  int64_t rows, cols, ld;
  at::ScalarType type;
  int dtype() const { return type == at::kFloat ? EFQAT_F32 : EFQAT_BF16; }
};
Rows rows_of(const at::Tensor& t) {
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) refuse_value("tensor must be two-dimensional with contiguous rows", "");
  const at::ScalarType type = t.scalar_type();
  if (type != at::kFloat && type != at::kBFloat16) {
    PyErr_SetString(PyExc_TypeError, "unsupported dtype");
    throw BadArgument();
  }
  const int64_t rows = t.size(0), cols = t.size(1);
  return {t.data_ptr(), rows, cols, rows > 1 ? t.stride(0) : cols, type};
}
Rows rows_like(PyObject* o, const Rows& x, const char* what) {
  const Rows r = rows_of(gpu_tensor(o));
  if (r.type != x.type) {
    PyErr_Format(PyExc_TypeError, "%s: another dtype than the call's", what);
    throw BadArgument();
  }
  if (r.rows != x.rows || r.cols != x.cols) refuse_value("%s: another shape than the call's", what);
  return r;
}
// a contiguous tensor of a given type and shape (cols < 0: one dimension)
void* dense(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, const char* what) {
  const at::Tensor& t = gpu_tensor(o);
  if (t.scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s: another dtype expected", what);
    throw BadArgument();
  }
  if (t.dim() != (cols < 0 ? 1 : 2) || t.size(0) != rows || (cols >= 0 && t.size(1) != cols)) refuse_value("%s: another shape expected", what);
  if (!t.is_contiguous()) refuse_value("%s: tensor must be contiguous", what);
  return t.data_ptr();
}
int64_t pitch_of(int64_t cols) { return (cols + 15) / 16 * 16; }
int64_t groups_of(int64_t cols) { return (cols + EFQAT_CKPT8_GROUP - 1) / EFQAT_CKPT8_GROUP; }
int8_t* codes_of(PyObject* o, const Rows& x, const char* what) { return (int8_t*)dense(o, at::kChar, x.rows, pitch_of(x.cols), what); }
float* scales_of(PyObject* o, const Rows& x, const char* what) { return (float*)dense(o, at::kFloat, x.rows, groups_of(x.cols), what); }

// the tensors that a call returns, given (not None) or new
struct Results {
  PyObject* tuple;
  const at::TensorOptions opt;
  Results(Py_ssize_t n, const at::Tensor& like) : tuple(PyTuple_New(n)), opt(like.options()) {
    if (!tuple) throw BadArgument();
    for (Py_ssize_t i = 0; i < n; ++i) {
      Py_INCREF(Py_None);
      PyTuple_SET_ITEM(tuple, i, Py_None);
    }
  }
  ~Results() { Py_XDECREF(tuple); }
  Results(const Results&) = delete;
  void put(Py_ssize_t i, PyObject* o) {               // takes the reference
    Py_DECREF(PyTuple_GET_ITEM(tuple, i));
    PyTuple_SET_ITEM(tuple, i, o);
  }
  at::Tensor make(at::ScalarType type, int64_t rows, int64_t cols) {
    const int64_t shape[2] = {rows, cols};
    return at::empty(at::IntArrayRef(shape, cols < 0 ? 1 : 2), opt.dtype(type));
  }
  Rows rows(Py_ssize_t i, PyObject* given, const Rows& x, const char* what) {
    if (given && given != Py_None) {
      const Rows r = rows_like(given, x, what);
      Py_INCREF(given);
      put(i, given);
      return r;
    }
    at::Tensor t = make(x.type, x.rows, x.cols);
    const Rows r = {t.data_ptr(), x.rows, x.cols, x.cols, x.type};
    put(i, THPVariable_Wrap(std::move(t)));
    return r;
  }
  void* dense_at(Py_ssize_t i, PyObject* given, at::ScalarType type, int64_t rows, int64_t cols, const char* what) {
    if (given && given != Py_None) {
      void* p = dense(given, type, rows, cols, what);
      Py_INCREF(given);
      put(i, given);
      return p;
    }
    at::Tensor t = make(type, rows, cols);
    void* p = t.data_ptr();
    put(i, THPVariable_Wrap(std::move(t)));
    return p;
  }
  int8_t* codes(Py_ssize_t i, PyObject* given, const Rows& x, const char* what) {
    return (int8_t*)dense_at(i, given, at::kChar, x.rows, pitch_of(x.cols), what);
  }
  float* scales(Py_ssize_t i, PyObject* given, const Rows& x, const char* what) {
    return (float*)dense_at(i, given, at::kFloat, x.rows, groups_of(x.cols), what);
  }
  PyObject* take(int rc) {
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* t = tuple;
    tuple = nullptr;
    return t;
  }
};
void* stream_now() { return (void*)c10::hip::getCurrentHIPStream().stream(); }
bool given(PyObject* o) { return o && o != Py_None; }

// FN(args, optional): n arguments, and `more` results that may be handed over (absent: nullptr)
template <auto FN, int N, int MORE>
PyObject* whole(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N && n != N + MORE) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %d or %d expected", n, N, N + MORE);
    return nullptr;
  }
  PyObject* out[MORE];
  for (int i = 0; i < MORE; ++i) out[i] = n == N ? nullptr : args[N + i];
  try {
    return FN(args, out);
  } catch (const BadArgument&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
template <class F>
int unlocked(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

// x -> codes, scales
PyObject* ckpt8_save(PyObject* const* a, PyObject* const* out) {
  const at::Tensor& t = gpu_tensor(a[0]);
  const Rows x = rows_of(t);
  Results r(2, t);
  int8_t* codes = r.codes(0, out[0], x, "x_codes");
  float* scales = r.scales(1, out[1], x, "x_scales");
  void* st = stream_now();
  return r.take(unlocked([&] { return efqat_ckpt8_save(x.p, x.ld, x.dtype(), x.rows, x.cols, codes, scales, st); }));
}
// codes, scales, cols, bf16 -> x
PyObject* ckpt8_load(PyObject* const* a, PyObject* const* out) {
  const at::Tensor& t = gpu_tensor(a[0]);
  const int64_t cols = integer(a[2], "integer");
  Rows x = {nullptr, t.dim() > 0 ? t.size(0) : 0, cols, cols, truth(a[3]) ? at::kBFloat16 : at::kFloat};
  const int8_t* codes = codes_of(a[0], x, "codes");
  const float* scales = scales_of(a[1], x, "scales");
  Results r(1, t);
  if (given(out[0])) x.type = gpu_tensor(out[0]).scalar_type();
  const Rows y = r.rows(0, out[0], x, "out");
  void* st = stream_now();
  return r.take(unlocked([&] { return efqat_ckpt8_load(codes, scales, y.rows, y.cols, y.p, y.ld, y.dtype(), st); }));
}
// x, kind, up, checkpoint -> y, x_codes, x_scales, up_codes, up_scales
PyObject* act_fwd(PyObject* const* a, PyObject* const* out) {
  const at::Tensor& t = gpu_tensor(a[0]);
  const Rows x = rows_of(t);
  const int kind = integer_as<int>(a[1], "kind");
  const bool gated = given(a[2]), keep = truth(a[3]);
  const Rows up = gated ? rows_like(a[2], x, "up") : Rows{};
  Results r(5, t);
  const Rows y = r.rows(0, out[0], x, "y");
  int8_t* xc = keep ? r.codes(1, out[1], x, "x_codes") : nullptr;
  float* xs = keep ? r.scales(2, out[2], x, "x_scales") : nullptr;
  int8_t* uc = keep && gated ? r.codes(3, out[3], x, "up_codes") : nullptr;
  float* us = keep && gated ? r.scales(4, out[4], x, "up_scales") : nullptr;
  void* st = stream_now();
  return r.take(unlocked([&] { return efqat_act_fwd(x.p, x.ld, up.p, up.ld, x.dtype(), x.rows, x.cols, kind, y.p, y.ld, xc, xs, uc, us, st); }));
}
// dy, kind, x_codes, x_scales, up_codes, up_scales -> dx, dup
PyObject* act_bwd(PyObject* const* a, PyObject* const* out) {
  const at::Tensor& t = gpu_tensor(a[0]);
  const Rows dy = rows_of(t);
  const int kind = integer_as<int>(a[1], "kind");
  const int8_t* xc = codes_of(a[2], dy, "x_codes");
  const float* xs = scales_of(a[3], dy, "x_scales");
  const bool gated = given(a[4]);
  if (gated != given(a[5])) refuse_value("up_codes and up_scales belong together", "");
  const int8_t* uc = gated ? codes_of(a[4], dy, "up_codes") : nullptr;
  const float* us = gated ? scales_of(a[5], dy, "up_scales") : nullptr;
  Results r(2, t);
  const Rows dx = r.rows(0, out[0], dy, "dx"), dup = gated ? r.rows(1, out[1], dy, "dup") : Rows{};
  void* st = stream_now();
  return r.take(unlocked([&] { return efqat_act_bwd(dy.p, dy.ld, dy.dtype(), dy.rows, dy.cols, kind, xc, xs, uc, us, dx.p, dx.ld, dup.p, dup.ld, st); }));
}
// x, weight, bias, eps, checkpoint -> y, mean, rstd, x_codes, x_scales
PyObject* layer_norm_fwd(PyObject* const* a, PyObject* const* out) {
  const at::Tensor& t = gpu_tensor(a[0]);
  const Rows x = rows_of(t);
  const float* w = given(a[1]) ? (const float*)dense(a[1], at::kFloat, x.cols, -1, "weight") : nullptr;
  const float* b = given(a[2]) ? (const float*)dense(a[2], at::kFloat, x.cols, -1, "bias") : nullptr;
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) throw BadArgument();
  const bool keep = truth(a[4]);
  Results r(5, t);
  const Rows y = r.rows(0, out[0], x, "y");
  float* mean = (float*)r.dense_at(1, out[1], at::kFloat, x.rows, -1, "mean");
  float* rstd = (float*)r.dense_at(2, out[2], at::kFloat, x.rows, -1, "rstd");
  int8_t* codes = keep ? r.codes(3, out[3], x, "x_codes") : nullptr;
  float* scales = keep ? r.scales(4, out[4], x, "x_scales") : nullptr;
  void* st = stream_now();
  return r.take(unlocked([&] {
    return efqat_layer_norm_fwd(x.p, x.ld, x.dtype(), x.rows, x.cols, w, b, (float)eps, y.p, y.ld, mean, rstd, codes, scales, st);
  }));
}
// dy, weight, mean, rstd, x, x_codes, x_scales, ws -> dx, dweight, dbias
PyObject* layer_norm_bwd(PyObject* const* a, PyObject* const* out) {
  const at::Tensor& t = gpu_tensor(a[0]);
  const Rows dy = rows_of(t);
  const float* w = given(a[1]) ? (const float*)dense(a[1], at::kFloat, dy.cols, -1, "weight") : nullptr;
  const float* mean = (const float*)dense(a[2], at::kFloat, dy.rows, -1, "mean");
  const float* rstd = (const float*)dense(a[3], at::kFloat, dy.rows, -1, "rstd");
  const bool kept = !given(a[4]);
  if (kept && (!given(a[5]) || !given(a[6]))) refuse_value("x, or x_codes and x_scales, expected", "");
  const Rows x = kept ? Rows{} : rows_like(a[4], dy, "x");
  const int8_t* codes = kept ? codes_of(a[5], dy, "x_codes") : nullptr;
  const float* scales = kept ? scales_of(a[6], dy, "x_scales") : nullptr;
  Results r(3, t);
  const Rows dx = r.rows(0, out[0], dy, "dx");
  float* dw = (float*)r.dense_at(1, out[1], at::kFloat, dy.cols, -1, "dweight");
  float* db = (float*)r.dense_at(2, out[2], at::kFloat, dy.cols, -1, "dbias");
  at::Tensor ws = given(a[7]) ? gpu_tensor(a[7]) : r.make(at::kByte, (int64_t)efqat_layer_norm_bwd_workspace_bytes(dy.rows, dy.cols), -1);
  if (!ws.is_contiguous()) refuse_value("%s: tensor must be contiguous", "ws");
  void *st = stream_now(), *p = ws.data_ptr();
  const size_t bytes = ws.nbytes();
  return r.take(unlocked([&] {
    return efqat_layer_norm_bwd(dy.p, dy.ld, dy.dtype(), x.p, x.ld, codes, scales, mean, rstd, w, dy.rows, dy.cols, dx.p, dx.ld, dw, db, p, bytes, st);
  }));
}

#define EFQAT_WHOLE(name, n, more) {#name, (PyCFunction)(void (*)(void))whole<name, n, more>, METH_FASTCALL, nullptr}
#define EFQAT_QUERY(name) {#name, (PyCFunction)(void (*)(void))query<efqat_##name>, METH_FASTCALL, nullptr}
#define EFQAT_ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<efqat_##name, false>, METH_FASTCALL, nullptr}
#define EFQAT_ENTRY_ROWS(name) {#name, (PyCFunction)(void (*)(void))entry<efqat_##name, true>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    EFQAT_ENTRY(fakequant_fwd),  EFQAT_ENTRY(channel_select), EFQAT_ENTRY(channel_select_static),
    EFQAT_ENTRY(weight_quant_select), EFQAT_ENTRY(network_select), EFQAT_ENTRY(layer_select),
    EFQAT_ENTRY(bias_grad),      EFQAT_ENTRY(linear_bwd_ex),  EFQAT_ENTRY(linear_bwd_weight_operand),
    EFQAT_ENTRY(conv_bwd_ex),    EFQAT_ENTRY(linear_fwd),
    EFQAT_WHOLE(ckpt8_save, 1, 2), EFQAT_WHOLE(ckpt8_load, 4, 1), EFQAT_WHOLE(act_fwd, 4, 5), EFQAT_WHOLE(act_bwd, 6, 2),
    EFQAT_WHOLE(layer_norm_fwd, 5, 5), EFQAT_WHOLE(layer_norm_bwd, 8, 3), EFQAT_ENTRY_ROWS(linear_xent_fwd),
    EFQAT_ENTRY_ROWS(linear_xent_bwd), EFQAT_QUERY(linear_xent_fwd_workspace_bytes),
    EFQAT_QUERY(linear_xent_bwd_workspace_bytes), {"empty", (PyCFunction)(void (*)(void))empty, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_efqat_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__efqat_torch() { return PyModule_Create(&module_def); }
