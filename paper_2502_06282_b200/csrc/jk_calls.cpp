// The target layer's calls (jk_add_norm, jk_quantize_rows, jk_linear, jk_rope_qkv) for Python: the checks of the tensors and
// the call.  They are made dozens of times a token, and small ones end on the GPU after 2 to 3 us: checked in Python and called
// through ctypes they took 5.9 to 8.4 us of the CPU each, of which the launch is 2.4.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <exception>

#include "jakiro.h"

namespace {

decltype(&jk_add_norm) add_norm_fn;
decltype(&jk_quantize_rows) quantize_fn;
decltype(&jk_linear) linear_fn;
decltype(&jk_rope_qkv) rope_fn;
PyTypeObject* mx8_type;
PyObject *codes_name, *scales_name;

struct refused {};                         // a Python exception has been set
[[noreturn]] void refuse(const char* format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(PyExc_ValueError, format, args);
  va_end(args);
  throw refused();
}
const char* name_of(at::ScalarType t) { return t == at::kBFloat16 ? "bfloat16" : t == at::kInt ? "int32" : "float32"; }

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse("%s: expected a tensor", name);
  return THPVariable_Unpack(o);
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw refused();
  return v;
}
jk_ctx* context(PyObject* o) { return o == Py_None ? nullptr : static_cast<jk_ctx*>(PyLong_AsVoidPtr(o)); }
at::ScalarType type_of(PyObject* o) { return o == Py_True ? at::kBFloat16 : at::kFloat; }

// A dense array [rows, n] (rows -1: [n]) on a CUDA device; None where it is not given.
void* dense(PyObject* o, const char* name, at::ScalarType type, int64_t rows, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  const bool shape = rows < 0 ? t.dim() == 1 && t.size(0) == n : t.dim() == 2 && t.size(0) == rows && t.size(1) == n;
  if (t.scalar_type() != type || !shape || !t.is_contiguous() || !t.is_cuda()) {
    if (rows < 0) refuse("%s: expected a contiguous %s tensor [%lld] on a CUDA device", name, name_of(type), (long long)n);
    refuse("%s: expected a contiguous %s tensor [%lld, %lld] on a CUDA device", name, name_of(type), (long long)rows, (long long)n);
  }
  return t.data_ptr();
}
// Rows that may lie apart, [rows, n] (-1: any): the pointer and the distance (0, which the library takes as dense, only for
// a single row: the rows of an expanded array are one, and lie no distance apart).
void* strided(const at::Tensor& t, const char* name, at::ScalarType type, int64_t rows, int64_t n, int64_t& stride) {
  if (t.scalar_type() != type || t.dim() != 2 || (rows >= 0 && t.size(0) != rows) || (n >= 0 && t.size(1) != n))
    refuse("%s: expected a %s tensor [%lld, %lld]", name, name_of(type), (long long)rows, (long long)n);
  stride = 0;
  if (t.stride(1) != 1 && t.size(1) > 1) refuse("%s: expected contiguous rows", name);
  if (t.size(0) > 1) {
    stride = t.stride(0);
    if (stride < t.size(1)) refuse("%s: its rows overlap", name);
  }
  if (!t.is_cuda()) refuse("%s is not on a CUDA device", name);
  return t.data_ptr();
}
// The codes and scales of an Mx8 [rows, n] (-1: any; its arrays were checked when it was made).
struct mx8 { void* codes = nullptr; uint8_t* scales = nullptr; int64_t rows = 0, n = 0; };
bool is_mx8(PyObject* o) { return PyObject_TypeCheck(o, mx8_type); }
mx8 open_mx8(PyObject* o, const char* name, int64_t rows, int64_t n) {
  mx8 m;
  if (!is_mx8(o)) refuse("%s: expected an Mx8", name);
  PyObject* c = PyObject_GetAttr(o, codes_name);
  PyObject* s = c ? PyObject_GetAttr(o, scales_name) : nullptr;
  if (s && THPVariable_Check(c) && THPVariable_Check(s)) {
    const at::Tensor& codes = THPVariable_Unpack(c);
    m.codes = codes.data_ptr();
    m.rows = codes.size(0);
    m.n = codes.size(1);
    m.scales = static_cast<uint8_t*>(THPVariable_Unpack(s).data_ptr());
  }
  Py_XDECREF(c);
  Py_XDECREF(s);
  if (!s) throw refused();
  if ((rows >= 0 && m.rows != rows) || (n >= 0 && m.n != n))
    refuse("%s: expected an array of [%lld, %lld]", name, (long long)rows, (long long)n);
  return m;
}
template <typename F> PyObject* guarded(F f) {
  try {
    return PyLong_FromLong(f());
  } catch (const refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
template <typename F, typename... A> int call(F f, jk_ctx* ctx, A... a) {
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f(ctx, stream, a...);
  Py_END_ALLOW_THREADS
  return rc;
}
void expect(Py_ssize_t have, Py_ssize_t want) {
  if (have != want) refuse("expected %zd arguments", want);
}

// (handle, bf16, x, weight, delta, out_sum, out, out_mx8)
PyObject* add_norm(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&] {
    expect(count, 8);
    const at::ScalarType T = type_of(a[1]);
    const at::Tensor& x = tensor(a[2], "x");
    if (x.dim() != 2) refuse("x: expected a tensor [rows, n]");
    const int64_t rows = x.size(0), n = x.size(1);
    if (rows > INT32_MAX || n > INT32_MAX) refuse("x: too large");
    void* px = dense(a[2], "x", T, rows, n);
    void* w = dense(a[3], "weight", T, -1, n);
    void* delta = dense(a[4], "delta", T, rows, n);
    void* sum = dense(a[5], "out_sum", T, rows, n);
    void* out = dense(a[6], "out", T, rows, n);
    const mx8 m = a[7] == Py_None ? mx8() : open_mx8(a[7], "out_mx8", rows, n);
    return call(add_norm_fn, context(a[0]), (int32_t)rows, (int32_t)n, px, delta, w, sum, out, m.codes, m.scales);
  });
}

// (handle, bf16, x, out)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&] {
    expect(count, 4);
    const mx8 m = open_mx8(a[3], "out", -1, -1);
    int64_t stride;
    void* x = strided(tensor(a[2], "x"), "x", type_of(a[1]), m.rows, m.n, stride);
    return call(quantize_fn, context(a[0]), m.rows, (int32_t)m.n, x, stride, m.codes, m.scales);
  });
}

// (handle, bf16, address of the jk_linear_op, x, out, residual)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&] {
    expect(count, 6);
    const at::ScalarType T = type_of(a[1]);
    const jk_linear_op* op = static_cast<const jk_linear_op*>(PyLong_AsVoidPtr(a[2]));
    if (!op) refuse("no projection");
    const bool in8 = op->operands == JK_ROWS_MX8;
    int64_t rows, xs = 0, rs = 0, os = 0;
    mx8 x8, o8;
    void *x, *out, *res = nullptr;
    if (in8 != is_mx8(a[3])) refuse(in8 ? "x: expected an Mx8" : "x: expected a tensor");
    if (in8) {
      x8 = open_mx8(a[3], "x", -1, op->n_in);
      x = x8.codes;
      rows = x8.rows;
    } else {
      const at::Tensor& t = tensor(a[3], "x");
      x = strided(t, "x", T, -1, op->n_in, xs);
      rows = t.size(0);
    }
    if (rows > INT32_MAX) refuse("x: too large");
    if (a[5] != Py_None) res = strided(tensor(a[5], "residual"), "residual", T, rows, op->n_out, rs);
    int32_t kind = JK_ROWS_MX8;
    if (is_mx8(a[4])) {
      o8 = open_mx8(a[4], "out", rows, op->n_out);
      out = o8.codes;
    } else {
      const at::Tensor& t = tensor(a[4], "out");
      kind = t.scalar_type() == at::kFloat ? JK_ROWS_F32 : JK_ROWS_T;
      out = strided(t, "out", kind == JK_ROWS_F32 ? at::kFloat : T, rows, op->n_out, os);
    }
    return call(linear_fn, context(a[0]), op, (int32_t)rows, x, x8.scales, xs, res, rs, out, kind, o8.scales, os);
  });
}

const int32_t* ints(PyObject* o, const char* name, int64_t least) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != at::kInt || t.numel() < least || !t.is_contiguous() || !t.is_cuda())
    refuse("%s: expected a contiguous int32 tensor of at least %lld elements on a CUDA device", name, (long long)least);
  return static_cast<const int32_t*>(t.data_ptr());
}

// (handle, bf16, Hq, Hkv, d, batch, n_tokens, qkv, pos, sections, theta, q_out, k_out, v_out, first_row)
PyObject* rope_qkv(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&] {
    expect(count, 15);
    const at::ScalarType T = type_of(a[1]);
    const int64_t Hq = integer(a[2]), Hkv = integer(a[3]), d = integer(a[4]), B = integer(a[5]), M = integer(a[6]);
    if (B < 0 || M < 0 || B > INT32_MAX || M > INT32_MAX) refuse("batch, n_tokens: out of range");
    const int64_t n = B * M, width = (Hq + 2 * Hkv) * d;
    const at::Tensor& qkv = tensor(a[7], "qkv");
    const int64_t dims = qkv.dim();
    if (qkv.scalar_type() != T || dims < 1 || qkv.size(-1) != width || qkv.numel() != n * width ||
        !(qkv.is_contiguous() || qkv.stride(-1) == 1))
      refuse("qkv: expected a %s tensor [batch, n_tokens, %lld]", name_of(T), (long long)width);
    int64_t stride = width;
    if (!qkv.is_contiguous() && n != 1) {
      const bool flat = dims == 2, deep = dims == 3 && qkv.size(0) == B && qkv.size(1) == M;
      if (!flat && !deep) refuse("qkv: expected a tensor [batch, n_tokens, %lld]", (long long)width);
      stride = deep && M > 1 ? qkv.stride(1) : qkv.stride(0);
      if (deep && B > 1 && M > 1 && qkv.stride(0) != M * stride) refuse("qkv: its rows do not lie evenly apart");
      if (stride < width) refuse("qkv: its rows overlap");
    }
    int32_t sections[16];
    PyObject* seq = PySequence_Fast(a[9], "sections: expected a sequence of counts");
    if (!seq) throw refused();
    const Py_ssize_t axes = PySequence_Fast_GET_SIZE(seq);
    for (Py_ssize_t i = 0; i < axes && i < 16; ++i) {
      const long long v = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq, i));
      sections[i] = v < 0 ? -1 : v > INT32_MAX ? INT32_MAX : (int32_t)v;
    }
    Py_DECREF(seq);
    if (PyErr_Occurred()) throw refused();
    if (axes > 16) refuse("sections: too many axes");
    // (positions made for more tokens would be read at the wrong distance from the second sequence on; more sequences, as in
    // k_out and first_row, do no harm)
    if (a[8] != Py_None) {
      const at::Tensor& t = tensor(a[8], "pos");
      const int64_t dim = t.dim();
      const bool deep = dim == 3 && t.size(0) >= B && t.size(1) == M && t.size(2) == axes;
      const bool flat = dim == 2 && t.size(0) == n && t.size(1) == axes;
      const bool one = axes == 1 && ((dim == 2 && t.size(0) >= B && t.size(1) == M) || (dim == 1 && t.size(0) == n));
      if (!deep && !flat && !one) refuse("pos: expected a tensor [batch, n_tokens, axes], here [%lld, %lld, %zd]", (long long)B, (long long)M, axes);
    }
    if (!qkv.is_cuda()) refuse("qkv is not on a CUDA device");
    const int32_t* pos = ints(a[8], "pos", n * axes);
    const double theta = PyFloat_AsDouble(a[10]);
    if (theta == -1. && PyErr_Occurred()) throw refused();
    const at::Tensor& q = tensor(a[11], "q_out");
    if (q.scalar_type() != T || q.numel() != n * Hq * d || !q.is_contiguous() || !q.is_cuda())
      refuse("q_out: expected a contiguous %s tensor [batch, n_tokens, %lld, %lld] on a CUDA device", name_of(T), (long long)Hq, (long long)d);
    const at::Tensor &k = tensor(a[12], "k_out"), &v = tensor(a[13], "v_out");
    if (k.scalar_type() != T || v.scalar_type() != T || k.dim() != 4 || k.sizes() != v.sizes() || k.size(0) < B || k.size(1) != Hkv ||
        k.size(2) < M || k.size(3) != d || !k.is_cuda() || !v.is_cuda())
      refuse("k_out, v_out: expected %s tensors of one shape, [batch, %lld, rows, %lld] on a CUDA device", name_of(T), (long long)Hkv, (long long)d);
    if (k.size(2) > INT32_MAX) refuse("k_out, v_out: too many rows");
    bool same = k.stride(3) == 1 && v.stride(3) == 1 && (k.stride(2) == d || k.size(2) == 1);
    for (int i = 0; i < 4; ++i) same = same && (k.stride(i) == v.stride(i) || k.size(i) == 1);
    if (!same) refuse("k_out and v_out must have the same strides and dense rows");
    const int32_t* first = ints(a[14], "first_row", B);
    return call(rope_fn, context(a[0]), (int32_t)B, (int32_t)M, qkv.data_ptr(), stride, pos, (int32_t)axes, sections, (float)theta,
                q.data_ptr(), k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), (int32_t)k.size(2), first);
  });
}

// (addresses of jk_add_norm, jk_quantize_rows, jk_linear, jk_rope_qkv; the class Mx8)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&] {
    expect(count, 5);
    if (!PyType_Check(a[4])) refuse("expected a class");
    add_norm_fn = reinterpret_cast<decltype(add_norm_fn)>(PyLong_AsVoidPtr(a[0]));
    quantize_fn = reinterpret_cast<decltype(quantize_fn)>(PyLong_AsVoidPtr(a[1]));
    linear_fn = reinterpret_cast<decltype(linear_fn)>(PyLong_AsVoidPtr(a[2]));
    rope_fn = reinterpret_cast<decltype(rope_fn)>(PyLong_AsVoidPtr(a[3]));
    Py_INCREF(a[4]);
    mx8_type = reinterpret_cast<PyTypeObject*>(a[4]);
    return 0;
  });
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(add_norm), METHOD(quantize), METHOD(linear), METHOD(rope_qkv), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  codes_name = PyUnicode_InternFromString("codes");
  scales_name = PyUnicode_InternFromString("scales");
  return PyModule_Create(&module);
}
