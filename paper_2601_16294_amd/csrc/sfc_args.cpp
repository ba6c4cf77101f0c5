// What the Python binding of the small operators asks of its tensors (sfcops.py), in one call
// each: pointers and leading dimensions of arguments that are as they should be, None for any
// other, whose fault the Python code then names.  A small call is bound by its host time, half
// of which went into asking a tensor for its type, device, shape and strides one by one
// (us a call, so / here: quantisation 7.1 / 5.2, linear layer 11.2 / 9.1, product 9.2 / 5.9).
#include <ATen/ops/empty.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sfcgemm.h"

namespace {

// The tensor behind `o` if it is a plain one (no subclass) on the current GPU, else null.
const at::Tensor* tensor(PyObject* o) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != THPVariableClass) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided) return nullptr;
  return t.device() == c10::impl::getDeviceGuardImpl(at::kCUDA)->getDevice() ? &t : nullptr;
}

PyObject* pointer(const at::Tensor& t) { return PyLong_FromVoidPtr(t.data_ptr()); }

// Integer arguments from args[at] on; false with a Python error set.
template <int N>
bool integers(PyObject* const* args, int64_t (&v)[N]) {
  for (int i = 0; i < N; ++i) {
    v[i] = PyLong_AsLongLong(args[i]);
    if (v[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// rows(t, r, c) -> (pointer, leading dimension, type) of a 2-D fp32 or bf16 matrix with
// unit column stride, r x c where r >= 0.
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int64_t v[2];
  if (n != 3) Py_RETURN_NONE;
  if (!integers(args + 1, v)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* t = tensor(args[0]);
    if (!t || t->dim() != 2) Py_RETURN_NONE;
    const auto type = t->scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) Py_RETURN_NONE;
    const int64_t r = t->size(0), c = t->size(1);
    if (v[0] >= 0 && (r != v[0] || c != v[1])) Py_RETURN_NONE;
    if (t->stride(1) != 1 && c > 1) Py_RETURN_NONE;
    return Py_BuildValue("NLi", pointer(*t), (long long)(r > 1 ? t->stride(0) : c ? c : 1),
                         type == at::kFloat ? SFC_OUT_F32 : SFC_OUT_BF16);
  });
}

// mx4(q, s, lead, r, blocks) -> (codes, row bytes, scales, row bytes) of a 4-bit matrix
// with `lead` (0 or 1) dimensions before it; r and blocks < 0: any.
PyObject* mx4(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int64_t v[3];
  if (n != 5) Py_RETURN_NONE;
  if (!integers(args + 2, v)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *q = tensor(args[0]), *s = tensor(args[1]);
    const int64_t lead = v[0], dims = 2 + lead;
    if (!q || !s || lead < 0 || lead > 1 || q->dim() != dims || s->dim() != dims) Py_RETURN_NONE;
    if (q->scalar_type() != at::kByte || s->scalar_type() != at::kByte) Py_RETURN_NONE;
    const auto sq = q->sizes(), ss = s->sizes(), dq = q->strides(), ds = s->strides();
    const int64_t r = sq[lead], half = sq[lead + 1], blocks = ss[lead + 1];
    if (half != 16 * blocks || ss[lead] != r || (lead && ss[0] != sq[0])) Py_RETURN_NONE;
    if ((v[1] >= 0 && r != v[1]) || (v[2] >= 0 && blocks != v[2])) Py_RETURN_NONE;
    if ((dq[lead + 1] != 1 && half > 1) || (ds[lead + 1] != 1 && blocks > 1)) Py_RETURN_NONE;
    const int64_t padded = (blocks + 3) & ~(int64_t)3;
    if (padded != blocks && q->numel()) {
      int64_t last = s->storage_offset();
      for (int64_t i = 0; i <= lead; ++i) last += (ss[i] - 1) * ds[i];
      if (last + padded > (int64_t)s->storage().nbytes()) Py_RETURN_NONE;
    }
    return Py_BuildValue("NLNL", pointer(*q), (long long)(r > 1 ? dq[lead] : half ? half : 16), pointer(*s),
                         (long long)(r > 1 ? ds[lead] : padded ? padded : 4));
  });
}

// vector(t, fp32, count) -> pointer of a contiguous fp32 or int32 tensor of `count`
// elements (< 0: any number).
PyObject* vector(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int64_t v[2];
  if (n != 3) Py_RETURN_NONE;
  if (!integers(args + 1, v)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* t = tensor(args[0]);
    if (!t || t->scalar_type() != (v[0] ? at::kFloat : at::kInt) || !t->is_contiguous()) Py_RETURN_NONE;
    if (v[1] >= 0 && t->numel() != v[1]) Py_RETURN_NONE;
    return pointer(*t);
  });
}

// stack(t, n, r, c) -> (pointer, leading dimension, stride, type) of a 3-D fp32 or bf16 tensor with unit
// column stride, n x r x c where they are >= 0.
PyObject* stack(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int64_t v[3];
  if (n != 4) Py_RETURN_NONE;
  if (!integers(args + 1, v)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* t = tensor(args[0]);
    if (!t || t->dim() != 3) Py_RETURN_NONE;
    const auto type = t->scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) Py_RETURN_NONE;
    const int64_t r = t->size(1), c = t->size(2);
    for (int i = 0; i < 3; ++i)
      if (v[i] >= 0 && t->size(i) != v[i]) Py_RETURN_NONE;
    if (t->stride(2) != 1 && c > 1) Py_RETURN_NONE;
    return Py_BuildValue("NLLi", pointer(*t), (long long)(r > 1 ? t->stride(1) : c ? c : 1), (long long)t->stride(0),
                         type == at::kFloat ? SFC_OUT_F32 : SFC_OUT_BF16);
  });
}

// empty(rows, cols) -> (codes, scales) on the current GPU, rows of scales padded to whole dwords.
PyObject* empty(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int64_t v[2];
  if (n != 2) Py_RETURN_NONE;
  if (!integers(args, v)) return nullptr;
  return guarded([&]() -> PyObject* {
    if (v[0] < 0 || v[1] < 0) Py_RETURN_NONE;
    const int64_t blocks = (v[1] + 31) >> 5, padded = (blocks + 3) & ~(int64_t)3;
    const auto options = at::TensorOptions().dtype(at::kByte).device(at::kCUDA);
    at::Tensor q = at::empty({v[0], 16 * blocks}, options), s = at::empty({v[0], padded}, options);
    if (padded != blocks) s = s.narrow(1, 0, blocks);
    return Py_BuildValue("NN", THPVariable_Wrap(std::move(q)), THPVariable_Wrap(std::move(s)));
  });
}

PyMethodDef kMethods[] = {
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows)), METH_FASTCALL, nullptr},
    {"mx4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx4)), METH_FASTCALL, nullptr},
    {"vector", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(vector)), METH_FASTCALL, nullptr},
    {"stack", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(stack)), METH_FASTCALL, nullptr},
    {"empty", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(empty)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_sfcargs", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sfcargs() { return PyModule_Create(&kModule); }
