// What the native bindings share: status and argument errors as ops.py raises
// them, and small conversions. Each binding is a module of its own.
#pragma once

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/utils/pybind.h>

#include "mra.h"

namespace py = pybind11;

namespace {

// ops.py's MraError factory; never destroyed (the interpreter ends first)
py::object& status_error = *new py::object();

// What fails here is raised as the Python function of ops.py raises it, also from
// the backward, whose errors reach the caller through the autograd engine: a
// refusal by the library as MraError, one by the checks as c10's ValueError and
// TypeError, which torch turns into Python's (as it does its own, an exhausted
// allocator's, and a saved-tensor hook's exception).
void ok(const char* fn, mra_status_t st) {
  if (st == MRA_OK) return;
  py::gil_scoped_acquire gil;
  const py::object err = status_error(fn, (int)st);
  PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(err.ptr())), err.ptr());
  python_error e;
  e.persist();
  throw e;
}

mra_dtype_t dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return MRA_F32;
  if (t.scalar_type() == at::kBFloat16) return MRA_BF16;
  TORCH_CHECK_TYPE(false, "unsupported dtype ", c10::toString(t.scalar_type()), "; expected float32 or bfloat16");
}

// A shape as Python writes it.
std::string tuple_of(at::IntArrayRef shape) {
  std::string s = "(";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + (shape.size() == 1 ? ",)" : ")");
}

void* ptr(const std::optional<at::Tensor>& t) { return t ? t->data_ptr() : nullptr; }

void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

template <class F>
void bind_one(const py::dict& a, const char* name, F& f) {
  f = reinterpret_cast<F>(a[name].cast<uintptr_t>());
}

}  // namespace
