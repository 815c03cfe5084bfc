// What the sources of the compiled Python module share: checks of the tensors, outputs and workspaces from torch's allocator, the
// tensors' device and its current stream, and the way in which a function is entered from Python.
#ifndef REGTOPK_BINDING_COMMON_H_
#define REGTOPK_BINDING_COMMON_H_

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/MemoryOverlap.h>
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <string>
#include <utility>
#include <vector>

#include "regtopk_experts.h"

namespace regtopk_binding {
inline PyObject* g_error = nullptr;          // called with (code, where); makes the exception that a failed call raises
inline PyObject* g_out_of_memory = nullptr;  // torch's type
}  // namespace regtopk_binding
using namespace regtopk_binding;

namespace {

using at::Tensor;

// Thrown where the Python error is already set.
struct Raised {};

[[noreturn]] void fail(PyObject* type, const std::string& what) {
  PyErr_SetString(type, what.c_str());
  throw Raised();
}
[[noreturn]] void type_error(const std::string& what) { fail(PyExc_TypeError, what); }
[[noreturn]] void value_error(const std::string& what) { fail(PyExc_ValueError, what); }

void check(int code, const char* where) {
  if (code == REGTOPK_OK) return;
  if (PyObject* e = PyObject_CallFunction(g_error, "is", code, where)) {
    PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e);
    Py_DECREF(e);
  }
  throw Raised();
}

const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) type_error(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
const Tensor* optional_tensor(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v;
}

int type_of(const Tensor& t, const char* name) {
  if (!t.is_cuda() || t.layout() != at::kStrided) type_error(std::string(name) + " must live on the device");
  switch (t.scalar_type()) {
    case at::kFloat: return REGTOPK_TYPE_F32;
    case at::kBFloat16: return REGTOPK_TYPE_BF16;
    case at::kHalf: return REGTOPK_TYPE_F16;
    default: type_error(std::string(name) + " is float32, bfloat16 or float16");
  }
}
int short_type_of(const Tensor& t, const char* name) {
  const int code = type_of(t, name);
  if (code == REGTOPK_TYPE_F32) type_error(std::string(name) + " is bfloat16 or float16");
  if (t.dim() != 2) value_error(std::string(name) + " is a matrix");
  return code;
}

// A tensor as rows: its last dimension is the row, and one distance leads from each row to the next.
struct Rows { int64_t rows, cols, ld; };
Rows rows_of(const Tensor& t, const char* name) {
  const auto size = t.sizes();
  const auto stride = t.strides();
  const int64_t n = t.dim();
  if (n == 0) value_error(std::string(name) + " needs at least one dimension");
  Rows r{1, size[n - 1], size[n - 1]};
  for (int64_t i = 0; i < n - 1; ++i) r.rows *= size[i];
  if (r.rows == 0 || r.cols == 0) return r;
  if (r.cols > 1 && stride[n - 1] != 1) value_error(std::string(name) + ": the elements of a row must be contiguous");
  int64_t span = 0;  // what one step of the dimension to the left has to be
  bool known = false;  // whether a dimension has given the row distance (0 too: an expanded one repeats its rows, and is refused)
  for (int64_t i = n - 2; i >= 0; --i) {
    if (size[i] == 1) continue;
    if (!known) r.ld = stride[i];
    else if (stride[i] != span) value_error(std::string(name) + ": no single distance leads from row to row (make it contiguous)");
    known = true;
    span = stride[i] * size[i];
  }
  if (r.ld < r.cols) value_error(std::string(name) + ": rows overlap");
  return r;
}

// Whether no two elements of a tensor lie in one place, for certain: sorted, each distance passes what the smaller ones span.
bool elements_apart(const Tensor& t) {
  std::vector<std::pair<int64_t, int64_t>> d;  // distance, count
  for (int64_t i = 0; i < t.dim(); ++i)
    if (t.size(i) > 1) d.emplace_back(t.stride(i), t.size(i));
  std::sort(d.begin(), d.end());
  int64_t span = 1;
  for (const auto& [stride, count] : d) {
    if (stride < span) return false;
    span += stride * (count - 1);
  }
  return true;
}

void same_shape(const Tensor& t, const Tensor& x, const char* name, bool or_float = false) {
  if (t.device() != x.device() || t.sizes() != x.sizes() || t.layout() != at::kStrided ||
      !(t.scalar_type() == x.scalar_type() || (or_float && t.scalar_type() == at::kFloat)))
    type_error(std::string(name) + " must match the input's shape, device and dtype" + (or_float ? " (or be float32)" : ""));
}
// A tensor that a call writes.  As with torch's own `out` arguments, one that autograd would have to follow is refused while it
// records, and its version goes up, so that a backward pass that has saved it for its own use notices.
void written(const Tensor& t, const char* name) {
  if (at::GradMode::is_enabled() && t.requires_grad()) value_error(std::string(name) + " requires a gradient, but autograd does not see this call (use torch.no_grad())");
  t.unsafeGetTensorImpl()->bump_version();
}
// Refuses an output that shares memory with an input, where torch can tell.  `same`: it may be the very input.
void apart(const Tensor& out, const Tensor& in, const char* name, bool same = false, const char* out_name = "out") {
  const at::MemOverlapStatus how = at::get_overlap_status(out, in);
  if (how == at::MemOverlapStatus::Partial || (how == at::MemOverlapStatus::Full && !same)) value_error(std::string(out_name) + " and " + name + " overlap");
}
const float* vector_of(const Tensor& t, int64_t n, const Tensor& x, const char* name) {
  if (t.device() != x.device() || t.scalar_type() != at::kFloat || t.numel() != n || !t.is_contiguous())
    type_error(std::string(name) + " must be " + std::to_string(n) + " contiguous float32 values on the input's device");
  return static_cast<const float*>(t.data_ptr());
}
int32_t groups_of(const Tensor& offsets, const Tensor& x) {
  if (offsets.device() != x.device() || offsets.scalar_type() != at::kLong || offsets.dim() != 1 || !offsets.is_contiguous() ||
      offsets.size(0) < 2 || offsets.size(0) > INT32_MAX)
    type_error("offsets must be a contiguous int64 vector of at least two values on the input's device");
  return static_cast<int32_t>(offsets.size(0) - 1);
}

uint64_t whole(PyObject* o, uint64_t most, const char* what) {
  PyObject* i = PyNumber_Index(o);
  if (!i) throw Raised();
  const unsigned long long v = PyLong_AsUnsignedLongLong(i);
  Py_DECREF(i);
  const bool bad = v == static_cast<unsigned long long>(-1) && PyErr_Occurred();
  if (bad) PyErr_Clear();
  if (bad || v > most) value_error(what);
  return v;
}
regtopk_dropout_params drop_params(PyObject* p, PyObject* seed, PyObject* subsequence) {
  regtopk_dropout_params d;
  d.p = number(p);
  if (!(d.p >= 0.0 && d.p <= 1.0)) value_error("p is a probability");
  d.seed = whole(seed, UINT64_MAX, "seed has 64 bits");
  d.subsequence = static_cast<uint32_t>(whole(subsequence, UINT32_MAX, "subsequence has 32 bits"));
  return d;
}

Tensor empty(at::IntArrayRef size, at::ScalarType type, const Tensor& like) {
  return at::detail::empty_cuda(size, type, like.device(), std::nullopt);
}
// Two float32 tensors of one size in one allocation: they live and die together, and every allocation costs 0.7 us.
std::pair<Tensor, Tensor> two_of(at::IntArrayRef size, const Tensor& like) {
  int64_t n = 1;
  for (const int64_t s : size) n *= s;
  const Tensor whole = empty({2 * n}, at::kFloat, like);
  const auto part = [&](int64_t at) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
    impl->set_storage_offset(at);
    impl->set_sizes_contiguous(size);
    return Tensor(std::move(impl));
  };
  return {part(0), part(n)};
}
// The same for two tensors of any sizes and types; the second begins at a multiple of 16 bytes.
std::pair<Tensor, Tensor> two_of(at::IntArrayRef size, at::ScalarType type, at::IntArrayRef other_size, at::ScalarType other_type, const Tensor& like) {
  const auto bytes_of = [](at::IntArrayRef s, at::ScalarType t) {
    int64_t n = static_cast<int64_t>(c10::elementSize(t));
    for (const int64_t i : s) n *= i;
    return n;
  };
  const int64_t second = (bytes_of(size, type) + 15) & ~int64_t(15);
  const Tensor whole = empty({second + bytes_of(other_size, other_type)}, at::kByte, like);
  const auto part = [&](at::IntArrayRef s, at::ScalarType t, int64_t at) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), c10::scalarTypeToTypeMeta(t));
    impl->set_storage_offset(at / static_cast<int64_t>(c10::elementSize(t)));
    impl->set_sizes_contiguous(s);
    return Tensor(std::move(impl));
  };
  return {part(size, type, 0), part(other_size, other_type, second)};
}
// Two tensors that need not live and die together: in one allocation only where they are so small (a megabyte) that what the longer one
// keeps alive of the other does not matter, but the 0.8 us of a second allocation do.
std::pair<Tensor, Tensor> two_if_small(at::IntArrayRef size, at::ScalarType type, at::IntArrayRef other_size, at::ScalarType other_type, const Tensor& like) {
  int64_t n = static_cast<int64_t>(c10::elementSize(type)), m = static_cast<int64_t>(c10::elementSize(other_type));
  for (const int64_t i : size) n *= i;
  for (const int64_t i : other_size) m *= i;
  if (n + m <= 1 << 20) return two_of(size, type, other_size, other_type, like);
  return {empty(size, type, like), empty(other_size, other_type, like)};
}
void* stream_of(const Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }
void* data(const Tensor* t) { return t ? t->data_ptr() : nullptr; }

// No C++ exception leaves the module: torch's errors become RuntimeErrors.
template <PyObject* (*F)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_Format(PyExc_TypeError, "expected %d arguments, got %d", kArgs, (int)n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised&) {
    return nullptr;
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(g_out_of_memory, e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

#define ENTRY(name, f, n) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<f, n>)), METH_FASTCALL, nullptr}

}  // namespace

// The functions of the operators around an expert sublayer (experts_binding.cpp), for the module's table.
extern PyMethodDef g_expert_methods[];
#endif
