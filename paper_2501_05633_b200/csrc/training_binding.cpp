// The training operators for Python: checks of the tensors, outputs and workspaces from torch's allocator, and the calls of
// include/regtopk_train.h on the tensors' device and its current stream.  Marshalling only.
//
// A compiled module and not ctypes, because the smallest calls are a few microseconds of GPU time: marshalling a layer
// norm's gradient through ctypes cost 40 us a call, this costs a fifth of that.
//
// The functions take positional arguments alone; training.py gives them their names, defaults and documentation.

#include "binding_common.h"

namespace {

// ---- the operators ----------------------------------------------------------------------------------------------------
PyObject* dropout(PyObject* const* a) {  // x, p, seed, subsequence, out
  const Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Rows in = rows_of(x, "x");
  const regtopk_dropout_params drop = drop_params(a[1], a[2], a[3]);
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor* given = optional_tensor(a[4], "out");
  if (given) same_shape(*given, x, "out");
  const Tensor out = given ? *given : empty(x.sizes(), x.scalar_type(), x);
  const Rows to = given ? rows_of(out, "out") : Rows{in.rows, in.cols, in.cols};
  if (given) apart(out, x, "x", true);
  if (given) written(out, "out");
  check(regtopk_dropout(x.data_ptr(), in.ld, out.data_ptr(), to.ld, in.rows, in.cols, type, &drop, stream_of(x)), "regtopk_dropout");
  return THPVariable_Wrap(out);
}

PyObject* layer_norm(PyObject* const* a) {  // x, weight, bias, eps, residual, p, seed, subsequence
  const Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Rows in = rows_of(x, "x");
  const float* weight = vector_of(tensor(a[1], "weight"), in.cols, x, "weight");
  const Tensor* bias = optional_tensor(a[2], "bias");
  if (bias) vector_of(*bias, in.cols, x, "bias");
  const Tensor* residual = optional_tensor(a[4], "residual");
  if (residual) same_shape(*residual, x, "residual", true);
  const Rows res = residual ? rows_of(*residual, "residual") : Rows{0, 0, 0};
  const regtopk_dropout_params drop = drop_params(a[5], a[6], a[7]);
  const bool drops = drop.p != 0.0, makes_h = residual || drops;
  const at::ScalarType stream_type = residual ? residual->scalar_type() : x.scalar_type();
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor y = empty(x.sizes(), x.scalar_type(), x), h = makes_h ? empty(x.sizes(), stream_type, x) : x;
  const auto [mean, rstd] = two_of(x.sizes().slice(0, x.dim() - 1), x);
  check(regtopk_layer_norm(x.data_ptr(), in.ld, data(residual), res.ld, weight, static_cast<const float*>(data(bias)),
                           static_cast<float>(number(a[3])), y.data_ptr(), in.cols, makes_h ? h.data_ptr() : nullptr, in.cols,
                           static_cast<float*>(mean.data_ptr()), static_cast<float*>(rstd.data_ptr()), in.rows, in.cols, type,
                           type_of(h, "h"), drops ? &drop : nullptr, stream_of(x)), "regtopk_layer_norm");
  return Py_BuildValue("NNNN", THPVariable_Wrap(y), makes_h ? THPVariable_Wrap(h) : Py_NewRef(a[0]), THPVariable_Wrap(mean), THPVariable_Wrap(rstd));
}

// dy, h, mean, rstd, weight, dh, p, seed, subsequence, offsets, dweight, dbias, accumulate
PyObject* layer_norm_backward(PyObject* const* a) {
  const Tensor &dy = tensor(a[0], "dy"), &h = tensor(a[1], "h");
  const int type = type_of(dy, "dy");
  const Rows in = rows_of(dy, "dy");
  same_shape(h, dy, "h", true);
  const Rows hr = rows_of(h, "h");
  const float* mean = vector_of(tensor(a[2], "mean"), in.rows, dy, "mean");
  const float* rstd = vector_of(tensor(a[3], "rstd"), in.rows, dy, "rstd");
  const float* weight = vector_of(tensor(a[4], "weight"), in.cols, dy, "weight");
  const Tensor* dh = optional_tensor(a[5], "dh");
  if (dh) same_shape(*dh, h, "dh");
  const Rows dhr = dh ? rows_of(*dh, "dh") : Rows{0, 0, 0};
  const regtopk_dropout_params drop = drop_params(a[6], a[7], a[8]);
  const bool drops = drop.p != 0.0, accumulate = truth(a[12]);
  const Tensor* offsets = optional_tensor(a[9], "offsets");
  const int32_t groups = offsets ? groups_of(*offsets, dy) : 1;
  const Tensor *dw = optional_tensor(a[10], "dweight"), *db = optional_tensor(a[11], "dbias");
  int64_t ld[2] = {in.cols, in.cols};
  const char* names[2] = {"dweight", "dbias"};
  for (int i = 0; i < 2; ++i) {
    const Tensor* t = i ? db : dw;
    if (!t) continue;
    if (t->device() != dy.device() || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != groups || t->size(1) != in.cols)
      type_error(std::string(names[i]) + " must be float32 [" + std::to_string(groups) + ", " + std::to_string(in.cols) + "] on the input's device");
    ld[i] = rows_of(*t, names[i]).ld;
  }
  if (accumulate && !dw && !db) value_error("accumulate needs dweight or dbias to add to");
  if (dw) written(*dw, "dweight");
  if (db) written(*db, "dbias");
  const c10::cuda::CUDAGuard guard(dy.device());
  Tensor made[2];
  if (!dw && !db) {
    std::tie(made[0], made[1]) = two_of({groups, in.cols}, dy);
    dw = &made[0];
    db = &made[1];
  }
  const bool same = !drops && h.scalar_type() == dy.scalar_type();
  const Tensor dx = empty(dy.sizes(), dy.scalar_type(), dy), dres = same ? dx : empty(dy.sizes(), h.scalar_type(), dy);
  const size_t bytes = regtopk_layer_norm_backward_workspace_bytes(in.rows, in.cols, groups);
  const Tensor ws = empty({static_cast<int64_t>(bytes)}, at::kByte, dy);
  check(regtopk_layer_norm_backward(dy.data_ptr(), in.ld, h.data_ptr(), hr.ld, mean, rstd, weight, data(dh), dhr.ld, dx.data_ptr(), in.cols,
                                    same ? nullptr : dres.data_ptr(), in.cols, static_cast<float*>(data(dw)), ld[0],
                                    static_cast<float*>(data(db)), ld[1], static_cast<const int64_t*>(data(offsets)), groups, accumulate,
                                    in.rows, in.cols, type, type_of(h, "h"), drops ? &drop : nullptr, ws.data_ptr(), bytes, stream_of(dy)),
        "regtopk_layer_norm_backward");
  PyObject* px = THPVariable_Wrap(dx);
  PyObject* pres = same ? Py_NewRef(px) : THPVariable_Wrap(dres);
  auto out = [&](int i) { return made[i].defined() ? THPVariable_Wrap(made[i]) : Py_NewRef(a[10 + i]); };
  return Py_BuildValue("NNNN", px, pres, out(0), out(1));
}

PyObject* grouped_matmul(PyObject* const* a) {  // x, w, offsets, out
  const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w"), &offsets = tensor(a[2], "offsets");
  const int type = short_type_of(x, "x");
  const Rows in = rows_of(x, "x");
  const int32_t groups = groups_of(offsets, x);
  if (w.device() != x.device() || w.scalar_type() != x.scalar_type() || w.dim() != 3 || w.size(2) != in.cols)
    type_error("w must be [experts, m, " + std::to_string(in.cols) + "] of x's dtype on x's device");
  const int64_t count = w.size(0), m = w.size(1), k = in.cols;
  if (count < 1 || groups % count) value_error("the number of groups must be a multiple of the number of matrices");
  const bool transposed = !(k <= 1 || w.stride(2) == 1);
  if (transposed && m > 1 && w.stride(1) != 1) value_error("w: one of its last two dimensions must be contiguous");
  const int64_t ldw = transposed ? w.stride(2) : m > 1 ? w.stride(1) : k, width = transposed ? m : k;
  if (ldw < width) value_error("w: rows overlap");
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor* given = optional_tensor(a[3], "out");
  if (given && (given->device() != x.device() || given->scalar_type() != x.scalar_type() || given->dim() != 2 ||
                given->size(0) != in.rows || given->size(1) != m))
    type_error("out must be [" + std::to_string(in.rows) + ", " + std::to_string(m) + "] of x's dtype on x's device");
  const Tensor y = given ? *given : empty({in.rows, m}, x.scalar_type(), x);
  const int64_t ldy = given ? rows_of(y, "out").ld : m;
  if (given) {
    apart(y, x, "x");
    apart(y, w, "w");
    written(y, "out");
  }
  const int32_t weights = static_cast<int32_t>(count);
  const int64_t stride = count > 1 ? w.stride(0) : ldw * (transposed ? k : m);
  const size_t bytes = regtopk_grouped_matmul_workspace_bytes(x.data_ptr(), in.ld, w.data_ptr(), ldw, stride, transposed, weights, groups, in.rows, k, m);
  Tensor ws;
  if (bytes) ws = empty({static_cast<int64_t>(bytes)}, at::kByte, x);
  check(regtopk_grouped_matmul(x.data_ptr(), in.ld, w.data_ptr(), ldw, stride, transposed, weights, y.data_ptr(), ldy,
                               static_cast<const int64_t*>(offsets.data_ptr()), groups, in.rows, k, m, type, bytes ? ws.data_ptr() : nullptr,
                               bytes, stream_of(x)), "regtopk_grouped_matmul");
  return given ? Py_NewRef(a[3]) : THPVariable_Wrap(y);
}

PyObject* grouped_matmul_dw(PyObject* const* a) {  // dy, x, offsets, out, accumulate
  const Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &offsets = tensor(a[2], "offsets");
  const int type = short_type_of(dy, "dy");
  const Rows up = rows_of(dy, "dy");
  const int32_t groups = groups_of(offsets, dy);
  if (x.device() != dy.device() || x.scalar_type() != dy.scalar_type() || x.dim() != 2 || x.size(0) != up.rows)
    type_error("x must be [" + std::to_string(up.rows) + ", k] of dy's dtype on dy's device");
  const Rows in = rows_of(x, "x");
  const Tensor* given = optional_tensor(a[3], "out");
  const bool accumulate = truth(a[4]);
  if (accumulate && !given) value_error("accumulate needs an out to add to");
  const int64_t m = up.cols, k = in.cols;
  const c10::cuda::CUDAGuard guard(dy.device());
  const Tensor out = given ? *given : empty({groups, m, k}, at::kFloat, dy);
  const int64_t n = out.dim();
  if (out.device() != dy.device() || out.scalar_type() != at::kFloat || (n != 3 && n != 4) || out.size(n - 2) != m || out.size(n - 1) != k ||
      (n == 3 ? out.size(0) : out.size(0) * out.size(1)) != groups)
    type_error("out must be float32 [" + std::to_string(groups) + ", " + std::to_string(m) + ", " + std::to_string(k) +
               "], or with the groups split into [workers, experts], on dy's device");
  const int64_t ld = m > 1 ? out.stride(n - 2) : k;
  if ((k > 1 && out.stride(n - 1) != 1) || ld < k) value_error("out: the elements of a row must be contiguous and rows must not overlap");
  if (out.numel() && !elements_apart(out)) value_error("out: matrices overlap");
  if (given) written(out, "out");
  const int32_t inner = n == 3 ? groups : static_cast<int32_t>(out.size(1));
  const int64_t inner_stride = out.stride(n - 3), outer_stride = n == 3 ? 0 : out.stride(0);
  const size_t bytes = regtopk_grouped_matmul_dw_workspace_bytes(dy.data_ptr(), up.ld, x.data_ptr(), in.ld, groups, up.rows, k, m);
  Tensor ws;
  if (bytes) ws = empty({static_cast<int64_t>(bytes)}, at::kByte, dy);
  check(regtopk_grouped_matmul_dw(dy.data_ptr(), up.ld, x.data_ptr(), in.ld, static_cast<float*>(out.data_ptr()), ld, inner_stride, outer_stride,
                                  inner, accumulate, static_cast<const int64_t*>(offsets.data_ptr()), groups, up.rows, k, m, type,
                                  bytes ? ws.data_ptr() : nullptr, bytes, stream_of(dy)), "regtopk_grouped_matmul_dw");
  return given ? Py_NewRef(a[3]) : THPVariable_Wrap(out);
}

PyObject* status(PyObject* const* a) {  // stream
  const unsigned long long s = whole(a[0], UINT64_MAX, "a stream's handle");
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = regtopk_train_status(reinterpret_cast<void*>(s));
  Py_END_ALLOW_THREADS
  check(rc, "regtopk_train_status");
  Py_RETURN_NONE;
}

PyObject* raise_with(PyObject* const* a) {
  Py_XSETREF(g_error, Py_NewRef(a[0]));
  Py_XSETREF(g_out_of_memory, Py_NewRef(a[1]));
  Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    ENTRY("dropout", dropout, 5), ENTRY("layer_norm", layer_norm, 8), ENTRY("layer_norm_backward", layer_norm_backward, 13),
    ENTRY("grouped_matmul", grouped_matmul, 4), ENTRY("grouped_matmul_dw", grouped_matmul_dw, 5), ENTRY("status", status, 1),
    ENTRY("raise_with", raise_with, 2), {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_training", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__training() {
  PyObject* m = PyModule_Create(&g_module);
  if (m && PyModule_AddFunctions(m, g_expert_methods) < 0) Py_CLEAR(m);
  return m;
}
