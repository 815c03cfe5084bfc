// The operators around an expert sublayer for Python: the calls of include/regtopk_experts.h.  Marshalling only; experts.py gives
// the functions their names, defaults and documentation.

#include "binding_common.h"

#include <torch/csrc/Dtype.h>

namespace {

int32_t small(PyObject* o, int32_t least, int32_t most, const char* what) {
  const uint64_t v = whole(o, static_cast<uint64_t>(most), what);
  if (v < static_cast<uint64_t>(least)) value_error(what);
  return static_cast<int32_t>(v);
}

at::ScalarType dtype_of(PyObject* o, const char* name) {
  if (!THPDtype_Check(o)) type_error(std::string(name) + " must be a torch.dtype");
  const at::ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
  if (t != at::kFloat && t != at::kBFloat16 && t != at::kHalf) type_error(std::string(name) + " is float32, bfloat16 or float16");
  return t;
}
int code_of(at::ScalarType t) { return t == at::kFloat ? REGTOPK_TYPE_F32 : t == at::kBFloat16 ? REGTOPK_TYPE_BF16 : REGTOPK_TYPE_F16; }

int64_t blocks_of(int64_t cols) { return (cols + 31) / 32; }

// 8-bit rows: a pair (values, scales) whose scales have a block for every 32 columns of each of a row's `halves`.
struct Packed {
  const Tensor *values, *scales;
  Rows v, s;
};
Packed packed_of(PyObject* o, const char* name, int halves) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) type_error(std::string(name) + " must be a tensor or a pair of values and scales");
  Packed p{&tensor(PyTuple_GET_ITEM(o, 0), "values"), &tensor(PyTuple_GET_ITEM(o, 1), "scales"), {}, {}};
  const Tensor &v = *p.values, &s = *p.scales;
  if (!v.is_cuda() || v.layout() != at::kStrided || v.scalar_type() != at::kFloat8_e4m3fn) type_error(std::string(name) + ": values are float8_e4m3fn on the device");
  if (s.device() != v.device() || s.layout() != at::kStrided || s.scalar_type() != at::kFloat8_e8m0fnu) type_error(std::string(name) + ": scales are float8_e8m0fnu on the values' device");
  p.v = rows_of(v, "values");
  p.s = rows_of(s, "scales");
  if (p.v.cols % halves) value_error(std::string(name) + ": a gated activation's input has an even number of columns");
  if (s.dim() != v.dim() || s.sizes().slice(0, s.dim() - 1) != v.sizes().slice(0, v.dim() - 1) || s.size(-1) != halves * blocks_of(p.v.cols / halves))
    type_error(std::string(name) + ": scales must be the rows' own, one for every 32 columns");
  return p;
}
const uint8_t* bytes_of(const Tensor* t) { return t ? static_cast<const uint8_t*>(t->data_ptr()) : nullptr; }

// New 8-bit rows for rows of `sizes`.
struct NewPacked {
  Tensor values, scales;
  int64_t ld_values, ld_scales;
  uint8_t* v() const { return static_cast<uint8_t*>(values.data_ptr()); }
  uint8_t* s() const { return static_cast<uint8_t*>(scales.data_ptr()); }
  PyObject* wrap() const { return Py_BuildValue("NN", THPVariable_Wrap(values), THPVariable_Wrap(scales)); }
};
NewPacked new_packed(at::IntArrayRef sizes, const Tensor& like, int halves) {
  std::vector<int64_t> s(sizes.begin(), sizes.end());
  const int64_t cols = s.back(), blocks = halves * blocks_of(cols / halves);
  s.back() = blocks;
  auto [v, e] = two_of(sizes, at::kFloat8_e4m3fn, s, at::kFloat8_e8m0fnu, like);
  return {std::move(v), std::move(e), cols, blocks};
}

// [..., k] values of one 32-bit type, contiguous, on x's device.
void index_like(const Tensor& t, at::ScalarType type, const Tensor& x, const char* name) {
  if (t.device() != x.device() || t.scalar_type() != type || t.dim() < 1 || !t.is_contiguous())
    type_error(std::string(name) + " must be contiguous " + (type == at::kInt ? "int32" : "float32") + " values on the input's device, with a token's in the last dimension");
}
int64_t tokens_of(const Tensor& place) { return place.size(-1) ? place.numel() / place.size(-1) : 0; }
int32_t choices_of(const Tensor& place, const char* name) {
  const int64_t k = place.size(-1);
  if (k < 1 || k > INT32_MAX) value_error(std::string(name) + ": a token has at least one");
  return static_cast<int32_t>(k);
}
const int64_t* filled_of(const Tensor& offsets, const Tensor& x) {
  return static_cast<const int64_t*>(offsets.data_ptr()) + groups_of(offsets, x);
}
std::vector<int64_t> with_cols(at::IntArrayRef sizes, int64_t cols) {
  std::vector<int64_t> s(sizes.begin(), sizes.end());
  s.back() = cols;
  return s;
}

// ---- 8-bit rows -------------------------------------------------------------------------------------------------------
PyObject* pack8(PyObject* const* a) {  // x
  const Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Rows in = rows_of(x, "x");
  const c10::cuda::CUDAGuard guard(x.device());
  const NewPacked p = new_packed(x.sizes(), x, 1);
  check(regtopk_pack8(x.data_ptr(), in.ld, p.v(), p.ld_values, p.s(), p.ld_scales, in.rows, in.cols, type, stream_of(x)), "regtopk_pack8");
  return p.wrap();
}

PyObject* unpack8(PyObject* const* a) {  // rows8, dtype
  const Packed p = packed_of(a[0], "rows8", 1);
  const at::ScalarType type = dtype_of(a[1], "dtype");
  const c10::cuda::CUDAGuard guard(p.values->device());
  const Tensor x = empty(p.values->sizes(), type, *p.values);
  check(regtopk_unpack8(bytes_of(p.values), p.v.ld, bytes_of(p.scales), p.s.ld, x.data_ptr(), p.v.cols, p.v.rows, p.v.cols, code_of(type), stream_of(x)),
        "regtopk_unpack8");
  return THPVariable_Wrap(x);
}

// ---- the router -------------------------------------------------------------------------------------------------------
int32_t scores_of(PyObject* o) {
  const char* s = PyUnicode_Check(o) ? PyUnicode_AsUTF8(o) : nullptr;
  if (s && std::string(s) == "softmax") return REGTOPK_SCORES_SOFTMAX;
  if (s && std::string(s) == "sigmoid") return REGTOPK_SCORES_SIGMOID;
  PyErr_Clear();
  value_error("scores are \"softmax\" or \"sigmoid\"");
}
Rows logits_of(const Tensor& logits, int* type) {
  *type = type_of(logits, "logits");
  const Rows in = rows_of(logits, "logits");
  if (in.cols < 1) value_error("logits: a token has at least one expert");
  return in;
}

PyObject* route(PyObject* const* a) {  // logits, k, scores, bias, groups, groups_kept, group_top, renormalise, scale
  const Tensor& logits = tensor(a[0], "logits");
  int type;
  const Rows in = logits_of(logits, &type);
  const int32_t most = static_cast<int32_t>(std::min<int64_t>(in.cols, INT32_MAX));
  const int32_t k = small(a[1], 1, most, "k is between 1 and the number of experts");
  const Tensor* bias = optional_tensor(a[3], "bias");
  if (bias) vector_of(*bias, in.cols, logits, "bias");
  regtopk_route_params p;
  p.scores = scores_of(a[2]);
  p.groups = small(a[4], 1, most, "groups is between 1 and the number of experts");
  if (in.cols % p.groups) value_error("the number of experts must be a multiple of the number of groups");
  p.groups_kept = small(a[5], 1, p.groups, "groups_kept is between 1 and groups");
  p.group_top = small(a[6], 1, 2, "group_top is 1 or 2");
  p.renormalise = truth(a[7]);
  p.scale = static_cast<float>(number(a[8]));
  if (!(p.scale - p.scale == 0.0f)) value_error("scale is a finite float32 number");
  const c10::cuda::CUDAGuard guard(logits.device());
  const std::vector<int64_t> size = with_cols(logits.sizes(), k);
  const auto [experts, weights] = two_if_small(size, at::kInt, size, at::kFloat, logits);
  check(regtopk_route(logits.data_ptr(), in.ld, static_cast<const float*>(data(bias)), static_cast<int32_t*>(experts.data_ptr()),
                      static_cast<float*>(weights.data_ptr()), in.rows, most, k, type, &p, stream_of(logits)), "regtopk_route");
  return Py_BuildValue("NN", THPVariable_Wrap(experts), THPVariable_Wrap(weights));
}

PyObject* route_backward(PyObject* const* a) {  // dweights, logits, experts, scores, renormalise, scale
  const Tensor &dweights = tensor(a[0], "dweights"), &logits = tensor(a[1], "logits"), &experts = tensor(a[2], "experts");
  int type;
  const Rows in = logits_of(logits, &type);
  index_like(experts, at::kInt, logits, "experts");
  index_like(dweights, at::kFloat, logits, "dweights");
  const int32_t k = choices_of(experts, "experts"), most = static_cast<int32_t>(std::min<int64_t>(in.cols, INT32_MAX));
  if (experts.sizes() != dweights.sizes() || experts.dim() != logits.dim() ||
      experts.sizes().slice(0, experts.dim() - 1) != logits.sizes().slice(0, logits.dim() - 1) || k > in.cols)
    type_error("experts and dweights must be [..., k] for the tokens of logits, k at most the number of experts");
  regtopk_route_params p{scores_of(a[3]), 1, 1, 1, truth(a[4]), static_cast<float>(number(a[5]))};
  if (!(p.scale - p.scale == 0.0f)) value_error("scale is a finite float32 number");
  const c10::cuda::CUDAGuard guard(logits.device());
  const Tensor out = empty(logits.sizes(), logits.scalar_type(), logits);
  check(regtopk_route_backward(static_cast<const float*>(dweights.data_ptr()), logits.data_ptr(), in.ld, static_cast<const int32_t*>(experts.data_ptr()),
                               out.data_ptr(), in.cols, in.rows, most, k, type, &p, stream_of(logits)), "regtopk_route_backward");
  return THPVariable_Wrap(out);
}

// ---- the tokens' way --------------------------------------------------------------------------------------------------
PyObject* sort_tokens(PyObject* const* a) {  // experts, n_experts, workers
  const Tensor& experts = tensor(a[0], "experts");
  if (!experts.is_cuda()) type_error("experts must live on the device");
  index_like(experts, at::kInt, experts, "experts");
  const int32_t k = choices_of(experts, "experts"), n = small(a[1], 1, INT32_MAX, "n_experts is at least 1");
  const Tensor* at = optional_tensor(a[2], "workers");
  const int32_t workers = at ? groups_of(*at, experts) : 1;
  const int64_t tokens = tokens_of(experts);
  if (static_cast<int64_t>(n) * workers > REGTOPK_MATMUL_MAX_GROUPS) check(REGTOPK_ERR_TOO_LARGE, "regtopk_sort_tokens");
  const c10::cuda::CUDAGuard guard(experts.device());
  const auto [offsets, place] = two_if_small({static_cast<int64_t>(n) * workers + 1}, at::kLong, experts.sizes(), at::kInt, experts);
  const size_t bytes = regtopk_sort_tokens_workspace_bytes(tokens, k, n, workers);
  Tensor ws;
  if (bytes) ws = empty({static_cast<int64_t>(bytes)}, at::kByte, experts);
  check(regtopk_sort_tokens(static_cast<const int32_t*>(experts.data_ptr()), static_cast<const int64_t*>(data(at)), workers,
                            static_cast<int64_t*>(offsets.data_ptr()), static_cast<int32_t*>(place.data_ptr()), tokens, k, n,
                            bytes ? ws.data_ptr() : nullptr, bytes, stream_of(experts)), "regtopk_sort_tokens");
  return Py_BuildValue("NN", THPVariable_Wrap(offsets), THPVariable_Wrap(place));
}

PyObject* spread_tokens(PyObject* const* a) {  // x, place, offsets, dtype
  const bool pair = PyTuple_Check(a[0]);
  Packed p{};
  if (pair) p = packed_of(a[0], "x", 1);
  const Tensor& x = pair ? *p.values : tensor(a[0], "x");
  if (!pair) type_of(x, "x");
  const Rows in = pair ? p.v : rows_of(x, "x");
  const at::ScalarType type = a[3] == Py_None ? (pair ? at::kBFloat16 : x.scalar_type()) : dtype_of(a[3], "dtype");
  if (!pair && type != x.scalar_type()) type_error("dtype must be x's own, but for 8-bit rows");
  const Tensor &place = tensor(a[1], "place"), &offsets = tensor(a[2], "offsets");
  index_like(place, at::kInt, x, "place");
  const int32_t k = choices_of(place, "place");
  if (tokens_of(place) != in.rows) type_error("place must be [..., k] for the tokens of x");
  const int64_t* filled = filled_of(offsets, x);
  const int64_t rows = place.numel();
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor out = empty({rows, in.cols}, type, x);
  check(regtopk_spread_tokens(x.data_ptr(), in.ld, bytes_of(p.scales), p.s.ld, static_cast<const int32_t*>(place.data_ptr()), filled, out.data_ptr(),
                              in.cols, in.rows, k, rows, in.cols, code_of(type), stream_of(x)), "regtopk_spread_tokens");
  return THPVariable_Wrap(out);
}

PyObject* join_tokens(PyObject* const* a) {  // rows, place, weights, residual
  const Tensor &from = tensor(a[0], "rows"), &place = tensor(a[1], "place");
  const int type = type_of(from, "rows");
  if (from.dim() != 2) value_error("rows is a matrix");
  const Rows in = rows_of(from, "rows");
  index_like(place, at::kInt, from, "place");
  const int32_t k = choices_of(place, "place");
  const Tensor* weights = optional_tensor(a[2], "weights");
  if (weights) index_like(*weights, at::kFloat, from, "weights");
  if (weights && weights->sizes() != place.sizes()) type_error("weights must have the shape of place");
  const int64_t tokens = tokens_of(place);
  const Tensor* residual = optional_tensor(a[3], "residual");
  Rows res{0, 0, 0};
  if (residual) {
    if (residual->device() != from.device() || residual->layout() != at::kStrided ||
        (residual->scalar_type() != from.scalar_type() && residual->scalar_type() != at::kFloat))
      type_error("residual must be of rows' dtype or float32, on its device");
    res = rows_of(*residual, "residual");
    if (res.rows != tokens || res.cols != in.cols) type_error("residual must have a row for each token of place");
  }
  const at::ScalarType out_type = residual ? residual->scalar_type() : from.scalar_type();
  const c10::cuda::CUDAGuard guard(from.device());
  const Tensor out = residual ? empty(residual->sizes(), out_type, from) : empty(with_cols(place.sizes(), in.cols), out_type, from);
  check(regtopk_join_tokens(from.data_ptr(), in.ld, static_cast<const int32_t*>(place.data_ptr()), static_cast<const float*>(data(weights)),
                            data(residual), res.ld, out.data_ptr(), in.cols, tokens, k, in.rows, in.cols, type, code_of(out_type), stream_of(from)),
        "regtopk_join_tokens");
  return THPVariable_Wrap(out);
}

PyObject* join_tokens_backward(PyObject* const* a) {  // dout, rows, place, weights, offsets
  const Tensor &dout = tensor(a[0], "dout"), &from = tensor(a[1], "rows"), &place = tensor(a[2], "place"), &weights = tensor(a[3], "weights"),
               &offsets = tensor(a[4], "offsets");
  const int type = type_of(from, "rows"), dtype = type_of(dout, "dout");
  if (from.dim() != 2) value_error("rows is a matrix");
  if (dout.device() != from.device() || (dtype != type && dtype != REGTOPK_TYPE_F32)) type_error("dout must be of rows' dtype or float32, on its device");
  const Rows in = rows_of(from, "rows"), up = rows_of(dout, "dout");
  index_like(place, at::kInt, from, "place");
  index_like(weights, at::kFloat, from, "weights");
  if (weights.sizes() != place.sizes()) type_error("weights must have the shape of place");
  const int32_t k = choices_of(place, "place");
  const int64_t tokens = tokens_of(place);
  if (up.rows != tokens || up.cols != in.cols) type_error("dout must have a row for each token of place, as wide as rows");
  const int64_t* filled = filled_of(offsets, from);
  const c10::cuda::CUDAGuard guard(from.device());
  const auto [drows, dweights] = two_if_small(from.sizes(), from.scalar_type(), place.sizes(), at::kFloat, from);
  check(regtopk_join_tokens_backward(dout.data_ptr(), up.ld, from.data_ptr(), in.ld, static_cast<const int32_t*>(place.data_ptr()),
                                     static_cast<const float*>(weights.data_ptr()), filled, drows.data_ptr(), in.cols,
                                     static_cast<float*>(dweights.data_ptr()), tokens, k, in.rows, in.cols, type, dtype, stream_of(from)),
        "regtopk_join_tokens_backward");
  return Py_BuildValue("NN", THPVariable_Wrap(drows), THPVariable_Wrap(dweights));
}

// ---- activations ------------------------------------------------------------------------------------------------------
int32_t kind_of(PyObject* o) {
  const char* s = PyUnicode_Check(o) ? PyUnicode_AsUTF8(o) : nullptr;
  if (s && std::string(s) == "silu") return REGTOPK_ACTIVATION_SILU;
  if (s && std::string(s) == "gelu") return REGTOPK_ACTIVATION_GELU;
  if (s && std::string(s) == "gelu_tanh") return REGTOPK_ACTIVATION_GELU_TANH;
  PyErr_Clear();
  value_error("kind is \"silu\", \"gelu\" or \"gelu_tanh\"");
}

PyObject* activation(PyObject* const* a) {  // a, kind, gated, keep8
  const Tensor& x = tensor(a[0], "a");
  const int type = type_of(x, "a");
  const Rows in = rows_of(x, "a");
  const int32_t kind = kind_of(a[1]);
  const bool gated = truth(a[2]), keeps = truth(a[3]);
  const int halves = gated ? 2 : 1;
  if (in.cols % halves) value_error("a: a gated activation's input has an even number of columns");
  const int64_t cols = in.cols / halves;
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor y = gated ? empty(with_cols(x.sizes(), cols), x.scalar_type(), x) : empty(x.sizes(), x.scalar_type(), x);
  NewPacked p{};
  if (keeps) p = new_packed(x.sizes(), x, halves);
  check(regtopk_activation(x.data_ptr(), in.ld, y.data_ptr(), cols, keeps ? p.v() : nullptr, p.ld_values, keeps ? p.s() : nullptr, p.ld_scales, in.rows,
                           cols, kind, gated, type, stream_of(x)), "regtopk_activation");
  return Py_BuildValue("NN", THPVariable_Wrap(y), keeps ? p.wrap() : Py_NewRef(Py_None));
}

PyObject* activation_backward(PyObject* const* a) {  // dy, kept, kind, gated, want_y
  const Tensor& dy = tensor(a[0], "dy");
  const int type = type_of(dy, "dy");
  const Rows up = rows_of(dy, "dy");
  const int32_t kind = kind_of(a[2]);
  const bool gated = truth(a[3]), wants_y = truth(a[4]), pair = PyTuple_Check(a[1]);
  const int halves = gated ? 2 : 1;
  Packed p{};
  if (pair) p = packed_of(a[1], "kept", halves);
  const Tensor& kept = pair ? *p.values : tensor(a[1], "kept");
  if (kept.device() != dy.device() || kept.layout() != at::kStrided || (!pair && kept.scalar_type() != dy.scalar_type()))
    type_error("kept must be 8-bit rows or a tensor of dy's dtype, on its device");
  if (kept.dim() != dy.dim() || kept.sizes().slice(0, kept.dim() - 1) != dy.sizes().slice(0, dy.dim() - 1) || kept.size(-1) != halves * up.cols)
    type_error(gated ? "kept must have dy's shape, with twice the columns" : "kept must have dy's shape");
  const Rows in = pair ? p.v : rows_of(kept, "kept");
  const c10::cuda::CUDAGuard guard(dy.device());
  Tensor da, y;
  if (wants_y) std::tie(da, y) = two_if_small(kept.sizes(), dy.scalar_type(), dy.sizes(), dy.scalar_type(), dy);
  else da = empty(kept.sizes(), dy.scalar_type(), dy);
  check(regtopk_activation_backward(dy.data_ptr(), up.ld, kept.data_ptr(), in.ld, bytes_of(p.scales), p.s.ld, da.data_ptr(), in.cols,
                                    wants_y ? y.data_ptr() : nullptr, up.cols, up.rows, up.cols, kind, gated, type, stream_of(dy)),
        "regtopk_activation_backward");
  return Py_BuildValue("NN", THPVariable_Wrap(da), wants_y ? THPVariable_Wrap(y) : Py_NewRef(Py_None));
}

// ---- the norm ---------------------------------------------------------------------------------------------------------
PyObject* rms_norm(PyObject* const* a) {  // x, weight, eps, residual, want_y, want_y8
  const Tensor& x = tensor(a[0], "x");
  const int type = type_of(x, "x");
  const Rows in = rows_of(x, "x");
  const float* weight = vector_of(tensor(a[1], "weight"), in.cols, x, "weight");
  const Tensor* residual = optional_tensor(a[3], "residual");
  if (residual) same_shape(*residual, x, "residual", true);
  const Rows res = residual ? rows_of(*residual, "residual") : Rows{0, 0, 0};
  const bool wants_y = truth(a[4]), wants_y8 = truth(a[5]);
  if (!wants_y && !wants_y8) value_error("at least one of want_y and want_y8");
  const c10::cuda::CUDAGuard guard(x.device());
  Tensor y;
  if (wants_y) y = empty(x.sizes(), x.scalar_type(), x);
  NewPacked p{};
  if (wants_y8) p = new_packed(x.sizes(), x, 1);
  Tensor h = x, rstd;
  const auto stats = x.sizes().slice(0, x.dim() - 1);
  if (residual) std::tie(h, rstd) = two_if_small(x.sizes(), residual->scalar_type(), stats, at::kFloat, x);
  else rstd = empty(stats, at::kFloat, x);
  check(regtopk_rms_norm(x.data_ptr(), in.ld, data(residual), res.ld, weight, static_cast<float>(number(a[2])), wants_y ? y.data_ptr() : nullptr, in.cols,
                         wants_y8 ? p.v() : nullptr, p.ld_values, wants_y8 ? p.s() : nullptr, p.ld_scales, residual ? h.data_ptr() : nullptr, in.cols,
                         static_cast<float*>(rstd.data_ptr()), in.rows, in.cols, type, type_of(h, "h"), stream_of(x)), "regtopk_rms_norm");
  return Py_BuildValue("NNNN", wants_y ? THPVariable_Wrap(y) : Py_NewRef(Py_None), wants_y8 ? p.wrap() : Py_NewRef(Py_None),
                       residual ? THPVariable_Wrap(h) : Py_NewRef(a[0]), THPVariable_Wrap(rstd));
}

PyObject* rms_norm_backward(PyObject* const* a) {  // dy, h, rstd, weight, dh, offsets, dweight, accumulate
  const Tensor &dy = tensor(a[0], "dy"), &h = tensor(a[1], "h");
  const int type = type_of(dy, "dy");
  const Rows in = rows_of(dy, "dy");
  same_shape(h, dy, "h", true);
  const Rows hr = rows_of(h, "h");
  const float* rstd = vector_of(tensor(a[2], "rstd"), in.rows, dy, "rstd");
  const float* weight = vector_of(tensor(a[3], "weight"), in.cols, dy, "weight");
  const Tensor* dh = optional_tensor(a[4], "dh");
  if (dh) same_shape(*dh, h, "dh");
  const Rows dhr = dh ? rows_of(*dh, "dh") : Rows{0, 0, 0};
  const Tensor* offsets = optional_tensor(a[5], "offsets");
  const int32_t groups = offsets ? groups_of(*offsets, dy) : 1;
  const Tensor* given = optional_tensor(a[6], "dweight");
  const bool accumulate = truth(a[7]);
  if (accumulate && !given) value_error("accumulate needs a dweight to add to");
  int64_t ld = in.cols;
  if (given) {
    if (given->device() != dy.device() || given->scalar_type() != at::kFloat || given->dim() != 2 || given->size(0) != groups || given->size(1) != in.cols)
      type_error("dweight must be float32 [" + std::to_string(groups) + ", " + std::to_string(in.cols) + "] on the input's device");
    ld = rows_of(*given, "dweight").ld;
    for (const Tensor* in : {&dy, &h, &tensor(a[2], "rstd"), &tensor(a[3], "weight"), dh})
      if (in) apart(*given, *in, "an input", false, "dweight");
    written(*given, "dweight");
  }
  const c10::cuda::CUDAGuard guard(dy.device());
  const size_t bytes = regtopk_rms_norm_backward_workspace_bytes(in.rows, in.cols, groups);
  Tensor dw, ws;
  if (given) dw = *given, ws = empty({static_cast<int64_t>(bytes)}, at::kByte, dy);
  else std::tie(dw, ws) = two_if_small({groups, in.cols}, at::kFloat, {static_cast<int64_t>(bytes)}, at::kByte, dy);
  const bool same = h.scalar_type() == dy.scalar_type();
  const Tensor dx = empty(dy.sizes(), dy.scalar_type(), dy), dres = same ? dx : empty(dy.sizes(), h.scalar_type(), dy);
  check(regtopk_rms_norm_backward(dy.data_ptr(), in.ld, h.data_ptr(), hr.ld, rstd, weight, data(dh), dhr.ld, dx.data_ptr(), in.cols,
                                  same ? nullptr : dres.data_ptr(), in.cols, static_cast<float*>(dw.data_ptr()), ld,
                                  static_cast<const int64_t*>(data(offsets)), groups, accumulate, in.rows, in.cols, type, type_of(h, "h"), ws.data_ptr(),
                                  bytes, stream_of(dy)), "regtopk_rms_norm_backward");
  PyObject* px = THPVariable_Wrap(dx);
  PyObject* pres = same ? Py_NewRef(px) : THPVariable_Wrap(dres);
  return Py_BuildValue("NNN", px, pres, given ? Py_NewRef(a[6]) : THPVariable_Wrap(dw));
}

}  // namespace

PyMethodDef g_expert_methods[] = {
    ENTRY("pack8", pack8, 1), ENTRY("unpack8", unpack8, 2), ENTRY("route", route, 9), ENTRY("route_backward", route_backward, 6),
    ENTRY("sort_tokens", sort_tokens, 3), ENTRY("spread_tokens", spread_tokens, 4), ENTRY("join_tokens", join_tokens, 4),
    ENTRY("join_tokens_backward", join_tokens_backward, 5), ENTRY("activation", activation, 4), ENTRY("activation_backward", activation_backward, 5),
    ENTRY("rms_norm", rms_norm, 6), ENTRY("rms_norm_backward", rms_norm_backward, 8), {nullptr, nullptr, 0, nullptr}};
