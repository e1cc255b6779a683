// torch_calls.cpp -- the common calls of the operators next to the sampler without Python in between:
// checks, output tensors and the C entry point in one step.  A call on a few rows takes the GPU some
// 10 us; ctypes and five allocations from Python take the host 20.
//
// Every function answers None for arguments that it does not take (another device than the current
// one, strides or types that need an error message, ..): binding.py then makes the call by its own
// path, which checks and refuses.  A status code of the library comes back as an integer.  The entry
// points' addresses are given once by binding.py, so that this module does not link to the library.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <climits>
#include <cmath>
#include <optional>
#include <type_traits>

#include "../../include/gls.h"

namespace {

decltype(&gls_token_logprobs) g_logprobs = nullptr;
decltype(&gls_emitted_logprobs) g_emitted = nullptr;
decltype(&gls_token_logprobs_backward) g_logprobs_backward = nullptr;
decltype(&gls_embed_tokens) g_embed = nullptr;
decltype(&gls_embed_tokens_backward_workspace_bytes) g_embed_backward_bytes = nullptr;
decltype(&gls_embed_tokens_backward) g_embed_backward = nullptr;
decltype(&gls_sample_tokens) g_sample = nullptr;
decltype(&gls_head_logits) g_head = nullptr;
decltype(&gls_head_logits_workspace_bytes) g_head_bytes = nullptr;
decltype(&gls_embed_tokens_int4) g_embed_int4 = nullptr;

constexpr int64_t kMaxTop = 256;  // the library's largest `top`

struct Decline {};  // thrown for what the general path should see

// other threads run while memory is found and the call is made, as they do under torch's operators
struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  NoGil() = default;
  NoGil(const NoGil&) = delete;
  ~NoGil() { PyEval_RestoreThread(state); }
};

// the tensor an argument holds, or an undefined one for None
at::Tensor tensor_or_none(PyObject* o) {
  if (o == Py_None) return at::Tensor();
  if (!THPVariable_Check(o)) throw Decline();
  return THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) throw Decline();
  return THPVariable_Unpack(o);
}
double number(PyObject* o) {
  if (!PyFloat_Check(o) && !PyLong_Check(o)) throw Decline();
  const double v = PyFloat_AsDouble(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Decline();
  }
  return v;
}
int64_t integer(PyObject* o) {
  if (!PyLong_Check(o)) throw Decline();
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Decline();
  }
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v == 1;
}
int dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return GLS_F32;
  if (t.scalar_type() == at::kBFloat16) return GLS_BF16;
  throw Decline();
}
// a dense strided tensor on the current device
c10::Device here(const at::Tensor& t) {
  if (!t.is_cuda() || t.layout() != at::kStrided || t.get_device() != c10::cuda::current_device()) throw Decline();
  return t.device();
}
// data of a contiguous tensor of this type and shape on `dev`; nullptr for an undefined one
template <class T>
T* data(const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape, c10::Device dev) {
  if (!t.defined()) return nullptr;
  if (t.scalar_type() != type || t.device() != dev || t.sizes() != shape || !t.is_contiguous()) throw Decline();
  return (T*)t.data_ptr();
}
gls_rows_t rows_of(const at::Tensor& t) {
  if (t.dim() != 4 || (t.stride(3) != 1 && t.size(3) > 1)) throw Decline();
  for (int i = 0; i < 3; ++i)
    if (t.size(i) <= 0 || t.size(i) > INT_MAX) throw Decline();
  gls_rows_t r;
  r.data = t.data_ptr();
  r.dtype = dtype_code(t);
  r.stride_b = t.stride(0);
  r.stride_k = t.stride(1);
  r.stride_j = t.stride(2);
  return r;
}
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
  return at::detail::empty_cuda(shape, type, dev, std::nullopt);
}
uint32_t* status_word(PyObject* o, c10::Device dev) {
  return data<uint32_t>(tensor_or_none(o), at::kInt, {1}, dev);
}
void* stream() { return (void*)c10::cuda::getCurrentCUDAStream().stream(); }

void put(PyObject* dict, const char* name, const at::Tensor& t) {
  PyObject* o = THPVariable_Wrap(t);
  if (!o) throw python_error();
  const int rc = PyDict_SetItemString(dict, name, o);
  Py_DECREF(o);
  if (rc) throw python_error();
}

struct ScoreOut {
  at::Tensor lp, lse, ent, ids, tlp;
  ScoreOut(at::IntArrayRef given, at::IntArrayRef lead, int64_t M, bool entropy, c10::Device dev) {
    lp = make(given, at::kFloat, dev);
    lse = make(lead, at::kFloat, dev);
    if (entropy) ent = make(lead, at::kFloat, dev);
    if (M > 0) {
      c10::SmallVector<int64_t, 5> top(lead.begin(), lead.end());
      top.push_back(M);
      ids = make(top, at::kInt, dev);
      tlp = make(top, at::kFloat, dev);
    }
  }
  float* entropy() { return ent.defined() ? (float*)ent.data_ptr() : nullptr; }
  int32_t* top_ids() { return ids.defined() ? (int32_t*)ids.data_ptr() : nullptr; }
  float* top_logprobs() { return tlp.defined() ? (float*)tlp.data_ptr() : nullptr; }
  PyObject* dict() {
    PyObject* d = PyDict_New();
    if (!d) throw python_error();  // put() failing means that memory ran out: the dict is not freed then
    put(d, "logprobs", lp);
    put(d, "lse", lse);
    if (ent.defined()) put(d, "entropy", ent);
    if (ids.defined()) {
      put(d, "top_ids", ids);
      put(d, "top_logprobs", tlp);
    }
    return d;
  }
};

#define CALL_BEGIN(count)  \
  HANDLE_TH_ERRORS         \
  if (n != (count)) {      \
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); \
    return nullptr;        \
  }                        \
  try {
#define CALL_END           \
  }                        \
  catch (const Decline&) { \
    Py_RETURN_NONE;        \
  }                        \
  END_HANDLE_TH_ERRORS

// token_logprobs(logits, tokens, top, inv_temp, want_entropy, status)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(6)
  const at::Tensor& x = tensor(a[0]);
  const at::Tensor& t = tensor(a[1]);
  const c10::Device dev = here(x);
  const gls_rows_t rows = rows_of(x);
  const int64_t M = integer(a[2]);
  const at::IntArrayRef lead = x.sizes().slice(0, 3);
  if (M < 0 || M > kMaxTop || (t.dim() != 3 && t.dim() != 4) || t.sizes().slice(0, 3) != lead) throw Decline();
  const int32_t* tokens = data<int32_t>(t, at::kInt, t.sizes(), dev);
  uint32_t* status = status_word(a[5], dev);
  const double inv_temp = number(a[3]);
  const int64_t G = t.dim() == 4 ? t.size(3) : 1;
  if (G < 0 || G > GLS_MAX_GIVEN || lead[1] > GLS_MAX_K) throw Decline();
  const bool entropy = truth(a[4]);
  std::optional<NoGil> free_others(std::in_place);
  ScoreOut o(t.sizes(), lead, M, entropy, dev);
  const int rc = g_logprobs(&rows, (int)lead[0], (int)lead[1], (int)lead[2], x.size(3), (float)inv_temp, nullptr, tokens,
                            (int)G, (int)M, (float*)o.lp.data_ptr(), (float*)o.lse.data_ptr(), nullptr, o.entropy(),
                            o.top_ids(), o.top_logprobs(), status, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return o.dict();
  CALL_END
}

// emitted_logprobs(target_logits, tokens, accept, top, inv_temp, flags, want_entropy, status)
PyObject* emitted_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(8)
  const at::Tensor& x = tensor(a[0]);
  const c10::Device dev = here(x);
  const gls_rows_t rows = rows_of(x);
  const int64_t B = x.size(0), K = x.size(1), J = x.size(2), M = integer(a[3]), flags = integer(a[5]);
  if (M < 0 || M > kMaxTop || flags < 0 || flags > 3 || K > GLS_MAX_K) throw Decline();
  const int64_t L = (flags & GLS_NO_BONUS) ? J : J - 1;
  const int64_t lead[2] = {B, J}, shape[3] = {B, K, L};
  const int32_t* tokens = data<int32_t>(tensor(a[1]), at::kInt, lead, dev);
  const uint8_t* accept = L > 0 ? data<uint8_t>(tensor(a[2]), at::kByte, shape, dev) : nullptr;
  uint32_t* status = status_word(a[7], dev);
  const double inv_temp = number(a[4]);
  const bool entropy = truth(a[6]);
  std::optional<NoGil> free_others(std::in_place);
  ScoreOut o(lead, lead, M, entropy, dev);
  const int rc = g_emitted(&rows, (int)B, (int)K, (int)L, x.size(3), (float)inv_temp, tokens, accept, (uint32_t)flags,
                           (int)M, (float*)o.lp.data_ptr(), (float*)o.lse.data_ptr(), o.entropy(), o.top_ids(),
                           o.top_logprobs(), status, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return o.dict();
  CALL_END
}

// token_logprobs_backward(logits, tokens, lse, entropy, lse_tail, top_ids, grad_logprobs, grad_lse,
//                         grad_entropy, grad_top_logprobs, inv_temp)
PyObject* token_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(11)
  const at::Tensor& x = tensor(a[0]);
  const at::Tensor t = tensor_or_none(a[1]), ids = tensor_or_none(a[5]);
  const c10::Device dev = here(x);
  const gls_rows_t rows = rows_of(x);
  const at::IntArrayRef lead = x.sizes().slice(0, 3);
  if (lead[1] > GLS_MAX_K) throw Decline();
  int64_t G = 0, M = 0;
  const int32_t *tokens = nullptr, *top = nullptr;
  if (t.defined()) {
    if ((t.dim() != 3 && t.dim() != 4) || t.sizes().slice(0, 3) != lead) throw Decline();
    tokens = data<int32_t>(t, at::kInt, t.sizes(), dev);
    G = t.dim() == 4 ? t.size(3) : 1;
  }
  if (ids.defined()) {
    if (ids.dim() != 4 || ids.sizes().slice(0, 3) != lead) throw Decline();
    top = data<int32_t>(ids, at::kInt, ids.sizes(), dev);
    M = ids.size(3);
  }
  if (G > GLS_MAX_GIVEN || M > kMaxTop || (a[6] != Py_None && !tokens) || (a[9] != Py_None && !top) ||
      (a[8] != Py_None && a[3] == Py_None))
    throw Decline();
  auto per_row = [&](PyObject* o) { return data<float>(tensor_or_none(o), at::kFloat, lead, dev); };
  const float *lse = per_row(a[2]), *ent = per_row(a[3]), *tail = per_row(a[4]), *g_lse = per_row(a[7]), *g_ent = per_row(a[8]);
  const float* g_lp = t.defined() ? data<float>(tensor_or_none(a[6]), at::kFloat, t.sizes(), dev) : nullptr;
  const float* g_top = ids.defined() ? data<float>(tensor_or_none(a[9]), at::kFloat, ids.sizes(), dev) : nullptr;
  const double inv_temp = number(a[10]);
  if (!lse) throw Decline();
  std::optional<NoGil> free_others(std::in_place);
  const at::Tensor grad = make(x.sizes(), x.scalar_type(), dev);
  const gls_rows_t out = rows_of(grad);
  const int rc = g_logprobs_backward(&rows, (int)lead[0], (int)lead[1], (int)lead[2], x.size(3), (float)inv_temp, nullptr,
                                     tokens, (int)G, top, (int)M, lse, tail, ent, g_lp, g_lse, g_ent, g_top, &out, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return THPVariable_Wrap(grad);
  CALL_END
}

// embed_tokens(table, tokens, scale, status)
PyObject* embed_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(4)
  const at::Tensor& table = tensor(a[0]);
  const at::Tensor& t = tensor(a[1]);
  const c10::Device dev = here(table);
  if (table.dim() != 2 || (table.stride(1) != 1 && table.size(1) > 1)) throw Decline();
  const int dt = dtype_code(table);
  const int32_t* tokens = data<int32_t>(t, at::kInt, t.sizes(), dev);
  uint32_t* status = status_word(a[3], dev);
  const double scale = number(a[2]);
  const int64_t D = table.size(1);
  c10::SmallVector<int64_t, 5> shape(t.sizes().begin(), t.sizes().end());
  shape.push_back(D);
  std::optional<NoGil> free_others(std::in_place);
  const at::Tensor out = make(shape, table.scalar_type(), dev);
  const int rc = g_embed(table.data_ptr(), dt, table.stride(0), table.size(0), D, tokens, t.numel(), (float)scale,
                         out.data_ptr(), D, status, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return THPVariable_Wrap(out);
  CALL_END
}

// embed_tokens_backward(grad_out, tokens, V, scale, status)
PyObject* embed_tokens_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(5)
  const at::Tensor& g = tensor(a[0]);
  const at::Tensor& t = tensor(a[1]);
  const c10::Device dev = here(g);
  const int dt = dtype_code(g);
  if (!g.is_contiguous() || g.dim() != t.dim() + 1 || g.sizes().slice(0, t.dim()) != t.sizes()) throw Decline();
  const int32_t* tokens = data<int32_t>(t, at::kInt, t.sizes(), dev);
  uint32_t* status = status_word(a[4], dev);
  const int64_t V = integer(a[2]), D = g.size(g.dim() - 1), N = t.numel();
  const double scale = number(a[3]);
  if (V <= 0 || D <= 0) throw Decline();
  std::optional<NoGil> free_others(std::in_place);
  const size_t need = g_embed_backward_bytes(N, V, D);
  const at::Tensor table = make({V, D}, g.scalar_type(), dev);
  const at::Tensor space = make({(int64_t)need}, at::kByte, dev);
  const int rc = g_embed_backward(g.data_ptr(), dt, D, tokens, N, V, D, (float)scale, table.data_ptr(), dt, D, 0u,
                                  space.data_ptr(), need, status, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return THPVariable_Wrap(table);
  CALL_END
}

// One sampling setting: a number, or a tensor [B], [B,K] or [B,K,J] whose sizes of 1 broadcast.
template <class T>
const T* setting(PyObject* o, at::ScalarType type, at::IntArrayRef lead, c10::Device dev, T* value, int64_t* stride) {
  if (!THPVariable_Check(o)) {
    if constexpr (std::is_integral_v<T>) {
      const int64_t v = integer(o);
      if (v < INT_MIN || v > INT_MAX) throw Decline();
      *value = (T)v;
    } else {
      const double v = number(o);
      *value = (T)v;
      if (std::isinf(*value) && !std::isinf(v)) throw Decline();  // beyond fp32
    }
    return nullptr;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || t.device() != dev || t.layout() != at::kStrided || t.dim() < 1 || t.dim() > 3) throw Decline();
  for (int i = 0; i < t.dim(); ++i) {
    if (t.size(i) != lead[i] && t.size(i) != 1) throw Decline();
    stride[i] = t.size(i) > 1 ? t.stride(i) : 0;
  }
  return (const T*)t.data_ptr();
}

// sample_tokens(logits, uniforms, inv_temp, top_k, top_p, min_p, want_logprobs, status)
PyObject* sample_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(8)
  const at::Tensor& x = tensor(a[0]);
  const c10::Device dev = here(x);
  const gls_rows_t rows = rows_of(x);
  const at::IntArrayRef lead = x.sizes().slice(0, 3);
  if (lead[1] > GLS_MAX_K) throw Decline();
  const float* u = data<float>(tensor(a[1]), at::kFloat, lead, dev);
  gls_sampling_t s = {};
  s.inv_temp_rows = setting(a[2], at::kFloat, lead, dev, &s.inv_temp, s.inv_temp_stride);
  s.top_k_rows = setting(a[3], at::kInt, lead, dev, &s.top_k, s.top_k_stride);
  s.top_p_rows = setting(a[4], at::kFloat, lead, dev, &s.top_p, s.top_p_stride);
  s.min_p_rows = setting(a[5], at::kFloat, lead, dev, &s.min_p, s.min_p_stride);
  const bool want = truth(a[6]);
  uint32_t* status = status_word(a[7], dev);
  std::optional<NoGil> free_others(std::in_place);
  const at::Tensor tokens = make(lead, at::kInt, dev);
  at::Tensor lp;
  if (want) lp = make(lead, at::kFloat, dev);
  const int rc = g_sample(&rows, (int)lead[0], (int)lead[1], (int)lead[2], x.size(3), &s, u, (int32_t*)tokens.data_ptr(),
                          want ? (float*)lp.data_ptr() : nullptr, status, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  PyObject* d = PyDict_New();
  if (!d) throw python_error();
  put(d, "tokens", tokens);
  if (want) put(d, "logprobs", lp);
  return d;
  CALL_END
}

// The table that codes, scales, zeros, columns and group make.
gls_int4_table_t table_of(PyObject* const* a, c10::Device dev) {
  const at::Tensor& codes = tensor(a[0]);
  const at::Tensor& scales = tensor(a[1]);
  const at::Tensor zeros = tensor_or_none(a[2]);
  gls_int4_table_t t;
  t.D = integer(a[3]);
  const int64_t group = integer(a[4]);
  if (group != 32 && group != 64 && group != 128) throw Decline();
  t.group = (int32_t)group;
  const int64_t G = (t.D + group - 1) / group;
  if (t.D <= 0 || codes.scalar_type() != at::kByte || codes.device() != dev || codes.layout() != at::kStrided ||
      codes.dim() != 2 || codes.stride(1) != 1 || codes.size(1) < (t.D + 31) / 32 * 16)
    throw Decline();
  t.V = codes.size(0);
  auto fits = [&](const at::Tensor& s) {
    return s.device() == dev && s.layout() == at::kStrided && s.dim() == 2 && s.size(0) == t.V && s.size(1) == G &&
           (s.stride(1) == 1 || G == 1);
  };
  if (!fits(scales) || (zeros.defined() && (!fits(zeros) || zeros.scalar_type() != at::kByte))) throw Decline();
  t.codes = (uint8_t*)codes.data_ptr();
  t.code_stride = codes.stride(0);
  t.scales = scales.data_ptr();
  t.scale_dtype = dtype_code(scales);
  t.scale_stride = scales.stride(0);
  t.zeros = zeros.defined() ? (uint8_t*)zeros.data_ptr() : nullptr;
  t.zero_stride = zeros.defined() ? zeros.stride(0) : 0;
  return t;
}
at::ScalarType type_of(int64_t code) {
  if (code == GLS_F32) return at::kFloat;
  if (code == GLS_BF16) return at::kBFloat16;
  throw Decline();
}

// head_logits(x, codes, scales, zeros, dim, group, type of the logits, -1 for x's)
PyObject* head_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(7)
  const at::Tensor& x = tensor(a[0]);
  const c10::Device dev = here(x);
  const int dt = dtype_code(x);
  const gls_int4_table_t t = table_of(a + 1, dev);
  const int64_t code = integer(a[6]);
  if (x.dim() < 1 || x.size(x.dim() - 1) != t.D || !x.is_contiguous()) throw Decline();
  const at::ScalarType type = type_of(code < 0 ? dt : code);
  c10::SmallVector<int64_t, 5> shape(x.sizes().begin(), x.sizes().end());
  shape.back() = t.V;
  std::optional<NoGil> free_others(std::in_place);
  const at::Tensor out = make(shape, type, dev);
  const int64_t N = x.numel() / t.D;
  const size_t need = g_head_bytes(N, t.D, dt);
  at::Tensor space;
  if (need) space = make({(int64_t)need}, at::kByte, dev);
  const int rc = g_head(x.data_ptr(), dt, t.D, N, &t, out.data_ptr(), type == at::kFloat ? GLS_F32 : GLS_BF16, t.V,
                        need ? space.data_ptr() : nullptr, need, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return THPVariable_Wrap(out);
  CALL_END
}

// embed_tokens_int4(codes, scales, zeros, dim, group, tokens, scale, type, status)
PyObject* embed_tokens_int4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN(9)
  const at::Tensor& k = tensor(a[5]);
  const c10::Device dev = here(k);
  const gls_int4_table_t t = table_of(a, dev);
  const int32_t* tokens = data<int32_t>(k, at::kInt, k.sizes(), dev);
  const double scale = number(a[6]);
  const at::ScalarType type = type_of(integer(a[7]));
  uint32_t* status = status_word(a[8], dev);
  c10::SmallVector<int64_t, 5> shape(k.sizes().begin(), k.sizes().end());
  shape.push_back(t.D);
  std::optional<NoGil> free_others(std::in_place);
  const at::Tensor out = make(shape, type, dev);
  const int rc = g_embed_int4(&t, tokens, k.numel(), (float)scale, out.data_ptr(), type == at::kFloat ? GLS_F32 : GLS_BF16, t.D,
                              status, stream());
  free_others.reset();
  if (rc) return PyLong_FromLong(rc);
  return THPVariable_Wrap(out);
  CALL_END
}

// entry_points(addresses of the ten entry points, in the order of the variables above)
PyObject* entry_points(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[10];
  if (n != 10) {
    PyErr_SetString(PyExc_TypeError, "ten addresses");
    return nullptr;
  }
  for (int i = 0; i < 10; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  g_logprobs = (decltype(g_logprobs))p[0];
  g_emitted = (decltype(g_emitted))p[1];
  g_logprobs_backward = (decltype(g_logprobs_backward))p[2];
  g_embed = (decltype(g_embed))p[3];
  g_embed_backward_bytes = (decltype(g_embed_backward_bytes))p[4];
  g_embed_backward = (decltype(g_embed_backward))p[5];
  g_sample = (decltype(g_sample))p[6];
  g_head = (decltype(g_head))p[7];
  g_head_bytes = (decltype(g_head_bytes))p[8];
  g_embed_int4 = (decltype(g_embed_int4))p[9];
  Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"entry_points", (PyCFunction)(void (*)(void))entry_points, METH_FASTCALL, nullptr},
    {"token_logprobs", (PyCFunction)(void (*)(void))token_logprobs, METH_FASTCALL, nullptr},
    {"emitted_logprobs", (PyCFunction)(void (*)(void))emitted_logprobs, METH_FASTCALL, nullptr},
    {"token_logprobs_backward", (PyCFunction)(void (*)(void))token_logprobs_backward, METH_FASTCALL, nullptr},
    {"embed_tokens", (PyCFunction)(void (*)(void))embed_tokens, METH_FASTCALL, nullptr},
    {"embed_tokens_backward", (PyCFunction)(void (*)(void))embed_tokens_backward, METH_FASTCALL, nullptr},
    {"sample_tokens", (PyCFunction)(void (*)(void))sample_tokens, METH_FASTCALL, nullptr},
    {"head_logits", (PyCFunction)(void (*)(void))head_logits, METH_FASTCALL, nullptr},
    {"embed_tokens_int4", (PyCFunction)(void (*)(void))embed_tokens_int4, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "gls_torch_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit_gls_torch_calls(void) { return PyModule_Create(&g_module); }
