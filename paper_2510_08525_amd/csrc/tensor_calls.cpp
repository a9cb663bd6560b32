// The operators' calls on torch tensors: argument checks and marshalling in front of the C-ABI, nothing else.  A Python module of its own,
// because a decode step makes these calls one after the other and each is a few microseconds of the GPU: looking at five tensors from
// Python takes as long as that (norm of one row: 7.8 us a call with the checks in Python and ctypes, 4.1 from here; the launch is 3.3).
// Every function returns the call's status; what is wrong with a tensor raises ValueError.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <initializer_list>

#include "rlkv.h"

namespace {

using c10::ScalarType;

constexpr int64_t kGroup = 128;
int64_t groups_of(int64_t n) { return (n + kGroup - 1) / kGroup; }

const char* name_of(ScalarType t) {
  switch (t) {
    case ScalarType::Float: return "float32";
    case ScalarType::BFloat16: return "bfloat16";
    case ScalarType::Float8_e4m3fn: return "float8_e4m3fn";
    case ScalarType::Int: return "int32";
    case ScalarType::Byte: return "uint8";
    default: return c10::toString(t);
  }
}
// rlkv_dtype_t of a tensor's type, or -1.
int kind_of(ScalarType t) {
  return t == ScalarType::Float ? RLKV_F32 : t == ScalarType::BFloat16 ? RLKV_BF16 : t == ScalarType::Float8_e4m3fn ? RLKV_E4M3 : -1;
}

// The device of a call, and its current stream; restored to what it was where that was another.
class OnDevice {
 public:
  explicit OnDevice(int index) : before_(c10::hip::current_device()), index_(index) {
    if (before_ != index_) c10::hip::set_device(static_cast<c10::DeviceIndex>(index_));
  }
  ~OnDevice() {
    if (before_ != index_) c10::hip::set_device(static_cast<c10::DeviceIndex>(before_));
  }
  void* stream() const { return c10::hip::getCurrentHIPStream(static_cast<c10::DeviceIndex>(index_)).stream(); }

 private:
  int before_, index_;
};

// As of torch's own operators into given outputs: while gradients are recorded no tensor may ask for one, since autograd does not see the call.
const at::Tensor* tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: need a tensor", what);
    return nullptr;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && c10::GradMode::is_enabled()) {
    PyErr_Format(PyExc_ValueError, "%s: requires a gradient, which the call does not record: detach it, or call under torch.no_grad()", what);
    return nullptr;
  }
  return &t;
}
// What the call has written: a version further, by which autograd knows that what it saved is no longer there.
void written(PyObject* o) {
  if (o == Py_None) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
bool on_device(const at::Tensor& t, const char* what, int index) {
  if (t.is_cuda() && (index < 0 || t.get_device() == index)) return true;
  if (index < 0) PyErr_Format(PyExc_ValueError, "%s: need a tensor on the GPU", what);
  else PyErr_Format(PyExc_ValueError, "%s: need a tensor on cuda:%d", what, index);
  return false;
}
bool of_type(const at::Tensor& t, const char* what, ScalarType type) {
  if (t.scalar_type() == type) return true;
  PyErr_Format(PyExc_ValueError, "%s: type %s, not %s", what, name_of(t.scalar_type()), name_of(type));
  return false;
}
bool of_size(const at::Tensor& t, const char* what, int dim, int64_t have, int64_t want) {
  if (have == want) return true;
  PyErr_Format(PyExc_ValueError, "%s: %lld at dimension %d, not %lld", what, (long long)have, dim, (long long)want);
  return false;
}

struct Matrix {
  void* p = nullptr;
  int64_t stride = 0, rows = 0, cols = 0;
  int device = -1;
  ScalarType type = ScalarType::Undefined;
};
// Two dimensions, contiguous columns, on a device (any, index < 0).  The distance of two rows of a matrix with one, which a tensor may
// report as anything, is its length.
bool any_matrix(PyObject* o, const char* what, int index, Matrix* m) {
  const at::Tensor* t = tensor(o, what);
  if (!t || !on_device(*t, what, index)) return false;
  if (t->dim() != 2 || (t->stride(1) != 1 && t->size(1) > 1)) {
    PyErr_Format(PyExc_ValueError, "%s: need a matrix with contiguous columns", what);
    return false;
  }
  m->p = t->data_ptr();
  m->rows = t->size(0);
  m->cols = t->size(1);
  m->stride = m->rows > 1 ? t->stride(0) : m->cols;
  m->device = t->get_device();
  m->type = t->scalar_type();
  return true;
}
bool matrix(PyObject* o, const char* what, int index, ScalarType type, int64_t rows, int64_t cols, Matrix* m) {
  if (!any_matrix(o, what, index, m)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return of_type(t, what, type) && of_size(t, what, 0, m->rows, rows) && of_size(t, what, 1, m->cols, cols);
}
// The same without a gap between rows.
bool matrix_whole(PyObject* o, const char* what, int index, ScalarType type, int64_t rows, int64_t cols, Matrix* m) {
  if (!matrix(o, what, index, type, rows, cols, m)) return false;
  if (rows <= 1 || cols == 0 || m->stride == cols) return true;
  PyErr_Format(PyExc_ValueError, "%s: need a contiguous tensor", what);
  return false;
}
// fp32 or bf16: activations and logits
bool activations(PyObject* o, const char* what, Matrix* m) {
  if (!any_matrix(o, what, -1, m)) return false;
  if (m->type == ScalarType::Float || m->type == ScalarType::BFloat16) return true;
  PyErr_Format(PyExc_ValueError, "%s: type %s is not one of float32, bfloat16", what, name_of(m->type));
  return false;
}
// A contiguous vector; None is a null pointer.
bool vector(PyObject* o, const char* what, int index, ScalarType type, int64_t n, void** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o, what);
  if (!t || !on_device(*t, what, index) || !of_type(*t, what, type)) return false;
  if (t->dim() != 1 || (t->size(0) > 1 && t->stride(0) != 1)) {
    PyErr_Format(PyExc_ValueError, "%s: need a contiguous vector", what);
    return false;
  }
  if (!of_size(*t, what, 0, t->size(0), n)) return false;
  *p = t->data_ptr();
  return true;
}
bool fits(int64_t n, const char* what) {
  if (n <= INT32_MAX) return true;
  PyErr_Format(PyExc_ValueError, "%s: %lld rows or columns", what, (long long)n);
  return false;
}
bool arguments(Py_ssize_t have, Py_ssize_t want) {
  if (have == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", have, want);
  return false;
}
bool number(PyObject* o, float* f) {
  const double d = PyFloat_AsDouble(o);
  *f = static_cast<float>(d);
  return !(d == -1.0 && PyErr_Occurred());
}

// The library's call, with the interpreter left to other threads meanwhile: a launch waits where the device's queue is full.  outputs: tensors
// and None.
template <typename F>
PyObject* status_of(std::initializer_list<PyObject*> outputs, F call) {
  int32_t status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  if (status == RLKV_OK)
    for (PyObject* o : outputs) written(o);
  return PyLong_FromLong(status);
}

#define RLKV_CALL_BEGIN try {
#define RLKV_CALL_END                                    \
  }                                                      \
  catch (const std::exception& e) {                      \
    PyErr_SetString(PyExc_RuntimeError, e.what());       \
    return nullptr;                                      \
  }

// x, weight, eps, out, scales, residual, sum_out
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  Matrix x, out, scales, residual, sum;
  void* weight;
  float eps;
  if (!arguments(n, 7) || !activations(a[0], "x", &x) || !fits(x.rows, "x") || !fits(x.cols, "x") || !number(a[2], &eps)) return nullptr;
  if (!vector(a[1], "weight", x.device, x.type, x.cols, &weight)) return nullptr;
  if (!any_matrix(a[3], "out", x.device, &out)) return nullptr;
  const bool eight = out.type == ScalarType::Float8_e4m3fn;
  if (!matrix(a[3], "out", x.device, eight ? out.type : x.type, x.rows, x.cols, &out)) return nullptr;
  if (a[4] != Py_None && !matrix(a[4], "scales", x.device, ScalarType::Float, groups_of(x.cols), x.rows, &scales)) return nullptr;
  if (a[5] != Py_None && !matrix(a[5], "residual", x.device, x.type, x.rows, x.cols, &residual)) return nullptr;
  if (a[6] != Py_None && !matrix(a[6], "sum_out", x.device, x.type, x.rows, x.cols, &sum)) return nullptr;
  const OnDevice on(x.device);
  return status_of({a[3], a[4], a[6]}, [&] {
    return rlkv_rms_norm(x.p, x.stride, residual.p, residual.stride, weight, eps, (int32_t)x.rows, (int32_t)x.cols, kind_of(x.type),
                         sum.p, sum.stride, out.p, out.stride, kind_of(out.type), static_cast<float*>(scales.p), scales.stride,
                         on.stream());
  });
  RLKV_CALL_END
}

// x, out, scales
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  Matrix x, out, scales;
  if (!arguments(n, 3) || !activations(a[0], "x", &x) || !fits(x.rows, "x") || !fits(x.cols, "x")) return nullptr;
  if (!matrix(a[1], "out", x.device, ScalarType::Float8_e4m3fn, x.rows, x.cols, &out)) return nullptr;
  if (!matrix(a[2], "scales", x.device, ScalarType::Float, groups_of(x.cols), x.rows, &scales)) return nullptr;
  const OnDevice on(x.device);
  return status_of({a[1], a[2]}, [&] {
    return rlkv_quantize(x.p, x.stride, (int32_t)x.rows, (int32_t)x.cols, kind_of(x.type), out.p, out.stride,
                         static_cast<float*>(scales.p), scales.stride, on.stream());
  });
  RLKV_CALL_END
}

// a, a_scales, b, b_scales, out
PyObject* scaled_matmul(PyObject*, PyObject* const* v, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  Matrix a, sa, b, sb, out;
  if (!arguments(n, 5) || !any_matrix(v[0], "a", -1, &a) || !any_matrix(v[2], "b", a.device, &b)) return nullptr;
  const ScalarType eight = ScalarType::Float8_e4m3fn;
  if (!matrix(v[0], "a", a.device, eight, a.rows, a.cols, &a) || !matrix(v[2], "b", a.device, eight, b.rows, a.cols, &b)) return nullptr;
  if (!fits(a.rows, "a") || !fits(a.cols, "a") || !fits(b.rows, "b")) return nullptr;
  const int64_t g = groups_of(a.cols);
  if (!matrix(v[1], "a_scales", a.device, ScalarType::Float, g, a.rows, &sa)) return nullptr;
  if (!matrix(v[3], "b_scales", a.device, ScalarType::Float, groups_of(b.rows), g, &sb)) return nullptr;
  if (!activations(v[4], "out", &out) || !matrix(v[4], "out", a.device, out.type, a.rows, b.rows, &out)) return nullptr;
  const OnDevice on(a.device);
  return status_of({v[4]}, [&] {
    return rlkv_scaled_matmul(a.p, a.stride, static_cast<float*>(sa.p), sa.stride, b.p, b.stride, static_cast<float*>(sb.p), sb.stride,
                              (int32_t)a.rows, (int32_t)b.rows, (int32_t)a.cols, out.p, out.stride, kind_of(out.type), on.stream());
  });
  RLKV_CALL_END
}

// logits, tokens, logprobs, scale, entropy, lse, top log probabilities, top tokens, workspace
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  Matrix x, values, ids;
  void *tokens, *logprobs, *entropy, *lse, *workspace;
  float scale;
  if (!arguments(n, 9) || !activations(a[0], "logits", &x) || !fits(x.rows, "logits") || !fits(x.cols, "logits")) return nullptr;
  if (!number(a[3], &scale)) return nullptr;
  if (!vector(a[1], "tokens", x.device, ScalarType::Int, x.rows, &tokens)) return nullptr;
  if (!vector(a[2], "logprobs", x.device, ScalarType::Float, x.rows, &logprobs)) return nullptr;
  if (!vector(a[4], "entropy", x.device, ScalarType::Float, x.rows, &entropy)) return nullptr;
  if (!vector(a[5], "lse", x.device, ScalarType::Float, x.rows, &lse)) return nullptr;
  if (a[6] != Py_None) {
    if (!any_matrix(a[6], "top log probabilities", x.device, &values)) return nullptr;
    if (!matrix(a[6], "top log probabilities", x.device, ScalarType::Float, x.rows, values.cols, &values)) return nullptr;
    if (!matrix(a[7], "top tokens", x.device, ScalarType::Int, x.rows, values.cols, &ids)) return nullptr;
    if (values.stride != values.cols || ids.stride != values.cols) {
      PyErr_SetString(PyExc_ValueError, "top: need contiguous tensors");
      return nullptr;
    }
  }
  const at::Tensor* w = tensor(a[8], "workspace");
  if (!w || !vector(a[8], "workspace", x.device, ScalarType::Byte, w->numel(), &workspace)) return nullptr;
  const OnDevice on(x.device);
  return status_of({a[2], a[4], a[5], a[6], a[6] == Py_None ? Py_None : a[7]}, [&] {
    return rlkv_token_logprobs(x.p, x.stride, (int32_t)x.rows, (int32_t)x.cols, kind_of(x.type), scale, static_cast<int32_t*>(tokens),
                               static_cast<float*>(logprobs), static_cast<float*>(entropy), static_cast<float*>(lse),
                               values.cols <= INT32_MAX ? (int32_t)values.cols : -1, static_cast<int32_t*>(ids.p),
                               static_cast<float*>(values.p), workspace, static_cast<size_t>(w->numel()), on.stream());
  });
  RLKV_CALL_END
}

// logits, tokens, lse, grad_logprobs, grad_logits, scale, entropy, grad_entropy
PyObject* token_logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  Matrix x, out;
  void *tokens, *lse, *g, *entropy, *gh;
  float scale;
  if (!arguments(n, 8) || !activations(a[0], "logits", &x) || !fits(x.rows, "logits") || !fits(x.cols, "logits")) return nullptr;
  if (!number(a[5], &scale)) return nullptr;
  if (!matrix(a[4], "grad_logits", x.device, x.type, x.rows, x.cols, &out)) return nullptr;
  if (!vector(a[1], "tokens", x.device, ScalarType::Int, x.rows, &tokens)) return nullptr;
  if (!vector(a[2], "lse", x.device, ScalarType::Float, x.rows, &lse)) return nullptr;
  if (!vector(a[3], "grad_logprobs", x.device, ScalarType::Float, x.rows, &g)) return nullptr;
  if (!vector(a[6], "entropy", x.device, ScalarType::Float, x.rows, &entropy)) return nullptr;
  if (!vector(a[7], "grad_entropy", x.device, ScalarType::Float, x.rows, &gh)) return nullptr;
  const OnDevice on(x.device);
  return status_of({a[4]}, [&] {
    return rlkv_token_logprobs_grad(x.p, x.stride, (int32_t)x.rows, (int32_t)x.cols, kind_of(x.type), scale,
                                    static_cast<int32_t*>(tokens), static_cast<float*>(lse), static_cast<float*>(entropy),
                                    static_cast<float*>(g), static_cast<float*>(gh), out.p, out.stride, on.stream());
  });
  RLKV_CALL_END
}

// ---- calls on a cache: what its owner knows of it ---------------------------------------------------------------------------------------
struct CacheShape {
  rlkv_cache_t* cache;
  int32_t layer;
  int device;
  ScalarType type;
  int64_t batch, q_heads, kv_heads, head_dim;
};
// handle, layer, (device, kind, batch, q heads, kv heads, head_dim)
bool cache_shape(PyObject* handle, PyObject* layer, PyObject* shape, CacheShape* s) {
  s->cache = handle == Py_None ? nullptr : static_cast<rlkv_cache_t*>(PyLong_AsVoidPtr(handle));   // (None: closed, which the library refuses)
  int beyond = 0;
  const long at = PyLong_AsLongAndOverflow(layer, &beyond);
  if (PyErr_Occurred()) return false;
  s->layer = (int32_t)at;
  if (beyond || s->layer != at) {
    PyErr_Format(PyExc_ValueError, "layer: %R is none", layer);
    return false;
  }
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 6) {
    PyErr_SetString(PyExc_TypeError, "shape of the cache");
    return false;
  }
  int64_t v[6];
  for (int i = 0; i < 6; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
  if (PyErr_Occurred()) return false;
  s->device = (int)v[0];
  s->type = v[1] == RLKV_F32 ? ScalarType::Float : ScalarType::BFloat16;
  s->batch = v[2]; s->q_heads = v[3]; s->kv_heads = v[4]; s->head_dim = v[5];
  return true;
}
struct Packed { void* p; int64_t token_stride, tokens; };
// [batch, tokens, (q + 2 kv heads) * head_dim], rows at equal distances
bool packed(PyObject* o, const CacheShape& s, Packed* q) {
  const at::Tensor* t = tensor(o, "qkv");
  if (!t || !on_device(*t, "qkv", s.device) || !of_type(*t, "qkv", s.type)) return false;
  const int64_t width = (s.q_heads + 2 * s.kv_heads) * s.head_dim;
  if (t->dim() != 3) {
    PyErr_SetString(PyExc_ValueError, "qkv: need [batch, tokens, (q heads + 2 kv heads) * head_dim]");
    return false;
  }
  if (!of_size(*t, "qkv", 0, t->size(0), s.batch) || !of_size(*t, "qkv", 2, t->size(2), width) || !fits(t->size(1), "qkv")) return false;
  q->p = t->data_ptr();
  q->tokens = t->size(1);
  q->token_stride = q->tokens > 1 ? t->stride(1) : s.batch > 1 ? t->stride(0) : width;
  if (t->stride(2) != 1 || q->token_stride < width ||
      (s.batch > 1 && q->tokens > 1 && t->stride(0) != q->tokens * q->token_stride)) {
    PyErr_SetString(PyExc_ValueError, "qkv: need contiguous rows at equal distances");
    return false;
  }
  return true;
}
// [batch, heads, tokens, head_dim], for one token also without that axis
bool heads_first(PyObject* o, const char* what, const CacheShape& s, int64_t heads, int64_t tokens, void** p) {
  const at::Tensor* t = tensor(o, what);
  if (!t || !on_device(*t, what, s.device) || !of_type(*t, what, s.type)) return false;
  const bool flat = t->dim() == 3 && tokens == 1;
  if ((t->dim() != 4 && !flat) || !t->is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s: need a contiguous [batch, heads, tokens, head_dim]", what);
    return false;
  }
  if (!of_size(*t, what, 0, t->size(0), s.batch) || !of_size(*t, what, 1, t->size(1), heads)) return false;
  if (!flat && !of_size(*t, what, 2, t->size(2), tokens)) return false;
  if (!of_size(*t, what, (int)t->dim() - 1, t->size(-1), s.head_dim)) return false;
  *p = t->data_ptr();
  return true;
}
// Address of the counts (an int32 array of the batch's size that the caller holds), 0: none.
bool address(PyObject* o, void** p) {
  *p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}

// handle, layer, shape, qkv, counts, rotary, q_out
PyObject* append_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  CacheShape s;
  Packed x;
  void *counts, *rotary, *q = nullptr;
  if (!arguments(n, 7) || !cache_shape(a[0], a[1], a[2], &s) || !packed(a[3], s, &x) || !address(a[4], &counts) || !address(a[5], &rotary))
    return nullptr;
  if (a[6] != Py_None && !heads_first(a[6], "q_out", s, s.q_heads, x.tokens, &q)) return nullptr;
  const OnDevice on(s.device);
  return status_of({a[6]}, [&] {
    return rlkv_append_rotary(s.cache, s.layer, x.p, x.token_stride, static_cast<int32_t*>(counts), (int32_t)x.tokens,
                              static_cast<rlkv_rotary_t*>(rotary), q, on.stream());
  });
  RLKV_CALL_END
}

// handle, layer, shape, qkv, counts, rotary, q_out, k_out, v_out
PyObject* rotary_split(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  CacheShape s;
  Packed x;
  void *counts, *rotary, *q, *k, *v;
  if (!arguments(n, 9) || !cache_shape(a[0], a[1], a[2], &s) || !packed(a[3], s, &x) || !address(a[4], &counts) || !address(a[5], &rotary))
    return nullptr;
  if (!heads_first(a[6], "q_out", s, s.q_heads, x.tokens, &q) || !heads_first(a[7], "k_out", s, s.kv_heads, x.tokens, &k) ||
      !heads_first(a[8], "v_out", s, s.kv_heads, x.tokens, &v))
    return nullptr;
  const OnDevice on(s.device);
  return status_of({a[6], a[7], a[8]}, [&] {
    return rlkv_rotary(s.cache, s.layer, x.p, x.token_stride, static_cast<int32_t*>(counts), (int32_t)x.tokens,
                       static_cast<rlkv_rotary_t*>(rotary), q, k, v, on.stream());
  });
  RLKV_CALL_END
}

bool integer(PyObject* o, const char* what, int32_t* v) {
  int beyond = 0;
  const long x = PyLong_AsLongAndOverflow(o, &beyond);
  if (PyErr_Occurred()) return false;
  *v = (int32_t)x;
  if (!beyond && *v == x) return true;
  PyErr_Format(PyExc_ValueError, "%s: %R is out of range", what, o);
  return false;
}
// A number, or a vector with one a row.
bool number_or_vector(PyObject* o, const char* what, int index, int64_t rows, double* f, const float** p) {
  void* at = nullptr;
  if (THPVariable_Check(o)) {
    if (!vector(o, what, index, ScalarType::Float, rows, &at)) return false;
    *p = static_cast<float*>(at);
    return true;
  }
  *f = PyFloat_AsDouble(o);
  return !(*f == -1.0 && PyErr_Occurred());
}

// logits, uniforms, tokens, temperature, top_k, top_p, min_p, logprobs, workspace
PyObject* sample_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  Matrix x;
  void *uniforms, *tokens, *logprobs, *workspace, *ks = nullptr;
  rlkv_sampling_t how = {};
  if (!arguments(n, 9) || !activations(a[0], "logits", &x) || !fits(x.rows, "logits") || !fits(x.cols, "logits")) return nullptr;
  if (!vector(a[1], "uniforms", x.device, ScalarType::Float, x.rows, &uniforms)) return nullptr;
  if (!vector(a[2], "tokens", x.device, ScalarType::Int, x.rows, &tokens)) return nullptr;
  if (!number_or_vector(a[3], "temperature", x.device, x.rows, &how.temperature, &how.temperatures)) return nullptr;
  if (THPVariable_Check(a[4])) {
    if (!vector(a[4], "top_k", x.device, ScalarType::Int, x.rows, &ks)) return nullptr;
    how.top_ks = static_cast<int32_t*>(ks);
  } else if (!integer(a[4], "top_k", &how.top_k)) {
    return nullptr;
  }
  if (!number_or_vector(a[5], "top_p", x.device, x.rows, &how.top_p, &how.top_ps)) return nullptr;
  if (!number_or_vector(a[6], "min_p", x.device, x.rows, &how.min_p, &how.min_ps)) return nullptr;
  if (!vector(a[7], "logprobs", x.device, ScalarType::Float, x.rows, &logprobs)) return nullptr;
  const at::Tensor* w = tensor(a[8], "workspace");
  if (!w || !vector(a[8], "workspace", x.device, ScalarType::Byte, w->numel(), &workspace)) return nullptr;
  const OnDevice on(x.device);
  return status_of({a[2], a[7]}, [&] {
    return rlkv_sample_tokens(x.p, x.stride, (int32_t)x.rows, (int32_t)x.cols, kind_of(x.type), &how, static_cast<float*>(uniforms),
                              static_cast<int32_t*>(tokens), static_cast<float*>(logprobs), workspace, static_cast<size_t>(w->numel()), on.stream());
  });
  RLKV_CALL_END
}

// ---- calls on packed sequences -----------------------------------------------------------------------------------------------------------
// [tokens, heads, head_dim] at any strides of tokens and heads; tokens and heads below 0: any.
bool head_rows(PyObject* o, const char* what, int index, ScalarType type, int64_t tokens, int64_t heads, rlkv_heads_t* r) {
  const at::Tensor* t = tensor(o, what);
  if (!t || !on_device(*t, what, index) || !of_type(*t, what, type)) return false;
  if (t->dim() != 3 || t->stride(2) != 1) {
    PyErr_Format(PyExc_ValueError, "%s: need [tokens, heads, head_dim] with contiguous rows", what);
    return false;
  }
  if ((tokens >= 0 && !of_size(*t, what, 0, t->size(0), tokens)) || (heads >= 0 && !of_size(*t, what, 1, t->size(1), heads)) ||
      !of_size(*t, what, 2, t->size(2), 128) || !fits(t->size(0), what) || !fits(t->size(1), what))
    return false;
  r->data = t->data_ptr();
  r->token_stride = t->size(0) > 1 ? t->stride(0) : 0;          // (the stride of an axis of one, which a tensor may report as anything)
  r->head_stride = t->size(1) > 1 ? t->stride(1) : 0;
  return true;
}
// q, k, v, offsets; scale, mask (bytes or None), sink, recent
bool packed_shape(PyObject* const* qkv, PyObject* const* how, rlkv_heads_t* q, rlkv_heads_t* k, rlkv_heads_t* v, rlkv_packed_t* s, int* index) {
  const ScalarType bf16 = ScalarType::BFloat16;
  if (!head_rows(qkv[0], "q", -1, bf16, -1, -1, q)) return false;
  const at::Tensor& t = THPVariable_Unpack(qkv[0]);
  *index = t.get_device();
  if (!head_rows(qkv[1], "k", *index, bf16, t.size(0), -1, k)) return false;
  const at::Tensor& u = THPVariable_Unpack(qkv[1]);
  if (!head_rows(qkv[2], "v", *index, bf16, t.size(0), u.size(1), v)) return false;
  const at::Tensor* at = tensor(qkv[3], "offsets");
  void* offsets;
  if (!at || !vector(qkv[3], "offsets", *index, ScalarType::Int, at->numel(), &offsets) || !fits(at->numel(), "offsets")) return false;
  if (at->numel() < 1) {
    PyErr_SetString(PyExc_ValueError, "offsets: need one more than there are sequences");
    return false;
  }
  *s = {};
  s->offsets = static_cast<int32_t*>(offsets);
  s->n_seqs = (int32_t)(at->numel() - 1);
  s->tokens = (int32_t)t.size(0);
  s->n_q_heads = (int32_t)t.size(1);
  s->n_kv_heads = (int32_t)u.size(1);
  if (how[1] != Py_None) {
    if (!PyBytes_Check(how[1]) || PyBytes_GET_SIZE(how[1]) != u.size(1)) {
      PyErr_SetString(PyExc_ValueError, "mask: need a 0 or 1 for each KV head");
      return false;
    }
    s->full_mask = reinterpret_cast<const uint8_t*>(PyBytes_AS_STRING(how[1]));
  }
  return number(how[0], &s->softmax_scale) && integer(how[2], "sink", &s->sink) && integer(how[3], "recent", &s->recent);
}

// q, k, v, offsets, out, lse, scale, mask, sink, recent
PyObject* packed_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  rlkv_heads_t q, k, v, out;
  rlkv_packed_t s;
  Matrix lse;
  int index;
  if (!arguments(n, 10) || !packed_shape(a, a + 6, &q, &k, &v, &s, &index)) return nullptr;
  if (!head_rows(a[4], "out", index, ScalarType::BFloat16, s.tokens, s.n_q_heads, &out)) return nullptr;
  if (a[5] != Py_None && !matrix_whole(a[5], "lse", index, ScalarType::Float, s.n_q_heads, s.tokens, &lse)) return nullptr;
  const OnDevice on(index);
  return status_of({a[4], a[5]}, [&] { return rlkv_packed_attention(&s, &q, &k, &v, &out, static_cast<float*>(lse.p), on.stream()); });
  RLKV_CALL_END
}

// q, k, v, offsets, out, lse, grad_out, grad_q, grad_k, grad_v, scale, mask, sink, recent, workspace
PyObject* packed_attention_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  rlkv_heads_t q, k, v, out, g, gq, gk, gv;
  rlkv_packed_t s;
  Matrix lse;
  int index;
  void* workspace;
  const ScalarType bf16 = ScalarType::BFloat16;
  if (!arguments(n, 15) || !packed_shape(a, a + 10, &q, &k, &v, &s, &index)) return nullptr;
  if (!head_rows(a[4], "out", index, bf16, s.tokens, s.n_q_heads, &out)) return nullptr;
  if (!matrix_whole(a[5], "lse", index, ScalarType::Float, s.n_q_heads, s.tokens, &lse)) return nullptr;
  if (!head_rows(a[6], "grad_out", index, bf16, s.tokens, s.n_q_heads, &g)) return nullptr;
  if (!head_rows(a[7], "grad_q", index, bf16, s.tokens, s.n_q_heads, &gq)) return nullptr;
  if (!head_rows(a[8], "grad_k", index, bf16, s.tokens, s.n_kv_heads, &gk)) return nullptr;
  if (!head_rows(a[9], "grad_v", index, bf16, s.tokens, s.n_kv_heads, &gv)) return nullptr;
  const at::Tensor* w = tensor(a[14], "workspace");
  if (!w || !vector(a[14], "workspace", index, ScalarType::Byte, w->numel(), &workspace)) return nullptr;
  const OnDevice on(index);
  return status_of({a[7], a[8], a[9]}, [&] {
    return rlkv_packed_attention_grad(&s, &q, &k, &v, &out, static_cast<float*>(lse.p), &g, &gq, &gk, &gv, workspace,
                                      static_cast<size_t>(w->numel()), on.stream());
  });
  RLKV_CALL_END
}

// What both directions of the heads' norm have: qkv, positions, rotary (address or None), then the rows of queries, keys and (or None) values;
// weights and eps (None: no norm).  The numbers of heads are those of the queries' and keys' rows.
struct HeadNormShape {
  Matrix qkv;
  void *positions, *rotary;
  rlkv_heads_t q, k, v;
  bool values;
  int32_t q_heads, kv_heads;
  rlkv_head_norm_t norm;
  bool normed;
};
bool head_norm_shape(PyObject* const* a, const char* const* names, PyObject* const* rows, PyObject* const* weights, HeadNormShape* s) {
  if (!activations(a[0], "qkv", &s->qkv) || !fits(s->qkv.rows, "qkv") || !vector(a[1], "positions", s->qkv.device, ScalarType::Int, s->qkv.rows, &s->positions))
    return false;
  if (!address(a[2], &s->rotary)) return false;
  const int at = s->qkv.device;
  if (!head_rows(rows[0], names[0], at, s->qkv.type, s->qkv.rows, -1, &s->q) || !head_rows(rows[1], names[1], at, s->qkv.type, s->qkv.rows, -1, &s->k))
    return false;
  s->q_heads = (int32_t)THPVariable_Unpack(rows[0]).size(1);
  s->kv_heads = (int32_t)THPVariable_Unpack(rows[1]).size(1);
  s->values = rows[2] != Py_None;
  if (s->values && !head_rows(rows[2], names[2], at, s->qkv.type, s->qkv.rows, s->kv_heads, &s->v)) return false;
  if (!of_size(THPVariable_Unpack(a[0]), "qkv", 1, s->qkv.cols, 128 * (s->q_heads + 2 * (int64_t)s->kv_heads))) return false;
  s->norm = {};
  s->normed = weights[2] != Py_None;
  void *wq, *wk;
  if (!vector(weights[0], "q_weight", at, s->qkv.type, 128, &wq) || !vector(weights[1], "k_weight", at, s->qkv.type, 128, &wk)) return false;
  if (!s->normed && (wq || wk)) {
    PyErr_SetString(PyExc_ValueError, "eps: weights are those of a norm, which needs one");
    return false;
  }
  s->norm.q_weight = wq;
  s->norm.k_weight = wk;
  return !s->normed || number(weights[2], &s->norm.eps);
}

// qkv, positions, rotary, q_out, k_out, v_out, q_weight, k_weight, eps
PyObject* head_norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  HeadNormShape s;
  const char* names[] = {"q_out", "k_out", "v_out"};
  if (!arguments(n, 9) || !head_norm_shape(a, names, a + 3, a + 6, &s)) return nullptr;
  const OnDevice on(s.qkv.device);
  return status_of({a[3], a[4], a[5]}, [&] {
    return rlkv_head_norm_rotary(s.qkv.p, s.qkv.stride, static_cast<int32_t*>(s.positions), static_cast<rlkv_rotary_t*>(s.rotary),
                                 s.normed ? &s.norm : nullptr, (int32_t)s.qkv.rows, s.q_heads, s.kv_heads, kind_of(s.qkv.type), &s.q, &s.k,
                                 s.values ? &s.v : nullptr, on.stream());
  });
  RLKV_CALL_END
}

// qkv, positions, rotary, grad_q, grad_k, grad_qkv, grad_v, q_weight, k_weight, eps, grad_q_weight, grad_k_weight, workspace
PyObject* head_norm_rotary_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  RLKV_CALL_BEGIN
  HeadNormShape s;
  Matrix grad;
  void *gq, *gk, *workspace;
  const char* names[] = {"grad_q", "grad_k", "grad_v"};
  if (!arguments(n, 13)) return nullptr;
  PyObject* const rows[] = {a[3], a[4], a[6]};
  if (!head_norm_shape(a, names, rows, a + 7, &s)) return nullptr;
  const int at = s.qkv.device;
  if (!matrix(a[5], "grad_qkv", at, s.qkv.type, s.qkv.rows, s.qkv.cols, &grad)) return nullptr;
  if (!vector(a[10], "grad_q_weight", at, ScalarType::Float, 128, &gq) || !vector(a[11], "grad_k_weight", at, ScalarType::Float, 128, &gk)) return nullptr;
  const at::Tensor* w = tensor(a[12], "workspace");
  if (!w || !vector(a[12], "workspace", at, ScalarType::Byte, w->numel(), &workspace)) return nullptr;
  const OnDevice on(at);
  return status_of({a[5], a[10], a[11]}, [&] {
    return rlkv_head_norm_rotary_grad(s.qkv.p, s.qkv.stride, static_cast<int32_t*>(s.positions), static_cast<rlkv_rotary_t*>(s.rotary),
                                      s.normed ? &s.norm : nullptr, (int32_t)s.qkv.rows, s.q_heads, s.kv_heads, kind_of(s.qkv.type), &s.q,
                                      &s.k, s.values ? &s.v : nullptr, grad.p, grad.stride, static_cast<float*>(gq), static_cast<float*>(gk),
                                      workspace, static_cast<size_t>(w->numel()), on.stream());
  });
  RLKV_CALL_END
}

#define RLKV_METHOD(name, function) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(function)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RLKV_METHOD("rms_norm", rms_norm),
                         RLKV_METHOD("quantize", quantize),
                         RLKV_METHOD("scaled_matmul", scaled_matmul),
                         RLKV_METHOD("token_logprobs", token_logprobs),
                         RLKV_METHOD("token_logprobs_grad", token_logprobs_grad),
                         RLKV_METHOD("append_rotary", append_rotary),
                         RLKV_METHOD("rotary", rotary_split),
                         RLKV_METHOD("sample_tokens", sample_tokens),
                         RLKV_METHOD("head_norm_rotary", head_norm_rotary),
                         RLKV_METHOD("head_norm_rotary_grad", head_norm_rotary_grad),
                         RLKV_METHOD("packed_attention", packed_attention),
                         RLKV_METHOD("packed_attention_grad", packed_attention_grad),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_tensor_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_calls() { return PyModule_Create(&definition); }
