// Python's side of the operators on tokens (norm, choice, rows and back): checks of the arguments, new outputs, the call, in one step.
//
// These calls are over in two or three microseconds on the GPU, and from Python through ctypes took 9 to 15 on the host, of which the launch is 3: every
// question to a tensor is 0.05 to 0.15, every allocation 1.3, every argument of the C function 0.1. Here they are 3 to 6 (one kernel, outputs given: 3.0 to 3.7). What is checked, and what is said
// where a check fails, is as elsewhere in the binding. The functions of the C ABI are those of the library that the package has loaded (bind).
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <optional>
#include <string>

#include "../../include/moesched.h"

namespace {

using at::ScalarType;
using at::Tensor;
using Shape = c10::SmallVector<int64_t, 6>;

constexpr int64_t MAX_INT = 0x7fffffff, MAX_WIDTH = 65536;

#define ENTRY_POINTS(X)                                                                                                                  \
  X(rms_norm) X(rms_norm_backward) X(route_choose) X(route_choose_backward) X(tokens_to_rows) X(rows_to_tokens) X(rows_to_tokens_backward) \
  X(rows_widen) X(norm_scratch_bytes) X(strerror) X(last_cuda_error)

struct Library {
#define X(name) decltype(&moesched_##name) name = nullptr;
  ENTRY_POINTS(X)
#undef X
} library;

PyObject *error_class = nullptr, *memory_class = nullptr;   // MoeschedError, torch's OutOfMemoryError

struct Refused {
  std::string why;
};
struct InPython {};                // an exception is set

[[noreturn]] void refuse(std::string why) { throw Refused{std::move(why)}; }

std::string text(at::IntArrayRef shape) {
  std::string s = "(";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + (shape.size() == 1 ? ",)" : ")");
}
const char* text(ScalarType t) {
  switch (t) {
    case ScalarType::BFloat16: return "torch.bfloat16";
    case ScalarType::Half: return "torch.float16";
    case ScalarType::Float: return "torch.float32";
    case ScalarType::Float8_e4m3fn: return "torch.float8_e4m3fn";
    case ScalarType::Int: return "torch.int32";
    default: return "torch.uint8";
  }
}

// MOESCHED_BF16, _FP16 or _FP32; -1 for another type
int type_of(ScalarType t) {
  return t == ScalarType::BFloat16 ? MOESCHED_BF16 : t == ScalarType::Half ? MOESCHED_FP16 : t == ScalarType::Float ? MOESCHED_FP32 : -1;
}

const Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a CUDA tensor (the library has no CPU path)");
  return THPVariable_Unpack(o);
}
void on_gpu(const Tensor& t, const char* what) {
  if (!t.is_cuda()) refuse(std::string(what) + " must be a CUDA tensor (the library has no CPU path)");
}
void dense(const Tensor& t, const char* what) {
  if (!t.is_contiguous()) refuse(std::string(what) + " must be contiguous " + text(t.scalar_type()));
}

// The tensor that decides about type, shape and GPU: [..., D], or [..., T, E] with another limit
const Tensor& leading(PyObject* o, const char* what, size_t least) {
  const Tensor& t = tensor(o, what);
  const auto s = t.sizes();
  if (s.size() < least || s.back() < 8 || s.back() > MAX_WIDTH || s.back() % 8 != 0)
    refuse(std::string(what) + " must be [..., D], D a multiple of 8 and 65536 at most");
  dense(t, what);
  return t;
}

// A tensor that has to be like that, on the GPU of `first`; in_out: an entry of the caller's dict of outputs
const Tensor& held(PyObject* o, ScalarType dtype, at::IntArrayRef shape, const Tensor& first, const char* what, bool in_out = false) {
  const auto name = [&] { return in_out ? std::string("out['") + what + "']" : std::string(what); };
  if (!THPVariable_Check(o)) refuse(name() + " must be a CUDA tensor (the library has no CPU path)");
  const Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != dtype || !t.is_contiguous()) refuse(name() + " must be contiguous " + text(dtype));
  if (t.sizes() != shape || t.device() != first.device())
    refuse(name() + " must have shape " + text(shape) + ", on the device of the others");
  return t;
}
const Tensor* held_or_none(PyObject* o, ScalarType dtype, at::IntArrayRef shape, const Tensor& first, const char* what) {
  return o == Py_None ? nullptr : &held(o, dtype, shape, first, what);
}
void* at_(const Tensor* t) { return t == nullptr ? nullptr : t->data_ptr(); }

// Not through the dispatcher, unless it has something to do: fill uninitialised memory (deterministic algorithms), or tell a dispatch mode
Tensor fresh(at::IntArrayRef shape, ScalarType dtype, const Tensor& first) {
  if (at::globalContext().deterministicAlgorithms() || c10::impl::TorchDispatchModeTLS::stack_len() > 0)
    return at::empty(shape, at::TensorOptions().dtype(dtype).device(first.device()));
  return at::detail::empty_cuda(shape, dtype, first.device(), std::nullopt);
}

// out[name] of the caller's dict, checked, or a new tensor
struct Outputs {
  PyObject* have;
  explicit Outputs(PyObject* out) : have(out == Py_None ? nullptr : out) {
    if (have != nullptr && !PyDict_Check(have)) refuse("out must be a dict of an earlier call");
  }
  Tensor take(PyObject* name, at::IntArrayRef shape, ScalarType dtype, const Tensor& first) const {
    PyObject* o = have == nullptr ? nullptr : PyDict_GetItemWithError(have, name);
    if (o == nullptr || o == Py_None) return fresh(shape, dtype, first);
    return held(o, dtype, shape, first, PyUnicode_AsUTF8(name), true);
  }
};
Tensor taken(PyObject* o, at::IntArrayRef shape, ScalarType dtype, const Tensor& first, const char* what) {
  return o == Py_None ? fresh(shape, dtype, first) : held(o, dtype, shape, first, what);
}

PyObject* wrapped(const Tensor& t) {
  PyObject* o = THPVariable_Wrap(t);
  if (o == nullptr) throw InPython{};
  return o;
}
struct Result {
  PyObject* dict = PyDict_New();
  ~Result() { Py_XDECREF(dict); }
  void put(PyObject* name, const Tensor& t) {
    PyObject* o = wrapped(t);
    const int rc = PyDict_SetItem(dict, name, o);
    Py_DECREF(o);
    if (rc != 0) throw InPython{};
  }
  PyObject* give() {
    PyObject* d = dict;
    dict = nullptr;
    return d;
  }
};

int64_t whole(PyObject* o, const char* what) {
  PyObject* n = PyNumber_Long(o);
  if (n == nullptr) throw InPython{};
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(n, &overflow);
  Py_DECREF(n);
  if (overflow != 0) refuse(std::string(what) + " is out of range");
  if (v == -1 && PyErr_Occurred()) throw InPython{};
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw InPython{};
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw InPython{};
  return v != 0;
}
int group_of(PyObject* o) {
  const int64_t g = whole(o, "group");
  if (g != 32 && g != 64 && g != 128) refuse("group must be 32, 64 or 128");
  return (int)g;
}

// Autograd does not record the calls: tensors that want a gradient are refused where it records, and those with a tangent of forward mode, which no_grad() leaves on,
// or gradient and tangent would be lost without a sign
void unrecorded(const char* what, const char* backward, std::initializer_list<PyObject*> arguments, PyObject* out = nullptr) {
  const bool records = c10::GradMode::is_enabled(), tangents = c10::AutogradState::get_tls_state().get_fw_grad_mode();
  const auto check = [&](PyObject* o) {
    if (!THPVariable_Check(o)) return;
    const Tensor& t = THPVariable_Unpack(o);
    if (records && t.requires_grad())
      refuse(std::string(what) + " is not recorded by autograd, but an argument requires a gradient: call it under torch.no_grad() "
             "(gradients come from " + backward + "), or detach the argument");
    if (tangents && t._fw_grad(0).defined())
      refuse(std::string(what) + " has no forward mode of autograd, but an argument has a tangent: call it with its primal");
  };
  for (PyObject* o : arguments) check(o);
  if (out != nullptr && PyDict_Check(out)) {                    // a caller's dict of outputs
    PyObject *name, *o;
    for (Py_ssize_t at = 0; PyDict_Next(out, &at, &name, &o);) check(o);
  }
}

int64_t rows_in(const Tensor& t) {
  const int64_t width = t.sizes().back(), rows = width == 0 ? 0 : t.numel() / width;
  if (rows > MOESCHED_MAX_ROWS) refuse("at most 2^30 rows");
  return rows;
}

// Other threads of the interpreter may run meanwhile
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// The call, with the GPU of `first` current and on its current stream. (An address may be refused too: a tensor without memory, as tracers have.)
template <typename Call>
void run(const char* what, const Tensor& first, Call call) {
  const c10::DeviceIndex index = first.device().index();
  const c10::cuda::OptionalCUDAGuard guard(first.device());
  void* stream = c10::cuda::getCurrentCUDAStream(index).stream();
  const int rc = [&] {
    const Unlocked unlocked;
    return call(stream);
  }();
  if (rc != 0)
    refuse(std::string("moesched_") + what + ": " + library.strerror(rc) + " (rc=" + std::to_string(rc) + ", cuda error " +
           std::to_string(library.last_cuda_error()) + ")");
}

#define NAMES(X) X(y) X(sum) X(q) X(scale) X(rstd) X(dx) X(dweight) X(experts) X(weights) X(drows) X(dweights)
struct Names {
#define X(name) PyObject* name = nullptr;
  NAMES(X)
#undef X
} names;

// x, weight, eps, residual, group, want_y, save, out
PyObject* rms_norm(PyObject* const* a) {
  unrecorded("rms_norm", "rms_norm_backward", {a[0], a[1], a[3]}, a[7]);
  const Tensor& x = leading(a[0], "x", 1);
  const ScalarType dtype = x.scalar_type();
  const int kind = type_of(dtype);
  if (kind < 0) refuse("x must be bfloat16, float16 or float32");
  const Shape shape(x.sizes().begin(), x.sizes().end());
  const int64_t D = shape.back(), rows = rows_in(x);
  const double eps = number(a[2]);
  if (!(eps >= 0.0 && eps < 3e38)) refuse("eps must be a number of at least 0");
  const bool want_y = truth(a[5]), save = truth(a[6]), bits8 = a[4] != Py_None;
  const int group = bits8 ? group_of(a[4]) : 0;
  if (!want_y && !bits8) refuse("y can only be left out where there is an output in 8 bits");
  const Tensor& weight = held(a[1], dtype, {D}, x, "weight");
  const Tensor* residual = held_or_none(a[3], dtype, shape, x, "residual");
  on_gpu(x, "x");
  const Outputs out(a[7]);
  Result result;
  Tensor y, sum, q, scale, rstd;
  if (want_y) result.put(names.y, y = out.take(names.y, shape, dtype, x));
  if (residual != nullptr) result.put(names.sum, sum = out.take(names.sum, shape, dtype, x));
  Shape less(shape.begin(), shape.end() - 1);
  if (save) result.put(names.rstd, rstd = out.take(names.rstd, less, ScalarType::Float, x));
  if (bits8) {
    result.put(names.q, q = out.take(names.q, shape, ScalarType::Float8_e4m3fn, x));
    less.push_back((D + group - 1) / group);
    result.put(names.scale, scale = out.take(names.scale, less, ScalarType::Float, x));
  }
  const auto at = [](const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
  run("rms_norm", x, [&](void* stream) {
    return library.rms_norm((int)rows, (int)D, kind, (float)eps, group, x.data_ptr(), at_(residual), weight.data_ptr(), at(sum), at(y),
                            static_cast<uint8_t*>(at(q)), static_cast<float*>(at(scale)), static_cast<float*>(at(rstd)), stream);
  });
  return result.give();
}

// dy, h, weight, rstd, dsum, out, scratch
PyObject* rms_norm_backward(PyObject* const* a) {
  unrecorded("rms_norm_backward", "rms_norm_backward", {a[0], a[1], a[2], a[3], a[4]}, a[5]);
  const Tensor& h = leading(a[1], "h", 1);
  const ScalarType dtype = h.scalar_type();
  const int kind = type_of(dtype);
  if (kind < 0) refuse("h must be bfloat16, float16 or float32");
  const Shape shape(h.sizes().begin(), h.sizes().end()), less(shape.begin(), shape.end() - 1);
  const int64_t D = shape.back(), rows = rows_in(h);
  const Tensor &dy = held(a[0], dtype, shape, h, "dy"), &weight = held(a[2], dtype, {D}, h, "weight"),
               &rstd = held(a[3], ScalarType::Float, less, h, "rstd");
  const Tensor* dsum = held_or_none(a[4], dtype, shape, h, "dsum");
  const int64_t need = (int64_t)library.norm_scratch_bytes((int)rows, (int)D);
  Tensor scratch;
  if (a[6] != Py_None) {
    scratch = tensor(a[6], "scratch");
    if (scratch.scalar_type() != ScalarType::Byte || !scratch.is_contiguous()) refuse("scratch must be contiguous torch.uint8");
    if (scratch.numel() < need || scratch.device() != h.device()) refuse("scratch is smaller than norm_scratch_bytes, or on another device");
  }
  on_gpu(h, "h");
  const Outputs out(a[5]);
  Result result;
  const Tensor dx = out.take(names.dx, shape, dtype, h), dweight = out.take(names.dweight, {D}, dtype, h);
  if (!scratch.defined()) scratch = fresh({need > 0 ? need : 1}, ScalarType::Byte, h);
  result.put(names.dx, dx);
  result.put(names.dweight, dweight);
  run("rms_norm_backward", h, [&](void* stream) {
    return library.rms_norm_backward((int)rows, (int)D, kind, dy.data_ptr(), h.data_ptr(), weight.data_ptr(), rstd.data_ptr<float>(), at_(dsum),
                                     dx.data_ptr(), dweight.data_ptr(), static_cast<float*>(scratch.data_ptr()), stream);
  });
  return result.give();
}

struct Choice {
  const Tensor& logits;
  int kind, score;
  int64_t rows, E, k;
  bool normalise;
  float factor;
  Shape choices;
};
Choice choice(PyObject* logits, int64_t k, PyObject* score, PyObject* normalise, PyObject* factor) {
  const Tensor& l = tensor(logits, "logits");
  const int kind = type_of(l.scalar_type());
  if (kind < 0) refuse("logits must be bfloat16, float16 or float32");
  const auto s = l.sizes();
  if (s.size() < 2 || s.back() < 1 || s.back() > MOESCHED_MAX_EXPERTS || k < 1 || k > s.back() || k > MOESCHED_MAX_TOP_K)
    refuse("logits must be [..., T, E] with 1024 experts at most, top_k 32 and E at most");
  dense(l, "logits");
  const char* name = PyUnicode_Check(score) ? PyUnicode_AsUTF8(score) : nullptr;
  const bool softmax = name != nullptr && std::strcmp(name, "softmax") == 0;
  if (!softmax && (name == nullptr || std::strcmp(name, "sigmoid") != 0)) refuse("score must be one of ['sigmoid', 'softmax']");
  const double f = number(factor);
  if (!(f > -3e38 && f < 3e38)) refuse("factor must be a number");
  Shape choices(s.begin(), s.end() - 1);
  if (choices.back() > MAX_INT / k) refuse("a source has less than 2^31 choices");
  choices.back() *= k;
  return {l, kind, softmax ? MOESCHED_SCORE_SOFTMAX : MOESCHED_SCORE_SIGMOID, rows_in(l), s.back(), k, truth(normalise), (float)f, std::move(choices)};
}

// logits, top_k, score, bias, normalise, factor, out
PyObject* route_choose(PyObject* const* a) {
  unrecorded("route_choose", "route_choose_backward", {a[0], a[3]}, a[6]);
  const Choice c = choice(a[0], whole(a[1], "top_k"), a[2], a[4], a[5]);
  const Tensor* bias = held_or_none(a[3], ScalarType::Float, {c.E}, c.logits, "bias");
  on_gpu(c.logits, "logits");
  const Outputs out(a[6]);
  Result result;
  const Tensor experts = out.take(names.experts, c.choices, ScalarType::Int, c.logits);
  const Tensor weights = out.take(names.weights, c.choices, ScalarType::Float, c.logits);
  result.put(names.experts, experts);
  result.put(names.weights, weights);
  run("route_choose", c.logits, [&](void* stream) {
    return library.route_choose((int)c.rows, (int)c.E, (int)c.k, c.kind, c.score, c.normalise, c.factor, c.logits.data_ptr(),
                                static_cast<float*>(at_(bias)), experts.data_ptr<int32_t>(), weights.data_ptr<float>(), stream);
  });
  return result.give();
}

// dweights, logits, experts, score, normalise, factor, out
PyObject* route_choose_backward(PyObject* const* a) {
  unrecorded("route_choose_backward", "route_choose_backward", {a[0], a[1], a[6]});
  const Tensor &logits = tensor(a[1], "logits"), &chosen = tensor(a[2], "experts");
  if (logits.dim() < 2 || chosen.dim() < 1) refuse("logits must be [..., T, E] and experts [..., T * top_k]");
  const int64_t T = logits.size(-2), k = T > 0 ? chosen.size(-1) / T : 1;
  const Choice c = choice(a[1], k, a[3], a[4], a[5]);
  const Tensor &experts = held(a[2], ScalarType::Int, c.choices, logits, "experts"), &dweights = held(a[0], ScalarType::Float, c.choices, logits, "dweights");
  on_gpu(logits, "logits");
  const Tensor out = taken(a[6], logits.sizes(), logits.scalar_type(), logits, "out");
  run("route_choose_backward", logits, [&](void* stream) {
    return library.route_choose_backward((int)c.rows, (int)c.E, (int)c.k, c.kind, c.score, c.normalise, c.factor, dweights.data_ptr<float>(),
                                         logits.data_ptr(), experts.data_ptr<int32_t>(), out.data_ptr(), stream);
  });
  return wrapped(out);
}

// Sources and choices a token, for tensors of the leading dimensions `lead` with T tokens each; k < 1: what slot has
struct Sources {
  int64_t G, T, k;
  Shape choices;                   // [..., T * k]
  const Tensor& slot;
};
Sources sources(at::IntArrayRef lead, int64_t T, PyObject* o, int64_t k, const Tensor& first) {
  const Tensor& slot = tensor(o, "slot");
  if (k < 1) {
    const int64_t S = slot.dim() > 0 ? slot.size(-1) : 0;
    k = T > 0 ? S / T : 1;
  }
  if (k < 1 || k > MOESCHED_MAX_TOP_K || T > MAX_INT / k) refuse("slot must have top_k entries for every token, top_k 32 at most");
  int64_t G = 1;
  for (const int64_t n : lead) G = n != 0 && G > MAX_INT / n ? MAX_INT + 1 : G * n;
  if (G > MAX_INT || (T > 0 && G > MOESCHED_MAX_ROWS / T)) refuse("at most 2^30 tokens");
  Shape choices(lead.begin(), lead.end());
  choices.push_back(T * k);
  held(o, ScalarType::Int, choices, first, "slot");
  return {G, T, k, std::move(choices), slot};
}
Shape with(Shape s, int64_t last) {
  s.push_back(last);
  return s;
}

// x, slot, scale, out, out_scale
PyObject* tokens_to_rows(PyObject* const* a) {
  unrecorded("tokens_to_rows", "rows_to_tokens", {a[0], a[2], a[3], a[4]});
  const Tensor& x = leading(a[0], "x", 2);
  const ScalarType dtype = x.scalar_type();
  if (type_of(dtype) < 0 && dtype != ScalarType::Float8_e4m3fn && dtype != ScalarType::Byte)
    refuse("x must be bfloat16, float16, float32, float8_e4m3fn or uint8");
  const auto s = x.sizes();
  const int64_t D = s.back();
  const Sources c = sources(s.slice(0, s.size() - 2), s[s.size() - 2], a[1], 0, x);
  int64_t P = 0;
  const Tensor* scale = nullptr;
  if (a[2] != Py_None) {
    const Tensor& t = tensor(a[2], "scale");
    P = t.dim() > 0 ? t.size(-1) : 0;
    if (P < 1 || P > D) refuse("scale must be [..., T, P], P between 1 and D");
    scale = &held(a[2], ScalarType::Float, with(Shape(s.begin(), s.end() - 1), P), x, "scale");
  } else if (a[4] != Py_None) {
    refuse("out_scale goes with scale");
  }
  on_gpu(x, "x");
  const Tensor out = taken(a[3], with(c.choices, D), dtype, x, "out");
  Tensor out_scale;
  if (scale != nullptr) out_scale = taken(a[4], with(c.choices, P), ScalarType::Float, x, "out_scale");
  run("tokens_to_rows", x, [&](void* stream) {
    return library.tokens_to_rows((int)c.G, (int)c.T, (int)c.k, (int)(D * (int64_t)x.element_size()), (int)P, x.data_ptr(),
                                  static_cast<float*>(at_(scale)), c.slot.data_ptr<int32_t>(), out.data_ptr(),
                                  scale != nullptr ? out_scale.data_ptr<float>() : nullptr, stream);
  });
  PyObject* rows = wrapped(out);
  if (scale == nullptr) return rows;
  PyObject* scales = wrapped(out_scale);
  PyObject* both = PyTuple_Pack(2, rows, scales);
  Py_DECREF(rows);
  Py_DECREF(scales);
  return both;
}

// rows, slot, top_k, weights, add, out
PyObject* rows_to_tokens(PyObject* const* a) {
  unrecorded("rows_to_tokens", "rows_to_tokens_backward", {a[0], a[3], a[4], a[5]});
  const Tensor& rows = leading(a[0], "rows", 2);
  const ScalarType dtype = rows.scalar_type();
  const int kind = type_of(dtype);
  if (kind < 0) refuse("rows must be bfloat16, float16 or float32");
  const auto s = rows.sizes();
  const int64_t D = s.back(), S = s[s.size() - 2], k = whole(a[2], "top_k");
  if (k < 1 || k > MOESCHED_MAX_TOP_K || S % k != 0) refuse("rows must be [..., T * top_k, D], top_k 32 at most");
  const Sources c = sources(s.slice(0, s.size() - 2), S / k, a[1], k, rows);
  const Tensor* weights = held_or_none(a[3], ScalarType::Float, c.choices, rows, "weights");
  Shape tokens(s.begin(), s.end());
  tokens[s.size() - 2] = c.T;
  const Tensor* add = held_or_none(a[4], dtype, tokens, rows, "add");
  on_gpu(rows, "rows");
  const Tensor out = taken(a[5], tokens, dtype, rows, "out");
  run("rows_to_tokens", rows, [&](void* stream) {
    return library.rows_to_tokens((int)c.G, (int)c.T, (int)c.k, (int)D, kind, rows.data_ptr(), c.slot.data_ptr<int32_t>(),
                                  static_cast<float*>(at_(weights)), at_(add), out.data_ptr(), stream);
  });
  return wrapped(out);
}

// dy, rows, slot, weights, out
PyObject* rows_to_tokens_backward(PyObject* const* a) {
  unrecorded("rows_to_tokens_backward", "rows_to_tokens_backward", {a[0], a[1], a[3]}, a[4]);
  const Tensor& dy = leading(a[0], "dy", 2);
  const ScalarType dtype = dy.scalar_type();
  const int kind = type_of(dtype);
  if (kind < 0) refuse("dy must be bfloat16, float16 or float32");
  const auto s = dy.sizes();
  const int64_t D = s.back();
  const Sources c = sources(s.slice(0, s.size() - 2), s[s.size() - 2], a[2], 0, dy);
  const Tensor &rows = held(a[1], dtype, with(c.choices, D), dy, "rows"), &weights = held(a[3], ScalarType::Float, c.choices, dy, "weights");
  on_gpu(dy, "dy");
  const Outputs out(a[4]);
  Result result;
  const Tensor drows = out.take(names.drows, with(c.choices, D), dtype, dy), dweights = out.take(names.dweights, c.choices, ScalarType::Float, dy);
  result.put(names.drows, drows);
  result.put(names.dweights, dweights);
  run("rows_to_tokens_backward", dy, [&](void* stream) {
    return library.rows_to_tokens_backward((int)c.G, (int)c.T, (int)c.k, (int)D, kind, dy.data_ptr(), rows.data_ptr(), c.slot.data_ptr<int32_t>(),
                                           weights.data_ptr<float>(), drows.data_ptr(), dweights.data_ptr<float>(), stream);
  });
  return result.give();
}

// rows, scale, group, dtype, out
PyObject* rows_widen(PyObject* const* a) {
  unrecorded("rows_widen", "dy times scale, and for scale from dy times rows", {a[0], a[1], a[4]});
  const int kind = THPDtype_Check(a[3]) ? type_of(reinterpret_cast<THPDtype*>(a[3])->scalar_type) : -1;
  if (kind < 0) refuse("dtype must be bfloat16, float16 or float32");
  const Tensor& rows = leading(a[0], "rows", 1);
  if (rows.scalar_type() != ScalarType::Float8_e4m3fn) refuse("rows must be float8_e4m3fn");
  const int group = group_of(a[2]);
  const auto s = rows.sizes();
  const int64_t D = s.back();
  const Tensor& scale = held(a[1], ScalarType::Float, with(Shape(s.begin(), s.end() - 1), (D + group - 1) / group), rows, "scale");
  const int64_t count = rows_in(rows);
  on_gpu(rows, "rows");
  const Tensor out = taken(a[4], s, reinterpret_cast<THPDtype*>(a[3])->scalar_type, rows, "out");
  run("rows_widen", rows, [&](void* stream) {
    return library.rows_widen((int)count, (int)D, group, kind, static_cast<uint8_t*>(rows.data_ptr()), scale.data_ptr<float>(), out.data_ptr(), stream);
  });
  return wrapped(out);
}

// What goes wrong becomes a Python exception: nothing leaves a C entry in another way
template <PyObject* (*FUNCTION)(PyObject* const*), int COUNT>
PyObject* entry(PyObject*, PyObject* const* arguments, Py_ssize_t count) {
  if (count != COUNT || library.strerror == nullptr) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or no library bound");
    return nullptr;
  }
  try {
    return FUNCTION(arguments);
  } catch (const Refused& r) {
    PyErr_SetString(error_class, r.why.c_str());
  } catch (const InPython&) {
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(memory_class, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// (error class, class of errors for want of memory, {name: address} of the library's functions)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (count != 3 || !PyDict_Check(a[2])) {
    PyErr_SetString(PyExc_TypeError, "bind(error class, memory class, {name: address})");
    return nullptr;
  }
  Library l;
#define X(name)                                                                                           \
  if (PyObject* o = PyDict_GetItemString(a[2], "moesched_" #name); o != nullptr)                          \
    l.name = reinterpret_cast<decltype(l.name)>(PyLong_AsVoidPtr(o));                                     \
  if (l.name == nullptr) {                                                                                \
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, "moesched_" #name);                            \
    return nullptr;                                                                                       \
  }
  ENTRY_POINTS(X)
#undef X
  Py_INCREF(a[0]);
  Py_XSETREF(error_class, a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(memory_class, a[1]);
  library = l;
  Py_RETURN_NONE;
}

template <PyObject* (*FUNCTION)(PyObject* const*), int COUNT>
constexpr PyCFunction method() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<FUNCTION, COUNT>));
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    {"rms_norm", method<rms_norm, 8>(), METH_FASTCALL, nullptr},
    {"rms_norm_backward", method<rms_norm_backward, 7>(), METH_FASTCALL, nullptr},
    {"route_choose", method<route_choose, 7>(), METH_FASTCALL, nullptr},
    {"route_choose_backward", method<route_choose_backward, 7>(), METH_FASTCALL, nullptr},
    {"tokens_to_rows", method<tokens_to_rows, 5>(), METH_FASTCALL, nullptr},
    {"rows_to_tokens", method<rows_to_tokens, 6>(), METH_FASTCALL, nullptr},
    {"rows_to_tokens_backward", method<rows_to_tokens_backward, 5>(), METH_FASTCALL, nullptr},
    {"rows_widen", method<rows_widen, 5>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

// What this file was compiled for and how, to be found in it before it is loaded
#ifndef MOESCHED_STAMP
#define MOESCHED_STAMP ""
#endif
const char stamp[] = MOESCHED_STAMP;

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
#define X(name) names.name = PyUnicode_InternFromString(#name);
  NAMES(X)
#undef X
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "stamp", stamp) != 0) Py_CLEAR(m);
  return m;
}
