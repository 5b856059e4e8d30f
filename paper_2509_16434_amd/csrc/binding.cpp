// The calls a training program makes once per environment step (buffer_write, act, buffer_write_outcome, gae), and the
// operators on caller-owned tensors (dropout, token_logp, ...), bound natively: argument checks and the call into libppo_learner.so in 0.4 us, where checking seven tensors through
// Python attributes and calling through ctypes cost 3.4 us beside the kernel launch behind it, which set the pace of
// small tasks (64 environments: 16 writes, 145 .. 161 -> 110 .. 114 us).  Marshalling only: the library's functions are
// handed in as addresses by learner.py, which loads the library and binds everything else.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>

#include "../../include/ppo_learner.h"

namespace {

decltype(&ppo_buffer_write) f_write = nullptr;
decltype(&ppo_buffer_write_range) f_write_range = nullptr;
decltype(&ppo_act) f_act = nullptr;
decltype(&ppo_buffer_write_outcome) f_outcome = nullptr;
decltype(&ppo_gae) f_gae = nullptr;
decltype(&ppo_dropout) f_dropout = nullptr;
decltype(&ppo_token_logp_ws_bytes) f_token_logp_ws = nullptr;
decltype(&ppo_token_logp) f_token_logp = nullptr;
decltype(&ppo_token_logp_backward) f_token_logp_backward = nullptr;
decltype(&ppo_token_loss_ws_bytes) f_token_loss_ws = nullptr;
decltype(&ppo_token_loss) f_token_loss = nullptr;
decltype(&ppo_pair_ws_bytes) f_pair_ws = nullptr;
decltype(&ppo_pair_loss) f_pair_loss = nullptr;
decltype(&ppo_token_gae_ws_bytes) f_token_gae_ws = nullptr;
decltype(&ppo_token_gae) f_token_gae = nullptr;

const char* dtype_name(at::ScalarType t) {
  return t == at::kFloat ? "torch.float32" : t == at::kBFloat16 ? "torch.bfloat16" : t == at::kByte ? "torch.uint8" : at::toString(t);
}

// Device pointer of a contiguous CUDA tensor of `numel` elements of type `dt`; None gives NULL.  False: error set.
bool device_ptr(PyObject* o, at::ScalarType dt, int64_t numel, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "expected a torch.Tensor or None, got %s", Py_TYPE(o)->tp_name); return false; }
  try {  // a tensor without storage of its own (a tracer's stand-in) throws when asked for its address
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) { PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor"); return false; }
    if (t.scalar_type() != dt) { PyErr_Format(PyExc_ValueError, "expected dtype %s, got %s", dtype_name(dt), dtype_name(t.scalar_type())); return false; }
    if (t.numel() != numel) { PyErr_Format(PyExc_ValueError, "expected %lld elements, got %lld", (long long)numel, (long long)t.numel()); return false; }
    *out = t.data_ptr();
    return true;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return false;
  }
}

bool integers(PyObject* const* args, int n, long long* out) {
  for (int i = 0; i < n; ++i) {
    PyObject* x = PyNumber_Index(args[i]);  // any integer type; a float is a TypeError, as it is through ctypes
    if (!x) return false;
    out[i] = PyLong_AsLongLong(x);
    Py_DECREF(x);
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

bool arity(Py_ssize_t got, Py_ssize_t want, const char* name) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, got);
  return false;
}

// setup(addresses of ppo_buffer_write, ppo_buffer_write_range, ppo_act, ppo_buffer_write_outcome, ppo_gae, then of the operators
// in the order of their declaration)
PyObject* py_setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long v[15];
  if (!arity(n, 15, "setup") || !integers(a, 15, v)) return nullptr;
  f_dropout = reinterpret_cast<decltype(f_dropout)>(v[5]); f_token_logp_ws = reinterpret_cast<decltype(f_token_logp_ws)>(v[6]);
  f_token_logp = reinterpret_cast<decltype(f_token_logp)>(v[7]); f_token_logp_backward = reinterpret_cast<decltype(f_token_logp_backward)>(v[8]);
  f_token_loss_ws = reinterpret_cast<decltype(f_token_loss_ws)>(v[9]); f_token_loss = reinterpret_cast<decltype(f_token_loss)>(v[10]);
  f_pair_ws = reinterpret_cast<decltype(f_pair_ws)>(v[11]); f_pair_loss = reinterpret_cast<decltype(f_pair_loss)>(v[12]);
  f_token_gae_ws = reinterpret_cast<decltype(f_token_gae_ws)>(v[13]); f_token_gae = reinterpret_cast<decltype(f_token_gae)>(v[14]);
  f_write = reinterpret_cast<decltype(f_write)>(v[0]); f_write_range = reinterpret_cast<decltype(f_write_range)>(v[1]);
  f_act = reinterpret_cast<decltype(f_act)>(v[2]); f_outcome = reinterpret_cast<decltype(f_outcome)>(v[3]); f_gae = reinterpret_cast<decltype(f_gae)>(v[4]);
  Py_RETURN_NONE;
}

// write(handle, fp32 images, elements per observation, P, A, t, env_offset or -1, count, obs, proprio, action, logp, value, reward, done) -> code
PyObject* py_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long v[8];
  if (!arity(n, 15, "write") || !integers(a, 8, v)) return nullptr;
  const long long cnt = v[7];
  void* p[7];
  if (!device_ptr(a[8], v[1] ? at::kFloat : at::kBFloat16, cnt * v[2], &p[0]) || !device_ptr(a[9], at::kFloat, cnt * v[3], &p[1]) ||
      !device_ptr(a[10], at::kFloat, cnt * v[4], &p[2]) || !device_ptr(a[11], at::kFloat, cnt, &p[3]) || !device_ptr(a[12], at::kFloat, cnt, &p[4]) ||
      !device_ptr(a[13], at::kFloat, cnt, &p[5]) || !device_ptr(a[14], at::kByte, cnt, &p[6]))
    return nullptr;
  ppo_ctx* c = reinterpret_cast<ppo_ctx*>(v[0]);
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  if (v[6] < 0)
    rc = f_write(c, (int32_t)v[5], p[0], (const float*)p[1], (const float*)p[2], (const float*)p[3], (const float*)p[4], (const float*)p[5], (const uint8_t*)p[6]);
  else
    rc = f_write_range(c, (int32_t)v[5], (int32_t)v[6], (int32_t)cnt, p[0], (const float*)p[1], (const float*)p[2], (const float*)p[3], (const float*)p[4],
                       (const float*)p[5], (const uint8_t*)p[6]);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// act(handle, fp32 images, elements per observation, P, A, t, N, obs, proprio, noise) -> (code, action [N][A], logp [N], value [N])
PyObject* py_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long v[7];
  if (!arity(n, 10, "act") || !integers(a, 7, v)) return nullptr;
  const long long N = v[6];
  void* p[3];
  if (!device_ptr(a[7], v[1] ? at::kFloat : at::kBFloat16, N * v[2], &p[0]) || !device_ptr(a[8], at::kFloat, N * v[3], &p[1]) ||
      !device_ptr(a[9], at::kFloat, N * v[4], &p[2]))
    return nullptr;
  try {
    const auto opt = at::TensorOptions().dtype(at::kFloat).device(at::kCUDA);
    at::Tensor action = at::empty({N, v[4]}, opt), logp = at::empty({N}, opt), value = at::empty({N}, opt);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f_act(reinterpret_cast<ppo_ctx*>(v[0]), (int32_t)v[5], p[0], (const float*)p[1], (const float*)p[2], (float*)action.data_ptr(), (float*)logp.data_ptr(),
               (float*)value.data_ptr());
    Py_END_ALLOW_THREADS;
    return Py_BuildValue("iNNN", rc, THPVariable_Wrap(std::move(action)), THPVariable_Wrap(std::move(logp)), THPVariable_Wrap(std::move(value)));
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// outcome(handle, t, N, reward, done) -> code
PyObject* py_outcome(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long v[3];
  void* p[2];
  if (!arity(n, 5, "outcome") || !integers(a, 3, v) || !device_ptr(a[3], at::kFloat, v[2], &p[0]) || !device_ptr(a[4], at::kByte, v[2], &p[1])) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = f_outcome(reinterpret_cast<ppo_ctx*>(v[0]), (int32_t)v[1], (const float*)p[0], (const uint8_t*)p[1]);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// gae(handle, N, last_value, gamma, lambda) -> code
PyObject* py_gae(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long v[2];
  void* p;
  if (!arity(n, 5, "gae") || !integers(a, 2, v) || !device_ptr(a[2], at::kFloat, v[1], &p)) return nullptr;
  const double gamma = PyFloat_AsDouble(a[3]), lam = PyFloat_AsDouble(a[4]);
  if (PyErr_Occurred()) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = f_gae(reinterpret_cast<ppo_ctx*>(v[0]), (const float*)p, (float)gamma, (float)lam);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// ---- operators on caller-owned tensors.  The first argument of each is the raw stream; results are allocated here, on the
// device of the inputs and under torch's current stream, which the caller has made the one that is passed.

// What is wrong with an argument, told as a Python exception of its kind.
struct Wrong { PyObject* type; std::string text; };

// The tensor in `o`; None gives an undefined one if it may be missing.
at::Tensor tensor(PyObject* o, const char* name, bool needed = true) {
  if (o == Py_None) {
    if (needed) throw Wrong{PyExc_TypeError, std::string(name) + " is missing"};
    return {};
  }
  if (!THPVariable_Check(o)) throw Wrong{PyExc_TypeError, std::string(name) + ": expected a torch.Tensor, got " + Py_TYPE(o)->tp_name};
  at::Tensor t = THPVariable_Unpack(o);
  if (!t.is_cuda()) throw Wrong{PyExc_ValueError, std::string(name) + ": expected a CUDA tensor"};
  return t;
}
void same_device(const at::Tensor& t, const at::Tensor& like, const char* name) {
  if (t.device() != like.device()) throw Wrong{PyExc_ValueError, std::string(name) + " is on " + t.device().str() + ", the call's first tensor on " + like.device().str()};
}
// Contiguous array of n elements of a type.
at::Tensor array(PyObject* o, const char* name, at::ScalarType dt, int64_t n, const at::Tensor& like, bool needed = true) {
  at::Tensor t = tensor(o, name, needed);
  if (!t.defined()) return t;
  same_device(t, like, name);
  if (!t.is_contiguous()) throw Wrong{PyExc_ValueError, std::string(name) + ": expected a contiguous tensor"};
  if (t.scalar_type() != dt) throw Wrong{PyExc_ValueError, std::string(name) + ": expected dtype " + at::toString(dt) + ", got " + at::toString(t.scalar_type())};
  if (t.numel() != n) throw Wrong{PyExc_ValueError, std::string(name) + ": expected " + std::to_string(n) + " elements, got " + std::to_string(t.numel())};
  return t;
}
int32_t dtype_code(const at::Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kFloat: return 0;
    case at::kBFloat16: return 1;
    case at::kHalf: return 2;
    default: throw Wrong{PyExc_ValueError, std::string(name) + ": expected float32, bfloat16 or float16, got " + at::toString(t.scalar_type())};
  }
}
// Matrix with adjacent columns; its row stride (that of a matrix of at most one row is its width).
int64_t row_stride(const at::Tensor& t, const char* name) {
  if (t.dim() != 2) throw Wrong{PyExc_ValueError, std::string(name) + ": expected two dimensions, got " + std::to_string(t.dim())};
  if (t.size(1) > 1 && t.stride(1) != 1) throw Wrong{PyExc_ValueError, std::string(name) + ": the columns of a row must be adjacent"};
  if (t.size(0) > 1 && t.stride(0) < t.size(1)) throw Wrong{PyExc_ValueError, std::string(name) + ": rows overlap"};
  return t.size(0) > 1 ? t.stride(0) : t.size(1);
}
// `out` if it is given (of the shape and type of `like`), else a new matrix.
at::Tensor out_matrix(PyObject* o, const at::Tensor& like) {
  at::Tensor t = tensor(o, "out", false);
  if (!t.defined()) return at::empty(like.sizes(), like.options().memory_format(at::MemoryFormat::Contiguous));
  same_device(t, like, "out");
  if (t.sizes() != like.sizes() || t.scalar_type() != like.scalar_type()) throw Wrong{PyExc_ValueError, "out: expected the shape and type of the input"};
  return t;
}
// `out` has been written: autograd is to know it, for a backward pass that needs what was there.
void changed(PyObject* out, const at::Tensor& t) {
  if (out != Py_None && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// Memory of `out` and of an input: apart, the same place with the same row stride, or side by side in rows of one stride.
void apart_or_same(const at::Tensor& out, int64_t ldo, const at::Tensor& in, int64_t ldi, const char* name) {
  if (!in.defined() || !out.numel()) return;
  const int64_t es = out.element_size(), rows = out.size(0), cols = out.size(1);
  const char *a = (const char*)out.data_ptr(), *b = (const char*)in.data_ptr();
  const char *ae = a + ((rows - 1) * ldo + cols) * es, *be = b + ((rows - 1) * ldi + cols) * es;
  if (a >= be || b >= ae || (a == b && ldo == ldi)) return;
  if (ldo == ldi && (a - b) % es == 0) {
    const int64_t d = (((a - b) / es) % ldo + ldo) % ldo;
    if (d >= cols && ldo - d >= cols) return;
  }
  throw Wrong{PyExc_ValueError, std::string("out overlaps ") + name + " without being it"};
}
template <class T> T* ptr(const at::Tensor& t) { return t.defined() ? (T*)t.data_ptr() : nullptr; }
PyObject* wrap(at::Tensor t) {
  if (t.defined()) return THPVariable_Wrap(std::move(t));
  Py_RETURN_NONE;
}
at::Tensor floats(int64_t n, const at::Tensor& like) { return at::empty({n}, like.options().dtype(at::kFloat).memory_format(at::MemoryFormat::Contiguous)); }
at::Tensor scratch(int64_t bytes, const at::Tensor& like) { return bytes > 0 ? at::empty({bytes}, like.options().dtype(at::kByte).memory_format(at::MemoryFormat::Contiguous)) : at::Tensor(); }
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Wrong{nullptr, ""};
  return v;
}
long long whole(PyObject* o) {
  long long v;
  if (!integers(&o, 1, &v)) throw Wrong{nullptr, ""};
  return v;
}
uint64_t whole64(PyObject* o) {
  PyObject* x = PyNumber_Index(o);
  if (!x) throw Wrong{nullptr, ""};
  const uint64_t v = PyLong_AsUnsignedLongLong(x);
  Py_DECREF(x);
  if (v == (uint64_t)-1 && PyErr_Occurred()) throw Wrong{nullptr, ""};
  return v;
}
void* stream_of(PyObject* o) { return reinterpret_cast<void*>((intptr_t)whole(o)); }

// Runs an operator's body; exceptions become Python errors.
template <class F>
PyObject* guarded(F body) {
  try {
    return body();
  } catch (const Wrong& w) {
    if (w.type) PyErr_SetString(w.type, w.text.c_str());
  } catch (const std::exception&) {
    torch::translate_exception_to_python(std::current_exception());   // as torch's own functions tell it, OutOfMemoryError among others
  }
  return nullptr;
}
// The library call without the interpreter's lock.
template <class F>
int without_lock(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call();
  Py_END_ALLOW_THREADS;
  return rc;
}

// dropout(stream, x, p, seed, layer, row_ids, residual, out) -> (code, y)
PyObject* py_dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 8, "dropout")) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor x = tensor(a[1], "x");
    const int32_t dt = dtype_code(x, "x");
    const int64_t ldx = row_stride(x, "x"), rows = x.size(0), cols = x.size(1);
    const at::Tensor ids = array(a[5], "row_ids", at::kLong, rows, x, false);
    const at::Tensor res = tensor(a[6], "residual", false);
    int64_t ldr = cols;
    if (res.defined()) {
      same_device(res, x, "residual");
      if (res.sizes() != x.sizes() || res.scalar_type() != x.scalar_type()) throw Wrong{PyExc_ValueError, "residual: expected the shape and type of x"};
      ldr = row_stride(res, "residual");
    }
    const double p = real(a[2]);
    const uint64_t seed = whole64(a[3]), layer = whole64(a[4]);
    void* st = stream_of(a[0]);
    const c10::DeviceGuard on(x.device());
    at::Tensor y = out_matrix(a[7], x);
    const int64_t ldy = row_stride(y, "out");
    apart_or_same(y, ldy, x, ldx, "x");
    apart_or_same(y, ldy, res, ldr, "residual");
    const int rc = without_lock([&] { return f_dropout(dt, rows, cols, x.data_ptr(), ldx, ptr<const int64_t>(ids), ptr<void>(res), ldr, p, seed, layer, y.data_ptr(), ldy, st); });
    if (rc == PPO_OK) changed(a[7], y);
    return Py_BuildValue("iN", rc, wrap(std::move(y)));
  });
}

// token_logp(stream, logits, target, temperature, want_entropy) -> (code, logp, entropy or None, stat)
PyObject* py_token_logp(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 5, "token_logp")) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor x = tensor(a[1], "logits");
    const int32_t dt = dtype_code(x, "logits");
    const int64_t ld = row_stride(x, "logits"), rows = x.size(0), V = x.size(1);
    const at::Tensor target = array(a[2], "target", at::kInt, rows, x);
    const double temperature = real(a[3]);
    const bool ent = whole(a[4]) != 0;
    void* st = stream_of(a[0]);
    const c10::DeviceGuard on(x.device());
    at::Tensor logp = floats(rows, x), entropy = ent ? floats(rows, x) : at::Tensor(), stat = at::empty({rows, 2}, logp.options());
    const int64_t wsb = f_token_logp_ws(rows, V);
    const at::Tensor ws = scratch(wsb, x);
    const int rc = without_lock([&] {
      return f_token_logp(dt, rows, V, x.data_ptr(), ld, ptr<const int32_t>(target), (float)temperature, ptr<float>(logp), ptr<float>(entropy), ptr<float>(stat), ptr<void>(ws), wsb, st);
    });
    return Py_BuildValue("iNNN", rc, wrap(std::move(logp)), wrap(std::move(entropy)), wrap(std::move(stat)));
  });
}

// token_logp_backward(stream, logits, target, stat, dlogp, temperature, entropy, dentropy, out) -> (code, dlogits)
PyObject* py_token_logp_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 9, "token_logp_backward")) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor x = tensor(a[1], "logits");
    const int32_t dt = dtype_code(x, "logits");
    const int64_t ld = row_stride(x, "logits"), rows = x.size(0), V = x.size(1);
    const at::Tensor target = array(a[2], "target", at::kInt, rows, x), stat = array(a[3], "stat", at::kFloat, 2 * rows, x),
                     dlogp = array(a[4], "dlogp", at::kFloat, rows, x), entropy = array(a[6], "entropy", at::kFloat, rows, x, a[7] != Py_None),
                     dentropy = array(a[7], "dentropy", at::kFloat, rows, x, false);
    const double temperature = real(a[5]);
    void* st = stream_of(a[0]);
    const c10::DeviceGuard on(x.device());
    at::Tensor d = out_matrix(a[8], x);
    const int64_t ldd = row_stride(d, "out");
    apart_or_same(d, ldd, x, ld, "logits");
    const int rc = without_lock([&] {
      return f_token_logp_backward(dt, rows, V, x.data_ptr(), ld, ptr<const int32_t>(target), (float)temperature, ptr<const float>(stat), ptr<const float>(dlogp),
                                   ptr<const float>(entropy), ptr<const float>(dentropy), d.data_ptr(), ldd, st);
    });
    if (rc == PPO_OK) changed(a[8], d);
    return Py_BuildValue("iN", rc, wrap(std::move(d)));
  });
}

// token_loss(stream, logits, target, logp_old, adv, logp_ref, weight, scale, temperature, clip_lo, clip_hi, kl_coef, ent_coef, out)
//   -> (code, dlogits, stats, logp)
PyObject* py_token_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 14, "token_loss")) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor x = tensor(a[1], "logits");
    const int32_t dt = dtype_code(x, "logits");
    const int64_t ld = row_stride(x, "logits"), rows = x.size(0), V = x.size(1);
    const at::Tensor target = array(a[2], "target", at::kInt, rows, x), old = array(a[3], "logp_old", at::kFloat, rows, x), adv = array(a[4], "adv", at::kFloat, rows, x),
                     ref = array(a[5], "logp_ref", at::kFloat, rows, x, false), weight = array(a[6], "weight", at::kFloat, rows, x, false);
    ppo_token_hparams hp;
    hp.scale = (float)real(a[7]); hp.temperature = (float)real(a[8]); hp.clip_lo = (float)real(a[9]); hp.clip_hi = (float)real(a[10]);
    hp.kl_coef = (float)real(a[11]); hp.ent_coef = (float)real(a[12]);
    void* st = stream_of(a[0]);
    const c10::DeviceGuard on(x.device());
    at::Tensor d = out_matrix(a[13], x);
    const int64_t ldd = row_stride(d, "out");
    apart_or_same(d, ldd, x, ld, "logits");
    at::Tensor logp = floats(rows, x), stats = floats(8, x);
    const int64_t wsb = f_token_loss_ws(rows, V);
    const at::Tensor ws = scratch(wsb, x);
    const int rc = without_lock([&] {
      return f_token_loss(dt, rows, V, x.data_ptr(), ld, ptr<const int32_t>(target), ptr<const float>(old), ptr<const float>(ref), ptr<const float>(adv), ptr<const float>(weight),
                          &hp, d.data_ptr(), ldd, ptr<float>(logp), ptr<float>(stats), ptr<void>(ws), wsb, st);
    });
    if (rc == PPO_OK) changed(a[13], d);
    return Py_BuildValue("iNNN", rc, wrap(std::move(d)), wrap(std::move(stats)), wrap(std::move(logp)));
  });
}

// pair_loss(stream, logp, offsets, logp_ref, mask, kind, length_mean, beta, label_smoothing, scale) -> (code, dlogp, margin, stats)
PyObject* py_pair_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 10, "pair_loss")) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor offsets = tensor(a[2], "offsets");
    const int64_t bounds = offsets.numel();
    if (bounds < 1 || bounds % 2 == 0) throw Wrong{PyExc_ValueError, "offsets: expected 2 * pairs + 1 elements, got " + std::to_string(bounds)};
    at::Tensor logp = tensor(a[1], "logp");
    const int64_t T = logp.numel(), pairs = bounds / 2;
    logp = array(a[1], "logp", at::kFloat, T, logp);
    array(a[2], "offsets", at::kLong, bounds, logp);
    const at::Tensor ref = array(a[3], "logp_ref", at::kFloat, T, logp, false), mask = array(a[4], "mask", at::kByte, T, logp, false);
    ppo_pair_hparams hp;
    hp.kind = (int32_t)whole(a[5]); hp.length_mean = whole(a[6]) != 0; hp.beta = (float)real(a[7]); hp.label_smoothing = (float)real(a[8]); hp.scale = (float)real(a[9]);
    void* st = stream_of(a[0]);
    const c10::DeviceGuard on(logp.device());
    at::Tensor dlogp = floats(T, logp), margin = floats(pairs, logp), stats = floats(7, logp);
    const int64_t wsb = f_pair_ws(pairs, T);
    const at::Tensor ws = scratch(wsb, logp);
    const int rc = without_lock([&] {
      return f_pair_loss(pairs, T, ptr<const float>(logp), ptr<const float>(ref), ptr<const uint8_t>(mask), ptr<const int64_t>(offsets), &hp, ptr<float>(dlogp), ptr<float>(margin),
                         ptr<float>(stats), ptr<void>(ws), wsb, st);
    });
    return Py_BuildValue("iNNN", rc, wrap(std::move(dlogp)), wrap(std::move(margin)), wrap(std::move(stats)));
  });
}

// token_gae(stream, reward, value, offsets, gamma, lambda, last_value, mask) -> (code, adv, ret)
PyObject* py_token_gae(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 8, "token_gae")) return nullptr;
  return guarded([&]() -> PyObject* {
    at::Tensor reward = tensor(a[1], "reward");
    const int64_t T = reward.numel();
    reward = array(a[1], "reward", at::kFloat, T, reward);
    const at::Tensor value = array(a[2], "value", at::kFloat, T, reward);
    at::Tensor offsets = tensor(a[3], "offsets");
    if (offsets.numel() < 1) throw Wrong{PyExc_ValueError, "offsets: expected sequences + 1 elements, got none"};
    offsets = array(a[3], "offsets", at::kLong, offsets.numel(), reward);
    const int64_t S = offsets.numel() - 1;
    const double gamma = real(a[4]), lambda = real(a[5]);
    const at::Tensor last = array(a[6], "last_value", at::kFloat, S, reward, false), mask = array(a[7], "mask", at::kByte, T, reward, false);
    void* st = stream_of(a[0]);
    const c10::DeviceGuard on(reward.device());
    at::Tensor adv = floats(T, reward), ret = floats(T, reward);
    const int64_t wsb = f_token_gae_ws(S, T);
    const at::Tensor ws = scratch(wsb, reward);
    const int rc = without_lock([&] {
      return f_token_gae(S, T, ptr<const float>(reward), ptr<const float>(value), ptr<const uint8_t>(mask), ptr<const int64_t>(offsets), ptr<const float>(last), gamma, lambda,
                         ptr<float>(adv), ptr<float>(ret), ptr<void>(ws), wsb, st);
    });
    return Py_BuildValue("iNN", rc, wrap(std::move(adv)), wrap(std::move(ret)));
  });
}

PyMethodDef methods[] = {{"setup", (PyCFunction)(void*)py_setup, METH_FASTCALL, nullptr}, {"write", (PyCFunction)(void*)py_write, METH_FASTCALL, nullptr},
                         {"act", (PyCFunction)(void*)py_act, METH_FASTCALL, nullptr}, {"outcome", (PyCFunction)(void*)py_outcome, METH_FASTCALL, nullptr},
                         {"gae", (PyCFunction)(void*)py_gae, METH_FASTCALL, nullptr}, {"dropout", (PyCFunction)(void*)py_dropout, METH_FASTCALL, nullptr},
                         {"token_logp", (PyCFunction)(void*)py_token_logp, METH_FASTCALL, nullptr}, {"token_logp_backward", (PyCFunction)(void*)py_token_logp_backward, METH_FASTCALL, nullptr},
                         {"token_loss", (PyCFunction)(void*)py_token_loss, METH_FASTCALL, nullptr}, {"pair_loss", (PyCFunction)(void*)py_pair_loss, METH_FASTCALL, nullptr},
                         {"token_gae", (PyCFunction)(void*)py_token_gae, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
