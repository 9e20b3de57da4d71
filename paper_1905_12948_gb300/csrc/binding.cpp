// Python module _tokens: the operators of tokens.py on torch tensors. It checks and
// marshals arguments, allocates outputs and calls the C ABI (through the addresses that
// init() is given); nothing is computed here. As compiled code it takes 4 to 12 us of
// host time a call, allocations and launch included, where ctypes and the same checks in
// Python took 10 to 20: small calls are bound by that.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "gmc.h"

namespace {

using at::Tensor;

struct Abi {
  decltype(&gmc_token_logp) token_logp = nullptr;
  decltype(&gmc_token_logp_backward) token_logp_backward = nullptr;
  decltype(&gmc_policy_loss) policy_loss = nullptr;
  decltype(&gmc_preference_loss) preference_loss = nullptr;
  decltype(&gmc_dropout) dropout = nullptr;
  decltype(&gmc_token_scores) token_scores = nullptr;
  decltype(&gmc_token_scores_backward) token_scores_backward = nullptr;
  decltype(&gmc_orthogonalize_workspace) orthogonalize_workspace = nullptr;
  decltype(&gmc_orthogonalize) orthogonalize = nullptr;
} g_abi;
PyObject* g_error = nullptr;  // GMCError

// Thrown with a Python error set.
struct PythonError {};

[[noreturn]] void fail(PyObject* type, const char* name, const char* what) {
  PyErr_Format(type, "%s %s", name, what);
  throw PythonError();
}
void check(int status, const char* what) {
  if (status == GMC_OK) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", status, what);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw PythonError();
}

const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, name, "must be a CUDA tensor");
  const Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) fail(PyExc_TypeError, name, "must be a CUDA tensor");
  return t;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError();
  return v;
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  return v;
}
uint64_t bits64(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw PythonError();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PythonError();
  return v != 0;
}

int32_t kind(const Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kFloat: return GMC_F32;
    case at::kBFloat16: return GMC_BF16;
    case at::kHalf: return GMC_F16;
    default: fail(PyExc_TypeError, name, "must be float32, bfloat16 or float16");
  }
}

// Rows of a 2-D tensor, each contiguous.
struct Rows {
  int64_t n, v, ld;
};
Rows rows(const Tensor& t, const char* name) {
  if (t.dim() != 2) fail(PyExc_TypeError, name, "must be 2-D");
  Rows r{t.size(0), t.size(1), t.stride(0)};
  if (r.v > 1 && t.stride(1) != 1) fail(PyExc_TypeError, name, "must have contiguous rows");
  if (r.n <= 1) r.ld = r.v;
  if (r.ld < r.v) fail(PyExc_TypeError, name, "must have rows that do not overlap");
  return r;
}

// The data of a contiguous tensor of n elements, NULL for None.
template <typename T>
T* vector(PyObject* o, int64_t n, at::ScalarType type, const Tensor& like, const char* name) {
  if (o == Py_None) return nullptr;
  const Tensor& t = tensor(o, name);
  if (t.device() != like.device()) fail(PyExc_TypeError, name, "must be on the logits' device");
  if (t.scalar_type() != type || !t.is_contiguous())
    fail(PyExc_TypeError, name, type == at::kLong ? "must be a contiguous int64 tensor" : "must be a contiguous float32 tensor");
  if (t.numel() != n) {
    PyErr_Format(PyExc_ValueError, "%s must have %lld elements", name, (long long)n);
    throw PythonError();
  }
  return static_cast<T*>(t.data_ptr());
}
const float* floats(PyObject* o, int64_t n, const Tensor& like, const char* name) {
  return vector<const float>(o, n, at::kFloat, like, name);
}
const int64_t* targets(PyObject* o, int64_t n, const Tensor& like) {
  return vector<const int64_t>(o, n, at::kLong, like, "targets");
}

// A new tensor of t's shape whose parts t[0], t[1], ... (n elements each, ld apart in t) lie
// at the offsets from a `whole`-byte boundary that t's do: contiguous but where t is a view with
// padded parts or an odd start. The kernels then store whole vectors.
Tensor empty_beside(const Tensor& t, int64_t parts, int64_t n, int64_t ld, int64_t whole) {
  const int64_t per = whole / t.element_size();
  const int64_t shift = (int64_t)(reinterpret_cast<uintptr_t>(t.data_ptr()) & (whole - 1)) / t.element_size();
  const int64_t pad = parts > 1 ? (ld - n) % per : 0;
  if (shift == 0 && pad == 0) return at::empty(t.sizes(), t.options());
  std::vector<int64_t> strides(t.dim());
  int64_t step = 1;
  for (int64_t d = t.dim() - 1; d > 0; --d) {
    strides[d] = step;
    step *= t.size(d);
  }
  strides[0] = n + pad;
  return at::empty({parts * (n + pad) + shift}, t.options()).as_strided(t.sizes(), strides, shift);
}

// The gradient's destination: `o`, or a new tensor for None; its row stride in *ld.
Tensor gradient(PyObject* o, const Tensor& logits, const Rows& r, int64_t* ld) {
  if (o == Py_None) {
    Tensor t = empty_beside(logits, r.n, r.v, r.ld, 32);
    *ld = r.n > 1 ? t.stride(0) : r.v;
    return t;
  }
  const Tensor& t = tensor(o, "out");
  if (t.sizes() != logits.sizes() || t.scalar_type() != logits.scalar_type() || t.device() != logits.device())
    fail(PyExc_TypeError, "out", "must have the logits' shape, dtype and device");
  *ld = rows(t, "out").ld;
  return t;
}

// What torch's own writes in place do: a backward pass that saved the tensor then refuses it.
// (Inference tensors have no version, and are never saved.)
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// `sizes` elements of a 1-D tensor from `at` on, as a tensor of its own.
Tensor part(const Tensor& whole, at::IntArrayRef sizes, int64_t at) {
  Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(at);
  t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
  return t;
}

void* stream_of(const Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }

void arguments(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return;
  PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", got, want);
  throw PythonError();
}

// Objects of a result, released if an exception is under way.
PyObject* wrap(Tensor t) {
  PyObject* o = THPVariable_Wrap(std::move(t));
  if (!o) throw PythonError();
  return o;
}
PyObject* tuple_of(std::initializer_list<PyObject*> parts) {
  PyObject* t = PyTuple_New((Py_ssize_t)parts.size());
  Py_ssize_t i = 0;
  for (PyObject* p : parts) {
    if (t) PyTuple_SET_ITEM(t, i++, p);
    else Py_DECREF(p);
  }
  if (!t) throw PythonError();
  return t;
}
PyObject* none() {
  Py_INCREF(Py_None);
  return Py_None;
}

using Args = PyObject* const*;

// (logits, targets, scale, return_stats)
PyObject* token_logp(Args a, Py_ssize_t na) {
  arguments(na, 4);
  const Tensor& x = tensor(a[0], "logits");
  const Rows r = rows(x, "logits");
  const int32_t k = kind(x, "logits");
  const int64_t* y = targets(a[1], r.n, x);
  const float scale = (float)number(a[2]);
  const bool with_stats = truth(a[3]);
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  const auto f32 = x.options().dtype(at::kFloat);
  Tensor logp = at::empty({r.n}, f32), stats;
  if (with_stats) stats = at::empty({r.n, 2}, f32);
  check(g_abi.token_logp(x.data_ptr(), k, r.n, r.v, r.ld, scale, y, logp.data_ptr<float>(),
                         with_stats ? stats.data_ptr<float>() : nullptr, stream_of(x)),
        "gmc_token_logp");
  if (!with_stats) return wrap(logp);
  return tuple_of({wrap(logp), wrap(stats)});
}

// (logits, targets, stats, dlogp, scale, out)
PyObject* token_logp_backward(Args a, Py_ssize_t na) {
  arguments(na, 6);
  const Tensor& x = tensor(a[0], "logits");
  const Rows r = rows(x, "logits");
  const int32_t k = kind(x, "logits");
  const int64_t* y = targets(a[1], r.n, x);
  const float* stats = floats(a[2], 2 * r.n, x, "stats");
  const float* g = floats(a[3], r.n, x, "dlogp");
  const float scale = (float)number(a[4]);
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  int64_t dld = 0;
  const Tensor out = gradient(a[5], x, r, &dld);
  check(g_abi.token_logp_backward(x.data_ptr(), k, r.n, r.v, r.ld, scale, y, stats, g, out.data_ptr(), dld, stream_of(x)),
        "gmc_token_logp_backward");
  if (a[5] != Py_None) written(out);
  return wrap(out);
}

gmc_loss_t handle(PyObject* o, const Tensor& x, PyObject* device) {
  void* h = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
  if (PyErr_Occurred()) throw PythonError();
  if (x.device().index() != integer(device)) fail(PyExc_TypeError, "logits", "must be on the TokenLoss's device");
  return static_cast<gmc_loss_t>(h);
}

// (handle, device index, logits, targets, old_logp, advantages, weights, ref_logp, clip_low,
// clip_high, kl, scale, grad, out)
PyObject* policy(Args a, Py_ssize_t na) {
  arguments(na, 14);
  const Tensor& x = tensor(a[2], "logits");
  gmc_loss_t h = handle(a[0], x, a[1]);
  const Rows r = rows(x, "logits");
  const int32_t k = kind(x, "logits");
  const int64_t* y = targets(a[3], r.n, x);
  const float* old_logp = floats(a[4], r.n, x, "old_logp");
  const float* adv = floats(a[5], r.n, x, "advantages");
  const float* w = floats(a[6], r.n, x, "weights");
  const float* ref = floats(a[7], r.n, x, "ref_logp");
  const float lo = (float)number(a[8]), hi = (float)number(a[9]), kl = (float)number(a[10]), scale = (float)number(a[11]);
  const bool grad = truth(a[12]);
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  int64_t dld = r.v;
  Tensor out;
  if (grad) out = gradient(a[13], x, r, &dld);
  const auto f32 = x.options().dtype(at::kFloat);
  const Tensor all = at::empty({2 * r.n + 1}, f32);  // one allocation: each one costs a microsecond
  const Tensor each = part(all, {r.n}, 0), logp = part(all, {r.n}, r.n), loss = part(all, {}, 2 * r.n);
  check(g_abi.policy_loss(h, x.data_ptr(), k, r.n, r.v, r.ld, scale, y, old_logp, ref, adv, w, lo, hi, kl,
                          loss.data_ptr<float>(), each.data_ptr<float>(), logp.data_ptr<float>(),
                          grad ? out.data_ptr() : nullptr, dld, stream_of(x)),
        "gmc_policy_loss");
  if (grad && a[13] != Py_None) written(out);
  return tuple_of({wrap(loss), wrap(each), wrap(logp), grad ? wrap(out) : none()});
}

// (handle, device index, logits, targets, offsets, beta, smoothing, ref_logp, weights, scale,
// grad, out)
PyObject* preference(Args a, Py_ssize_t na) {
  arguments(na, 12);
  const Tensor& x = tensor(a[2], "logits");
  gmc_loss_t h = handle(a[0], x, a[1]);
  const Rows r = rows(x, "logits");
  const int32_t k = kind(x, "logits");
  const int64_t* y = targets(a[3], r.n, x);
  const int64_t ends = tensor(a[4], "offsets").numel();
  if (ends % 2 != 1) fail(PyExc_ValueError, "offsets", "must have 2 * pairs + 1 elements");
  const int64_t pairs = ends / 2;
  const int64_t* offsets = vector<const int64_t>(a[4], ends, at::kLong, x, "offsets");
  const float beta = (float)number(a[5]), smoothing = (float)number(a[6]);
  const float* ref = floats(a[7], r.n, x, "ref_logp");
  const float* w = floats(a[8], pairs, x, "weights");
  const float scale = (float)number(a[9]);
  const bool grad = truth(a[10]);
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  int64_t dld = r.v;
  Tensor out;
  if (grad) out = gradient(a[11], x, r, &dld);
  const auto f32 = x.options().dtype(at::kFloat);
  const Tensor all = at::empty({r.n + 3 * pairs + 1}, f32);  // one allocation, as above
  const Tensor logp = part(all, {r.n}, 0), ratio = part(all, {2 * pairs}, r.n),
               each = part(all, {pairs}, r.n + 2 * pairs), loss = part(all, {}, r.n + 3 * pairs);
  check(g_abi.preference_loss(h, x.data_ptr(), k, r.n, r.v, r.ld, scale, y, offsets, pairs, ref, w, beta, smoothing,
                              loss.data_ptr<float>(), each.data_ptr<float>(), ratio.data_ptr<float>(),
                              logp.data_ptr<float>(), grad ? out.data_ptr() : nullptr, dld, stream_of(x)),
        "gmc_preference_loss");
  if (grad && a[11] != Py_None) written(out);
  return tuple_of({wrap(loss), wrap(each), wrap(ratio), wrap(logp), grad ? wrap(out) : none()});
}

// The distance between the workers' parts of one of dropout's tensors.
int64_t worker_stride(const Tensor& t, const Tensor& x, int64_t K, int64_t n, const char* name) {
  if (t.sizes() != x.sizes() || t.scalar_type() != x.scalar_type() || t.device() != x.device())
    fail(PyExc_TypeError, name, "must be a tensor of x's shape, dtype and device");
  if (t.is_contiguous()) return n;
  int64_t step = 1;
  for (int64_t d = t.dim() - 1; d > 0; --d) {
    if (t.size(d) > 1 && t.stride(d) != step) fail(PyExc_TypeError, name, "must have contiguous parts for each worker");
    step *= t.size(d);
  }
  if (K > 1 && t.stride(0) < n) fail(PyExc_TypeError, name, "must have parts that do not overlap");
  return K > 1 ? t.stride(0) : n;
}

// (x, p, seed, t, worker, site, residual, out)
PyObject* dropout(Args a, Py_ssize_t na) {
  arguments(na, 8);
  const Tensor& x = tensor(a[0], "x");
  if (x.dim() < 2) fail(PyExc_TypeError, "x", "must have the workers as its first dimension");
  const int32_t k = kind(x, "x");
  const double p = number(a[1]);
  const uint64_t seed = bits64(a[2]);
  const int64_t t = integer(a[3]), worker = integer(a[4]), site = integer(a[5]);
  const int64_t K = x.size(0), n = K ? x.numel() / K : 0, ldx = worker_stride(x, x, K, n, "x");
  const void* res = nullptr;
  int64_t ldr = 0;
  if (a[6] != Py_None) {
    const Tensor& r = tensor(a[6], "residual");
    ldr = worker_stride(r, x, K, n, "residual");
    res = r.data_ptr();
  }
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  const Tensor out = a[7] == Py_None ? empty_beside(x, K, n, ldx, 32) : tensor(a[7], "out");
  const int64_t ldo = worker_stride(out, x, K, n, "out");
  check(g_abi.dropout(x.data_ptr(), ldx, res, ldr, out.data_ptr(), ldo, k, worker, K, n, p, seed, t, site, stream_of(x)),
        "gmc_dropout");
  if (a[7] != Py_None) written(out);
  return wrap(out);
}

// The targets of n rows: (n,) or (n, given) int64, or None.
struct Given {
  const int64_t* y = nullptr;
  int32_t given = 0;
  std::vector<int64_t> shape;
};
Given given_of(PyObject* o, int64_t n, const Tensor& like) {
  Given g;
  if (o == Py_None) return g;
  const Tensor& t = tensor(o, "targets");
  if (t.dim() < 1 || t.dim() > 2 || t.size(0) != n) fail(PyExc_ValueError, "targets", "must be (n,) or (n, given)");
  const int64_t each = t.dim() == 1 ? 1 : t.size(1);
  if (each < 1 || each > 64) fail(PyExc_ValueError, "targets", "must be 1 to 64 a row");
  g.y = vector<const int64_t>(o, n * each, at::kLong, like, "targets");
  g.given = (int32_t)each;
  g.shape.assign(t.sizes().begin(), t.sizes().end());
  return g;
}

// (logits, targets, top, scale, return_stats)
PyObject* token_scores(Args a, Py_ssize_t na) {
  arguments(na, 5);
  const Tensor& x = tensor(a[0], "logits");
  const Rows r = rows(x, "logits");
  const int32_t k = kind(x, "logits");
  const Given g = given_of(a[1], r.n, x);
  const int64_t top = integer(a[2]);
  if (top < 0 || top > 64 || top > r.v) fail(PyExc_ValueError, "top", "must be 0 to 64, and at most the vocabulary");
  const float scale = (float)number(a[3]);
  const bool with_stats = truth(a[4]);
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  // one allocation for all floats, the numbers of 16 bytes a row first; the indices in one of their own: torch.save
  // takes no storage that holds two types
  const int64_t best_at = with_stats ? 4 * r.n : 0, logp_at = best_at + r.n * top, entropy_at = logp_at + r.n * g.given;
  const Tensor all = at::empty({entropy_at + r.n}, x.options().dtype(at::kFloat));
  Tensor logp, best, index, stats;
  const Tensor entropy = part(all, {r.n}, entropy_at);
  if (g.given) logp = part(all, g.shape, logp_at);
  if (top) best = part(all, {r.n, top}, best_at), index = at::empty({r.n, top}, x.options().dtype(at::kLong));
  if (with_stats) stats = part(all, {r.n, 4}, 0);
  check(g_abi.token_scores(x.data_ptr(), k, r.n, r.v, r.ld, scale, g.y, g.given, (int32_t)top,
                           g.given ? logp.data_ptr<float>() : nullptr, entropy.data_ptr<float>(),
                           top ? best.data_ptr<float>() : nullptr, top ? index.data_ptr<int64_t>() : nullptr,
                           with_stats ? stats.data_ptr<float>() : nullptr, stream_of(x)),
        "gmc_token_scores");
  return tuple_of({g.given ? wrap(logp) : none(), wrap(entropy), top ? wrap(best) : none(), top ? wrap(index) : none(),
                   with_stats ? wrap(stats) : none()});
}

// (logits, targets, stats, dlogp, dentropy, scale, out)
PyObject* token_scores_backward(Args a, Py_ssize_t na) {
  arguments(na, 7);
  const Tensor& x = tensor(a[0], "logits");
  const Rows r = rows(x, "logits");
  const int32_t k = kind(x, "logits");
  const Given g = given_of(a[1], r.n, x);
  const float* stats = floats(a[2], 4 * r.n, x, "stats");
  if (a[3] == Py_None && a[4] == Py_None) fail(PyExc_ValueError, "dlogp", "or dentropy must be given");
  if (!g.given && a[3] != Py_None) fail(PyExc_ValueError, "dlogp", "is that of targets: there are none");
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  const float* dlogp = floats(a[3], r.n * g.given, x, "dlogp");
  const float* dentropy = floats(a[4], r.n, x, "dentropy");
  const float scale = (float)number(a[5]);
  int64_t dld = 0;
  const Tensor out = gradient(a[6], x, r, &dld);
  check(g_abi.token_scores_backward(x.data_ptr(), k, r.n, r.v, r.ld, scale, g.y, g.given, stats, dlogp, dentropy,
                                    out.data_ptr(), dld, stream_of(x)),
        "gmc_token_scores_backward");
  if (a[6] != Py_None) written(out);
  return wrap(out);
}

// Strides of K matrices (one: a 2-D tensor), their rows contiguous.
struct Matrices {
  int64_t K, m, n, ldk, ld;
};
Matrices matrices(const Tensor& t, const char* name) {
  const int64_t d = t.dim();
  if (d != 2 && d != 3) fail(PyExc_TypeError, name, "must be a matrix, or the workers' matrices");
  Matrices s{d == 3 ? t.size(0) : 1, t.size(d - 2), t.size(d - 1), d == 3 ? t.stride(0) : 0, t.stride(d - 2)};
  if (s.n > 1 && t.stride(d - 1) != 1) fail(PyExc_TypeError, name, "must have contiguous rows");
  if (s.m <= 1) s.ld = s.n;
  if (s.K <= 1) s.ldk = s.m * s.ld;
  const bool apart = s.ld >= s.n && s.ldk >= (s.m - 1) * s.ld + s.n;  // a matrix after the other
  const bool in_turn = s.m > 1 && s.ldk >= s.n && s.ld >= (s.K - 1) * s.ldk + s.n;  // a row of each
  if (!apart && !in_turn) fail(PyExc_TypeError, name, "must have rows that do not overlap");
  return s;
}

// (x, steps, coefficients, scale, out)
PyObject* orthogonalize(Args a, Py_ssize_t na) {
  arguments(na, 5);
  const Tensor& x = tensor(a[0], "x");
  const int32_t k = kind(x, "x");
  const Matrices s = matrices(x, "x");
  const int64_t steps = integer(a[1]);
  if (steps < 1 || steps > 16) fail(PyExc_ValueError, "steps", "must be 1 to 16");
  float coef[48];
  PyObject* seq = PySequence_Fast(a[2], "coefficients must be (a, b, c), or one such triple for each step");
  if (!seq) throw PythonError();
  struct Release {
    PyObject* o;
    ~Release() { Py_DECREF(o); }
  } release{seq};
  const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq);
  bool single = false;  // three numbers (a row of an array is one too, by its methods, but has a length)
  if (count == 3 && PyObject_Size(PySequence_Fast_GET_ITEM(seq, 0)) < 0) {
    PyErr_Clear();
    single = true;
  }
  if (!single && count != steps) fail(PyExc_ValueError, "coefficients", "must be (a, b, c), or one such triple for each step");
  for (int64_t i = 0; i < steps; ++i) {
    PyObject* three = single ? (Py_INCREF(seq), seq)
                             : PySequence_Fast(PySequence_Fast_GET_ITEM(seq, i), "coefficients must hold triples");
    if (!three) throw PythonError();
    Release also{three};
    if (PySequence_Fast_GET_SIZE(three) != 3) fail(PyExc_ValueError, "coefficients", "must hold triples");
    for (int j = 0; j < 3; ++j) coef[3 * i + j] = (float)number(PySequence_Fast_GET_ITEM(three, j));
  }
  const float scale = (float)number(a[3]);
  const c10::cuda::OptionalCUDAGuard guard(x.device());
  Tensor out;
  Matrices o = s;
  if (a[4] == Py_None) {
    out = at::empty(x.sizes(), x.options());
    o.ld = s.n, o.ldk = s.m * s.n;
  } else {
    out = tensor(a[4], "out");
    if (out.sizes() != x.sizes() || out.scalar_type() != x.scalar_type() || out.device() != x.device())
      fail(PyExc_TypeError, "out", "must have x's shape, dtype and device");
    o = matrices(out, "out");
  }
  const int64_t bytes = g_abi.orthogonalize_workspace(k, s.K, s.m, s.n);
  if (bytes < 0) check(GMC_EINVAL, "gmc_orthogonalize");
  const Tensor work = at::empty({bytes}, x.options().dtype(at::kByte));
  check(g_abi.orthogonalize(x.data_ptr(), s.ldk, s.ld, out.data_ptr(), o.ldk, o.ld, k, s.K, s.m, s.n, (int32_t)steps, coef,
                            scale, work.data_ptr(), bytes, stream_of(x)),
        "gmc_orthogonalize");
  if (a[4] != Py_None) written(out);
  return wrap(out);
}

// (GMCError, the first five entry points' addresses in Abi's order)
PyObject* init(Args a, Py_ssize_t na) {
  arguments(na, 6);
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[1 + i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a NULL entry point");
      throw PythonError();
    }
  }
  g_abi.token_logp = reinterpret_cast<decltype(g_abi.token_logp)>(p[0]);
  g_abi.token_logp_backward = reinterpret_cast<decltype(g_abi.token_logp_backward)>(p[1]);
  g_abi.policy_loss = reinterpret_cast<decltype(g_abi.policy_loss)>(p[2]);
  g_abi.preference_loss = reinterpret_cast<decltype(g_abi.preference_loss)>(p[3]);
  g_abi.dropout = reinterpret_cast<decltype(g_abi.dropout)>(p[4]);
  Py_INCREF(a[0]);
  Py_XSETREF(g_error, a[0]);
  return none();
}

// (the other entry points' addresses in Abi's order)
PyObject* init_more(Args a, Py_ssize_t na) {
  arguments(na, 4);
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a NULL entry point");
      throw PythonError();
    }
  }
  g_abi.token_scores = reinterpret_cast<decltype(g_abi.token_scores)>(p[0]);
  g_abi.token_scores_backward = reinterpret_cast<decltype(g_abi.token_scores_backward)>(p[1]);
  g_abi.orthogonalize_workspace = reinterpret_cast<decltype(g_abi.orthogonalize_workspace)>(p[2]);
  g_abi.orthogonalize = reinterpret_cast<decltype(g_abi.orthogonalize)>(p[3]);
  return none();
}

// No C++ exception leaves the module: a Python error that is set, or torch's own.
template <PyObject* (*F)(Args, Py_ssize_t)>
PyObject* entry(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    if (F != init && !(g_error && (F == init_more || g_abi.orthogonalize))) {
      PyErr_SetString(PyExc_RuntimeError, "init() and init_more() come first");
      return nullptr;
    }
    return F(a, n);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

#define GMC_METHOD(f) \
  {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<f>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {GMC_METHOD(init),       GMC_METHOD(token_logp), GMC_METHOD(token_logp_backward),
                           GMC_METHOD(policy),     GMC_METHOD(preference), GMC_METHOD(dropout),
                           GMC_METHOD(init_more),  GMC_METHOD(token_scores), GMC_METHOD(token_scores_backward),
                           GMC_METHOD(orthogonalize),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_tokens", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tokens() { return PyModule_Create(&g_module); }
