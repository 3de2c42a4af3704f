// Python entry points of the passes as a native extension: argument checks, output allocation, the current stream and
// the call into libsmat, for the methods of binding.SmatPlan and for the operators around the pass.  It holds no state besides the plan handle and shape it
// is given; the Python form of the same checks (attribute look-ups, shape tuples, ctypes conversions) cost about 8 us a
// decoding step and 25 us a forward + backward, more than the kernels of a small problem.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <initializer_list>
#include <optional>
#include <string>
#include <vector>

#include "../../include/smat.h"

namespace {

struct Plan {
  PyObject_HEAD
  const smat_plan* handle;
  int64_t b, h, T, dk, dv, n, m;
  at::ScalarType dtype;
};

PyObject* smat_error = nullptr;   // binding.SmatError

bool fail_status(int code, const char* what) {
  if (code == SMAT_OK) return true;
  PyObject* e = PyObject_CallFunction(smat_error, "is", code, what);
  if (e) {
    PyErr_SetObject(smat_error, e);
    Py_DECREF(e);
  }
  return false;
}

std::string shape_text(at::IntArrayRef s) {
  std::string t = "(";
  for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + ")";
}

// The tensor behind `o`, checked: CUDA, dtype, contiguous, exactly this shape.
const at::Tensor* tensor(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor", name);
    return nullptr;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) {
    PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", name);
    return nullptr;
  }
  if (t.scalar_type() != dtype || t.sizes() != shape || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous CUDA tensor of %s and shape %s, got %s %s", name,
                 c10::toString(dtype), shape_text(shape).c_str(), c10::toString(t.scalar_type()),
                 shape_text(t.sizes()).c_str());
    return nullptr;
  }
  return &t;
}

// Memory that a call works in.  The passes and the decoding steps take what the device can reach, pinned memory of the host and strided views among
// it (as many bytes as the tensor has elements, from its first one on); `plain`: contiguous memory of the device alone.
bool workspace(PyObject* o, const char* name, void** ptr, size_t* bytes, bool plain) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor", name);
    return false;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (plain ? !t.is_cuda() || !t.is_contiguous() : !t.is_cuda() && !t.is_pinned()) {
    PyErr_Format(PyExc_ValueError, plain ? "%s: expected a contiguous CUDA tensor" : "%s: expected memory that the device can reach", name);
    return false;
  }
  *ptr = t.data_ptr();
  *bytes = (size_t)t.numel();
  return true;
}

bool stream(PyObject* o, void** st) {
  if (o == Py_None) {
    *st = c10::cuda::getCurrentCUDAStream().stream();
    return true;
  }
  PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
  if (!v) return false;
  *st = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

// The interpreter lock is released for a call into the library (a full launch queue may block it).  The library throws
// nothing; what can throw, the data pointers of tensors without storage among it, is asked for before.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
int unlocked(F call) {
  Unlocked lock;
  return call();
}

// Anything int() takes (a position kept as a float or as an array scalar among it).
bool token_index(PyObject* o, long long* t) {
  if (PyLong_CheckExact(o)) {
    *t = PyLong_AsLongLong(o);
    return !(*t == -1 && PyErr_Occurred());
  }
  PyObject* n = PyNumber_Long(o);
  if (!n) return false;
  *t = PyLong_AsLongLong(n);
  Py_DECREF(n);
  return !(*t == -1 && PyErr_Occurred());
}

bool arity(Py_ssize_t got, Py_ssize_t want, const char* name) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, got);
  return false;
}

// An output: the caller's tensor, or a new one like `like`.  A tensor handed in has the same element type, is contiguous
// and holds at least as many elements: another view of the same rows, or a larger buffer whose first part is written.
bool output(PyObject* o, const char* name, const at::Tensor& like, at::Tensor* out) {
  if (o == Py_None) {
    *out = at::empty_like(like);
    return true;
  }
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.scalar_type() == like.scalar_type() && t.numel() >= like.numel() && t.is_contiguous()) {
      *out = t;
      return true;
    }
  }
  PyErr_Format(PyExc_ValueError, "%s: expected a contiguous CUDA tensor of %s that holds shape %s", name,
               c10::toString(like.scalar_type()), shape_text(like.sizes()).c_str());
  return false;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

PyObject* wrap_all(std::initializer_list<at::Tensor> ts) {
  PyObject* tuple = PyTuple_New((Py_ssize_t)ts.size());
  if (!tuple) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) PyTuple_SET_ITEM(tuple, i++, wrap(t));
  return tuple;
}

// The exception in flight as the one torch raises for it (an exhausted device: torch.OutOfMemoryError).
PyObject* raise() {
  torch::translate_exception_to_python(std::current_exception());
  return nullptr;
}

// forward(kind, Q, K, V, log_a, O, workspace, stream, prof, type): kind 0 plain or routed, 1 gated, 2 normalised
PyObject* plan_forward(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 10, "forward")) return nullptr;
    const Plan& p = *reinterpret_cast<Plan*>(self);
    const long kind = PyLong_AsLong(a[0]);
    const int64_t sk[4] = {p.b, p.h, p.T, p.dk}, sv[4] = {p.b, p.h, p.T, p.dv};
    const at::Tensor *Q = tensor(a[1], "Q", p.dtype, sk), *K = Q ? tensor(a[2], "K", p.dtype, sk) : nullptr;
    const at::Tensor* V = K ? tensor(a[3], "V", p.dtype, sv) : nullptr;
    if (!V) return nullptr;
    const int64_t sg[2] = {p.b * p.h, p.T};
    const at::Tensor* la = kind == 1 ? tensor(a[4], "log_a", at::kFloat, sg) : nullptr;
    if (kind == 1 && !la) return nullptr;
    at::Tensor O;
    void *ws, *st;
    size_t bytes;
    if (kind == 0 && a[5] != Py_None && !tensor(a[5], "O", p.dtype, sv)) return nullptr;
    if (!output(a[5], "O", *V, &O) || !workspace(a[6], "workspace", &ws, &bytes, false) || !stream(a[7], &st)) return nullptr;
    const void *q = Q->data_ptr(), *k = K->data_ptr(), *v = V->data_ptr();
    void* o = O.data_ptr();
    int rc;
    const char* what;
    if (kind == 1) {
      what = "smat_forward_gated";
      const float* log_a = la->data_ptr<float>();
      rc = unlocked([&] { return smat_forward_gated(p.handle, q, k, v, log_a, o, ws, bytes, st); });
    } else if (kind == 2) {
      what = "smat_forward_normalized";
      rc = unlocked([&] { return smat_forward_normalized(p.handle, q, k, v, o, ws, bytes, st); });
    } else if (a[8] != Py_None || a[9] != Py_None) {
      const int64_t sp[2] = {p.b * p.h, p.n}, stp[2] = {p.b * p.h, p.m};
      const at::Tensor *prof = tensor(a[8], "prof", at::kInt, sp), *type = prof ? tensor(a[9], "type", at::kInt, stp) : nullptr;
      if (!type) return nullptr;
      what = "smat_forward_routed";
      const int32_t *cells = prof->data_ptr<int>(), *types = type->data_ptr<int>();
      rc = unlocked([&] { return smat_forward_routed(p.handle, q, k, v, o, cells, types, ws, bytes, st); });
    } else {
      what = "smat_forward";
      rc = unlocked([&] { return smat_forward(p.handle, q, k, v, o, ws, bytes, st); });
    }
    return fail_status(rc, what) ? wrap(O) : nullptr;
  } catch (...) {
    return raise();
  }
}

// backward(kind, Q, K, V, log_a, O, dO, dQ, dK, dV, dlog_a, workspace, stream, prof, type)
PyObject* plan_backward(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 15, "backward")) return nullptr;
    const Plan& p = *reinterpret_cast<Plan*>(self);
    const long kind = PyLong_AsLong(a[0]);
    const int64_t sk[4] = {p.b, p.h, p.T, p.dk}, sv[4] = {p.b, p.h, p.T, p.dv};
    const at::Tensor *Q = tensor(a[1], "Q", p.dtype, sk), *K = Q ? tensor(a[2], "K", p.dtype, sk) : nullptr;
    const at::Tensor* V = K ? tensor(a[3], "V", p.dtype, sv) : nullptr;
    const at::Tensor* O = V && kind == 2 ? tensor(a[5], "O", p.dtype, sv) : V;
    const at::Tensor* dO = O ? tensor(a[6], "dO", p.dtype, sv) : nullptr;
    if (!dO) return nullptr;
    const int64_t sg[2] = {p.b * p.h, p.T};
    const at::Tensor* la = kind == 1 ? tensor(a[4], "log_a", at::kFloat, sg) : nullptr;
    if (kind == 1 && !la) return nullptr;
    at::Tensor dQ, dK, dV, dla;
    void *ws, *st;
    size_t bytes;
    if (!output(a[7], "dQ", *Q, &dQ) || !output(a[8], "dK", *K, &dK) || !output(a[9], "dV", *V, &dV) ||
        (la && !output(a[10], "dlog_a", *la, &dla)) || !workspace(a[11], "workspace", &ws, &bytes, false) || !stream(a[12], &st))
      return nullptr;
    const void *q = Q->data_ptr(), *k = K->data_ptr(), *v = V->data_ptr(), *go = dO->data_ptr();
    void *gq = dQ.data_ptr(), *gk = dK.data_ptr(), *gv = dV.data_ptr();
    int rc;
    const char* what;
    if (kind == 1) {
      what = "smat_backward_gated";
      const float* log_a = la->data_ptr<float>();
      float* glog_a = dla.data_ptr<float>();
      rc = unlocked([&] { return smat_backward_gated(p.handle, q, k, v, log_a, go, gq, gk, gv, glog_a, ws, bytes, st); });
    } else if (kind == 2) {
      what = "smat_backward_normalized";
      const void* o = O->data_ptr();
      rc = unlocked([&] { return smat_backward_normalized(p.handle, q, k, v, o, go, gq, gk, gv, ws, bytes, st); });
    } else if (a[13] != Py_None || a[14] != Py_None) {
      const int64_t sp[2] = {p.b * p.h, p.n}, stp[2] = {p.b * p.h, p.m};
      const at::Tensor *prof = tensor(a[13], "prof", at::kInt, sp), *type = prof ? tensor(a[14], "type", at::kInt, stp) : nullptr;
      if (!type) return nullptr;
      what = "smat_backward_routed";
      const int32_t *cells = prof->data_ptr<int>(), *types = type->data_ptr<int>();
      rc = unlocked([&] { return smat_backward_routed(p.handle, q, k, v, go, gq, gk, gv, cells, types, ws, bytes, st); });
    } else {
      what = "smat_backward";
      rc = unlocked([&] { return smat_backward(p.handle, q, k, v, go, gq, gk, gv, ws, bytes, st); });
    }
    if (!fail_status(rc, what)) return nullptr;
    return la ? wrap_all({dQ, dK, dV, dla}) : wrap_all({dQ, dK, dV});
  } catch (...) {
    return raise();
  }
}

// decode_step(q, k, v, log_a_t, t, cache, o, stream, packed): log_a_t None for the ungated step; packed: `cache` is a packed one
PyObject* plan_decode_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 9, "decode_step")) return nullptr;
    const bool packed = a[8] == Py_True;
    const Plan& p = *reinterpret_cast<Plan*>(self);
    const int64_t sk[3] = {p.b, p.h, p.dk}, sv[3] = {p.b, p.h, p.dv};
    const at::Tensor *q = tensor(a[0], "q", p.dtype, sk), *k = q ? tensor(a[1], "k", p.dtype, sk) : nullptr;
    const at::Tensor* v = k ? tensor(a[2], "v", p.dtype, sv) : nullptr;
    if (!v) return nullptr;
    const at::Tensor* la = nullptr;
    if (a[3] != Py_None) {
      if (!THPVariable_Check(a[3])) {
        PyErr_SetString(PyExc_ValueError, "log_a_t: expected a tensor");
        return nullptr;
      }
      la = &THPVariable_Unpack(a[3]);
      if (!la->is_cuda() || !la->is_contiguous() || la->scalar_type() != at::kFloat || la->numel() != p.b * p.h) {
        PyErr_Format(PyExc_ValueError, "log_a_t: expected a contiguous CUDA fp32 tensor of %lld log-gates", (long long)(p.b * p.h));
        return nullptr;
      }
    }
    long long t;
    if (!token_index(a[4], &t)) return nullptr;
    at::Tensor o;
    void *cache, *st;
    size_t bytes;
    if (!workspace(a[5], "cache", &cache, &bytes, packed) || !output(a[6], "o", *v, &o) || !stream(a[7], &st)) return nullptr;
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
    void* op = o.data_ptr();
    const float* log_a = la ? la->data_ptr<float>() : nullptr;
    const int rc = unlocked([&] {
      if (packed) return smat_decode_step_packed(p.handle, qp, kp, vp, log_a, t, op, cache, bytes, st);
      return la ? smat_decode_step_gated(p.handle, qp, kp, vp, log_a, t, op, cache, bytes, st)
                : smat_decode_step(p.handle, qp, kp, vp, t, op, cache, bytes, st);
    });
    const char* what = packed ? "smat_decode_step_packed" : la ? "smat_decode_step_gated" : "smat_decode_step";
    return fail_status(rc, what) ? wrap(o) : nullptr;
  } catch (...) {
    return raise();
  }
}

// ---- operators around the pass -------------------------------------------------------------------------------------------
// Their tensors may have any strides as long as the last dimension is contiguous.  They run on the tensors' own device, which
// need not be the current one, and on its current stream unless one is given.

// The tensor behind `o`, checked: CUDA, this element type and device, contiguous features.  `shape` (empty: any).
const at::Tensor* rows_tensor(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape, const at::Tensor* like) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor", name);
    return nullptr;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.layout() != at::kStrided) {
    PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", name);
    return nullptr;
  }
  const bool features = t.dim() >= 1 && (t.stride(-1) == 1 || t.size(-1) == 1);
  if (t.scalar_type() != dtype || (like && t.sizes() != shape) || !features || t.numel() == 0) {
    const std::string want = like ? " and shape " + shape_text(shape) : std::string();
    PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor of %s%s with contiguous features, got %s %s", name,
                 c10::toString(dtype), want.c_str(), c10::toString(t.scalar_type()), shape_text(t.sizes()).c_str());
    return nullptr;
  }
  if (like && t.device() != like->device()) {
    PyErr_Format(PyExc_ValueError, "%s: on another device than the first tensor", name);
    return nullptr;
  }
  return &t;
}

// A contiguous array of exactly this shape on the same device (states, weights).
const at::Tensor* array_tensor(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape, const at::Tensor& like) {
  const at::Tensor* t = rows_tensor(o, name, dtype, shape, &like);
  if (t && !t->is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous tensor", name);
    return nullptr;
  }
  return t;
}

bool float_type(PyObject* o, const char* name, at::ScalarType* dtype) {
  if (THPVariable_Check(o)) {
    *dtype = THPVariable_Unpack(o).scalar_type();
    if (*dtype == at::kFloat || *dtype == at::kBFloat16) return true;
  }
  PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor of Float or BFloat16", name);
  return false;
}
smat_dtype smat_type(at::ScalarType t) { return t == at::kBFloat16 ? SMAT_BF16 : SMAT_F32; }

// Where a call runs: on the tensors' device, and on its current stream or on the one that is given.  A given stream is the
// current one while the call takes memory: what it takes belongs to that stream, so that a workspace is free again behind the kernels
// that use it, and no block is written while the caller's stream still uses it for what it held before.
struct Running {
  c10::cuda::CUDAGuard device;
  c10::cuda::OptionalCUDAStreamGuard given;
  std::optional<c10::cuda::CUDAStream> caller;      // the caller's stream, where it is another
  void* st = nullptr;

  explicit Running(const at::Tensor& t) : device(t.device()) {}
  bool on(PyObject* o) {
    if (!stream(o, &st)) return false;
    if (o == Py_None) return true;
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream();
    if (st == current.stream()) return true;
    caller = current;
    given.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), current.device_index()));
    return true;
  }
  // A new contiguous tensor.  (Straight from the allocator's front end: two outputs through the dispatcher cost a single-token call
  // 1 us of 5.)
  at::Tensor fresh(at::IntArrayRef shape, at::ScalarType dtype) const {
    return at::Tensor(at::detail::empty_cuda(shape, dtype, device.current_device(), c10::nullopt));
  }
  // ... that the caller gets, and may give back while its own stream reads it
  at::Tensor output(at::IntArrayRef shape, at::ScalarType dtype) const {
    at::Tensor t = fresh(shape, dtype);
    if (caller) t.record_stream(caller->unwrap());
    return t;
  }
};

// An output: the caller's tensor (this shape, any strides), or a new contiguous one.
bool rows_output(PyObject* o, const char* name, const at::Tensor& like, const Running& run, at::Tensor* out) {
  if (o == Py_None) {
    *out = run.output(like.sizes(), like.scalar_type());
    return true;
  }
  const at::Tensor* t = rows_tensor(o, name, like.scalar_type(), like.sizes(), &like);
  if (t) *out = *t;
  return t != nullptr;
}
bool array_output(PyObject* o, const char* name, at::IntArrayRef shape, const at::Tensor& like, const Running& run, at::Tensor* out) {
  if (o == Py_None) {
    *out = run.output(shape, at::kFloat);
    return true;
  }
  const at::Tensor* t = array_tensor(o, name, at::kFloat, shape, like);
  if (t) *out = *t;
  return t != nullptr;
}

// Which dimensions of a tensor are the batch, the heads (or groups) and the tokens; -1: there is none, it counts as one.
struct Axes {
  int batch, head, token;
};
smat_rows rows_of(const at::Tensor& t, const Axes& x) {
  const auto step = [&](int d) { return d < 0 ? (int64_t)0 : t.stride(d); };
  return smat_rows{t.data_ptr(), step(x.batch), step(x.head), step(x.token)};
}
int64_t size_of(const at::Tensor& t, int d) { return d < 0 ? 1 : t.size(d); }

bool fits_int(int64_t v, const char* name) {
  if (v <= INT32_MAX) return true;
  PyErr_Format(PyExc_ValueError, "%s: a dimension is too large", name);
  return false;
}

// rotary(Q, K, frequencies, positions, first, interleaved, scale, adjoint, Q_out, K_out, stream)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 11, "rotary")) return nullptr;
    at::ScalarType dtype;
    if (!float_type(a[0], "Q", &dtype)) return nullptr;
    const at::Tensor* Q = rows_tensor(a[0], "Q", dtype, {}, nullptr);
    if (!Q) return nullptr;
    if (Q->dim() != 3 && Q->dim() != 4) {
      PyErr_SetString(PyExc_ValueError, "Q: expected [batch, heads, T, d] or [batch, heads, d]");
      return nullptr;
    }
    const Axes axes{0, 1, Q->dim() == 4 ? 2 : -1};
    const int64_t batch = Q->size(0), T = size_of(*Q, axes.token);
    const at::Tensor* K = nullptr;
    if (a[1] != Py_None) {
      std::vector<int64_t> shape(Q->sizes().begin(), Q->sizes().end());
      if (THPVariable_Check(a[1]) && THPVariable_Unpack(a[1]).dim() == Q->dim()) shape[1] = THPVariable_Unpack(a[1]).size(1);
      K = rows_tensor(a[1], "K", dtype, shape, Q);
      if (!K) return nullptr;
    }
    if (!THPVariable_Check(a[2]) || THPVariable_Unpack(a[2]).dim() != 1) {
      PyErr_SetString(PyExc_ValueError, "frequencies: expected a CUDA fp64 tensor [rotated / 2]");
      return nullptr;
    }
    const at::Tensor* F = array_tensor(a[2], "frequencies", at::kDouble, THPVariable_Unpack(a[2]).sizes(), *Q);
    if (!F) return nullptr;
    smat_rotary_problem p{};
    if (a[3] != Py_None) {
      if (!THPVariable_Check(a[3])) {
        PyErr_SetString(PyExc_ValueError, "positions: expected a tensor");
        return nullptr;
      }
      const at::Tensor& P = THPVariable_Unpack(a[3]);
      const bool one = P.dim() == 1 && P.size(0) == T;                                            // the same for every sequence
      const bool rows = P.dim() == 2 && P.size(0) == batch && P.size(1) == T;
      const bool column = axes.token < 0 && P.dim() == 1 && P.size(0) == batch;                   // one token of each sequence
      if (!P.is_cuda() || P.device() != Q->device() || P.scalar_type() != at::kLong || !(one || rows || column) ||
          (!column && T > 1 && P.stride(-1) != 1)) {
        PyErr_Format(PyExc_ValueError, "positions: expected a CUDA int64 tensor of shape (%lld) or (%lld, %lld) with contiguous tokens",
                     (long long)T, (long long)batch, (long long)T);
        return nullptr;
      }
      p.positions = P.data_ptr<int64_t>();
      p.positions_batch = column || rows ? P.stride(0) : 0;
    }
    long long first;
    if (!token_index(a[4], &first)) return nullptr;
    const int interleaved = PyObject_IsTrue(a[5]), adjoint = PyObject_IsTrue(a[7]);
    const double scale = PyFloat_AsDouble(a[6]);
    if (interleaved < 0 || adjoint < 0 || (scale == -1.0 && PyErr_Occurred())) return nullptr;
    if (!fits_int(batch, "Q") || !fits_int(Q->size(1), "Q") || (K && !fits_int(K->size(1), "K")) || !fits_int(Q->size(-1), "Q") ||
        !fits_int(F->size(0) * 2, "frequencies"))
      return nullptr;
    Running run(*Q);
    at::Tensor Qo, Ko;
    if (!run.on(a[10]) || !rows_output(a[8], "Q_out", *Q, run, &Qo) || (K && !rows_output(a[9], "K_out", *K, run, &Ko))) return nullptr;
    p.batch = (int)batch;
    p.q_heads = (int)Q->size(1);
    p.k_heads = K ? (int)K->size(1) : 0;
    p.T = T;
    p.d = (int)Q->size(-1);
    p.rotated = (int)F->size(0) * 2;
    p.interleaved = interleaved;
    p.adjoint = adjoint;
    p.scale = (float)scale;
    p.dtype = smat_type(dtype);
    p.frequencies = F->data_ptr<double>();
    p.first = first;
    const smat_rows q = rows_of(*Q, axes), qo = rows_of(Qo, axes);
    smat_rows k{}, ko{};
    if (K) { k = rows_of(*K, axes); ko = rows_of(Ko, axes); }
    const int rc = unlocked([&] { return smat_rotary(&p, &q, K ? &k : nullptr, &qo, K ? &ko : nullptr, run.st); });
    if (!fail_status(rc, "smat_rotary")) return nullptr;
    return K ? wrap_all({Qo, Ko}) : wrap(Qo);
  } catch (...) {
    return raise();
  }
}

// Shapes that the norm takes: [batch, T, groups, width], [batch, T, width], [rows, width]; with a weight of every group also
// [batch, groups, width].
bool norm_problem(const at::Tensor& x, PyObject* weight, PyObject* scale, PyObject* eps, PyObject* sigmoid, Axes* axes,
                  smat_norm_problem* p, const at::Tensor** W, const at::Tensor** S) {
  const int dim = (int)x.dim();
  const bool grouped = THPVariable_Check(weight) && THPVariable_Unpack(weight).dim() == 2;
  if (dim < 2 || dim > 4 || (grouped && dim == 2)) {
    PyErr_SetString(PyExc_ValueError, "rows: expected [batch, T, groups, width], [batch, T, width] or [rows, width]");
    return false;
  }
  *axes = dim == 4 ? Axes{0, 2, 1} : dim == 2 ? Axes{0, -1, -1} : grouped ? Axes{0, 1, -1} : Axes{0, -1, 1};
  const int64_t width = x.size(-1), groups = size_of(x, axes->head);
  const int64_t of_group[2] = {groups, width}, of_all[1] = {width};
  *W = array_tensor(weight, "weight", at::kFloat, grouped ? at::IntArrayRef(of_group) : at::IntArrayRef(of_all), x);
  *S = *W && scale != Py_None ? array_tensor(scale, "scale", at::kFloat, of_all, x) : nullptr;
  if (!*W || (scale != Py_None && !*S)) return false;
  const double e = PyFloat_AsDouble(eps);
  if (e == -1.0 && PyErr_Occurred()) return false;
  if (!fits_int(x.size(0), "rows") || !fits_int(groups, "rows") || !fits_int(width, "rows")) return false;
  p->batch = (int)x.size(0);
  p->T = size_of(x, axes->token);
  p->groups = (int)groups;
  p->width = (int)width;
  p->dtype = smat_type(x.scalar_type());
  p->activation = sigmoid == Py_True ? SMAT_ACT_SIGMOID : SMAT_ACT_SILU;
  p->eps = (float)e;
  p->weight = (*W)->data_ptr<float>();
  p->weight_group = grouped ? width : 0;
  p->scale = *S ? (*S)->data_ptr<float>() : nullptr;
  return true;
}

// norm_forward(X, weight, eps, residual, scale, gate, sigmoid, Y, H, stream)
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 10, "norm_forward")) return nullptr;
    at::ScalarType dtype;
    if (!float_type(a[0], "X", &dtype)) return nullptr;
    const at::Tensor* X = rows_tensor(a[0], "X", dtype, {}, nullptr);
    Axes axes;
    smat_norm_problem p{};
    const at::Tensor *W, *S;
    if (!X || !norm_problem(*X, a[1], a[4], a[2], a[6], &axes, &p, &W, &S)) return nullptr;
    const at::Tensor *R = nullptr, *G = nullptr;
    if (a[3] != Py_None && !(R = rows_tensor(a[3], "residual", dtype, X->sizes(), X))) return nullptr;
    if (a[5] != Py_None && !(G = rows_tensor(a[5], "gate", dtype, X->sizes(), X))) return nullptr;
    const bool keeps = R || S || a[8] != Py_None;
    Running run(*X);
    at::Tensor Y, H;
    if (!run.on(a[9]) || !rows_output(a[7], "Y", *X, run, &Y) || (keeps && !rows_output(a[8], "H", *X, run, &H))) return nullptr;
    const smat_rows x = rows_of(*X, axes), y = rows_of(Y, axes);
    smat_rows r{}, g{}, h{};
    if (R) r = rows_of(*R, axes);
    if (G) g = rows_of(*G, axes);
    if (keeps) h = rows_of(H, axes);
    const int rc = unlocked([&] { return smat_norm_forward(&p, &x, R ? &r : nullptr, G ? &g : nullptr, &y, keeps ? &h : nullptr, run.st); });
    if (!fail_status(rc, "smat_norm_forward")) return nullptr;
    return keeps ? wrap_all({Y, H}) : wrap(Y);
  } catch (...) {
    return raise();
  }
}

PyObject* wrap_or_none(const at::Tensor& t) {
  if (t.defined()) return wrap(t);
  Py_RETURN_NONE;
}

// norm_backward(dY, H, weight, eps, gate, sigmoid, dH, X, scale, dH_out, dX, dgate, workspace, stream)
// -> (dH, dX, dweight, dscale, dgate)
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 14, "norm_backward")) return nullptr;
    at::ScalarType dtype;
    if (!float_type(a[1], "H", &dtype)) return nullptr;
    const at::Tensor* H = rows_tensor(a[1], "H", dtype, {}, nullptr);
    Axes axes;
    smat_norm_problem p{};
    const at::Tensor *W, *S;
    if (!H || !norm_problem(*H, a[2], a[8], a[3], a[5], &axes, &p, &W, &S)) return nullptr;
    const at::Tensor *dY = rows_tensor(a[0], "dY", dtype, H->sizes(), H), *G = nullptr, *dI = nullptr, *X = nullptr;
    if (!dY || (a[4] != Py_None && !(G = rows_tensor(a[4], "gate", dtype, H->sizes(), H))) ||
        (a[6] != Py_None && !(dI = rows_tensor(a[6], "dH", dtype, H->sizes(), H))) ||
        (S && !(X = rows_tensor(a[7], "X", dtype, H->sizes(), H))))
      return nullptr;
    Running run(*H);
    at::Tensor dH, dX, dG, dW, dS, own;
    void* ws = nullptr;
    size_t bytes = smat_norm_workspace_bytes(&p);
    if (!run.on(a[13]) || !rows_output(a[9], "dH_out", *H, run, &dH) || (S && !rows_output(a[10], "dX", *H, run, &dX)) ||
        (G && !rows_output(a[11], "dgate", *H, run, &dG)))
      return nullptr;
    dW = run.output(W->sizes(), at::kFloat);
    if (S) dS = run.output(S->sizes(), at::kFloat);
    if (a[12] == Py_None) {
      own = run.fresh({(int64_t)bytes}, at::kByte);
      ws = own.data_ptr();
    } else if (!workspace(a[12], "workspace", &ws, &bytes, true)) {
      return nullptr;
    } else if (THPVariable_Unpack(a[12]).device() != H->device()) {
      PyErr_SetString(PyExc_ValueError, "workspace: on another device than H");
      return nullptr;
    }
    const smat_rows dy = rows_of(*dY, axes), h = rows_of(*H, axes), dh = rows_of(dH, axes);
    smat_rows g{}, dg{}, di{}, x{}, dx{};
    if (G) { g = rows_of(*G, axes); dg = rows_of(dG, axes); }
    if (dI) di = rows_of(*dI, axes);
    if (S) { x = rows_of(*X, axes); dx = rows_of(dX, axes); }
    float *dw = dW.data_ptr<float>(), *ds = S ? dS.data_ptr<float>() : nullptr;
    const int rc = unlocked([&] {
      return smat_norm_backward(&p, &dy, &h, G ? &g : nullptr, S ? &x : nullptr, dI ? &di : nullptr, &dh, S ? &dx : nullptr,
                                G ? &dg : nullptr, dw, ds, ws, bytes, run.st);
    });
    if (!fail_status(rc, "smat_norm_backward")) return nullptr;
    PyObject* tuple = PyTuple_New(5);
    if (!tuple) return nullptr;
    PyTuple_SET_ITEM(tuple, 0, wrap(dH));
    PyTuple_SET_ITEM(tuple, 1, wrap(S ? dX : dH));
    PyTuple_SET_ITEM(tuple, 2, wrap(dW));
    PyTuple_SET_ITEM(tuple, 3, wrap_or_none(dS));
    PyTuple_SET_ITEM(tuple, 4, wrap_or_none(dG));
    return tuple;
  } catch (...) {
    return raise();
  }
}

// x, h and their gradients [batch, T, channels], or [batch, channels] for one token.
bool recurrence_problem(const at::Tensor& x, at::ScalarType gates, Axes* axes, smat_recurrence_problem* p) {
  if ((x.dim() != 2 && x.dim() != 3) || !fits_int(x.size(0), "rows") || !fits_int(x.size(-1), "rows")) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "rows: expected [batch, T, channels] or [batch, channels]");
    return false;
  }
  *axes = Axes{0, -1, x.dim() == 3 ? 1 : -1};
  p->batch = (int)x.size(0);
  p->T = size_of(x, axes->token);
  p->channels = (int)x.size(-1);
  p->dtype = smat_type(x.scalar_type());
  p->gate_dtype = smat_type(gates);
  return true;
}

// recurrence_forward(X, log_a, h0, H, hT, stream) -> (H, hT)
PyObject* recurrence_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 6, "recurrence_forward")) return nullptr;
    at::ScalarType dtype, gates;
    if (!float_type(a[0], "X", &dtype) || !float_type(a[1], "log_a", &gates)) return nullptr;
    const at::Tensor* X = rows_tensor(a[0], "X", dtype, {}, nullptr);
    const at::Tensor* A = X ? rows_tensor(a[1], "log_a", gates, X->sizes(), X) : nullptr;
    Axes axes;
    smat_recurrence_problem p{};
    if (!A || !recurrence_problem(*X, gates, &axes, &p)) return nullptr;
    const int64_t state[2] = {p.batch, p.channels};
    const at::Tensor* h0 = nullptr;
    if (a[2] != Py_None && !(h0 = array_tensor(a[2], "h0", at::kFloat, state, *X))) return nullptr;
    Running run(*X);
    at::Tensor H, hT;
    if (!run.on(a[5]) || !rows_output(a[3], "H", *X, run, &H) || !array_output(a[4], "hT", state, *X, run, &hT)) return nullptr;
    const smat_rows x = rows_of(*X, axes), la = rows_of(*A, axes), h = rows_of(H, axes);
    const float* from = h0 ? h0->data_ptr<float>() : nullptr;
    float* to = hT.data_ptr<float>();
    const int rc = unlocked([&] { return smat_recurrence_forward(&p, &x, &la, from, &h, to, run.st); });
    return fail_status(rc, "smat_recurrence_forward") ? wrap_all({H, hT}) : nullptr;
  } catch (...) {
    return raise();
  }
}

// recurrence_backward(log_a, H, dH, h0, dhT, dX, dlog_a, dh0, stream) -> (dX, dlog_a, dh0)
PyObject* recurrence_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 9, "recurrence_backward")) return nullptr;
    at::ScalarType dtype, gates;
    if (!float_type(a[1], "H", &dtype) || !float_type(a[0], "log_a", &gates)) return nullptr;
    const at::Tensor* H = rows_tensor(a[1], "H", dtype, {}, nullptr);
    const at::Tensor* A = H ? rows_tensor(a[0], "log_a", gates, H->sizes(), H) : nullptr;
    const at::Tensor* dH = A ? rows_tensor(a[2], "dH", dtype, H->sizes(), H) : nullptr;
    Axes axes;
    smat_recurrence_problem p{};
    if (!dH || !recurrence_problem(*H, gates, &axes, &p)) return nullptr;
    const int64_t state[2] = {p.batch, p.channels};
    const at::Tensor *h0 = nullptr, *dhT = nullptr;
    if ((a[3] != Py_None && !(h0 = array_tensor(a[3], "h0", at::kFloat, state, *H))) ||
        (a[4] != Py_None && !(dhT = array_tensor(a[4], "dhT", at::kFloat, state, *H))))
      return nullptr;
    Running run(*H);
    at::Tensor dX, dA, dh0;
    if (!run.on(a[8]) || !rows_output(a[5], "dX", *H, run, &dX) || !rows_output(a[6], "dlog_a", *A, run, &dA) ||
        !array_output(a[7], "dh0", state, *H, run, &dh0))
      return nullptr;
    const smat_rows la = rows_of(*A, axes), h = rows_of(*H, axes), dh = rows_of(*dH, axes), dx = rows_of(dX, axes), da = rows_of(dA, axes);
    const float *start = h0 ? h0->data_ptr<float>() : nullptr, *from = dhT ? dhT->data_ptr<float>() : nullptr;
    float* to = dh0.data_ptr<float>();
    const int rc = unlocked([&] { return smat_recurrence_backward(&p, &la, &h, &dh, start, from, &dx, &da, to, run.st); });
    return fail_status(rc, "smat_recurrence_backward") ? wrap_all({dX, dA, dh0}) : nullptr;
  } catch (...) {
    return raise();
  }
}

// repack(cache, packed, stream, packs): smat_decode_pack, or smat_decode_unpack
PyObject* plan_repack(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    if (!arity(n, 4, "repack")) return nullptr;
    const Plan& p = *reinterpret_cast<Plan*>(self);
    void *cache, *packed, *st;
    size_t bytes, packed_bytes;
    if (!workspace(a[0], "cache", &cache, &bytes, true) || !workspace(a[1], "packed", &packed, &packed_bytes, true) || !stream(a[2], &st)) return nullptr;
    const bool packs = a[3] == Py_True;
    const int rc = unlocked([&] {
      return packs ? smat_decode_pack(p.handle, cache, bytes, packed, packed_bytes, st)
                   : smat_decode_unpack(p.handle, packed, packed_bytes, cache, bytes, st);
    });
    if (!fail_status(rc, packs ? "smat_decode_pack" : "smat_decode_unpack")) return nullptr;
    Py_RETURN_NONE;
  } catch (...) {
    return raise();
  }
}

// Plan(handle, batch, heads, T, d_k, d_v, bf16)
PyObject* plan_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long handle;
  long long b, h, T, dk, dv;
  int bf16;
  if (!PyArg_ParseTuple(args, "KLLLLLi", &handle, &b, &h, &T, &dk, &dv, &bf16)) return nullptr;
  smat_geometry g;
  const smat_plan* plan = reinterpret_cast<const smat_plan*>(handle);
  if (!fail_status(smat_get_geometry(plan, &g), "smat_get_geometry")) return nullptr;
  Plan* p = reinterpret_cast<Plan*>(type->tp_alloc(type, 0));
  if (!p) return nullptr;
  p->handle = plan;
  p->b = b; p->h = h; p->T = T; p->dk = dk; p->dv = dv; p->n = g.n; p->m = g.m;
  p->dtype = bf16 ? at::kBFloat16 : at::kFloat;
  return reinterpret_cast<PyObject*>(p);
}

PyMethodDef plan_methods[] = {
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(plan_forward)), METH_FASTCALL, nullptr},
    {"backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(plan_backward)), METH_FASTCALL, nullptr},
    {"decode_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(plan_decode_step)), METH_FASTCALL, nullptr},
    {"repack", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(plan_repack)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject plan_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XSETREF(smat_error, cls);
  Py_RETURN_NONE;
}

#define FASTCALL(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr
PyMethodDef module_methods[] = {{"set_error", set_error, METH_O, nullptr},
                                {"rotary", FASTCALL(rotary)},
                                {"norm_forward", FASTCALL(norm_forward)},
                                {"norm_backward", FASTCALL(norm_backward)},
                                {"recurrence_forward", FASTCALL(recurrence_forward)},
                                {"recurrence_backward", FASTCALL(recurrence_backward)},
                                {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_smat_torch", nullptr, -1, module_methods};

}  // namespace

PyMODINIT_FUNC PyInit__smat_torch(void) {
  plan_type.tp_name = "_smat_torch.Plan";
  plan_type.tp_basicsize = sizeof(Plan);
  plan_type.tp_flags = Py_TPFLAGS_DEFAULT;
  plan_type.tp_new = plan_new;
  plan_type.tp_methods = plan_methods;
  if (PyType_Ready(&plan_type) < 0) return nullptr;
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  Py_INCREF(&plan_type);
  if (PyModule_AddObject(m, "Plan", reinterpret_cast<PyObject*>(&plan_type)) < 0) {
    Py_DECREF(&plan_type);
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
