// The single calls of the Python binding in native code: arguments are read from the tensors directly and handed to the C
// ABI.  A few-token forward keeps the GPU busy for 4 us; reading its arguments in Python and marshalling them through ctypes
// took about 10 us, so the host was what such a call waited for.
//
// Checks and conversions are those of a plain ctypes call: matrices are 2-d with unit column stride (AssertionError), storage is
// bf16 or fp32 (TypeError), integers wrap to 64 bits, None is a null pointer.  Every function returns the status of
// the call; the interpreter lock is released while the library runs.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/flop.h"

namespace {

struct Stop {};   // a Python exception is set

const at::Tensor* tensor(PyObject* o) {   // nullptr for None
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a torch.Tensor, got %s", Py_TYPE(o)->tp_name);
    throw Stop{};
  }
  return &THPVariable_Unpack(o);
}
const at::Tensor& required(PyObject* o) {
  const at::Tensor* t = tensor(o);
  if (!t) { PyErr_SetString(PyExc_AttributeError, "'NoneType' object has no attribute 'shape'"); throw Stop{}; }
  return *t;
}
template <typename T = void> T* ptr(PyObject* o) {
  const at::Tensor* t = tensor(o);
  return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}

struct Mat { void* p = nullptr; int64_t ld = 0, rows = 0, cols = 0; };
int storage(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return FLOP_BF16;
  if (t.scalar_type() == at::kFloat) return FLOP_F32;
  PyErr_Format(PyExc_TypeError, "unsupported dtype %s", at::toString(t.scalar_type()));
  throw Stop{};
}
Mat matrix(PyObject* o) {
  const at::Tensor& t = required(o);
  if (t.dim() != 2 || t.stride(1) != 1) {
    PyErr_SetString(PyExc_AssertionError, "matrices must be row-major with unit column stride");
    throw Stop{};
  }
  Mat m;
  m.p = t.data_ptr();
  m.rows = t.size(0); m.cols = t.size(1);
  m.ld = m.rows > 1 ? t.stride(0) : std::max(t.stride(0), m.cols);
  return m;
}
Mat optional_matrix(PyObject* o) { return o == Py_None ? Mat{} : matrix(o); }

int64_t integer(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Stop{};
  return (int64_t)v;
}
int flag(PyObject* o) {   // int(o)
  PyObject* v = PyNumber_Long(o);
  if (!v) throw Stop{};
  const unsigned long m = PyLong_AsUnsignedLongMask(v);
  Py_DECREF(v);
  return (int)m;
}
flop_hc_params_t hard_concrete(PyObject* o) {
  float v[3];
  for (int i = 0; i < 3; ++i) {
    PyObject* at = PyLong_FromLong(i);
    PyObject* e = at ? PyObject_GetItem(o, at) : nullptr;   // float(o[i]), whatever o is
    Py_XDECREF(at);
    PyObject* d = e ? PyNumber_Float(e) : nullptr;
    Py_XDECREF(e);
    if (!d) throw Stop{};
    v[i] = (float)PyFloat_AS_DOUBLE(d);
    Py_DECREF(d);
  }
  return flop_hc_params_t{v[0], v[1], v[2]};
}
void* stream() { return (void*)c10::cuda::getCurrentCUDAStream().stream(); }
size_t numel(PyObject* o) { const at::Tensor* t = tensor(o); return t ? (size_t)t->numel() : 0; }

// Runs the library call without the interpreter lock and returns its status as a Python integer.  The lock is back before an
// exception (the library's planners allocate on the host) leaves the call and becomes a Python one.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F> PyObject* call(F&& f) {
  int status;
  {
    Unlocked u;
    status = f();
  }
  return PyLong_FromLong(status);
}

#define FLOP_METHOD(name, count)                                                        \
  PyObject* name##_body(PyObject* const* a);                                            \
  PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n) {                         \
    HANDLE_TH_ERRORS                                                                    \
    if (n != (count)) {                                                                 \
      PyErr_Format(PyExc_TypeError, #name ": %d arguments expected", (int)(count));     \
      return nullptr;                                                                   \
    }                                                                                   \
    try { return name##_body(a); } catch (const Stop&) { return nullptr; }              \
    END_HANDLE_TH_ERRORS                                                                \
  }                                                                                     \
  PyObject* name##_body(PyObject* const* a)

FLOP_METHOD(gate_sample, 7) {   // log_alpha, hc, seed, offset, z, mask, dz_dla
  const float* la = static_cast<const float*>(required(a[0]).data_ptr());
  const int64_t n = (int64_t)numel(a[0]);
  const flop_hc_params_t hc = hard_concrete(a[1]);
  const uint64_t seed = (uint64_t)integer(a[2]), offset = (uint64_t)integer(a[3]);
  float* z = ptr<float>(a[4]); uint8_t* mask = ptr<uint8_t>(a[5]); float* dz = ptr<float>(a[6]);
  void* st = stream();
  return call([&] { return flop_gate_sample(la, n, hc, seed, offset, z, mask, dz, st); });
}

FLOP_METHOD(gated_lowrank_fwd, 7) {   // X, Q, P, z, Y, H_save, ws
  const Mat X = matrix(a[0]), Q = matrix(a[1]), P = matrix(a[2]), Y = matrix(a[4]), H = optional_matrix(a[5]);
  const int dt = storage(required(a[0]));
  const float* z = ptr<float>(a[3]); void* ws = ptr(a[6]); const size_t wb = numel(a[6]);
  void* st = stream();
  return call([&] { return flop_gated_lowrank_fwd(X.p, X.ld, Q.p, Q.ld, P.p, P.ld, z, Y.p, Y.ld, H.p, H.ld, X.rows, X.cols, P.rows, P.cols, dt, ws, wb, st); });
}

FLOP_METHOD(gated_lowrank_bwd, 13) {   // dY, X, Q, P, z, dz_dla, H_save, dX, dP, dQ, dlog_alpha, ws, accumulate
  const Mat dY = matrix(a[0]), X = matrix(a[1]), Q = matrix(a[2]), P = matrix(a[3]), H = matrix(a[6]);
  const Mat dX = optional_matrix(a[7]), dP = optional_matrix(a[8]), dQ = optional_matrix(a[9]);
  const int dt = storage(required(a[1]));
  const int wdt = a[8] != Py_None ? storage(required(a[8])) : a[9] != Py_None ? storage(required(a[9])) : dt;
  const float *z = ptr<float>(a[4]), *dz = ptr<float>(a[5]); float* dla = ptr<float>(a[10]);
  void* ws = ptr(a[11]); const size_t wb = numel(a[11]); const int acc = flag(a[12]);
  void* st = stream();
  return call([&] {
    return flop_gated_lowrank_bwd(dY.p, dY.ld, X.p, X.ld, Q.p, Q.ld, P.p, P.ld, z, dz, H.p, H.ld, dX.p, dX.ld, dP.p, dP.ld, dQ.p, dQ.ld, dla, acc,
                                  X.rows, X.cols, P.rows, P.cols, dt, wdt, ws, wb, st);
  });
}

FLOP_METHOD(expected_l0_lagrangian, 10) {   // log_alpha, seg_off, seg_size, hc, target, lam, out4, seg_expected, dlog_alpha, ws
  const float* la = static_cast<const float*>(required(a[0]).data_ptr());
  const int64_t n = (int64_t)numel(a[0]);
  const int32_t n_seg = (int32_t)required(a[2]).numel();
  const int64_t* off = ptr<int64_t>(a[1]); const float* size = ptr<float>(a[2]);
  const flop_hc_params_t hc = hard_concrete(a[3]);
  const float *target = ptr<float>(a[4]), *lam = ptr<float>(a[5]);
  float *out4 = ptr<float>(a[6]), *seg = ptr<float>(a[7]), *dla = ptr<float>(a[8]);
  void* ws = ptr(a[9]); const size_t wb = numel(a[9]);
  void* st = stream();
  return call([&] { return flop_expected_l0_lagrangian(la, n, off, size, n_seg, hc, target, lam, out4, seg, dla, ws, wb, st); });
}

FLOP_METHOD(gated_embedding_fwd, 6) {   // ids, E, O, z, Y, H_save
  const Mat E = matrix(a[1]), O = matrix(a[2]), Y = matrix(a[4]), H = matrix(a[5]);
  const int dt = storage(required(a[1]));
  const int64_t T = required(a[0]).numel();
  const int32_t* ids = ptr<int32_t>(a[0]); const float* z = ptr<float>(a[3]);
  void* st = stream();
  return call([&] { return flop_gated_embedding_fwd(ids, T, E.p, E.ld, E.rows, O.p, O.ld, z, Y.p, Y.ld, H.p, H.ld, E.cols, O.cols, dt, st); });
}

FLOP_METHOD(gated_embedding_bwd, 12) {   // dY, ids, E, O, z, dz_dla, H_save, dE, dO, dlog_alpha, ws, accumulate
  const Mat dY = matrix(a[0]), E = matrix(a[2]), O = matrix(a[3]), H = matrix(a[6]), dE = optional_matrix(a[7]), dO = optional_matrix(a[8]);
  const int dt = storage(required(a[2])), wdt = a[8] != Py_None ? storage(required(a[8])) : (int)FLOP_BF16;
  const int64_t T = required(a[1]).numel();
  const int32_t* ids = ptr<int32_t>(a[1]); const float *z = ptr<float>(a[4]), *dz = ptr<float>(a[5]); float* dla = ptr<float>(a[9]);
  void* ws = ptr(a[10]); const size_t wb = numel(a[10]); const int acc = flag(a[11]);
  void* st = stream();
  return call([&] {
    return flop_gated_embedding_bwd(dY.p, dY.ld, ids, T, E.p, E.ld, E.rows, O.p, O.ld, z, dz, H.p, H.ld, (float*)dE.p, dE.ld, dO.p, dO.ld, dla, acc,
                                    E.cols, O.cols, dt, wdt, ws, wb, st);
  });
}

FLOP_METHOD(compact_ranks, 10) {   // log_alpha_or_z, mode, hc, idx, k_dev, z_det, P, Q, Pc, Qc
  const float* in = static_cast<const float*>(required(a[0]).data_ptr());
  const int64_t r = (int64_t)numel(a[0]);
  const int mode = (int)integer(a[1]);
  const flop_hc_params_t hc = hard_concrete(a[2]);
  int32_t *idx = ptr<int32_t>(a[3]), *k = ptr<int32_t>(a[4]); float* z = ptr<float>(a[5]);
  const Mat P = optional_matrix(a[6]), Q = optional_matrix(a[7]), Pc = optional_matrix(a[8]), Qc = optional_matrix(a[9]);
  const int dt = a[6] != Py_None ? storage(required(a[6])) : (int)FLOP_F32;
  void* st = stream();
  return call([&] {
    return flop_compact_ranks(in, mode, hc, r, P.p, P.ld, Q.p, Q.ld, Q.cols, P.rows, dt, idx, k, z, Pc.p, Pc.ld, Qc.p, Qc.ld, nullptr, 0, st);
  });
}

FLOP_METHOD(compact_fwd, 6) {   // X, Qc, Pc, Y, k, ws
  const Mat X = matrix(a[0]), Qc = matrix(a[1]), Pc = matrix(a[2]), Y = matrix(a[3]);
  const int dt = storage(required(a[0]));
  const int64_t k = integer(a[4]);
  void* ws = ptr(a[5]); const size_t wb = numel(a[5]);
  void* st = stream();
  return call([&] { return flop_compact_fwd(X.p, X.ld, Qc.p, Qc.ld, Pc.p, Pc.ld, Y.p, Y.ld, X.rows, X.cols, Pc.rows, k, dt, ws, wb, st); });
}

// ---- the 8-bit products and the distillation loss (module _operators)
float number(PyObject* o) {   // float(o)
  PyObject* v = PyNumber_Float(o);
  if (!v) throw Stop{};
  const double d = PyFloat_AS_DOUBLE(v);
  Py_DECREF(v);
  return (float)d;
}
// A tensor of another type than the call reads would be read as that type: refused here, the library sees addresses only.
void need(PyObject* o, at::ScalarType type, int64_t count, const char* what) {
  const at::Tensor* t = tensor(o);
  if (!t) return;
  if (t->scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s: expected %s, got %s", what, at::toString(type), at::toString(t->scalar_type()));
    throw Stop{};
  }
  if (count >= 0 && (!t->is_contiguous() || t->numel() < count)) {
    PyErr_Format(PyExc_AssertionError, "%s: expected %lld contiguous values", what, (long long)count);
    throw Stop{};
  }
}
void same(int64_t a, int64_t b, const char* what) {
  if (a == b) return;
  PyErr_Format(PyExc_AssertionError, "%s: %lld against %lld", what, (long long)a, (long long)b);
  throw Stop{};
}

FLOP_METHOD(quantize_rows, 3) {   // X, Xq, scale
  const Mat X = matrix(a[0]), Xq = matrix(a[1]);
  const int dt = storage(required(a[0]));
  need(a[1], at::kChar, -1, "Xq"); need(a[2], at::kFloat, X.rows, "scale");
  same(X.rows, Xq.rows, "rows of X and Xq"); same(X.cols, Xq.cols, "columns of X and Xq");
  float* scale = ptr<float>(a[2]);
  void* st = stream();
  return call([&] { return flop_quantize_rows(X.p, X.ld, X.rows, X.cols, dt, (int8_t*)Xq.p, Xq.ld, scale, st); });
}

FLOP_METHOD(gemm_i8, 5) {   // A, B, a_scale, b_scale, Y
  const Mat A = matrix(a[0]), B = matrix(a[1]), Y = matrix(a[4]);
  const int dt = storage(required(a[4]));
  need(a[0], at::kChar, -1, "A"); need(a[1], at::kChar, -1, "B");
  need(a[2], at::kFloat, A.rows, "a_scale"); need(a[3], at::kFloat, B.rows, "b_scale");
  same(A.cols, B.cols, "columns of A and B"); same(Y.rows, A.rows, "rows of Y and A"); same(Y.cols, B.rows, "columns of Y and rows of B");
  const float *sa = ptr<float>(a[2]), *sb = ptr<float>(a[3]);
  void* st = stream();
  return call([&] { return flop_gemm_i8((const int8_t*)A.p, A.ld, sa, (const int8_t*)B.p, B.ld, sb, Y.p, Y.ld, A.rows, B.rows, A.cols, dt, st); });
}

FLOP_METHOD(compact_fwd_i8, 8) {   // X, Qq, q_scale, Pq, p_scale, Y, k, ws
  const Mat X = matrix(a[0]), Q = matrix(a[1]), P = matrix(a[3]), Y = matrix(a[5]);
  const int dt = storage(required(a[0]));
  const int64_t k = integer(a[6]);
  need(a[1], at::kChar, -1, "Qq"); need(a[3], at::kChar, -1, "Pq");
  need(a[2], at::kFloat, k, "q_scale"); need(a[4], at::kFloat, P.rows, "p_scale");
  same(storage(required(a[5])), dt, "types of Y and X"); same(Y.rows, X.rows, "rows of Y and X"); same(Y.cols, P.rows, "columns of Y and rows of Pq");
  same(Q.cols, X.cols, "columns of Qq and X");
  same(Q.rows >= k && P.cols >= k, 1, "k fits Qq and Pq");
  const float *qs = ptr<float>(a[2]), *ps = ptr<float>(a[4]);
  void* ws = ptr(a[7]); const size_t wb = numel(a[7]);
  void* st = stream();
  return call([&] {
    return flop_compact_fwd_i8(X.p, X.ld, (const int8_t*)Q.p, Q.ld, qs, (const int8_t*)P.p, P.ld, ps, Y.p, Y.ld, X.rows, X.cols, P.rows, k, dt, ws, wb, st);
  });
}

struct Distill { Mat S, t, idx; int dt; const float *lse, *weight; float tau; };
Distill distill(PyObject* const* a) {   // S, t_logits, t_idx, t_lse, weight, temperature
  Distill d;
  d.S = matrix(a[0]); d.t = matrix(a[1]); d.idx = matrix(a[2]);
  d.dt = storage(required(a[0]));
  need(a[1], at::kFloat, -1, "t_logits"); need(a[2], at::kInt, -1, "t_idx");
  need(a[3], at::kFloat, d.S.rows, "t_lse"); need(a[4], at::kFloat, d.S.rows, "weight");
  same(d.t.rows, d.S.rows, "rows of t_logits and S"); same(d.idx.rows, d.S.rows, "rows of t_idx and S"); same(d.idx.cols, d.t.cols, "columns of t_idx and t_logits");
  d.lse = ptr<float>(a[3]); d.weight = ptr<float>(a[4]);
  d.tau = number(a[5]);
  return d;
}
Mat gradient(PyObject* o, const Distill& d) {
  const Mat g = matrix(o);
  same(storage(required(o)), d.dt, "types of dS and S"); same(g.rows, d.S.rows, "rows of dS and S"); same(g.cols, d.S.cols, "columns of dS and S");
  return g;
}

FLOP_METHOD(distill_topk_fwd, 8) {   // S, t_logits, t_idx, t_lse, weight, temperature, loss, stats
  const Distill d = distill(a);
  need(a[6], at::kFloat, d.S.rows, "loss"); need(a[7], at::kFloat, 4 * d.S.rows, "stats");
  float *loss = ptr<float>(a[6]), *stats = ptr<float>(a[7]);
  void* st = stream();
  return call([&] {
    return flop_distill_topk_fwd(d.S.p, d.S.ld, d.S.rows, d.S.cols, d.dt, (const float*)d.t.p, d.t.ld, (const int32_t*)d.idx.p, d.idx.ld, d.t.cols, d.lse, d.weight,
                                 d.tau, loss, stats, st);
  });
}

FLOP_METHOD(distill_topk_bwd, 9) {   // S, t_logits, t_idx, t_lse, weight, temperature, stats, dloss, dS
  const Distill d = distill(a);
  const Mat dS = gradient(a[8], d);
  need(a[6], at::kFloat, 4 * d.S.rows, "stats"); need(a[7], at::kFloat, d.S.rows, "dloss");
  const float *stats = ptr<float>(a[6]), *dloss = ptr<float>(a[7]);
  void* st = stream();
  return call([&] {
    return flop_distill_topk_bwd(d.S.p, d.S.ld, d.S.rows, d.S.cols, d.dt, (const float*)d.t.p, d.t.ld, (const int32_t*)d.idx.p, d.idx.ld, d.t.cols, d.lse, d.weight,
                                 d.tau, stats, dloss, dS.p, dS.ld, st);
  });
}

FLOP_METHOD(distill_topk_fwd_bwd, 8) {   // S, t_logits, t_idx, t_lse, weight, temperature, loss, dS
  const Distill d = distill(a);
  const Mat dS = gradient(a[7], d);
  need(a[6], at::kFloat, d.S.rows, "loss");
  float* loss = ptr<float>(a[6]);
  void* st = stream();
  return call([&] {
    return flop_distill_topk_fwd_bwd(d.S.p, d.S.ld, d.S.rows, d.S.cols, d.dt, (const float*)d.t.p, d.t.ld, (const int32_t*)d.idx.p, d.idx.ld, d.t.cols, d.lse,
                                     d.weight, d.tau, loss, dS.p, dS.ld, st);
  });
}

// ---- embedding lookup, dropout and layer norm (module _rows)
// The library works on the current device and sees addresses only: a tensor of the host or of another device is refused here, and the call runs
// on the device of its tensors, on that device's current stream.
struct Place {
  c10::DeviceIndex device = -1;
  c10::cuda::OptionalCUDAGuard guard;
  Place(std::initializer_list<PyObject*> tensors) {
    for (PyObject* o : tensors) {
      const at::Tensor* t = tensor(o);
      if (!t) continue;
      if (!t->is_cuda()) {
        PyErr_Format(PyExc_TypeError, "expected tensors on a CUDA device, got one on %s", t->device().str().c_str());
        throw Stop{};
      }
      if (device < 0) device = t->device().index();
      same(t->device().index(), device, "devices of the tensors");
    }
    if (device >= 0) guard.set_index(device);
  }
  void* stream() const { return (void*)c10::cuda::getCurrentCUDAStream(device).stream(); }
};
Mat like(PyObject* o, const Mat& m, int dt, const char* what) {   // a matrix of m's size and type; None: none
  const Mat r = optional_matrix(o);
  if (o == Py_None) return r;
  same(storage(required(o)), dt, what); same(r.rows, m.rows, what); same(r.cols, m.cols, what);
  return r;
}
struct Mask { float p; uint64_t seed, offset; const uint64_t* dev; };
Mask mask(PyObject* const* a) {   // p, seed, offset, offset_dev
  Mask m{number(a[0]), (uint64_t)integer(a[1]), (uint64_t)integer(a[2]), nullptr};
  need(a[3], at::kLong, 1, "offset_dev");
  m.dev = ptr<const uint64_t>(a[3]);
  return m;
}

FLOP_METHOD(embedding_fwd, 4) {   // ids, E, scale, Y
  const Mat E = matrix(a[1]), Y = matrix(a[3]);
  const int dt = storage(required(a[1]));
  const float scale = number(a[2]);
  same(storage(required(a[3])), dt, "types of Y and E"); same(Y.cols, E.cols, "columns of Y and E");
  required(a[0]); need(a[0], at::kInt, Y.rows, "ids"); same((int64_t)numel(a[0]), Y.rows, "ids and rows of Y");
  const int32_t* ids = ptr<int32_t>(a[0]);
  const Place at{a[0], a[1], a[3]};
  return call([&] { return flop_embedding_fwd(ids, Y.rows, E.p, E.ld, E.rows, scale, Y.p, Y.ld, Y.cols, dt, at.stream()); });
}

FLOP_METHOD(embedding_bwd, 6) {   // dY, ids, scale, dE, ws, accumulate
  const Mat dY = matrix(a[0]), dE = matrix(a[3]);
  const int dt = storage(required(a[0])), wdt = storage(required(a[3]));
  const float scale = number(a[2]);
  same(dE.cols, dY.cols, "columns of dE and dY");
  required(a[1]); need(a[1], at::kInt, dY.rows, "ids"); same((int64_t)numel(a[1]), dY.rows, "ids and rows of dY");
  const int32_t* ids = ptr<int32_t>(a[1]);
  need(a[4], at::kByte, 0, "ws");
  void* ws = ptr(a[4]); const size_t wb = numel(a[4]);
  const int accumulate = flag(a[5]);
  const Place at{a[0], a[1], a[3], a[4]};
  return call([&] { return flop_embedding_bwd(dY.p, dY.ld, ids, dY.rows, dE.rows, scale, dE.p, dE.ld, accumulate, dY.cols, dt, wdt, ws, wb, at.stream()); });
}

FLOP_METHOD(dropout_fwd, 7) {   // X, R, p, seed, offset, offset_dev, Y
  const Mat X = matrix(a[0]);
  const int dt = storage(required(a[0]));
  const Mat R = like(a[1], X, dt, "R and X"), Y = like((required(a[6]), a[6]), X, dt, "Y and X");
  const Mask m = mask(a + 2);
  const Place at{a[0], a[1], a[5], a[6]};
  return call([&] { return flop_dropout_fwd(X.p, X.ld, R.p, R.ld, m.p, m.seed, m.offset, m.dev, Y.p, Y.ld, X.rows, X.cols, dt, at.stream()); });
}

FLOP_METHOD(dropout_bwd, 6) {   // dY, p, seed, offset, offset_dev, dX
  const Mat dY = matrix(a[0]);
  const int dt = storage(required(a[0]));
  const Mat dX = like((required(a[5]), a[5]), dY, dt, "dX and dY");
  const Mask m = mask(a + 1);
  const Place at{a[0], a[4], a[5]};
  return call([&] { return flop_dropout_bwd(dY.p, dY.ld, m.p, m.seed, m.offset, m.dev, dX.p, dX.ld, dY.rows, dY.cols, dt, at.stream()); });
}

FLOP_METHOD(layer_norm_fwd, 12) {   // X, R, p, seed, offset, offset_dev, weight, bias, eps, S, Y, stats
  const Mat X = matrix(a[0]);
  const int dt = storage(required(a[0]));
  const Mat R = like(a[1], X, dt, "R and X"), S = like(a[9], X, dt, "S and X"), Y = like((required(a[10]), a[10]), X, dt, "Y and X");
  const Mask m = mask(a + 2);
  need(a[6], at::kFloat, X.cols, "weight"); need(a[7], at::kFloat, X.cols, "bias"); need(a[11], at::kFloat, 2 * X.rows, "stats");
  const float *w = ptr<float>(a[6]), *b = ptr<float>(a[7]), eps = number(a[8]);
  float* stats = ptr<float>(a[11]);
  const Place at{a[0], a[1], a[5], a[6], a[7], a[9], a[10], a[11]};
  return call([&] {
    return flop_layer_norm_fwd(X.p, X.ld, R.p, R.ld, m.p, m.seed, m.offset, m.dev, w, b, eps, S.p, S.ld, Y.p, Y.ld, stats, X.rows, X.cols, dt, at.stream());
  });
}

FLOP_METHOD(layer_norm_bwd, 15) {   // dY, S, stats, weight, dS, p, seed, offset, offset_dev, dX, dR, dweight, dbias, ws, accumulate
  const Mat dY = matrix(a[0]);
  const int dt = storage(required(a[0]));
  const Mat S = like((required(a[1]), a[1]), dY, dt, "S and dY"), dS = like(a[4], dY, dt, "dS and dY"), dX = like(a[9], dY, dt, "dX and dY"),
            dR = like(a[10], dY, dt, "dR and dY");
  const Mask m = mask(a + 5);
  need(a[2], at::kFloat, 2 * dY.rows, "stats"); need(a[3], at::kFloat, dY.cols, "weight");
  need(a[11], at::kFloat, dY.cols, "dweight"); need(a[12], at::kFloat, dY.cols, "dbias"); need(a[13], at::kByte, 0, "ws");
  const float *stats = ptr<float>(a[2]), *w = ptr<float>(a[3]);
  float *dw = ptr<float>(a[11]), *db = ptr<float>(a[12]);
  void* ws = ptr(a[13]); const size_t wb = numel(a[13]);
  const int accumulate = flag(a[14]);
  const Place at{a[0], a[1], a[2], a[3], a[4], a[8], a[9], a[10], a[11], a[12], a[13]};
  return call([&] {
    return flop_layer_norm_bwd(dY.p, dY.ld, S.p, S.ld, stats, w, dS.p, dS.ld, m.p, m.seed, m.offset, m.dev, dX.p, dX.ld, dR.p, dR.ld, dw, db, accumulate, dY.rows,
                               dY.cols, dt, ws, wb, at.stream());
  });
}

#define FLOP_ENTRY(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FLOP_ENTRY(gate_sample), FLOP_ENTRY(gated_lowrank_fwd), FLOP_ENTRY(gated_lowrank_bwd), FLOP_ENTRY(expected_l0_lagrangian),
                         FLOP_ENTRY(gated_embedding_fwd), FLOP_ENTRY(gated_embedding_bwd), FLOP_ENTRY(compact_ranks), FLOP_ENTRY(compact_fwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
PyMethodDef operator_methods[] = {FLOP_ENTRY(quantize_rows), FLOP_ENTRY(gemm_i8), FLOP_ENTRY(compact_fwd_i8), FLOP_ENTRY(distill_topk_fwd),
                                  FLOP_ENTRY(distill_topk_bwd), FLOP_ENTRY(distill_topk_fwd_bwd), {nullptr, nullptr, 0, nullptr}};
PyMethodDef row_methods[] = {FLOP_ENTRY(embedding_fwd), FLOP_ENTRY(embedding_bwd), FLOP_ENTRY(dropout_fwd), FLOP_ENTRY(dropout_bwd),
                             FLOP_ENTRY(layer_norm_fwd), FLOP_ENTRY(layer_norm_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef rows = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, row_methods, nullptr, nullptr, nullptr, nullptr};
PyModuleDef operators = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, operator_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The calls beside the layer's own path are modules of their own inside this one.
PyMODINIT_FUNC PyInit__binding_native(void) {
  PyObject* m = PyModule_Create(&module);
  for (PyModuleDef* def : {&operators, &rows}) {
    PyObject* o = m ? PyModule_Create(def) : nullptr;
    if (!o || PyModule_AddObject(m, def->m_name, o) < 0) {
      Py_XDECREF(o);
      Py_XDECREF(m);
      return nullptr;
    }
  }
  return m;
}
