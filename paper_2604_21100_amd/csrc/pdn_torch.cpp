// The calls on a pool of states and those around the rule, from torch tensors: what the binding does for
// them, compiled.  A server makes these calls once a token, and with a few dozen
// arguments the checks alone take an interpreter three times as long as the launch
// (a decode call: 14.0 us of the host in Python, 7.0 here, of which the library 3.4).
// Checks of dtypes, shapes, strides and devices, and the packing of pdn.h's
// structures; everything else is the library's.  Host code only; the library's
// functions come as addresses.
#include <Python.h>
#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/pdn.h"

namespace {

struct Refused {};   // a Python error is set

[[noreturn]] void refuse(PyObject* kind, const std::string& what) {
  PyErr_SetString(kind, what.c_str());
  throw Refused{};
}

const at::Tensor* tensor(PyObject* o, const char* name) {   // None: nullptr
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + " must be a tensor");
  return &THPVariable_Unpack(o);
}
const at::Tensor& given(PyObject* o, const char* name) {
  const at::Tensor* t = tensor(o, name);
  if (!t) refuse(PyExc_TypeError, std::string(name) + " must be a tensor");
  return *t;
}

std::string text(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

void check(const char* name, const at::Tensor& t, at::Device device, at::ScalarType dtype, at::IntArrayRef shape) {
  if (t.scalar_type() != dtype)
    refuse(PyExc_TypeError, std::string(name) + " must be " + c10::toString(dtype) + ", got " + c10::toString(t.scalar_type()));
  if (t.sizes() != shape)
    refuse(PyExc_ValueError, std::string(name) + " must be " + text(shape) + ", got " + text(t.sizes()));
  if (t.device() != device)
    refuse(PyExc_ValueError, std::string(name) + " is on " + t.device().str() + ", not on " + device.str());
}

// address of a dense tensor of this dtype and shape on `device` (None: NULL)
template <typename T = void>
T* on(const char* name, PyObject* o, at::Device device, at::ScalarType dtype, at::IntArrayRef shape) {
  const at::Tensor* t = tensor(o, name);
  if (!t) return nullptr;
  check(name, *t, device, dtype, shape);
  if (!t->is_contiguous()) refuse(PyExc_ValueError, std::string(name) + " must be contiguous");
  return static_cast<T*>(t->data_ptr());
}

// a [tokens, heads, d] tensor with dense rows; stride: from one token to the next (0: dense,
// so a row that is expanded over the tokens must not get there as it is)
const void* token_rows(const char* name, PyObject* o, at::Device device, at::ScalarType dtype, at::IntArrayRef shape,
                       int64_t* stride) {
  const at::Tensor& t = given(o, name);
  check(name, t, device, dtype, shape);
  *stride = 0;
  if (!t.is_contiguous()) {
    if (t.stride(2) != 1 || (t.stride(1) != shape[2] && shape[1] > 1))
      refuse(PyExc_ValueError, std::string("a token's row of ") + name + " must be dense");
    if (shape[0] > 1 && t.stride(0) < shape[1] * shape[2])
      refuse(PyExc_ValueError, std::string("a token's row of ") + name + " must not overlap another's (stride " +
                                   std::to_string(t.stride(0)) + ")");
    *stride = t.stride(0);
  }
  return t.data_ptr();
}

int64_t whole(PyObject* o) {
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused{};
  return x;
}
double real(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Refused{};
  return x;
}
template <typename F>
F function(PyObject* o) {
  return reinterpret_cast<F>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLong(o)));
}
pdn_dtype io_of(const at::Tensor& t) {
  if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16)
    refuse(PyExc_TypeError, std::string("tensors must be float32 or bfloat16, got ") + c10::toString(t.scalar_type()));
  return t.scalar_type() == at::kFloat ? PDN_F32 : PDN_BF16;
}
at::Tensor empty(at::IntArrayRef shape, at::Device device, at::ScalarType dtype) {
  return at::empty(shape, at::TensorOptions().device(device).dtype(dtype));
}

// pdn_slot_fwd or pdn_slot_draft: o, or a status that is not PDN_OK
PyObject* slot(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kQ, kK, kV, kBeta, kS, kTape, kPending, kAccepted, kRecord, kStarts, kSlots, kSlotsOut, kFresh, kMaxTokens, kG,
           kGate, kPrecond, kBetaP, kGP, kLogA, kA, kKtilde, kX, kScale, kRidge, kKnorm, kO, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor &S = given(a[kS], "S"), &q = given(a[kQ], "q"), &v = given(a[kV], "v");
    if (S.dim() != 4 || q.dim() != 3 || v.dim() != 3)
      refuse(PyExc_ValueError, "S must be [slots, H, dk, dv], q, k [tokens, Hk, dk] and v [tokens, H, dv]");
    const at::Device dev = S.device();
    const int64_t P = S.size(0), H = S.size(1), dk = S.size(2), dv = S.size(3), M = q.size(0), Hk = q.size(1);
    const at::ScalarType dt = q.scalar_type(), f32 = at::kFloat, i32 = at::kInt;
    const at::Tensor *starts = tensor(a[kStarts], "starts"), *slots = tensor(a[kSlots], "slots");
    const bool counted = a[kMaxTokens] != Py_None;
    int64_t T = counted ? whole(a[kMaxTokens]) : 0, N;
    if (starts) N = starts->numel() - 1;
    else if (slots) N = slots->numel();
    else N = T ? M / T : M;   // rows shared out evenly
    if (N < 0) refuse(PyExc_ValueError, "starts must hold one entry more than sequences");
    if (!counted) T = starts ? M : N ? M / N : 0;

    pdn_problem p{};
    p.B = N; p.T = T; p.H = H;
    p.dk = static_cast<int32_t>(std::min<int64_t>(dk, INT32_MAX));
    p.dv = static_cast<int32_t>(std::min<int64_t>(dv, INT32_MAX));
    p.chunk = 64;
    p.io = io_of(q);
    p.gate = static_cast<pdn_gate>(whole(a[kGate]));
    p.precond = static_cast<pdn_precond>(whole(a[kPrecond]));
    p.knorm = static_cast<pdn_knorm>(whole(a[kKnorm]));
    p.x = static_cast<float>(real(a[kX]));
    p.scale = static_cast<float>(real(a[kScale]));
    p.ridge = static_cast<float>(real(a[kRidge]));

    pdn_inputs in{};
    pdn_slots s{};
    const int64_t keys[] = {M, Hk, dk}, values[] = {M, H, dv}, scalars[] = {M, H}, channels[] = {M, H, dk}, heads[] = {H},
                  seqs[] = {N}, ends[] = {N + 1}, states[] = {P, H, dk};
    in.q = token_rows("q", a[kQ], dev, dt, keys, &s.q_stride);
    in.k = token_rows("k", a[kK], dev, dt, keys, &s.k_stride);
    in.v = token_rows("v", a[kV], dev, dt, values, &s.v_stride);
    given(a[kBeta], "beta");
    in.beta = on<float>("beta", a[kBeta], dev, f32, scalars);
    in.g = on<float>("g", a[kG], dev, f32, p.gate == PDN_GATE_CHANNEL ? at::IntArrayRef(channels) : at::IntArrayRef(scalars));
    in.beta_p = on<float>("beta_p", a[kBetaP], dev, f32, scalars);
    in.g_p = on<float>("g_p", a[kGP], dev, f32, scalars);
    in.log_a_scale = on<float>("log_a_scale", a[kLogA], dev, f32, heads);
    in.ktilde = on("ktilde", a[kKtilde], dev, dt, keys);
    s.tokens = M; s.slots = P; s.Hk = Hk;
    s.starts = on<int32_t>("starts", a[kStarts], dev, i32, ends);
    s.slot = on<int32_t>("slots", a[kSlots], dev, i32, seqs);
    s.slot_out = on<int32_t>("slots_out", a[kSlotsOut], dev, i32, seqs);
    s.fresh = on<int32_t>("fresh", a[kFresh], dev, i32, seqs);
    s.S = on<float>("S", a[kS], dev, f32, S.sizes());
    s.A = on<float>("A", a[kA], dev, f32, states);
    if (a[kTape] != Py_None) {
      const at::Tensor& tape = given(a[kTape], "tape");
      if (tape.dim() != 4) refuse(PyExc_ValueError, "tape must be [slots, tokens, H, record]");
      const int64_t records[] = {P, tape.size(1), H, whole(a[kRecord])}, counts[] = {P, H};
      s.tape = on<float>("tape", a[kTape], dev, f32, records);
      s.tape_tokens = tape.size(1);
      s.pending = on<int32_t>("pending", a[kPending], dev, i32, counts);
      s.accepted = on<int32_t>("accepted", a[kAccepted], dev, i32, seqs);
    }
    if (!dev.is_cuda()) refuse(PyExc_ValueError, "S is on " + dev.str());
    at::Tensor made;
    void* o;
    if (a[kO] == Py_None) {
      made = empty(values, dev, dt);
      o = made.data_ptr();
    } else {
      o = on("o", a[kO], dev, dt, values);
    }
    const auto fn = function<decltype(&pdn_slot_fwd)>(a[kFn]);
    void* const stream = function<void*>(a[kStream]);
    pdn_status st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(&p, &in, &s, o, stream);
    Py_END_ALLOW_THREADS
    if (st != PDN_OK) return PyLong_FromLong(st);
    if (made.defined()) return THPVariable_Wrap(made);
    Py_INCREF(a[kO]);
    return a[kO];
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// pdn_draft_verify: (accepted, token), or a status that is not PDN_OK
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kSizeFn, kP, kQ, kIds, kU, kR, kStarts, kAccepted, kToken, kWorkspace, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor &p = given(a[kP], "p"), &r = given(a[kR], "r");
    if (p.dim() != 2) refuse(PyExc_ValueError, "p must be [rows, V]");
    const at::Device dev = p.device();
    if (!dev.is_cuda()) refuse(PyExc_ValueError, "p is on " + dev.str());
    const int64_t M = p.size(0), V = p.size(1), N = r.numel();
    const pdn_dtype io = io_of(p);
    const at::ScalarType f32 = at::kFloat, i32 = at::kInt;
    const int64_t rows[] = {M}, seqs[] = {N}, ends[] = {N + 1};
    given(a[kIds], "ids");
    given(a[kU], "u");
    const void* const pp = on("p", a[kP], dev, p.scalar_type(), p.sizes());
    const void* const qp = on("q", a[kQ], dev, p.scalar_type(), p.sizes());
    const int32_t *const ids = on<int32_t>("ids", a[kIds], dev, i32, rows), *const starts = on<int32_t>("starts", a[kStarts], dev, i32, ends);
    const float *const u = on<float>("u", a[kU], dev, f32, rows), *const rp = on<float>("r", a[kR], dev, f32, seqs);
    at::Tensor accepted, token, ws;
    if (a[kAccepted] == Py_None) accepted = empty(seqs, dev, i32);
    if (a[kToken] == Py_None) token = empty(seqs, dev, i32);
    size_t bytes = 0;
    pdn_status st = PDN_OK;
    if (a[kWorkspace] == Py_None) {
      st = function<decltype(&pdn_draft_verify_workspace_size)>(a[kSizeFn])(N, V, &bytes);
      if (st != PDN_OK) return PyLong_FromLong(st);
      ws = empty({static_cast<int64_t>(bytes)}, dev, at::kByte);
    } else {
      ws = given(a[kWorkspace], "workspace");
      on("workspace", a[kWorkspace], dev, at::kByte, ws.sizes());
      bytes = static_cast<size_t>(ws.numel());
    }
    int32_t* const ap = accepted.defined() ? accepted.data_ptr<int32_t>() : on<int32_t>("accepted", a[kAccepted], dev, i32, seqs);
    int32_t* const tp = token.defined() ? token.data_ptr<int32_t>() : on<int32_t>("token", a[kToken], dev, i32, seqs);
    const auto fn = function<decltype(&pdn_draft_verify)>(a[kFn]);
    void *const stream = function<void*>(a[kStream]), *const wp = ws.data_ptr();
    Py_BEGIN_ALLOW_THREADS
    st = fn(N, M, V, io, pp, qp, ids, u, rp, starts, ap, tp, wp, bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PDN_OK) return PyLong_FromLong(st);
    PyObject *x = accepted.defined() ? THPVariable_Wrap(accepted) : a[kAccepted], *y = token.defined() ? THPVariable_Wrap(token) : a[kToken];
    if (!accepted.defined()) Py_INCREF(x);
    if (!token.defined()) Py_INCREF(y);
    PyObject* const both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// a given tensor's address, or a new one of that kind in `made`
void* out_or_new(const char* name, PyObject* o, at::Device device, at::ScalarType dtype, at::IntArrayRef shape, at::Tensor* made) {
  if (o != Py_None) return on(name, o, device, dtype, shape);
  *made = empty(shape, device, dtype);
  return made->data_ptr();
}
// what a call returns for it (a new reference)
PyObject* result(PyObject* given, const at::Tensor& made) {
  if (made.defined()) return THPVariable_Wrap(made);
  Py_INCREF(given);
  return given;
}
at::ScalarType scalar_of(pdn_dtype t) { return t == PDN_BF16 ? at::kBFloat16 : at::kFloat; }
bool truth(PyObject* o) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw Refused{};
  return x != 0;
}
void on_device(const char* name, at::Device dev) {
  if (!dev.is_cuda()) refuse(PyExc_ValueError, std::string(name) + " is on " + dev.str());
}
at::Tensor workspace_of(PyObject* o, at::Device dev, size_t bytes, size_t* has) {
  if (o == Py_None) {
    *has = bytes;
    return empty({static_cast<int64_t>(bytes)}, dev, at::kByte);
  }
  const at::Tensor& ws = given(o, "workspace");
  on("workspace", o, dev, at::kByte, ws.sizes());
  *has = static_cast<size_t>(ws.numel());
  return ws;
}
int64_t rows_before(const at::Tensor& t, int64_t dims) {   // the product of the sizes but the last `dims`
  int64_t n = 1;
  for (int64_t i = 0; i + dims < t.dim(); ++i) n *= t.size(i);
  return n;
}
// name -> tensor, for what there is
PyObject* grads(std::initializer_list<std::pair<const char*, std::pair<PyObject*, const at::Tensor*>>> items) {
  PyObject* const d = PyDict_New();
  if (!d) return nullptr;
  for (const auto& it : items) {
    if (it.second.first == Py_None && !it.second.second->defined()) continue;
    PyObject* const v = result(it.second.first, *it.second.second);
    if (!v || PyDict_SetItemString(d, it.first, v) < 0) {
      Py_XDECREF(v);
      Py_DECREF(d);
      return nullptr;
    }
    Py_DECREF(v);
  }
  return d;
}

pdn_rnorm rnorm_of(const at::Tensor& y, pdn_dtype stream, PyObject* post, PyObject* alpha, PyObject* eps) {
  pdn_rnorm p{};
  p.D = y.size(-1);
  p.rows = rows_before(y, 1);
  p.io = io_of(y);
  p.stream = stream;
  p.post_norm = truth(post);
  p.alpha = static_cast<float>(real(alpha));
  p.eps = static_cast<float>(real(eps));
  return p;
}

// pdn_residual_norm: (u, h or None), or a status that is not PDN_OK
PyObject* residual_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kY, kResidual, kWeight, kPostWeight, kScale, kPost, kAlpha, kEps, kStreamType, kWantH, kU, kH, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor& y = given(a[kY], "y");
    const at::Tensor* const residual = tensor(a[kResidual], "residual");
    if (y.dim() < 1) refuse(PyExc_ValueError, "y must be [..., D]");
    const at::Device dev = y.device();
    const int64_t named = whole(a[kStreamType]);   // (-1: not named)
    pdn_dtype sm = residual ? io_of(*residual) : named >= 0 ? static_cast<pdn_dtype>(named) : io_of(y);
    if (named >= 0 && named != sm) refuse(PyExc_TypeError, "h_dtype must be residual's dtype");
    const pdn_rnorm p = rnorm_of(y, sm, a[kPost], a[kAlpha], a[kEps]);
    const at::ScalarType io = y.scalar_type(), st = scalar_of(sm), f32 = at::kFloat;
    const int64_t vec[] = {p.D};
    const void* const yp = on("y", a[kY], dev, io, y.sizes());
    const void* const rp = on("residual", a[kResidual], dev, st, y.sizes());
    const float *const w = on<float>("weight", a[kWeight], dev, f32, vec), *const pw = on<float>("post_weight", a[kPostWeight], dev, f32, vec),
                *const sc = on<float>("scale", a[kScale], dev, f32, vec);
    at::Tensor u, h;
    void* const up = out_or_new("u", a[kU], dev, io, y.sizes(), &u);
    void* const hp = a[kH] != Py_None || truth(a[kWantH]) ? out_or_new("h", a[kH], dev, st, y.sizes(), &h) : nullptr;
    on_device("y", dev);
    const auto fn = function<decltype(&pdn_residual_norm)>(a[kFn]);
    void* const stream = function<void*>(a[kStream]);
    pdn_status status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(&p, yp, rp, w, pw, sc, up, hp, stream);
    Py_END_ALLOW_THREADS
    if (status != PDN_OK) return PyLong_FromLong(status);
    PyObject *const x = result(a[kU], u), *const z = result(a[kH], h);
    PyObject* const both = x && z ? PyTuple_Pack(2, x, z) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(z);
    return both;
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// pdn_residual_norm_bwd: a dict of gradients, or a status that is not PDN_OK
PyObject* residual_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kSizeFn, kDu, kH, kY, kDh, kWeight, kPostWeight, kScale, kPost, kAlpha, kEps, kWantResidual, kWantVectors, kDy, kDres,
           kDw, kDp, kDs, kWorkspace, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor &du = given(a[kDu], "du"), &h = given(a[kH], "h");
    if (du.dim() < 1) refuse(PyExc_ValueError, "du must be [..., D]");
    const at::Device dev = du.device();
    const pdn_rnorm p = rnorm_of(du, io_of(h), a[kPost], a[kAlpha], a[kEps]);
    const at::ScalarType io = du.scalar_type(), st = h.scalar_type(), f32 = at::kFloat;
    const int64_t vec[] = {p.D};
    const void *const dup = on("du", a[kDu], dev, io, du.sizes()), *const hp = on("h", a[kH], dev, st, du.sizes()),
               *const yp = on("y", a[kY], dev, io, du.sizes()), *const dhp = on("dh", a[kDh], dev, st, du.sizes());
    const float *const w = on<float>("weight", a[kWeight], dev, f32, vec), *const pw = on<float>("post_weight", a[kPostWeight], dev, f32, vec),
                *const sc = on<float>("scale", a[kScale], dev, f32, vec);
    at::Tensor dy, dres, dw, dp, ds;
    const bool vectors = truth(a[kWantVectors]);
    void* const dyp = out_or_new("dy", a[kDy], dev, io, du.sizes(), &dy);
    void* const drp = a[kDres] != Py_None || truth(a[kWantResidual]) ? out_or_new("dresidual", a[kDres], dev, st, du.sizes(), &dres) : nullptr;
    auto vector = [&](const char* name, int at, const float* of, at::Tensor* made) -> float* {
      if (a[at] == Py_None && !(vectors && of)) return nullptr;
      return static_cast<float*>(out_or_new(name, a[at], dev, f32, vec, made));
    };
    float *const dwp = vector("dweight", kDw, w, &dw), *const dpp = vector("dpost_weight", kDp, pw, &dp), *const dsp = vector("dscale", kDs, sc, &ds);
    on_device("du", dev);
    size_t bytes = 0, has = 0;
    pdn_status status = function<decltype(&pdn_residual_norm_bwd_workspace_size)>(a[kSizeFn])(&p, &bytes);
    if (status != PDN_OK) return PyLong_FromLong(status);
    const at::Tensor ws = workspace_of(a[kWorkspace], dev, dwp || dpp || dsp ? bytes : 0, &has);
    const auto fn = function<decltype(&pdn_residual_norm_bwd)>(a[kFn]);
    void *const stream = function<void*>(a[kStream]), *const wp = ws.data_ptr();
    Py_BEGIN_ALLOW_THREADS
    status = fn(&p, dup, dhp, hp, yp, w, pw, sc, dyp, drp, dwp, dpp, dsp, wp, has, stream);
    Py_END_ALLOW_THREADS
    if (status != PDN_OK) return PyLong_FromLong(status);
    return grads({{"dy", {a[kDy], &dy}}, {"dresidual", {a[kDres], &dres}}, {"dweight", {a[kDw], &dw}}, {"dpost_weight", {a[kDp], &dp}},
                  {"dscale", {a[kDs], &ds}}});
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// a [..., H, d] tensor whose tokens' rows are dense and evenly spaced; stride as in token_rows
void* head_rows(const char* name, PyObject* o, at::Device device, at::ScalarType dtype, at::IntArrayRef shape, int64_t* stride) {
  *stride = 0;
  const at::Tensor* const tp = tensor(o, name);
  if (!tp) return nullptr;
  const at::Tensor& t = *tp;
  check(name, t, device, dtype, shape);
  if (!t.is_contiguous()) {
    const int64_t D = t.dim(), H = shape[D - 2], d = shape[D - 1];
    if ((t.stride(D - 1) != 1 && d > 1) || (t.stride(D - 2) != d && H > 1))
      refuse(PyExc_ValueError, std::string("a token's row of ") + name + " must be dense");
    int64_t tokens = 1;
    for (int64_t i = D - 3; i >= 0; --i) {
      if (shape[i] == 1) continue;
      if (tokens == 1) *stride = t.stride(i);
      else if (t.stride(i) != *stride * tokens)
        refuse(PyExc_ValueError, std::string("the tokens' rows of ") + name + " must be evenly spaced");
      tokens *= shape[i];
    }
    if (tokens > 1 && *stride < H * d)
      refuse(PyExc_ValueError, std::string("a token's row of ") + name + " must not overlap another's (stride " + std::to_string(*stride) + ")");
  }
  return t.data_ptr();
}

pdn_hnorm hnorm_of(const at::Tensor& x, PyObject* norm, const at::Tensor* weight, PyObject* act, PyObject* eps) {
  if (x.dim() < 2) refuse(PyExc_ValueError, "x must be [..., H, d]");
  pdn_hnorm p{};
  p.tokens = rows_before(x, 2);
  p.H = x.size(-2);
  if (x.size(-1) > INT32_MAX) refuse(PyExc_ValueError, "too many channels");
  p.d = static_cast<int32_t>(x.size(-1));
  p.io = io_of(x);
  p.norm = static_cast<pdn_norm>(whole(norm));
  p.act = static_cast<pdn_act>(whole(act));
  p.head_weight = weight && weight->dim() == 2;
  p.eps = static_cast<float>(real(eps));
  return p;
}
float* head_vector(const char* name, PyObject* o, at::Device dev, const pdn_hnorm& p) {
  const int64_t each[] = {p.H, p.d}, shared[] = {p.d};
  return on<float>(name, o, dev, at::kFloat, p.head_weight ? at::IntArrayRef(each) : at::IntArrayRef(shared));
}

// pdn_head_norm: y, or a status that is not PDN_OK
PyObject* head_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kX, kNorm, kWeight, kZ, kAct, kEps, kY, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor& x = given(a[kX], "x");
    pdn_hnorm p = hnorm_of(x, a[kNorm], tensor(a[kWeight], "weight"), a[kAct], a[kEps]);
    const at::Device dev = x.device();
    const at::ScalarType io = x.scalar_type();
    const void *const xp = head_rows("x", a[kX], dev, io, x.sizes(), &p.x_stride), *const zp = head_rows("z", a[kZ], dev, io, x.sizes(), &p.z_stride);
    const float* const w = head_vector("weight", a[kWeight], dev, p);
    at::Tensor y;
    void* yp = head_rows("y", a[kY], dev, io, x.sizes(), &p.y_stride);
    if (a[kY] == Py_None) {
      y = empty(x.sizes(), dev, io);
      yp = y.data_ptr();
    }
    on_device("x", dev);
    const auto fn = function<decltype(&pdn_head_norm)>(a[kFn]);
    void* const stream = function<void*>(a[kStream]);
    pdn_status status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(&p, xp, zp, w, yp, stream);
    Py_END_ALLOW_THREADS
    if (status != PDN_OK) return PyLong_FromLong(status);
    return result(a[kY], y);
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// pdn_head_norm_bwd: a dict of gradients, or a status that is not PDN_OK
PyObject* head_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kSizeFn, kDy, kX, kNorm, kWeight, kZ, kAct, kEps, kWantVectors, kDx, kDz, kDw, kWorkspace, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor& x = given(a[kX], "x");
    given(a[kDy], "dy");
    pdn_hnorm p = hnorm_of(x, a[kNorm], tensor(a[kWeight], "weight"), a[kAct], a[kEps]);
    const at::Device dev = x.device();
    const at::ScalarType io = x.scalar_type();
    const void *const dyp = head_rows("dy", a[kDy], dev, io, x.sizes(), &p.dy_stride), *const xp = head_rows("x", a[kX], dev, io, x.sizes(), &p.x_stride),
               *const zp = head_rows("z", a[kZ], dev, io, x.sizes(), &p.z_stride);
    const float* const w = head_vector("weight", a[kWeight], dev, p);
    at::Tensor dx, dz, dw;
    void* dxp = head_rows("dx", a[kDx], dev, io, x.sizes(), &p.dx_stride);
    if (!dxp && a[kDx] == Py_None) {
      dx = empty(x.sizes(), dev, io);
      dxp = dx.data_ptr();
    }
    void* dzp = head_rows("dz", a[kDz], dev, io, x.sizes(), &p.dz_stride);
    if (a[kDz] == Py_None && a[kZ] != Py_None) {
      dz = empty(x.sizes(), dev, io);
      dzp = dz.data_ptr();
    }
    float* dwp = head_vector("dweight", a[kDw], dev, p);
    if (a[kDw] == Py_None && a[kWeight] != Py_None && truth(a[kWantVectors])) {
      dw = empty(THPVariable_Unpack(a[kWeight]).sizes(), dev, at::kFloat);
      dwp = dw.data_ptr<float>();
    }
    on_device("x", dev);
    size_t bytes = 0, has = 0;
    pdn_status status = function<decltype(&pdn_head_norm_bwd_workspace_size)>(a[kSizeFn])(&p, &bytes);
    if (status != PDN_OK) return PyLong_FromLong(status);
    const at::Tensor ws = workspace_of(a[kWorkspace], dev, dwp ? bytes : 0, &has);
    const auto fn = function<decltype(&pdn_head_norm_bwd)>(a[kFn]);
    void *const stream = function<void*>(a[kStream]), *const wp = ws.data_ptr();
    Py_BEGIN_ALLOW_THREADS
    status = fn(&p, dyp, xp, zp, w, dxp, dzp, dwp, wp, has, stream);
    Py_END_ALLOW_THREADS
    if (status != PDN_OK) return PyLong_FromLong(status);
    return grads({{"dx", {a[kDx], &dx}}, {"dz", {a[kDz], &dz}}, {"dweight", {a[kDw], &dw}}});
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// pdn_logits: out, or a status that is not PDN_OK
PyObject* logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kSizeFn, kLogits, kProbs, kTemperature, kRepetition, kPresence, kFrequency, kCounts, kSlots, kIds, kStarts, kBiasStarts,
           kBiasIds, kBiasValues, kMask, kMaskRows, kOut, kOutType, kWorkspace, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor& l = given(a[kLogits], "logits");
    if (l.dim() != 2) refuse(PyExc_ValueError, "logits must be [rows, V]");
    const at::Device dev = l.device();
    pdn_logits_args p{};
    p.rows = l.size(0);
    p.V = l.size(1);
    p.dtype = io_of(l);
    p.probs = truth(a[kProbs]);
    p.logits = l.data_ptr();
    if (!l.is_contiguous()) {
      if (l.stride(1) != 1 && p.V > 1) refuse(PyExc_ValueError, "a row of logits must be dense");
      if (p.rows > 1 && l.stride(0) < p.V) refuse(PyExc_ValueError, "a row of logits must not overlap another's");
      p.stride = p.rows > 1 ? l.stride(0) : 0;
    }
    // how many sequences: by what there is one of for each
    int64_t N = p.rows;
    for (int i : {kFrequency, kPresence, kRepetition, kTemperature, kSlots})
      if (const at::Tensor* t = tensor(a[i], "a list of the sequences")) N = t->numel();
    if (const at::Tensor* t = tensor(a[kStarts], "starts")) N = t->numel() - 1;
    if (N < 0) refuse(PyExc_ValueError, "starts must hold one entry more than sequences");
    p.N = N;
    const at::ScalarType f32 = at::kFloat, i32 = at::kInt;
    const int64_t seqs[] = {N}, ends[] = {N + 1}, rows[] = {p.rows}, words = (p.V + 31) / 32;
    p.starts = on<int32_t>("starts", a[kStarts], dev, i32, ends);
    p.temperature = on<float>("temperature", a[kTemperature], dev, f32, seqs);
    p.repetition = on<float>("repetition", a[kRepetition], dev, f32, seqs);
    p.presence = on<float>("presence", a[kPresence], dev, f32, seqs);
    p.frequency = on<float>("frequency", a[kFrequency], dev, f32, seqs);
    if (const at::Tensor* t = tensor(a[kCounts], "counts")) {
      if (t->dim() != 2) refuse(PyExc_ValueError, "counts must be [slots, V]");
      p.slots = t->size(0);
      const int64_t table[] = {p.slots, p.V};
      p.counts = on<int32_t>("counts", a[kCounts], dev, i32, table);
    }
    p.slot = on<int32_t>("slots", a[kSlots], dev, i32, seqs);
    p.ids = on<int32_t>("ids", a[kIds], dev, i32, rows);
    if (a[kBiasStarts] != Py_None) {
      p.biases = given(a[kBiasIds], "bias ids").numel();
      given(a[kBiasValues], "bias values");
      const int64_t list[] = {p.biases};
      p.bias_starts = on<int32_t>("bias starts", a[kBiasStarts], dev, i32, ends);
      p.bias_ids = on<int32_t>("bias ids", a[kBiasIds], dev, i32, list);
      p.bias_values = on<float>("bias values", a[kBiasValues], dev, f32, list);
    }
    if (const at::Tensor* t = tensor(a[kMask], "mask")) {
      if (t->dim() != 2) refuse(PyExc_ValueError, "mask must be [masks, words]");
      p.masks = t->size(0);
      const int64_t bits[] = {p.masks, words};
      p.mask = on<int32_t>("mask", a[kMask], dev, i32, bits);
    }
    p.mask_rows = on<int32_t>("mask_rows", a[kMaskRows], dev, i32, rows);
    const int64_t named = whole(a[kOutType]);   // (-1: not named)
    const at::Tensor* const o = tensor(a[kOut], "out");
    p.out_dtype = o ? io_of(*o) : named >= 0 ? static_cast<pdn_dtype>(named) : p.probs ? PDN_F32 : p.dtype;
    if (named >= 0 && named != p.out_dtype) refuse(PyExc_TypeError, "dtype must be out's");
    const int64_t shape[] = {p.rows, p.V};
    at::Tensor made;
    void* const op = out_or_new("out", a[kOut], dev, scalar_of(p.out_dtype), shape, &made);
    on_device("logits", dev);
    size_t bytes = 0, has = 0;
    pdn_status status = function<decltype(&pdn_logits_workspace_size)>(a[kSizeFn])(p.rows, p.V, &bytes);
    if (status != PDN_OK) return PyLong_FromLong(status);
    const at::Tensor ws = workspace_of(a[kWorkspace], dev, p.probs ? bytes : 0, &has);
    const auto fn = function<decltype(&pdn_logits)>(a[kFn]);
    void *const stream = function<void*>(a[kStream]), *const wp = ws.data_ptr();
    Py_BEGIN_ALLOW_THREADS
    status = fn(&p, op, wp, has, stream);
    Py_END_ALLOW_THREADS
    if (status != PDN_OK) return PyLong_FromLong(status);
    return result(a[kOut], made);
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// pdn_token_counts: counts, or a status that is not PDN_OK
PyObject* token_counts(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    enum { kFn, kIds, kCounts, kStarts, kSlots, kSlotsOut, kFresh, kAccepted, kPrompt, kStream, kCount };
    if (n != kCount) refuse(PyExc_TypeError, "wrong number of arguments");
    const at::Tensor &ids = given(a[kIds], "ids"), &counts = given(a[kCounts], "counts");
    if (counts.dim() != 2) refuse(PyExc_ValueError, "counts must be [slots, V]");
    const at::Device dev = counts.device();
    const int64_t M = ids.numel(), P = counts.size(0), V = counts.size(1);
    int64_t N = M;
    for (int i : {kAccepted, kFresh, kSlotsOut, kSlots})
      if (const at::Tensor* t = tensor(a[i], "a list of the sequences")) N = t->numel();
    if (const at::Tensor* t = tensor(a[kStarts], "starts")) N = t->numel() - 1;
    if (N < 0) refuse(PyExc_ValueError, "starts must hold one entry more than sequences");
    const at::ScalarType i32 = at::kInt;
    const int64_t rows[] = {M}, seqs[] = {N}, ends[] = {N + 1};
    const int32_t *const ip = on<int32_t>("ids", a[kIds], dev, i32, rows), *const sp = on<int32_t>("starts", a[kStarts], dev, i32, ends),
                  *const from = on<int32_t>("slots", a[kSlots], dev, i32, seqs), *const to = on<int32_t>("slots_out", a[kSlotsOut], dev, i32, seqs),
                  *const fresh = on<int32_t>("fresh", a[kFresh], dev, i32, seqs), *const acc = on<int32_t>("accepted", a[kAccepted], dev, i32, seqs);
    int32_t* const cp = on<int32_t>("counts", a[kCounts], dev, i32, counts.sizes());
    on_device("counts", dev);
    const bool prompt = truth(a[kPrompt]);
    const auto fn = function<decltype(&pdn_token_counts)>(a[kFn]);
    void* const stream = function<void*>(a[kStream]);
    pdn_status status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(N, M, V, P, prompt, ip, sp, from, to, fresh, acc, cp, stream);
    Py_END_ALLOW_THREADS
    if (status != PDN_OK) return PyLong_FromLong(status);
    Py_INCREF(a[kCounts]);
    return a[kCounts];
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"slot", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slot)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, nullptr},
    {"residual_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(residual_norm)), METH_FASTCALL, nullptr},
    {"residual_norm_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(residual_norm_bwd)), METH_FASTCALL, nullptr},
    {"head_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_norm)), METH_FASTCALL, nullptr},
    {"head_norm_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_norm_bwd)), METH_FASTCALL, nullptr},
    {"logits", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(logits)), METH_FASTCALL, nullptr},
    {"token_counts", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_counts)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pdn_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pdn_torch() { return PyModule_Create(&module); }
