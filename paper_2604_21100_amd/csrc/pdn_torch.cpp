// The calls on a pool of states, from torch tensors: what the binding does for
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

PyMethodDef methods[] = {
    {"slot", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slot)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pdn_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pdn_torch() { return PyModule_Create(&module); }
