// C ABI of libpdn: argument validation (host only, before any HIP call),
// workspace sizing and kernel sequencing.  See include/pdn.h.
#include "../../include/pdn.h"

#include <hip/hip_runtime.h>

#include <array>
#include <cmath>
#include <cstdint>
#include <vector>

#include "pdn_checks.hpp"
#include "pdn_internal.hpp"

namespace {

using namespace pdn;   // (the checks)

static_assert(PDN_NOALLOC_SCRATCH_BYTES == pdn::kNoallocScratchBytes,
              "the header's scratch size and the library's must agree");

struct Sizes {
  int64_t BH, NT, tok;        // tok = B*T*H
  int64_t nq, nv, nscal, ngate, nS, nA;
  int esz;
};

// types, head sizes, modes and their numbers; `chunked`: the chunk too
pdn_status check_mode(const pdn_problem* p, bool chunked) {
  if (!p) return PDN_ERR_NULL;
  if (p->B < 0 || p->T < 0 || p->H < 0) return PDN_ERR_SHAPE;
  if (p->io != PDN_F32 && p->io != PDN_BF16) return PDN_ERR_DTYPE;
  if ((p->dk != 64 && p->dk != 128) || (p->dv != 64 && p->dv != 128)) return PDN_ERR_UNSUPPORTED;
  if (chunked && !pdn::chunk_supported(p->chunk)) return PDN_ERR_UNSUPPORTED;
  if (p->gate != PDN_GATE_NONE && p->gate != PDN_GATE_SCALAR && p->gate != PDN_GATE_CHANNEL)
    return PDN_ERR_VALUE;
  if (p->precond != PDN_PRECOND_SQUASH && p->precond != PDN_PRECOND_IDENTITY &&
      p->precond != PDN_PRECOND_EXTERNAL && p->precond != PDN_PRECOND_DIAG_SM &&
      p->precond != PDN_PRECOND_ATQ)
    return PDN_ERR_VALUE;
  if (!std::isfinite(p->x) || !(p->x >= 1.0f) || !std::isfinite(p->scale)) return PDN_ERR_VALUE;
  if ((p->precond == PDN_PRECOND_DIAG_SM || p->precond == PDN_PRECOND_ATQ) &&
      (!std::isfinite(p->ridge) || !(p->ridge > 0.0f)))
    return PDN_ERR_VALUE;
  if (p->knorm < PDN_KNORM_NONE || p->knorm > PDN_KNORM_BETA) return PDN_ERR_VALUE;
  if (p->knorm != PDN_KNORM_NONE && p->precond != PDN_PRECOND_SQUASH) return PDN_ERR_VALUE;
  if (p->knorm == PDN_KNORM_BETA && p->gate == PDN_GATE_CHANNEL) return PDN_ERR_UNSUPPORTED;
  return PDN_OK;
}

pdn_status check_problem(const pdn_problem* p, Sizes* sz) {
  const pdn_status st = check_mode(p, true);
  if (st != PDN_OK) return st;
  Sizes s{};
  int64_t bt;
  if (!mul_ok(p->B, p->H, &s.BH) || !mul_ok(p->B, p->T, &bt) || !mul_ok(bt, p->H, &s.tok))
    return PDN_ERR_SHAPE;
  s.NT = (p->T + p->chunk - 1) / p->chunk;
  int64_t tpad;
  if (!mul_ok(s.NT, p->chunk, &tpad)) return PDN_ERR_SHAPE;
  // every element count used below must fit in int64 (with a generous margin
  // for the workspace's byte counts)
  int64_t tmp;
  if (!mul_ok(s.tok, 128, &s.nq) || !mul_ok(s.BH, tpad, &tmp) || !mul_ok(tmp, 128 * 8, &tmp) ||
      !mul_ok(s.BH, 128 * 128 * 4, &tmp))
    return PDN_ERR_SHAPE;
  if (s.NT > (int64_t)1 << 30 || s.BH * s.NT > (int64_t)INT32_MAX) return PDN_ERR_SHAPE;
  s.nq = s.tok * p->dk;
  s.nv = s.tok * p->dv;
  s.nscal = s.tok;
  s.ngate = p->gate == PDN_GATE_NONE ? 0 : (p->gate == PDN_GATE_SCALAR ? s.tok : s.tok * p->dk);
  s.nS = s.BH * p->dk * p->dv;
  s.nA = s.BH * p->dk;
  s.esz = p->io == PDN_BF16 ? 2 : 4;
  *sz = s;
  return PDN_OK;
}

pdn_status check_inputs(const pdn_problem* p, const pdn_inputs* in, const Sizes& s,
                        std::vector<Buf>* bufs) {
  if (!in) return PDN_ERR_NULL;
  const bool empty = s.tok == 0;
  // per-token tensors are only dereferenced when there are tokens
  if (!empty) {
    if (!in->q || !in->k || !in->v || !in->beta) return PDN_ERR_NULL;
    if (p->gate != PDN_GATE_NONE && !in->g) return PDN_ERR_NULL;
    if (pdn::has_gram(p->precond) && !in->beta_p) return PDN_ERR_NULL;
    if (p->precond == PDN_PRECOND_SQUASH && !in->log_a_scale) return PDN_ERR_NULL;
    if (p->precond == PDN_PRECOND_EXTERNAL && !in->ktilde) return PDN_ERR_NULL;
  }
  if (p->gate == PDN_GATE_NONE && in->g) return PDN_ERR_VALUE;
  const int64_t e = s.esz;
  std::vector<Buf> b = {
      {in->q, s.nq * e}, {in->k, s.nq * e}, {in->v, s.nv * e}, {in->beta, s.nscal * 4},
      {in->g, s.ngate * 4}, {in->S0, s.nS * 4},
  };
  if (pdn::has_gram(p->precond)) {
    b.push_back({in->beta_p, s.nscal * 4});
    b.push_back({in->g_p, s.nscal * 4});
    b.push_back({in->A0, s.nA * 4});
  }
  if (p->precond == PDN_PRECOND_SQUASH) b.push_back({in->log_a_scale, p->H * 4});
  if (p->precond == PDN_PRECOND_EXTERNAL) b.push_back({in->ktilde, s.nq * e});
  for (const Buf& x : b)
    if (x.p && !aligned16(x.p)) return PDN_ERR_ALIGN;
  *bufs = b;
  return PDN_OK;
}

// the backward covers every gate kind and the SQUASH / IDENTITY / EXTERNAL
// write keys; fp32 io at head dims 64
pdn_status check_bwd_support(const pdn_problem* p) {
  if (p->io == PDN_F32 && (p->dk != 64 || p->dv != 64)) return PDN_ERR_UNSUPPORTED;
  if (p->precond == PDN_PRECOND_DIAG_SM || p->precond == PDN_PRECOND_ATQ) return PDN_ERR_UNSUPPORTED;
  if (p->knorm != PDN_KNORM_NONE) return PDN_ERR_UNSUPPORTED;
  return PDN_OK;
}

// ---- calls on a pool of states
struct SlotSizes {
  int64_t nq, nk, nv, no, nx;       // bytes the token tensors span
  int64_t nscal, ngate, ngram;      // per-token fp32 tensors, bytes
  int64_t nS, nA, ntape, npend, nseq;
  int64_t qs, ks, vs;               // token strides
};

// rows x stride (the last row: its own width), in bytes
bool span_ok(int64_t rows, int64_t stride, int64_t width, int esz, int64_t* out) {
  if (rows == 0) {
    *out = 0;
    return true;
  }
  int64_t x;
  if (!mul_ok(rows - 1, stride, &x) || x > INT64_MAX / 16 - width) return false;
  *out = (x + width) * esz;
  return true;
}

pdn_status check_slots(const pdn_problem* p, const pdn_slots* s, bool draft, SlotSizes* out) {
  const pdn_status st = check_mode(p, false);
  if (st != PDN_OK) return st;
  if (!s) return PDN_ERR_NULL;
  if (s->tokens < 0 || s->slots < 0 || s->Hk < 0) return PDN_ERR_SHAPE;
  const int64_t Hk = s->Hk ? s->Hk : p->H;
  if (p->H > 0 && p->H % Hk != 0) return PDN_ERR_SHAPE;
  // row numbers and slots are 32-bit on the device; one workgroup of at most 768
  // work items a head, of which a launch holds fewer than 2^32.  (T is only where a
  // sequence is cut: any number.)
  int64_t heads;
  if (s->tokens > INT32_MAX || s->slots > INT32_MAX || p->B > INT32_MAX || !mul_ok(p->B, p->H, &heads) ||
      heads >= (int64_t)1 << 22)
    return PDN_ERR_SHAPE;
  int64_t even;
  if (!s->starts && (!mul_ok(p->B, p->T, &even) || even != s->tokens)) return PDN_ERR_SHAPE;
  if (!s->slot && p->B > s->slots) return PDN_ERR_SHAPE;
  SlotSizes z{};
  const int esz = p->io == PDN_BF16 ? 2 : 4;
  int64_t wq, wv, tok, slots_h, rec;
  if (!mul_ok(Hk, p->dk, &wq) || !mul_ok(p->H, p->dv, &wv) || !mul_ok(s->tokens, p->H, &tok) ||
      !mul_ok(s->slots, p->H, &slots_h))
    return PDN_ERR_SHAPE;
  z.qs = s->q_stride ? s->q_stride : wq;
  z.ks = s->k_stride ? s->k_stride : wq;
  z.vs = s->v_stride ? s->v_stride : wv;
  // (a few rows are seen through a buffer of 32-bit offsets)
  const int64_t far = (int64_t)1 << 25;
  if (z.qs < wq || z.ks < wq || z.vs < wv || z.qs > far || z.ks > far || z.vs > far || wq > far || wv > far ||
      p->H * (int64_t)p->dk > far)
    return PDN_ERR_SHAPE;
  if (z.qs * esz % 16 || z.ks * esz % 16 || z.vs * esz % 16) return PDN_ERR_ALIGN;
  if (!span_ok(s->tokens, z.qs, wq, esz, &z.nq) || !span_ok(s->tokens, z.ks, wq, esz, &z.nk) ||
      !span_ok(s->tokens, z.vs, wv, esz, &z.nv) || !span_ok(s->tokens, wv, wv, esz, &z.no) ||
      !span_ok(s->tokens, wq, wq, esz, &z.nx) || !mul_ok(tok, 4 * 128, &z.nscal) ||
      !mul_ok(slots_h, (int64_t)4 * 128 * 128, &z.nS))
    return PDN_ERR_SHAPE;
  z.nscal = tok * 4;
  z.ngate = p->gate == PDN_GATE_NONE ? 0 : p->gate == PDN_GATE_SCALAR ? tok * 4 : tok * 4 * p->dk;
  z.nS = slots_h * p->dk * p->dv * 4;
  z.nA = slots_h * p->dk * 4;
  z.nseq = p->B * 4;
  if (draft) {
    if (s->tape_tokens > INT32_MAX || p->T > s->tape_tokens || s->tape_tokens < 1) return PDN_ERR_SHAPE;
    if (!mul_ok(slots_h, s->tape_tokens, &rec) || !mul_ok(rec, 4 * 512, &z.ntape)) return PDN_ERR_SHAPE;
    z.ntape = rec * 4 * (p->dk + p->dv + (p->gate == PDN_GATE_CHANNEL ? p->dk : 4) +
                         (pdn::has_gram(p->precond) ? p->dk : 0));
    z.npend = slots_h * 4;
  }
  *out = z;
  return PDN_OK;
}

pdn_status slot_call(const pdn_problem* p, const pdn_inputs* in, const pdn_slots* s, void* o, bool draft,
                     void* hip_stream) {
  SlotSizes z;
  pdn_status st = check_slots(p, s, draft, &z);
  if (st != PDN_OK) return st;
  if (!in) return PDN_ERR_NULL;
  const bool gram = pdn::has_gram(p->precond), some = s->tokens > 0 && p->H > 0;
  const bool work = p->B > 0 && p->H > 0 && s->slots > 0;
  if (some) {
    if (!in->q || !in->k || !in->v || !in->beta || !o) return PDN_ERR_NULL;
    if (p->gate != PDN_GATE_NONE && !in->g) return PDN_ERR_NULL;
    if (gram && !in->beta_p) return PDN_ERR_NULL;
    if (p->precond == PDN_PRECOND_EXTERNAL && !in->ktilde) return PDN_ERR_NULL;
  }
  if (work) {
    if (!s->S || (gram && !s->A)) return PDN_ERR_NULL;
    if (p->precond == PDN_PRECOND_SQUASH && !in->log_a_scale) return PDN_ERR_NULL;
    if (draft && (!s->pending || !s->tape)) return PDN_ERR_NULL;
  }
  if (p->gate == PDN_GATE_NONE && in->g) return PDN_ERR_VALUE;
  // the states are the pool's
  if (in->S0 || in->A0) return PDN_ERR_VALUE;
  if (!gram && s->A) return PDN_ERR_VALUE;
  if (!draft && (s->tape || s->pending || s->accepted)) return PDN_ERR_VALUE;
  const Buf none{nullptr, 0};   // (what a mode does not read is not looked at)
  constexpr size_t kTensors = 9;
  const std::array<Buf, kTensors + 5> ins = {{
      {in->q, z.nq}, {in->k, z.nk}, {in->v, z.nv}, {in->beta, z.nscal}, {in->g, z.ngate},
      gram ? Buf{in->beta_p, z.nscal} : none, gram ? Buf{in->g_p, z.nscal} : none,
      p->precond == PDN_PRECOND_SQUASH ? Buf{in->log_a_scale, p->H * 4} : none,
      p->precond == PDN_PRECOND_EXTERNAL ? Buf{in->ktilde, z.nx} : none,
      // lists
      {s->starts, (p->B + 1) * 4}, {s->slot, z.nseq}, {s->slot_out, z.nseq}, {s->fresh, z.nseq}, {s->accepted, z.nseq}}};
  const std::array<Buf, 5> outs = {{{o, z.no}, {s->S, z.nS}, {s->A, z.nA}, {s->tape, z.ntape}, {s->pending, z.npend}}};
  for (size_t i = 0; i < ins.size(); ++i)
    if (ins[i].p && (reinterpret_cast<uintptr_t>(ins[i].p) & (i < kTensors ? 15u : 3u))) return PDN_ERR_ALIGN;
  for (const Buf& x : outs)
    if (x.p && !aligned16(x.p)) return PDN_ERR_ALIGN;
  if ((st = check_aliasing(ins, outs, Buf{nullptr, 0})) != PDN_OK) return st;
  if (!work) return PDN_OK;

  pdn::SlotArgs a{};
  a.B = p->B; a.T = p->T < INT32_MAX ? p->T : INT32_MAX; a.H = p->H; a.Hk = s->Hk ? s->Hk : p->H;
  a.tokens = s->tokens; a.slots = s->slots;
  a.q_stride = z.qs; a.k_stride = z.ks; a.v_stride = z.vs;
  a.dk = p->dk; a.dv = p->dv;
  a.gate = p->gate; a.precond = p->precond; a.knorm = p->knorm;
  a.lnx = std::log(p->x);
  a.scale = p->scale;
  a.ridge = p->ridge;
  a.q = in->q; a.k = in->k; a.v = in->v; a.ktilde = in->ktilde;
  a.beta = in->beta; a.g = in->g; a.beta_p = in->beta_p; a.g_p = in->g_p;
  a.log_a_scale = in->log_a_scale;
  a.starts = s->starts; a.slot = s->slot; a.slot_out = s->slot_out; a.fresh = s->fresh;
  a.S = s->S; a.A = s->A; a.o = o;
  if (draft) {
    a.tape = s->tape;
    a.pending = s->pending;
    a.accepted = s->accepted;
    a.tape_tokens = s->tape_tokens;
  }
  return pdn::launch_slots(a, p->io == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK
                                                                                                     : PDN_ERR_HIP;
}

}  // namespace

extern "C" {

const char* pdn_status_string(pdn_status st) {
  switch (st) {
    case PDN_OK: return "ok";
    case PDN_ERR_NULL: return "a required pointer is NULL";
    case PDN_ERR_SHAPE: return "invalid or overflowing shape";
    case PDN_ERR_DTYPE: return "unknown io dtype";
    case PDN_ERR_UNSUPPORTED: return "head dimension, chunk size or mode not supported (dk, dv in {64, 128}; chunk 32 or 64)";
    case PDN_ERR_ALIGN: return "a tensor is not 16-byte aligned";
    case PDN_ERR_ALIAS: return "an output overlaps an input, another output or the workspace";
    case PDN_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case PDN_ERR_VALUE: return "invalid scalar, enum or gate pointer";
    case PDN_ERR_HIP: return "HIP launch failed";
    case PDN_ERR_SCRATCH:
      return "problem needs more workspace than the no-allocation entry point's fixed scratch "
             "(pdn_noalloc_scratch_bytes(), 64 MiB per device)";
  }
  return "unknown status";
}

int pdn_abi_version(void) { return PDN_ABI_VERSION; }

pdn_status pdn_workspace_size(const pdn_problem* p, int with_bwd, size_t* bytes) {
  if (!bytes) return PDN_ERR_NULL;
  Sizes s;
  const pdn_status st = check_problem(p, &s);
  if (st != PDN_OK) return st;
  if (with_bwd) {
    const pdn_status sb = check_bwd_support(p);
    if (sb != PDN_OK) return sb;
    *bytes = pdn::bwd_ws_layout(s.BH, static_cast<int>(s.NT), p->dk, p->dv, s.esz, p->gate, p->precond, p->chunk).total;
    return PDN_OK;
  }
  const pdn::WsLayout L = pdn::fwd_ws_layout(s.BH, static_cast<int>(s.NT), p->dk, p->dv, s.esz, p->gate,
                                             p->precond, p->chunk);
  *bytes = L.total;
  return PDN_OK;
}

pdn_status pdn_scan_segments(const pdn_problem* p, int* segments) {
  if (!segments) return PDN_ERR_NULL;
  Sizes s;
  const pdn_status st = check_problem(p, &s);
  if (st != PDN_OK) return st;
  *segments = s.tok > 0 ? pdn::scan_split(s.BH, static_cast<int>(s.NT), p->dk, p->dv).S : 1;
  return PDN_OK;
}

// Forward intermediates the backward kernels read: the forward workspace
// plus the residual arrays of the backward layout.
static void set_forward_ws(pdn::FwdArgs& a, const pdn::WsLayout& L, const pdn_problem* p, char* w) {
  if (p->precond == PDN_PRECOND_ATQ) a.Qt = w + L.Qt;
  if (p->gate == PDN_GATE_CHANNEL) {
    a.QL = w + L.QL;
    a.KL = w + L.KL;
  }
  if (pdn::has_gram(p->precond)) {
    a.sumL = reinterpret_cast<float*>(w + L.sumL);
    a.sumD = reinterpret_cast<float*>(w + L.sumD);
    a.Abound = reinterpret_cast<float*>(w + L.Abound);
  }
  if (p->io == PDN_BF16) {
    a.Kd = w + L.KtG;
    a.forms_p = pdn::scan_forms_p(a.BH, a.NT, a.dv, a.gate, a.precond);
  }
  else a.KtG = w + L.KtG;
  a.Tm = w + L.Tm;
  a.Pm = w + L.Pm;
  if (p->gate != PDN_GATE_NONE) a.G = reinterpret_cast<float*>(w + L.G);
  if (L.split.S > 1) {
    a.seg_cnt = L.split.S;
    a.seg_len = L.split.L;
    a.seg_end = reinterpret_cast<float*>(w + L.seg_end);
    a.seg_phi = reinterpret_cast<float*>(w + L.seg_phi);
    a.seg_start = reinterpret_cast<float*>(w + L.seg_start);
  }
}

static void set_residuals(pdn::FwdArgs& f, const pdn::BwdWsLayout& L, char* w) {
  f.Hs = w + L.Hs; f.Er = w + L.Er;
  f.Ktr = w + L.Ktr;
  if (!f.Kd) {   // fp32
    if (f.gate == pdn::kGateChannel) f.Kw = w + L.Kw;
    f.PtT = w + L.PtT; f.MtT = w + L.MtT; f.QlT = w + L.QlT; f.KnT = w + L.KnT;
  }
}

// train: the training forward (also leaves the backward's intermediates in
// the workspace, which then has the backward's size).  noalloc: ws and
// ws_bytes are ignored; the workspace is the device's fixed scratch array,
// looked up only after every argument has been validated.
static pdn_status chunk_fwd_impl(const pdn_problem* p, const pdn_inputs* in, pdn_fwd_out* out,
                                 void* ws, size_t ws_bytes, void* hip_stream,
                                 hipEvent_t const* ev, bool train, bool noalloc = false) {
  Sizes s;
  pdn_status st = check_problem(p, &s);
  if (st != PDN_OK) return st;
  std::vector<Buf> ins;
  if ((st = check_inputs(p, in, s, &ins)) != PDN_OK) return st;
  if (train && (st = check_bwd_support(p)) != PDN_OK) return st;
  if (!out) return PDN_ERR_NULL;
  if (s.tok > 0 && !out->o) return PDN_ERR_NULL;
  if (!pdn::has_gram(p->precond) && out->A_T) return PDN_ERR_VALUE;
  const std::vector<Buf> outs = {{out->o, s.nv * s.esz}, {out->S_T, s.nS * 4}, {out->A_T, s.nA * 4}};
  for (const Buf& x : outs)
    if (x.p && !aligned16(x.p)) return PDN_ERR_ALIGN;
  const pdn::WsLayout L = pdn::fwd_ws_layout(s.BH, static_cast<int>(s.NT), p->dk, p->dv, s.esz, p->gate,
                                             p->precond, p->chunk);
  const pdn::BwdWsLayout LB =
      pdn::bwd_ws_layout(s.BH, static_cast<int>(s.NT), p->dk, p->dv, s.esz, p->gate, p->precond, p->chunk);
  const size_t need_bytes = train ? LB.total : L.total;
  const bool need_ws = s.tok > 0;
  if (noalloc) {
    ws = nullptr;
    ws_bytes = 0;
    if (need_ws && need_bytes > pdn::kNoallocScratchBytes) return PDN_ERR_SCRATCH;
  }
  // the whole declared workspace range must be disjoint from inputs/outputs;
  // its size is checked last
  if ((st = check_aliasing(ins, outs, Buf{ws, need_ws ? static_cast<int64_t>(ws_bytes) : 0})) != PDN_OK)
    return st;
  if (noalloc && need_ws) {
    // every argument is valid: the first HIP call of this entry point (the
    // scratch array belongs to the library, so it overlaps no caller buffer)
    if (pdn::noalloc_scratch(&ws) != hipSuccess) return PDN_ERR_HIP;
    ws_bytes = pdn::kNoallocScratchBytes;
  }
  if (need_ws && (!ws || ws_bytes < need_bytes || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0))
    return PDN_ERR_WORKSPACE;

  pdn::FwdArgs a{};
  a.B = p->B; a.T = p->T; a.H = p->H; a.BH = s.BH;
  a.chunk = p->chunk;
  a.NT = static_cast<int>(s.NT);
  a.Tpad = s.NT * p->chunk;
  a.dk = p->dk; a.dv = p->dv;
  a.gate = p->gate; a.precond = p->precond;
  a.lnx = std::log(p->x);
  a.scale = p->scale;
  a.ridge = p->ridge;
  a.knorm = p->knorm;
  a.q = in->q; a.k = in->k; a.v = in->v; a.ktilde = in->ktilde;
  a.beta = in->beta; a.g = in->g; a.beta_p = in->beta_p; a.g_p = in->g_p;
  a.log_a_scale = in->log_a_scale; a.A0 = in->A0; a.S0 = in->S0;
  a.o = out->o; a.S_T = out->S_T; a.A_T = out->A_T;
  char* w = static_cast<char*>(ws);
  if (need_ws) {
    set_forward_ws(a, train ? LB.f : L, p, w);
    if (train) set_residuals(a, LB, w);
  }
  const hipError_t e =
      pdn::launch_forward(a, p->io == PDN_BF16, static_cast<hipStream_t>(hip_stream), ev, train);
  return e == hipSuccess ? PDN_OK : PDN_ERR_HIP;
}

pdn_status pdn_chunk_fwd(const pdn_problem* p, const pdn_inputs* in, pdn_fwd_out* out, void* ws,
                         size_t ws_bytes, void* hip_stream) {
  return chunk_fwd_impl(p, in, out, ws, ws_bytes, hip_stream, nullptr, false);
}

pdn_status pdn_chunk_fwd_noalloc(const pdn_problem* p, const pdn_inputs* in, pdn_fwd_out* out,
                                 void* hip_stream) {
  return chunk_fwd_impl(p, in, out, nullptr, 0, hip_stream, nullptr, false, true);
}

size_t pdn_noalloc_scratch_bytes(void) { return pdn::kNoallocScratchBytes; }

pdn_status pdn_chunk_fwd_events(const pdn_problem* p, const pdn_inputs* in, pdn_fwd_out* out,
                                void* ws, size_t ws_bytes, void* hip_stream,
                                void* const* stage_events, int n_events) {
  if (!stage_events) return PDN_ERR_NULL;
  if (n_events != PDN_FWD_STAGE_EVENTS) return PDN_ERR_VALUE;
  return chunk_fwd_impl(p, in, out, ws, ws_bytes, hip_stream,
                        reinterpret_cast<hipEvent_t const*>(stage_events), false);
}

// saved: the forward intermediates are in ws already (training forward)
static pdn_status chunk_bwd_impl(const pdn_problem* p, const pdn_inputs* in, const void* dO,
                                 const float* dS_T, pdn_bwd_out* out, void* ws, size_t ws_bytes,
                                 void* hip_stream, hipEvent_t const* ev, bool saved) {
  Sizes s;
  pdn_status st = check_problem(p, &s);
  if (st != PDN_OK) return st;
  std::vector<Buf> ins;
  if ((st = check_inputs(p, in, s, &ins)) != PDN_OK) return st;
  if ((st = check_bwd_support(p)) != PDN_OK) return st;
  if (!out) return PDN_ERR_NULL;
  const bool tok = s.tok > 0;
  if (tok && (!dO || !out->dq || !out->dk || !out->dv || !out->dbeta)) return PDN_ERR_NULL;
  if (tok && p->gate != PDN_GATE_NONE && !out->dg) return PDN_ERR_NULL;
  if (p->gate == PDN_GATE_NONE && out->dg) return PDN_ERR_VALUE;
  const bool sq = p->precond == PDN_PRECOND_SQUASH;
  if (!sq && (out->dbeta_p || out->dg_p || out->dlog_a_scale || out->dA0)) return PDN_ERR_VALUE;
  if (p->precond != PDN_PRECOND_EXTERNAL && out->dktilde) return PDN_ERR_VALUE;
  ins.push_back({dO, s.nv * s.esz});
  ins.push_back({dS_T, s.nS * 4});
  const int64_t e = s.esz;
  const std::vector<Buf> outs = {
      {out->dq, s.nq * e},        {out->dk, s.nq * e},          {out->dv, s.nv * e},
      {out->dbeta, s.nscal * 4},  {out->dg, s.ngate * 4},       {out->dS0, s.nS * 4},
      {out->dbeta_p, s.nscal * 4}, {out->dg_p, s.nscal * 4},    {out->dlog_a_scale, p->H * 4},
      {out->dA0, s.nA * 4},       {out->dktilde, s.nq * e}};
  for (const Buf& x : outs)
    if (x.p && !aligned16(x.p)) return PDN_ERR_ALIGN;
  for (const Buf& x : ins)
    if (x.p && !aligned16(x.p)) return PDN_ERR_ALIGN;
  const pdn::BwdWsLayout L =
      pdn::bwd_ws_layout(s.BH, static_cast<int>(s.NT), p->dk, p->dv, s.esz, p->gate, p->precond, p->chunk);
  if ((st = check_aliasing(ins, outs, Buf{ws, tok ? static_cast<int64_t>(ws_bytes) : 0})) != PDN_OK)
    return st;
  if (tok && (!ws || ws_bytes < L.total || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0))
    return PDN_ERR_WORKSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (s.BH == 0 || !tok) {
    if (ev)  // nothing to time: the stage events still mark the empty stages
      for (int k = 0; k < PDN_BWD_STAGE_EVENTS; ++k)
        if (ev[k] && hipEventRecord(ev[k], stream) != hipSuccess) return PDN_ERR_HIP;
  }
  if (s.BH == 0) return PDN_OK;
  if (!tok) {
    // T == 0: the state passes through unchanged
    pdn::FwdArgs f{};
    f.BH = s.BH; f.dk = p->dk; f.dv = p->dv;
    f.S0 = dS_T; f.S_T = out->dS0; f.A0 = nullptr; f.A_T = out->dA0;
    const hipError_t he = pdn::launch_forward(f, p->io == PDN_BF16, stream);
    return he == hipSuccess ? PDN_OK : PDN_ERR_HIP;
  }
  pdn::BwdArgs a{};
  pdn::FwdArgs& f = a.f;
  f.B = p->B; f.T = p->T; f.H = p->H; f.BH = s.BH;
  f.chunk = p->chunk;
  f.NT = static_cast<int>(s.NT);
  f.Tpad = s.NT * p->chunk;
  f.dk = p->dk; f.dv = p->dv;
  f.gate = p->gate; f.precond = p->precond;
  f.lnx = std::log(p->x);
  f.scale = p->scale;
  f.q = in->q; f.k = in->k; f.v = in->v; f.ktilde = in->ktilde;
  f.beta = in->beta; f.g = in->g; f.beta_p = in->beta_p; f.g_p = in->g_p;
  f.log_a_scale = in->log_a_scale; f.A0 = in->A0; f.S0 = in->S0;
  f.o = nullptr; f.S_T = nullptr; f.A_T = nullptr;
  char* w = static_cast<char*>(ws);
  set_forward_ws(f, L.f, p, w);
  set_residuals(f, L, w);
  a.dO = dO; a.dS_T = dS_T;
  a.dq = out->dq; a.dk = out->dk; a.dv = out->dv; a.dbeta = out->dbeta; a.dg = out->dg;
  a.dS0 = out->dS0; a.dbeta_p = out->dbeta_p; a.dg_p = out->dg_p; a.dlog_a_scale = out->dlog_a_scale;
  a.dA0 = out->dA0; a.dktilde = out->dktilde;
  a.dHs = w + L.dHs; a.Zr = w + L.Zr;
  a.dKt = w + L.dKt;
  a.dKm = w + L.dKm;
  a.pcL = reinterpret_cast<float*>(w + L.pcL);
  a.pcS = reinterpret_cast<float*>(w + L.pcS);
  a.pcA = reinterpret_cast<float*>(w + L.pcA);
  a.pcC = reinterpret_cast<float*>(w + L.pcC);
  a.pcMu = reinterpret_cast<float*>(w + L.pcMu);
  const hipError_t he = pdn::launch_backward(a, p->io == PDN_BF16, stream, ev, !saved);
  return he == hipSuccess ? PDN_OK : PDN_ERR_HIP;
}

pdn_status pdn_chunk_bwd(const pdn_problem* p, const pdn_inputs* in, const void* dO,
                         const float* dS_T, pdn_bwd_out* out, void* ws, size_t ws_bytes,
                         void* hip_stream) {
  return chunk_bwd_impl(p, in, dO, dS_T, out, ws, ws_bytes, hip_stream, nullptr, false);
}

pdn_status pdn_chunk_bwd_events(const pdn_problem* p, const pdn_inputs* in, const void* dO,
                                const float* dS_T, pdn_bwd_out* out, void* ws, size_t ws_bytes,
                                void* hip_stream, void* const* stage_events, int n_events) {
  if (!stage_events) return PDN_ERR_NULL;
  if (n_events != PDN_BWD_STAGE_EVENTS) return PDN_ERR_VALUE;
  return chunk_bwd_impl(p, in, dO, dS_T, out, ws, ws_bytes, hip_stream,
                        reinterpret_cast<hipEvent_t const*>(stage_events), false);
}

// stage_events: NULL (n_events 0) or an array of n_events == n entries
// (NULL entries are skipped)
static pdn_status check_events(void* const* ev, int n_events, int n) {
  if (!ev) return n_events == 0 ? PDN_OK : PDN_ERR_NULL;
  if (n_events != n) return PDN_ERR_VALUE;
  return PDN_OK;
}

pdn_status pdn_chunk_fwd_train(const pdn_problem* p, const pdn_inputs* in, pdn_fwd_out* out,
                               void* ws, size_t ws_bytes, void* hip_stream,
                               void* const* stage_events, int n_events) {
  const pdn_status st = check_events(stage_events, n_events, PDN_FWD_STAGE_EVENTS);
  if (st != PDN_OK) return st;
  return chunk_fwd_impl(p, in, out, ws, ws_bytes, hip_stream,
                        reinterpret_cast<hipEvent_t const*>(stage_events), true);
}

pdn_status pdn_chunk_bwd_train(const pdn_problem* p, const pdn_inputs* in, const void* dO,
                               const float* dS_T, pdn_bwd_out* out, void* ws, size_t ws_bytes,
                               void* hip_stream, void* const* stage_events, int n_events) {
  const pdn_status st = check_events(stage_events, n_events, PDN_BWD_STAGE_EVENTS);
  if (st != PDN_OK) return st;
  return chunk_bwd_impl(p, in, dO, dS_T, out, ws, ws_bytes, hip_stream,
                        reinterpret_cast<hipEvent_t const*>(stage_events), true);
}

pdn_status pdn_slot_fwd(const pdn_problem* p, const pdn_inputs* in, const pdn_slots* s, void* o,
                        void* hip_stream) {
  return slot_call(p, in, s, o, false, hip_stream);
}

pdn_status pdn_slot_draft(const pdn_problem* p, const pdn_inputs* in, const pdn_slots* s, void* o,
                          void* hip_stream) {
  return slot_call(p, in, s, o, true, hip_stream);
}

static pdn_status check_verify(int64_t N, int64_t rows, int64_t V, pdn_dtype dtype, bool even, int64_t* row_bytes,
                               int64_t* ws_bytes) {
  if (N < 0 || rows < 0 || V < 0) return PDN_ERR_SHAPE;
  if (dtype != PDN_F32 && dtype != PDN_BF16) return PDN_ERR_DTYPE;
  // ids and row numbers are 32-bit; a workgroup a segment and sequence
  int64_t blocks, bytes;
  if (N > INT32_MAX || rows > INT32_MAX || V > INT32_MAX || (V == 0 && rows > 0)) return PDN_ERR_SHAPE;
  if (!mul_ok(N, pdn::verify_blocks(V), &blocks) || blocks >= (int64_t)1 << 24 || N >= (int64_t)1 << 24)
    return PDN_ERR_SHAPE;
  if (!mul_ok(rows, V, &bytes) || !mul_ok(bytes, 4, &bytes)) return PDN_ERR_SHAPE;
  if (even && N > 0 && rows % N != 0) return PDN_ERR_SHAPE;
  *row_bytes = rows * V * (dtype == PDN_BF16 ? 2 : 4);
  *ws_bytes = blocks * 16;
  return PDN_OK;
}

pdn_status pdn_draft_verify_workspace_size(int64_t N, int64_t V, size_t* bytes) {
  if (!bytes) return PDN_ERR_NULL;
  int64_t rb, wb;
  const pdn_status st = check_verify(N, V > 0 ? N : 0, V, PDN_F32, false, &rb, &wb);
  if (st == PDN_OK) *bytes = static_cast<size_t>(wb);
  return st;
}

pdn_status pdn_draft_verify(int64_t N, int64_t rows, int64_t V, pdn_dtype dtype, const void* p, const void* q,
                            const int32_t* ids, const float* u, const float* r, const int32_t* starts,
                            int32_t* accepted, int32_t* token, void* ws, size_t ws_bytes, void* hip_stream) {
  int64_t rb, wb;
  pdn_status st = check_verify(N, rows, V, dtype, !starts, &rb, &wb);
  if (st != PDN_OK) return st;
  if (N > 0 && (!accepted || !token)) return PDN_ERR_NULL;
  if (N > 0 && rows > 0 && (!p || !ids || !u || !r)) return PDN_ERR_NULL;
  const std::array<Buf, 6> ins = {
      {{p, rb}, {q, rb}, {ids, rows * 4}, {u, rows * 4}, {r, N * 4}, {starts, (N + 1) * 4}}};
  const std::array<Buf, 2> outs = {{{accepted, N * 4}, {token, N * 4}}};
  for (size_t i = 0; i < ins.size(); ++i)   // (probabilities: to an element, as a row of an odd V is)
    if (reinterpret_cast<uintptr_t>(ins[i].p) & (dtype == PDN_BF16 && i < 2 ? 1u : 3u)) return PDN_ERR_ALIGN;
  for (const Buf& x : outs)
    if (reinterpret_cast<uintptr_t>(x.p) & 3u) return PDN_ERR_ALIGN;
  if ((st = check_aliasing(ins, outs, Buf{ws, N > 0 ? static_cast<int64_t>(ws_bytes) : 0})) != PDN_OK) return st;
  if (N == 0) return PDN_OK;
  if (wb > 0 && (!ws || ws_bytes < static_cast<size_t>(wb) || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0))
    return PDN_ERR_WORKSPACE;
  pdn::VerifyArgs a{};
  a.N = N; a.rows = rows; a.V = V;
  a.p = p; a.q = q; a.ids = ids; a.u = u; a.r = r; a.starts = starts;
  a.accepted = accepted; a.token = token;
  a.sums = static_cast<double*>(ws);
  return pdn::launch_verify(a, dtype == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK
                                                                                                      : PDN_ERR_HIP;
}

}  // extern "C"
