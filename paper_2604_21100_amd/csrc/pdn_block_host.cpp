// The calls around the rule (norms, logits, token counts): argument validation on the
// host before any HIP call, workspace sizes.  See include/pdn.h.
#include <array>
#include <cmath>

#include "pdn_checks.hpp"
#include "pdn_internal.hpp"

namespace {

using namespace pdn;

constexpr int64_t kMost = (int64_t)1 << 48;   // elements: byte counts stay far inside 64 bits

int size_of(pdn_dtype t) { return t == PDN_BF16 ? 2 : 4; }
bool known(pdn_dtype t) { return t == PDN_F32 || t == PDN_BF16; }
bool element_aligned(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(size - 1)) == 0; }
bool ws_ok(const void* ws, size_t has, int64_t needs) {
  return needs == 0 || (ws && has >= static_cast<size_t>(needs) && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0);
}

pdn_status check_rnorm(const pdn_rnorm* p, int64_t* n) {
  if (!p) return PDN_ERR_NULL;
  if (p->rows < 0 || p->D < 1) return PDN_ERR_SHAPE;
  if (p->D > kRnormMaxD) return PDN_ERR_UNSUPPORTED;
  if (!known(p->io) || !known(p->stream)) return PDN_ERR_DTYPE;
  if (!std::isfinite(p->alpha) || !std::isfinite(p->eps) || !(p->eps > 0.f)) return PDN_ERR_VALUE;
  if (!mul_ok(p->rows, p->D, n) || *n > kMost) return PDN_ERR_SHAPE;
  return PDN_OK;
}

pdn_status check_hnorm(const pdn_hnorm* p, int64_t* n) {
  if (!p) return PDN_ERR_NULL;
  if (p->tokens < 0 || p->H < 0 || p->d < 1) return PDN_ERR_SHAPE;
  if (p->d > kHnormMaxD) return PDN_ERR_UNSUPPORTED;
  if (!known(p->io)) return PDN_ERR_DTYPE;
  if (p->norm != PDN_NORM_RMS && p->norm != PDN_NORM_L2) return PDN_ERR_VALUE;
  if (p->act != PDN_ACT_NONE && p->act != PDN_ACT_SILU && p->act != PDN_ACT_SIGMOID) return PDN_ERR_VALUE;
  if (!std::isfinite(p->eps) || !(p->eps > 0.f)) return PDN_ERR_VALUE;
  // a workgroup a head at least, and of a weight's gradient one for every 32 of its elements
  if (p->H >= (int64_t)1 << 24 || p->H * p->d > (int64_t)1 << 26) return PDN_ERR_SHAPE;
  if (!mul_ok(p->tokens, p->H * p->d, n) || *n > kMost) return PDN_ERR_SHAPE;
  return PDN_OK;
}

// Rows of `width` bytes, `stride` bytes apart.
struct Rows {
  const void* p;
  int64_t n, width, stride;
};
// elements of a stride as it is given -> Rows; false: rows overlap, or sizes that do not fit
bool rows_of(const void* p, int64_t tokens, int64_t row, int64_t stride, int size, Rows* r) {
  if (stride == 0) stride = row;
  if (stride < 0 || stride > kMost || (tokens > 1 && stride < row)) return false;
  int64_t all;
  if (!mul_ok(tokens, stride, &all) || all > kMost) return false;
  *r = Rows{p, tokens, row * size, stride * size};
  return true;
}
bool same_rows(const Rows& a, const Rows& b) { return a.p == b.p && (a.n <= 1 || a.stride == b.stride); }
bool rows_overlap(const Rows& a, const Rows& b) {
  if (!a.p || !b.p || a.n == 0 || b.n == 0 || a.width == 0 || b.width == 0) return false;
  const Range ra = rng(a.p, (a.n - 1) * a.stride + a.width), rb = rng(b.p, (b.n - 1) * b.stride + b.width);
  if (!overlap(ra, rb)) return false;
  if (a.n > 1 && b.n > 1 && a.stride == b.stride) {   // slices of one tensor's rows: apart if their columns are
    const uintptr_t s = static_cast<uintptr_t>(a.stride);
    const uintptr_t d = ra.lo <= rb.lo ? (rb.lo - ra.lo) % s : (s - (ra.lo - rb.lo) % s) % s;
    if (d >= static_cast<uintptr_t>(a.width) && s - d >= static_cast<uintptr_t>(b.width)) return false;
  }
  return true;
}
Rows flat(const void* p, int64_t bytes) { return Rows{p, 1, bytes, bytes}; }

// outputs against inputs, each other and the workspace
template <size_t I, size_t O>
pdn_status check_rows(const std::array<Rows, I>& ins, const std::array<Rows, O>& outs, const Rows& ws) {
  for (size_t i = 0; i < O; ++i) {
    for (const Rows& in : ins)
      if (rows_overlap(outs[i], in)) return PDN_ERR_ALIAS;
    for (size_t j = i + 1; j < O; ++j)
      if (rows_overlap(outs[i], outs[j])) return PDN_ERR_ALIAS;
    if (rows_overlap(outs[i], ws)) return PDN_ERR_ALIAS;
  }
  for (const Rows& in : ins)
    if (rows_overlap(in, ws)) return PDN_ERR_ALIAS;
  return PDN_OK;
}

HnormArgs hnorm_args(const pdn_hnorm* p) {
  HnormArgs a{};
  a.M = p->tokens; a.H = p->H; a.d = p->d; a.act = p->act;
  a.l2 = p->norm == PDN_NORM_L2;
  a.head_weight = p->head_weight != 0;
  a.eps = p->eps;
  const int64_t row = p->H * p->d;
  a.sx = p->x_stride ? p->x_stride : row;
  a.sz = p->z_stride ? p->z_stride : row;
  a.sy = p->y_stride ? p->y_stride : row;
  a.sdy = p->dy_stride ? p->dy_stride : row;
  a.sdx = p->dx_stride ? p->dx_stride : row;
  a.sdz = p->dz_stride ? p->dz_stride : row;
  return a;
}

}  // namespace

extern "C" {

pdn_status pdn_residual_norm(const pdn_rnorm* p, const void* y, const void* residual, const float* weight,
                             const float* post_weight, const float* scale, void* u, void* h, void* hip_stream) {
  int64_t n;
  pdn_status st = check_rnorm(p, &n);
  if (st != PDN_OK) return st;
  if (n > 0 && (!y || !u)) return PDN_ERR_NULL;
  if (post_weight && !p->post_norm) return PDN_ERR_VALUE;
  const int io = size_of(p->io), sm = size_of(p->stream);
  if (!element_aligned(y, io) || !element_aligned(u, io) || !element_aligned(residual, sm) || !element_aligned(h, sm) ||
      !element_aligned(weight, 4) || !element_aligned(post_weight, 4) || !element_aligned(scale, 4))
    return PDN_ERR_ALIGN;
  const int64_t v = p->D * 4;
  const std::array<Buf, 5> ins = {{{y, n * io}, {h == residual ? nullptr : residual, n * sm}, {weight, v}, {post_weight, v}, {scale, v}}};
  const std::array<Buf, 2> outs = {{{u, n * io}, {h, n * sm}}};
  if ((st = check_aliasing(ins, outs, Buf{nullptr, 0})) != PDN_OK) return st;
  if (n == 0) return PDN_OK;
  RnormArgs a{};
  a.rows = p->rows; a.D = p->D; a.alpha = p->alpha; a.eps = p->eps; a.post_norm = p->post_norm != 0;
  a.y = y; a.residual = residual; a.weight = weight; a.post_weight = post_weight; a.scale = scale;
  a.u = u; a.h = h;
  return launch_rnorm_fwd(a, p->io == PDN_BF16, p->stream == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK
                                                                                                                  : PDN_ERR_HIP;
}

pdn_status pdn_residual_norm_bwd_workspace_size(const pdn_rnorm* p, size_t* bytes) {
  if (!bytes) return PDN_ERR_NULL;
  int64_t n;
  const pdn_status st = check_rnorm(p, &n);
  if (st == PDN_OK) *bytes = static_cast<size_t>(rnorm_parts(p->rows, p->D) * p->D * 3 * 4);
  return st;
}

pdn_status pdn_residual_norm_bwd(const pdn_rnorm* p, const void* du, const void* dh, const void* h, const void* y,
                                 const float* weight, const float* post_weight, const float* scale, void* dy, void* dresidual,
                                 float* dweight, float* dpost_weight, float* dscale, void* ws, size_t ws_bytes, void* hip_stream) {
  int64_t n;
  pdn_status st = check_rnorm(p, &n);
  if (st != PDN_OK) return st;
  if (n > 0 && (!du || !h || !dy || (!y && (p->post_norm || dscale)))) return PDN_ERR_NULL;
  if ((post_weight && !p->post_norm) || (dweight && !weight) || (dpost_weight && !post_weight) || (dscale && !scale)) return PDN_ERR_VALUE;
  const int io = size_of(p->io), sm = size_of(p->stream);
  for (const void* x : {du, y, static_cast<const void*>(dy)})
    if (!element_aligned(x, io)) return PDN_ERR_ALIGN;
  for (const void* x : {dh, h, static_cast<const void*>(dresidual)})
    if (!element_aligned(x, sm)) return PDN_ERR_ALIGN;
  for (const float* x : {weight, post_weight, scale, static_cast<const float*>(dweight), static_cast<const float*>(dpost_weight),
                         static_cast<const float*>(dscale)})
    if (!element_aligned(x, 4)) return PDN_ERR_ALIGN;
  const int64_t v = p->D * 4, needs = dweight || dpost_weight || dscale ? rnorm_parts(p->rows, p->D) * v * 3 : 0;
  const std::array<Buf, 7> ins = {{{du, n * io}, {dh == dresidual ? nullptr : dh, n * sm}, {h, n * sm}, {y, n * io}, {weight, v},
                                   {post_weight, v}, {scale, v}}};
  const std::array<Buf, 5> outs = {{{dy, n * io}, {dresidual, n * sm}, {dweight, v}, {dpost_weight, v}, {dscale, v}}};
  if ((st = check_aliasing(ins, outs, Buf{ws, needs > 0 ? static_cast<int64_t>(ws_bytes) : 0})) != PDN_OK) return st;
  if (!ws_ok(ws, ws_bytes, needs)) return PDN_ERR_WORKSPACE;
  RnormArgs a{};
  a.rows = p->rows; a.D = p->D; a.alpha = p->alpha; a.eps = p->eps; a.post_norm = p->post_norm != 0;
  a.weight = weight; a.post_weight = post_weight; a.scale = scale;
  a.y = y; a.du = du; a.dh = dh; a.h_in = h;
  a.dy = dy; a.dresidual = dresidual; a.dweight = dweight; a.dpost_weight = dpost_weight; a.dscale = dscale;
  a.part = static_cast<float*>(ws);
  return launch_rnorm_bwd(a, p->io == PDN_BF16, p->stream == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK
                                                                                                                  : PDN_ERR_HIP;
}

pdn_status pdn_head_norm(const pdn_hnorm* p, const void* x, const void* z, const float* weight, void* y, void* hip_stream) {
  int64_t n;
  pdn_status st = check_hnorm(p, &n);
  if (st != PDN_OK) return st;
  if (n > 0 && (!x || !y || (!z && p->act != PDN_ACT_NONE))) return PDN_ERR_NULL;
  if (z && p->act == PDN_ACT_NONE) return PDN_ERR_VALUE;
  const int io = size_of(p->io);
  if (!element_aligned(x, io) || !element_aligned(z, io) || !element_aligned(y, io) || !element_aligned(weight, 4)) return PDN_ERR_ALIGN;
  const int64_t row = p->H * p->d;
  Rows rx, rz, ry;
  if (!rows_of(x, p->tokens, row, p->x_stride, io, &rx) || !rows_of(z, p->tokens, row, p->z_stride, io, &rz) ||
      !rows_of(y, p->tokens, row, p->y_stride, io, &ry))
    return PDN_ERR_SHAPE;
  if (same_rows(rx, ry)) rx.p = nullptr;   // in place
  const std::array<Rows, 3> ins = {rx, rz, flat(weight, (p->head_weight ? row : p->d) * 4)};
  const std::array<Rows, 1> outs = {ry};
  if ((st = check_rows(ins, outs, flat(nullptr, 0))) != PDN_OK) return st;
  if (n == 0) return PDN_OK;
  HnormArgs a = hnorm_args(p);
  a.x = x; a.z = z; a.weight = weight; a.y = y;
  return launch_hnorm_fwd(a, p->io == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK : PDN_ERR_HIP;
}

pdn_status pdn_head_norm_bwd_workspace_size(const pdn_hnorm* p, size_t* bytes) {
  if (!bytes) return PDN_ERR_NULL;
  int64_t n;
  const pdn_status st = check_hnorm(p, &n);
  if (st == PDN_OK) *bytes = static_cast<size_t>(hnorm_parts(hnorm_args(p)) * p->d * 4);
  return st;
}

pdn_status pdn_head_norm_bwd(const pdn_hnorm* p, const void* dy, const void* x, const void* z, const float* weight, void* dx,
                             void* dz, float* dweight, void* ws, size_t ws_bytes, void* hip_stream) {
  int64_t n;
  pdn_status st = check_hnorm(p, &n);
  if (st != PDN_OK) return st;
  const bool gated = p->act != PDN_ACT_NONE;
  if (n > 0 && (!dy || !x || !dx || (gated && (!z || !dz)))) return PDN_ERR_NULL;
  if ((!gated && (z || dz)) || (dweight && !weight)) return PDN_ERR_VALUE;
  const int io = size_of(p->io);
  for (const void* t : {dy, x, z, static_cast<const void*>(dx), static_cast<const void*>(dz)})
    if (!element_aligned(t, io)) return PDN_ERR_ALIGN;
  if (!element_aligned(weight, 4) || !element_aligned(dweight, 4)) return PDN_ERR_ALIGN;
  const int64_t row = p->H * p->d, v = (p->head_weight ? row : p->d) * 4;
  Rows rdy, rx, rz, rdx, rdz;
  if (!rows_of(dy, p->tokens, row, p->dy_stride, io, &rdy) || !rows_of(x, p->tokens, row, p->x_stride, io, &rx) ||
      !rows_of(z, p->tokens, row, p->z_stride, io, &rz) || !rows_of(dx, p->tokens, row, p->dx_stride, io, &rdx) ||
      !rows_of(dz, p->tokens, row, p->dz_stride, io, &rdz))
    return PDN_ERR_SHAPE;
  if (same_rows(rdy, rdx)) rdy.p = nullptr;   // in place
  const int64_t needs = dweight ? hnorm_parts(hnorm_args(p)) * p->d * 4 : 0;
  const std::array<Rows, 4> ins = {rdy, rx, rz, flat(weight, v)};
  const std::array<Rows, 3> outs = {rdx, rdz, flat(dweight, v)};
  if ((st = check_rows(ins, outs, flat(needs > 0 ? ws : nullptr, static_cast<int64_t>(ws_bytes)))) != PDN_OK) return st;
  if (!ws_ok(ws, ws_bytes, needs)) return PDN_ERR_WORKSPACE;
  if (p->H == 0 && p->head_weight) return PDN_OK;
  HnormArgs a = hnorm_args(p);
  a.dy = dy; a.x = x; a.z = z; a.weight = weight;
  a.dx = dx; a.dz = dz; a.dweight = dweight;
  a.part = static_cast<float*>(ws);
  return launch_hnorm_bwd(a, p->io == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK : PDN_ERR_HIP;
}

static pdn_status check_vocab(int64_t rows, int64_t V, int64_t* blocks) {
  if (rows < 0 || V < 0 || rows > INT32_MAX || V > INT32_MAX || (V == 0 && rows > 0)) return PDN_ERR_SHAPE;
  if (!mul_ok(rows, logits_segments(V), blocks) || *blocks >= (int64_t)1 << 24) return PDN_ERR_SHAPE;   // (a launch's work items)
  return PDN_OK;
}

pdn_status pdn_logits_workspace_size(int64_t rows, int64_t V, size_t* bytes) {
  if (!bytes) return PDN_ERR_NULL;
  int64_t blocks;
  const pdn_status st = check_vocab(rows, V, &blocks);
  if (st == PDN_OK) *bytes = static_cast<size_t>(blocks * 16);
  return st;
}

pdn_status pdn_logits(const pdn_logits_args* p, void* out, void* ws, size_t ws_bytes, void* hip_stream) {
  if (!p) return PDN_ERR_NULL;
  int64_t blocks, table, bits;
  pdn_status st = check_vocab(p->rows, p->V, &blocks);
  if (st != PDN_OK) return st;
  if (!known(p->dtype) || !known(p->out_dtype)) return PDN_ERR_DTYPE;
  const int64_t rows = p->rows, V = p->V, N = p->N, words = (V + 31) / 32;
  if (N < 0 || N > INT32_MAX || p->slots < 0 || p->slots > INT32_MAX || p->biases < 0 || p->biases > INT32_MAX || p->masks < 0 ||
      p->masks > INT32_MAX)
    return PDN_ERR_SHAPE;
  if (!p->starts && (N > 0 ? rows % N != 0 : rows > 0)) return PDN_ERR_SHAPE;
  if (!mul_ok(p->slots, V, &table) || table > kMost || !mul_ok(p->masks, words, &bits) || bits > kMost) return PDN_ERR_SHAPE;
  if (p->counts && !p->slot && N > p->slots) return PDN_ERR_SHAPE;
  if (p->mask && !p->mask_rows && p->masks < rows) return PDN_ERR_SHAPE;
  const int in = size_of(p->dtype), on = size_of(p->out_dtype);
  Rows logits;
  if (!rows_of(p->logits, rows, V, p->stride, in, &logits)) return PDN_ERR_SHAPE;
  if (N > 0 && rows > 0 && (!p->logits || !out)) return PDN_ERR_NULL;
  if ((p->bias_starts != nullptr) != (p->bias_ids != nullptr) || (p->bias_ids != nullptr) != (p->bias_values != nullptr)) {
    if (p->biases > 0 || !p->bias_starts) return PDN_ERR_NULL;   // (an empty list may have no address)
  }
  if ((p->slot && !p->counts) || (p->mask_rows && !p->mask)) return PDN_ERR_VALUE;
  if (!element_aligned(p->logits, in) || !element_aligned(out, on)) return PDN_ERR_ALIGN;
  const std::array<Rows, 14> ins = {
      Rows{}, flat(p->starts, (N + 1) * 4), flat(p->temperature, N * 4), flat(p->repetition, N * 4), flat(p->presence, N * 4),
      flat(p->frequency, N * 4), flat(p->counts, table * 4), flat(p->slot, N * 4), flat(p->ids, rows * 4),
      flat(p->bias_starts, (N + 1) * 4), flat(p->bias_ids, p->biases * 4), flat(p->bias_values, p->biases * 4),
      flat(p->mask, bits * 4), flat(p->mask_rows, rows * 4)};
  for (const Rows& r : ins)
    if (!element_aligned(r.p, 4)) return PDN_ERR_ALIGN;
  const Rows o = Rows{out, rows, V * on, V * on};
  std::array<Rows, 14> all = ins;
  if (!(same_rows(logits, o) && p->dtype == p->out_dtype)) all[0] = logits;   // (else in place)
  const int64_t needs = p->probs && N > 0 ? blocks * 16 : 0;
  const std::array<Rows, 1> outs = {o};
  const Rows space = flat(needs > 0 ? ws : nullptr, static_cast<int64_t>(ws_bytes));
  if ((st = check_rows(all, outs, space)) != PDN_OK) return st;
  if (!ws_ok(ws, ws_bytes, needs)) return PDN_ERR_WORKSPACE;
  if (rows == 0 || N == 0) return PDN_OK;
  LogitsArgs a{};
  a.rows = rows; a.V = V; a.N = N; a.stride = p->stride ? p->stride : V;
  a.slots = p->slots; a.biases = p->biases; a.masks = p->masks; a.probs = p->probs != 0;
  a.logits = p->logits; a.out = out; a.starts = p->starts;
  a.temperature = p->temperature; a.repetition = p->repetition; a.presence = p->presence; a.frequency = p->frequency;
  a.counts = p->counts; a.slot = p->slot; a.ids = p->ids;
  if (p->biases > 0) {
    a.bias_starts = p->bias_starts; a.bias_ids = p->bias_ids; a.bias_values = p->bias_values;
  }
  a.mask = p->mask; a.mask_rows = p->mask_rows;
  a.parts = ws;
  return launch_logits(a, p->dtype == PDN_BF16, p->out_dtype == PDN_BF16, static_cast<hipStream_t>(hip_stream)) == hipSuccess
             ? PDN_OK : PDN_ERR_HIP;
}

pdn_status pdn_token_counts(int64_t N, int64_t rows, int64_t V, int64_t slots, int32_t prompt, const int32_t* ids,
                            const int32_t* starts, const int32_t* slot, const int32_t* slot_out, const int32_t* fresh,
                            const int32_t* accepted, int32_t* counts, void* hip_stream) {
  int64_t blocks, table;
  if (N < 0 || rows < 0 || V < 0 || slots < 0 || N >= (int64_t)1 << 24 || rows > INT32_MAX || V > INT32_MAX || slots > INT32_MAX)
    return PDN_ERR_SHAPE;
  if (!mul_ok(N, count_segments(V), &blocks) || blocks >= (int64_t)1 << 24) return PDN_ERR_SHAPE;
  if (!mul_ok(slots, V, &table) || table > kMost) return PDN_ERR_SHAPE;
  if (!starts && (N > 0 ? rows % N != 0 : rows > 0)) return PDN_ERR_SHAPE;
  if (!slot && N > slots) return PDN_ERR_SHAPE;
  if (N > 0 && ((rows > 0 && !ids) || (table > 0 && !counts))) return PDN_ERR_NULL;
  const std::array<Buf, 6> ins = {{{ids, rows * 4}, {starts, (N + 1) * 4}, {slot, N * 4}, {slot_out, N * 4}, {fresh, N * 4},
                                   {accepted, N * 4}}};
  const std::array<Buf, 1> outs = {{{counts, table * 4}}};
  for (const Buf& b : ins)
    if (!element_aligned(b.p, 4)) return PDN_ERR_ALIGN;
  if (!element_aligned(counts, 4)) return PDN_ERR_ALIGN;
  const pdn_status st = check_aliasing(ins, outs, Buf{nullptr, 0});
  if (st != PDN_OK) return st;
  if (N == 0 || table == 0) return PDN_OK;
  CountArgs a{};
  a.N = N; a.rows = rows; a.V = V; a.slots = slots; a.prompt = prompt != 0;
  a.ids = ids; a.starts = starts; a.slot = slot; a.slot_out = slot_out; a.fresh = fresh; a.accepted = accepted;
  a.counts = counts;
  return launch_counts(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PDN_OK : PDN_ERR_HIP;
}

}  // extern "C"
