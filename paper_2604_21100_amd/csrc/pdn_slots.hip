// The gated delta rule over packed sequences whose states live in slots of a pool:
// single tokens (slot_step), two to eight tokens and drafted ones, which are scored
// without moving the state (slot_blocks).  Longer runs are pdn_slot_chunks.hip's and
// pdn_slot_runs.hip's.  Per sequence and value head, with S^T the state and G the
// inclusive prefix of the log-decay over a block of up to eight tokens (lam = exp(G)):
//   L[t][s] = beta_t k_t Lam_t/Lam_s . kt_s  (s < t)    P[t][s] = q_t Lam_t/Lam_s . kt_s  (s <= t)
//   X = Diag(beta) (V - Diag(lam) K S^T)                E = (I + L)^{-1} X
//   O = scale (Diag(lam) Q S^T + P E)                   S'^T = lam_C S^T + Kt^T Diag(lam_C / lam) E
// All of it in fp32: states, operands and products (the fp32 matrix
// instruction), so a state comes out as exact as a token-by-token one.
//
// A workgroup holds one head's state in registers: a wave 16 or 32 columns of it, a
// lane the rows 16 m + 4 (l / 16) + i of its one or two.  That is at once the
// accumulator layout of the update (16 x 16 tiles of S^T)
// and, contracted in the order (m, i), the right operand of the products with
// S^T, so the state goes from one block to the next without leaving its
// registers.  The left operand of those products stacks the eight key rows
// on the eight query rows: 16, a whole tile.
//
// Drafted tokens: a record of each (write key, correction e, prefix of the
// log-decay, preconditioner state) stays on the tape; the next call's first
// pass over the state applies the accepted ones,
//   S'^T = lam_n S^T + sum_{s <= n} (lam_n / lam_s) kt_s e_s.
// One workgroup holds a whole head, so a slot's tape and states may be read
// and written by the same call.
#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_slots.hpp"
#include "pdn_tile.hpp"

namespace pdn {

namespace {

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// a wave's 32 columns of it, two a lane (from element `at` of the head)
template <int DK, int DV>
struct Columns2 {
  static constexpr int MB = DK / 16;
  floatx4 t[MB][2];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int m = 0; m < MB; ++m) t[m][0] = t[m][1] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int at) {
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const floatx2 x =
            __builtin_bit_cast(floatx2, __builtin_amdgcn_raw_buffer_load_b64(r, 4 * at, (16 * m + i) * DV * 4, 0));
        t[m][0][i] = x[0];
        t[m][1][i] = x[1];
      }
  }
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, int at) const {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, floatx2{t[m][0][i], t[m][1][i]}), r, 4 * at,
                                              (16 * m + i) * DV * 4, 0);
  }
};
// the write key of a token's channel, but for the factor of slot_sum_factor
__device__ __forceinline__ float write_key(const SlotArgs& a, float k, float x, float A, float Ap, float mu) {
  if (a.precond == kSquash) return squash_gain(A, mu, a.lnx) * k;
  if (a.precond == kDiagSM) return k / (Ap + a.ridge);
  return a.precond == kExternal ? x : k;
}
// ---------------------------------------------------------------- one token
//   S' = alpha S + e kt^T,  e = beta (v - (alpha S) k),  o = scale ((alpha S) q + (kt . q) e)
// on the vector unit: six operations a state element, which no matrix instruction
// would make fewer.  What bounds it is reading and writing the state, so the rest is
// kept small: at most 108 registers and 2 KB of LDS, four workgroups a compute unit, the
// loads of some in flight beside the work of others (64 sequences x 16 heads of 128 x
// 128: 26 us, 5.2 TB/s; 256 x 32: 214 us, 5.0 TB/s; a 1 GiB copy makes 5.1).  One
// sequence of 16 heads: 6 us, a launch and four dependent memory latencies.
template <typename T, int DK, int DV, bool CH>
__global__ __launch_bounds__(DV * 2, 4) void slot_step(SlotArgs a) {
  constexpr int NTHR = DV * 2, NW = DV / 32, MB = DK / 16;
  __shared__ __attribute__((aligned(16))) float sK[DK], sQ[DK], sKt[DK], sLam[CH ? DK : 4];
  __shared__ float sSum[NW];
  const SlotWhere where = slot_where(a);
  const int64_t seq = where.seq, h = where.h, hk = where.hk;
  const int64_t src = a.slot ? a.slot[seq] : seq, dst = a.slot_out ? a.slot_out[seq] : src;
  if (src < 0 || src >= a.slots || dst < 0 || dst >= a.slots) return;
  const SlotRows rows = slot_rows(a, seq);
  const bool fresh = a.fresh && a.fresh[seq] != 0, gram = has_gram(a.precond);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, lg = l >> 4;
  const int v0 = 32 * w + 2 * (l & 15), at = 4 * lg * DV + v0;
  const bool key = tid < DK, qry = NTHR >= 2 * DK ? tid / DK == 1 : key, both = a.precond == kATQ;
  const int c = tid % DK;
  Columns2<DK, DV> S;
  if (fresh) S.zero();
  else S.load(slot_head<DK, DV>(a, src, h), at);
  float A = gram && key && !fresh ? a.A[(src * a.H + h) * DK + c] : 0.f;
  if (rows.n > 0) {
    const int64_t row = rows.lo, sc = row * a.H + h;
    const float kv = key ? to_f(static_cast<const T*>(a.k)[row * a.k_stride + hk * DK + c]) : 0.f;
    float qv = qry || (both && key) ? to_f(static_cast<const T*>(a.q)[row * a.q_stride + hk * DK + c]) : 0.f;
    const float xv = a.precond == kExternal && key ? to_f(static_cast<const T*>(a.ktilde)[(row * a.Hk + hk) * DK + c]) : 0.f;
    const floatx2 vv = ld2<T>(static_cast<const T*>(a.v) + row * a.v_stride + h * DV + v0);
    const float beta = a.beta[sc], g = CH ? a.g[sc * DK + c] : a.gate == kGateScalar ? a.g[sc] : 0.f;
    const float Ap = A;
    if (gram) A = (a.g_p ? fast_exp(a.g_p[sc]) : 1.f) * A + a.beta_p[sc] * kv * kv;
    float kt = write_key(a, kv, xv, A, Ap, a.precond == kSquash ? fast_exp(a.log_a_scale[h]) : 0.f);
    if (both) qv /= A + a.ridge;
    if (slot_needs_sum(a)) {
      const float x = wave_sum(key ? kv * kt : 0.f);
      if (l == 0) sSum[w] = x;
      __syncthreads();
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) m += sSum[i];
      kt *= slot_sum_factor(a, m, beta, g);
    }
    if (key) {
      sK[c] = both ? 0.f : kv;   // (a linear-attention update has no correction by the state)
      sKt[c] = kt;
      if (CH) sLam[c] = fast_exp(g);
    }
    if (both ? key : qry) sQ[c] = qv;
    __syncthreads();
    const float lam0 = CH ? 1.f : fast_exp(g);
    floatx2 y = {0.f, 0.f}, z = y;
    float kq = 0.f;
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const floatx4 k4 = *reinterpret_cast<const floatx4*>(&sK[16 * m + 4 * lg]);
      const floatx4 q4 = *reinterpret_cast<const floatx4*>(&sQ[16 * m + 4 * lg]);
      const floatx4 t4 = *reinterpret_cast<const floatx4*>(&sKt[16 * m + 4 * lg]);
      if (CH) {
        const floatx4 f = *reinterpret_cast<const floatx4*>(&sLam[16 * m + 4 * lg]);
        S.t[m][0] *= f;
        S.t[m][1] *= f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[0] += k4[i] * S.t[m][0][i];
        y[1] += k4[i] * S.t[m][1][i];
        z[0] += q4[i] * S.t[m][0][i];
        z[1] += q4[i] * S.t[m][1][i];
        kq += q4[i] * t4[i];
      }
    }
#pragma unroll
    for (int off = 16; off < 64; off <<= 1) {
      y[0] += __shfl_xor(y[0], off, 64);
      y[1] += __shfl_xor(y[1], off, 64);
      z[0] += __shfl_xor(z[0], off, 64);
      z[1] += __shfl_xor(z[1], off, 64);
      kq += __shfl_xor(kq, off, 64);
    }
    const floatx2 e = beta * (vv - lam0 * y), o = a.scale * (lam0 * z + kq * e);
    if (lg == 0) st2<T>(static_cast<T*>(a.o) + row * a.H * DV + h * DV + v0, o[0], o[1]);
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const floatx4 t4 = *reinterpret_cast<const floatx4*>(&sKt[16 * m + 4 * lg]);
      S.t[m][0] = lam0 * S.t[m][0] + t4 * e[0];
      S.t[m][1] = lam0 * S.t[m][1] + t4 * e[1];
    }
  }
  S.store(slot_head<DK, DV>(a, dst, h), at);
  if (gram && key) a.A[(dst * a.H + h) * DK + c] = A;
}

// ---------------------------------------------------------------- blocks of tokens
// Everything that does not need the state is loaded first and worked on while
// the state is on its way: a block's rows (16 bytes a thread), from them L and
// P, and the accepted records.  A wave has 16 columns here, a lane one (with two,
// the state and the rest of it take more registers than there are).
//
// What bounds it is the chain of a workgroup, of which a compute unit holds two: rows,
// L and P (two barriers), the state's arrival, records, products, solve.  Drafts of
// 64 sequences x 16 heads: 44 us for 152 MB, 3.5 TB/s; 96 x 16 of four tokens with
// per-channel decays 63 us, 3.4 TB/s; five tokens of one sequence 10 us.  Eight
// tokens of 64 x 16 heads without a tape 35 us.  (With pending counts read ahead of
// the rows drafts took 45 and 64 us, with the state first 46 and 66; a third workgroup
// would leave a lane 80 of the 128 registers that it takes.)
template <typename T, int DK, int DV, bool CH, bool DRAFT>
__global__ __launch_bounds__(DV * 4, 4) void slot_blocks(SlotArgs a) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  constexpr int NTHR = DV * 4, NW = DV / 16, MB = DK / 16, LD = DK + 4;
  constexpr int RP = kSlotBlock * DK * sizeof(T) / 16, NRP = (RP + NTHR - 1) / NTHR;   // 16-byte pieces of a block's key rows
  constexpr int GP = kSlotBlock * DK * 4 / 16, NGP = (GP + NTHR - 1) / NTHR;           // of a block's rows of fp32
  __shared__ __attribute__((aligned(16))) T sRaw[3][kSlotBlock][DK];   // keys, queries, the caller's write keys
  __shared__ __attribute__((aligned(16))) float sKQ[2 * kSlotBlock][LD], sKt[kSlotBlock][LD];
  // CH: g; the write keys with the decay to the block's end; operands of the products
  // of channel_rows (the columns of the second are the write keys).
  // Drafts: the accepted records' write keys and, with CH, their log-decays and the
  // decay over them; A after each token.
  __shared__ __attribute__((aligned(16))) float sG[CH ? kSlotBlock : 1][LD], sKw[CH ? kSlotBlock : 1][LD], sGr[CH && DRAFT ? kSlotBlock : 1][LD];
  __shared__ __attribute__((aligned(16))) float sR1[CH ? 16 : 1][LD], sR2[CH ? 16 : 1][LD], sC1[CH ? kPairCols : 1][LD];
  __shared__ __attribute__((aligned(16))) float sC[DRAFT ? kSlotBlock : 1][LD], sAt[DRAFT ? kSlotBlock : 1][LD];
  __shared__ __attribute__((aligned(16))) float sPart[NW][16][kSlotBlock], sLP[16][kSlotBlock + 4], sE[NW][kSlotBlock][16];
  __shared__ __attribute__((aligned(16))) float sLam[CH ? DK : 4], sGt[CH && DRAFT ? kSlotBlock : 1][LD], sSum[NW][kSlotBlock], sLr[CH && DRAFT ? DK : 4];
  // of each token: log-decay, its sum from the first token, the decay to and from
  // the token within the block as factors (1 with a per-channel gate), write strength,
  // preconditioner gain and decay
  __shared__ __attribute__((aligned(16))) float sg[kSlotBlock], sGp[kSlotBlock], sTo[kSlotBlock], sOn[kSlotBlock], sB[kSlotBlock], sBp[kSlotBlock], sDp[kSlotBlock];
  const SlotWhere where = slot_where(a);
  const int64_t seq = where.seq, h = where.h, hk = where.hk;
  const int64_t src = a.slot ? a.slot[seq] : seq, dst = a.slot_out ? a.slot_out[seq] : src;
  if (src < 0 || src >= a.slots || dst < 0 || dst >= a.slots) return;
  const SlotRows rows = slot_rows(a, seq);
  const bool fresh = a.fresh && a.fresh[seq] != 0;
  const int prec = a.precond, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool both = prec == kATQ, gram = has_gram(prec);
  // The thread's number, made anew for each part: what is formed from it, addresses
  // above all, is then formed where it is used (held throughout, all of them
  // together take more registers than there are).
  int tid = threadIdx.x;
  auto anew = [&]() { asm volatile("" : "+v"(tid)); };
  struct Place {
    int l, lr, lg, tb, v0, c;   // c: the channel whose rows a thread forms
    bool key, qry;              // the key's and write key's, the query's
  };
  auto place = [&]() {
    const int l = tid & 63, lg = l >> 4;
    const bool key = tid < DK;
    return Place{l, l & 15, lg, 4 * (lg & 1), 16 * w + (l & 15), tid % DK, key, NTHR >= 2 * DK ? tid / DK == 1 : key};
  };
  const int64_t R = DK + DV + (CH ? DK : 4) + (gram ? DK : 0), rs = a.H * R;   // a record; from one token's to the next

  // ---- A block's rows, from memory into registers, then into LDS.  Rows are seen
  // through a buffer that ends with the sequence (past it: zeros); what a call does
  // not have is a buffer of no bytes.  (No branches: one would wait for its loads.)
  u32x4 rk[NRP], rq[NRP], rx[NRP], rg[NGP];
  float vn[4], vv[4];   // values: those under way, the block's
  float s_b = 0.f, s_g = 0.f, s_bp = 0.f, s_gp = 0.f;
  const bool scalar = a.gate == kGateScalar;
  const float *const gb = scalar ? a.g : a.beta, *const bpb = gram ? a.beta_p : a.beta,
              *const gpb = gram && a.g_p ? a.g_p : a.beta;
  auto load_rows = [&](int64_t t0) {
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
    const int n = static_cast<int>(min<int64_t>(kSlotBlock, rows.n - t0));
    const int64_t row = rows.lo + t0;
    auto view = [&](const void* p, int64_t stride, int64_t first, int width, int esz, bool there) {
      return buf_rsrc(static_cast<const char*>(p) + (row * stride + first) * esz,
                      there ? static_cast<uint32_t>(((n - 1) * stride + width) * esz) : 0);
    };
    auto piece = [&](__amdgpu_buffer_rsrc_t r, int64_t stride, int row_bytes, int esz, int x) {
      const uint32_t at = x * NTHR + tid, t = at * 16 / row_bytes, o = at * 16 % row_bytes;
      return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                           r, static_cast<int>(t * static_cast<uint32_t>(stride * esz) + o), 0, 0));
    };
    const __amdgpu_buffer_rsrc_t vk = view(a.k, a.k_stride, hk * DK, DK, sizeof(T), true),
                                 vq = view(a.q, a.q_stride, hk * DK, DK, sizeof(T), true),
                                 vx = view(a.ktilde, a.Hk * DK, hk * DK, DK, sizeof(T), prec == kExternal),
                                 vw = view(a.v, a.v_stride, h * DV, DV, sizeof(T), true);
#pragma unroll
    for (int x = 0; x < NRP; ++x) {
      rk[x] = piece(vk, a.k_stride, DK * sizeof(T), sizeof(T), x);
      rq[x] = piece(vq, a.q_stride, DK * sizeof(T), sizeof(T), x);
      rx[x] = piece(vx, a.Hk * DK, DK * sizeof(T), sizeof(T), x);
    }
    if (CH) {
      const __amdgpu_buffer_rsrc_t vg = view(a.g, a.H * DK, h * DK, DK, 4, true);
#pragma unroll
      for (int x = 0; x < NGP; ++x) rg[x] = piece(vg, a.H * DK, DK * 4, 4, x);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int o = (tb + i) * static_cast<uint32_t>(a.v_stride * sizeof(T)) + v0 * sizeof(T);
      vn[i] = buf_get<T>(vw, o);
    }
    const int64_t sc = (row + min(tid & (kSlotBlock - 1), n - 1)) * a.H + h;
    const bool in = (tid & (kSlotBlock - 1)) < n;
    const float x_b = a.beta[sc], x_g = gb[sc], x_bp = bpb[sc], x_gp = gpb[sc];
    s_b = in ? x_b : 0.f;
    s_g = in && scalar ? sum_decay(x_g) : 0.f;
    s_bp = in && gram ? x_bp : 0.f;
    s_gp = in && gram && a.g_p ? x_gp : 0.f;
  };
  // Drafts: log-decay summed over the tokens before (the scalar's over the blocks before;
  // a channel's) in 64 bits, so that a record's sum is rounded once.
  double gacc = 0.0;
  auto put_rows = [&]() {
    auto put = [&](void* p, const u32x4& v, int x, int pieces, int row_bytes, int ld_bytes) {
      const int at = x * NTHR + tid;
      if (at < pieces)
        *reinterpret_cast<u32x4*>(static_cast<char*>(p) + at * 16 / row_bytes * ld_bytes + at * 16 % row_bytes) = v;
    };
#pragma unroll
    for (int x = 0; x < NRP; ++x) {
      put(sRaw[0], rk[x], x, RP, DK * sizeof(T), DK * sizeof(T));
      put(sRaw[1], rq[x], x, RP, DK * sizeof(T), DK * sizeof(T));
      if (prec == kExternal) put(sRaw[2], rx[x], x, RP, DK * sizeof(T), DK * sizeof(T));
    }
    if (CH)
#pragma unroll
      for (int x = 0; x < NGP; ++x) put(sG, rg[x], x, GP, DK * 4, LD * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) vv[i] = vn[i];
    float to, on;
    block_sums(s_g, tid, &to, &on);
    if (tid < kSlotBlock) {
      sg[tid] = s_g;
      sTo[tid] = fast_exp(to);
      sOn[tid] = fast_exp(on);
      sB[tid] = s_b;
      sBp[tid] = s_bp;
      sDp[tid] = fast_exp(s_gp);
      if (DRAFT && !CH) {
        double sum = s_g;
#pragma unroll
        for (int off = 1; off < kSlotBlock; off <<= 1) {
          const double y = __shfl_up(sum, off, kSlotBlock);
          if (tid >= off) sum += y;
        }
        sGp[tid] = static_cast<float>(gacc + sum);
        gacc += __shfl(sum, kSlotBlock - 1, kSlotBlock);
      }
    }
  };
  if (rows.n > 0) load_rows(0);

  // ---- drafts: the first accepted records
  const float* const rec = DRAFT ? a.tape + (src * a.tape_tokens * a.H + h) * R : nullptr;
  u32x4 ck[NGP], cg[NGP];
  float ce[2], cs = 0.f;
  auto load_records = [&](int b0) {   // (whether accepted or not; never past the tape)
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
    const int n = static_cast<int>(min(a.tape_tokens - b0, (int64_t)kSlotBlock));
#pragma unroll
    for (int x = 0; x < NGP; ++x) {
      const int at = x * NTHR + tid, t = at / (DK / 4), cc = 4 * (at % (DK / 4));
      ck[x] = cg[x] = u32x4{0, 0, 0, 0};
      if (t < n) {
        ck[x] = *reinterpret_cast<const u32x4*>(rec + (b0 + t) * rs + cc);
        if (CH) cg[x] = *reinterpret_cast<const u32x4*>(rec + (b0 + t) * rs + DK + DV + cc);
      }
    }
    cs = !CH && (l & 7) < n ? rec[(b0 + (l & 7)) * rs + DK + DV] : 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = 4 * j + lg;
      ce[j] = t < n ? rec[(b0 + t) * rs + DK + v0] : 0.f;
    }
  };
  int cnt = 0;
  if (DRAFT && a.accepted && !fresh) {
    load_records(0);
    const int64_t pend = min((int64_t)a.pending[src * a.H + h], a.tape_tokens);
    cnt = static_cast<int>(max(min((int64_t)a.accepted[seq], pend), (int64_t)0));
  }
  const float* const last = DRAFT ? rec + max(cnt - 1, 0) * rs : nullptr;

  // ---- the state (A first: what is loaded after the state is there after it)
  SlotColumns<DK, DV> S;
  float A = 0.f;
  {
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
    if (gram && key && !fresh) A = cnt > 0 ? last[DK + DV + (CH ? DK : 4) + c] : a.A[(src * a.H + h) * DK + c];
    if (fresh) S.zero();
    else S.load(slot_head<DK, DV>(a, src, h), 4 * lg * DV + v0);
  }
  auto store_state = [&](float A) {
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
    S.store(slot_head<DK, DV>(a, dst, h), 4 * lg * DV + v0);
    if (gram && key) a.A[(dst * a.H + h) * DK + c] = A;
  };
  const float A0 = A;
  const float mu = prec == kSquash ? fast_exp(a.log_a_scale[h]) : 0.f;

  // ---- a block's operands: key, query and write-key rows, L and P
  auto operands = [&](int nt) {
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
    {
      float kt[kSlotBlock], kv[kSlotBlock], At[kSlotBlock];
      float ex[kSlotBlock], up[kSlotBlock], lam = 1.f;   // CH: a token's decay, that from the block's start
      const float Ab = A;   // before the block
#pragma unroll
      for (int t = 0; t < kSlotBlock; ++t) {
        kv[t] = to_f(sRaw[0][t][c]);
        if (CH) {
          ex[t] = fast_exp(sG[t][c]);
          lam *= ex[t];
          up[t] = lam;
        }
      }
      if (gram) {   // (a token past the end leaves A: no gain, no decay)
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) {
          A = sDp[t] * A + sBp[t] * kv[t] * kv[t];
          At[t] = A;
        }
        if (DRAFT && key)
#pragma unroll
          for (int t = 0; t < kSlotBlock; ++t) sAt[t][c] = At[t];
      }
      if (prec == kSquash) {
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) kt[t] = squash_gain(At[t], mu, a.lnx) * kv[t];
      } else if (prec == kDiagSM) {
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) kt[t] = kv[t] / ((t ? At[t - 1] : Ab) + a.ridge);
      } else {
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) kt[t] = prec == kExternal ? to_f(sRaw[2][t][c]) : kv[t];
      }
      if (both ? key : qry) {
        float q[kSlotBlock];
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) {
          q[t] = to_f(sRaw[1][t][c]);
          if (both) q[t] /= At[t] + a.ridge;
          if (!CH) sKQ[kSlotBlock + t][c] = q[t];
        }
        if constexpr (CH) channel_rows(q, ex, up, 1, c, sKQ, sR1, sR2);
      }
      if (slot_needs_sum(a)) {   // the write key's row sums
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) {
          const float x = wave_sum(key ? kv[t] * kt[t] : 0.f);
          if (l == 0) sSum[w][t] = x;
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) {
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < NW; ++i) m += sSum[i][t];
          kt[t] = t < nt ? slot_sum_factor(a, m, sB[t], sg[t]) * kt[t] : 0.f;
        }
      }
      if (key) {
        // (a linear-attention update has no correction by the state: no key rows)
        if (both)
#pragma unroll
          for (int t = 0; t < kSlotBlock; ++t) kv[t] = 0.f;
        if constexpr (CH) {
          channel_rows(kv, ex, up, 0, c, sKQ, sR1, sR2);
          channel_cols(kt, ex, c, sC1, sKt, sKw);
          sLam[c] = lam;
        } else {
#pragma unroll
          for (int t = 0; t < kSlotBlock; ++t) {
            sKQ[t][c] = kv[t];
            sKt[t][c] = kt[t];
          }
        }
      }
      if (CH && DRAFT) {   // (a token's log-decay as where a scalar gate's are summed)
#pragma unroll
        for (int t = 0; t < kSlotBlock; ++t) {
          gacc += sum_decay(sG[t][c]);
          if (key) sGt[t][c] = static_cast<float>(gacc);
        }
      }
    }
    __syncthreads();
    // (rows of K over rows of Q) times Kt^T, a share of the channels a wave; CH: half
    // the waves each of the two products
    constexpr int NP = CH ? NW / 2 : NW;
    const int pass = w / NP, m1 = w % NP;
    const float(*const rows16)[LD] = !CH ? sKQ : pass ? sR2 : sR1;
    const float(*const cols8)[LD] = !CH || pass ? sKt : sC1;
    floatx4 g4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m0 = 0; m0 < MB; m0 += NP) {
      const int m = m0 + m1;
      if (MB < NP && m >= MB) break;
      const floatx4 r4 = *reinterpret_cast<const floatx4*>(&rows16[lr][16 * m + 4 * lg]);
      const floatx4 t4 = *reinterpret_cast<const floatx4*>(&cols8[lr & 7][16 * m + 4 * lg]);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma4(g4, r4[i], t4[i]);
    }
    settled(g4);
    if (lr < kSlotBlock)
#pragma unroll
      for (int i = 0; i < 4; ++i) sPart[w][4 * lg + i][lr] = g4[i];
    __syncthreads();
    if (tid < 16 * kSlotBlock) {
      const int r = tid / kSlotBlock, s = tid % kSlotBlock, t = r % kSlotBlock;
      float x = 0.f;
      int row = r, col = s;
      if (CH) row = channel_pair(r, s, &col);
#pragma unroll
      for (int i = 0; i < NP; ++i) x += sPart[i + (CH ? row / 16 * NP : 0)][row % 16][col];
      if (!CH) {   // (summed token by token: a difference of two long sums would lose a short one)
        float g = 0.f;
#pragma unroll
        for (int j = 1; j < kSlotBlock; ++j) g += j > s && j <= t ? sg[j] : 0.f;
        x *= fast_exp(g);
      }
      sLP[r][s] = r < kSlotBlock ? (s < t ? sB[t] * x : 0.f) : (s <= t ? x : 0.f);
    }
    __syncthreads();
  };

  // ---- eight accepted records: write keys or, without the per-channel gate, corrections
  // with their decay to the last accepted token (one of the first eight, as a rule:
  // its sum is then at hand, where a load would wait for the state's)
  float lam_r = 1.f;   // the decay over all of them (CH: sLr)
  auto put_records = [&](int b0) {   // into LDS; what was not accepted as zeros
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
#pragma unroll
    for (int x = 0; x < NGP; ++x) {
      const int at = x * NTHR + tid, t = at / (DK / 4), cc = 4 * (at % (DK / 4));
      if (at < GP) {
        *reinterpret_cast<u32x4*>(&sC[t][cc]) = b0 + t < cnt ? ck[x] : u32x4{0, 0, 0, 0};
        if (CH) *reinterpret_cast<u32x4*>(&sGr[t][cc]) = cg[x];
      }
    }
    float f = 0.f;
    if (!CH) {
      const float Gn = cnt > kSlotBlock ? last[DK + DV] : __shfl(cs, max(cnt - 1, 0), 64);
      lam_r = fast_exp(Gn);
      f = fast_exp(Gn - cs);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (!CH) ce[j] *= __shfl(f, 4 * j + lg, 64);
      if (b0 + 4 * j + lg >= cnt) ce[j] = 0.f;
    }
  };
  auto decay_records = [&](int b0) {   // (CH; after a barrier)
#pragma unroll
    for (int x = 0; x < NGP; ++x) {
      const int at = x * NTHR + tid, t = at / (DK / 4), cc = 4 * (at % (DK / 4));
      if (at < GP) {
        floatx4 gn;
        if (cnt > kSlotBlock) gn = *reinterpret_cast<const floatx4*>(last + DK + DV + cc);
        else gn = *reinterpret_cast<const floatx4*>(&sGr[cnt - 1][cc]);
        const floatx4 g = *reinterpret_cast<const floatx4*>(&sGr[t][cc]);
        floatx4 kt = *reinterpret_cast<const floatx4*>(&sC[t][cc]), f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (b0 + t < cnt) kt[i] *= fast_exp(gn[i] - g[i]);
          f[i] = fast_exp(gn[i]);
        }
        *reinterpret_cast<floatx4*>(&sC[t][cc]) = kt;
        if (t == 0) *reinterpret_cast<floatx4*>(&sLr[cc]) = f;
      }
    }
  };
  auto apply_records = [&](int b0) {
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (b0 + 4 * j >= cnt) break;
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const float x = sC[4 * j + lg][16 * m + lr];
        mma4(S.t[m], x, ce[j]);
      }
    }
    settled(S.t);
  };

  // (more than one block: drafts only, which come here without tokens too, their
  // accepted records being applied in the first round)
  for (int64_t t0 = 0; t0 < rows.n || (DRAFT && t0 == 0); t0 += kSlotBlock) {
    const int nt = static_cast<int>(max(min<int64_t>(kSlotBlock, rows.n - t0), (int64_t)0));
    const int64_t row0 = rows.lo + t0;
    anew();
    if (nt > 0) put_rows();
    if (DRAFT && t0 == 0 && cnt > 0) put_records(0);
    __syncthreads();
    anew();
    if (DRAFT && rows.n > t0 + kSlotBlock) load_rows(t0 + kSlotBlock);
    anew();
    if (CH && DRAFT && t0 == 0 && cnt > 0) decay_records(0);
    anew();
    if (nt > 0) operands(nt);
    anew();
    if (DRAFT && t0 == 0) {
      if (cnt > 0) {
        if (CH && nt == 0) __syncthreads();
        [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          floatx4 lam = {lam_r, lam_r, lam_r, lam_r};
          if (CH) lam = *reinterpret_cast<const floatx4*>(&sLr[16 * m + 4 * lg]);
          S.t[m] *= lam;
        }
        apply_records(0);
        for (int b0 = kSlotBlock; b0 < cnt; b0 += kSlotBlock) {
          load_records(b0);
          __syncthreads();
          put_records(b0);
          __syncthreads();
          if (CH) {
            decay_records(b0);
            __syncthreads();
          }
          apply_records(b0);
        }
      }
      if (cnt > 0 || fresh || src != dst) {
        store_state(A0);
      }
      __syncthreads();   // (what is read of the tape has been read)
      if (tid == 0) a.pending[dst * a.H + h] = static_cast<int>(rows.n);
      if (nt == 0) break;
    }
    anew();
    [[maybe_unused]] const auto [l, lr, lg, tb, v0, c, key, qry] = place();
    T* const ob = static_cast<T*>(a.o) + h * DV + v0;
    if (DRAFT) {   // the records, but for e
      float* r0 = a.tape + ((dst * a.tape_tokens + t0) * a.H + h) * R;
      for (int x = tid; x < nt * DK / 4; x += NTHR) {
        const int t = x / (DK / 4), cc = 4 * (x % (DK / 4));
        float* r = r0 + t * rs;
        *reinterpret_cast<floatx4*>(r + cc) = *reinterpret_cast<const floatx4*>(&sKt[t][cc]);
        if (CH) *reinterpret_cast<floatx4*>(r + DK + DV + cc) = *reinterpret_cast<const floatx4*>(&sGt[t][cc]);
        if (gram) *reinterpret_cast<floatx4*>(r + DK + DV + (CH ? DK : 4) + cc) = *reinterpret_cast<const floatx4*>(&sAt[t][cc]);
      }
      if (!CH && tid < 4 * nt) r0[tid / 4 * rs + DK + DV + tid % 4] = sGp[tid / 4];
    }
    // ---- (rows of K over rows of Q) times S^T
    floatx4 yz = {0.f, 0.f, 0.f, 0.f}, yz1 = yz;   // (two sums: each product would wait for the one before)
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const floatx4 r4 = *reinterpret_cast<const floatx4*>(&sKQ[lr][16 * m + 4 * lg]);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma4(i & 1 ? yz1 : yz, r4[i], S.t[m][i]);
    }
    settled(yz, yz1);
    yz += yz1;
    // ---- E: tokens 0-3 in the first 16 lanes, 4-7 in the next
    floatx4 e;
    {
      floatx4 ld[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) ld[i] = *reinterpret_cast<const floatx4*>(&sLP[tb + i][tb]);
      const floatx4 be = *reinterpret_cast<const floatx4*>(&sB[tb]), lam = *reinterpret_cast<const floatx4*>(&sTo[tb]);
      floatx4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = be[i] * (vv[i] - lam[i] * yz[i]);
      yz *= lam;
      e = slot_solve4(ld, x);
      if (nt > 4) {
        floatx4 f;   // e of tokens 0-3
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = __shfl(e[j], lr, 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 lx = *reinterpret_cast<const floatx4*>(&sLP[4 + i][0]);
          x[i] -= (lx[0] * f[0] + lx[1] * f[1]) + (lx[2] * f[2] + lx[3] * f[3]);
        }
        x = slot_solve4(ld, x);
        if (lg == 1) e = x;
      }
      if (lg >= 2) e = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    // ---- O: rows 8-15 of the products, plus P E
    {
      floatx4 p4 = *reinterpret_cast<const floatx4*>(&sLP[lr][tb]);
      if (lr < kSlotBlock || lg >= 2) p4 = floatx4{0.f, 0.f, 0.f, 0.f};
      const bool hurt = __any(!all_numbers(e));
      floatx4 en = e;
      int first = kSlotBlock;
      if (hurt) first = first_of(take_out(en, tb, kSlotBlock));
#pragma unroll
      for (int i = 0; i < 4; ++i) mma4(yz, p4[i], en[i]);
      settled(yz);
      if (hurt) put_from(yz, tb, first, __builtin_nanf(""));
      if (lg >= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (tb + i < nt) ob[(row0 + tb + i) * a.H * DV] = from_f<T>(a.scale * yz[i]);
    }
    if (DRAFT && lg < 2)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (tb + i < nt)
          a.tape[((dst * a.tape_tokens + t0 + tb + i) * a.H + h) * R + DK + v0] = e[i];
    // ---- the state after the block (drafts: only for the block after it)
    if (!DRAFT || t0 + kSlotBlock < rows.n) {
      const floatx4 wt = *reinterpret_cast<const floatx4*>(&sOn[tb]);
      if (lg < 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) sE[w][tb + i][lr] = wt[i] * e[i];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const float lc = sTo[kSlotBlock - 1];
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        floatx4 f = {lc, lc, lc, lc};
        if (CH) f = *reinterpret_cast<const floatx4*>(&sLam[16 * m + 4 * lg]);
        S.t[m] *= f;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (4 * j >= nt) break;
        const float ej = sE[w][4 * j + lg][lr];
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          const float x = CH ? sKw[4 * j + lg][16 * m + lr] : sKt[4 * j + lg][16 * m + lr];
          mma4(S.t[m], x, ej);
        }
      }
      settled(S.t);
    }
    __syncthreads();
  }
  if constexpr (!DRAFT) {
    store_state(A);
  }
}

template <typename T, int DK, int DV, bool CH>
hipError_t launch_form(const SlotArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.B * a.H));
  if (a.tape) hipLaunchKernelGGL((slot_blocks<T, DK, DV, CH, true>), grid, dim3(DV * 4), 0, s, a);
  else if (a.T <= 1) hipLaunchKernelGGL((slot_step<T, DK, DV, CH>), grid, dim3(DV * 2), 0, s, a);
  else hipLaunchKernelGGL((slot_blocks<T, DK, DV, CH, false>), grid, dim3(DV * 4), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DK, int DV>
hipError_t launch_gate(const SlotArgs& a, hipStream_t s) {
  return a.gate == kGateChannel ? launch_form<T, DK, DV, true>(a, s) : launch_form<T, DK, DV, false>(a, s);
}

template <typename T>
hipError_t launch_dims(const SlotArgs& a, hipStream_t s) {
  if (a.dk == 64) return a.dv == 64 ? launch_gate<T, 64, 64>(a, s) : launch_gate<T, 64, 128>(a, s);
  return a.dv == 64 ? launch_gate<T, 128, 64>(a, s) : launch_gate<T, 128, 128>(a, s);
}

}  // namespace

hipError_t launch_slots(const SlotArgs& a, int io_bf16, hipStream_t s) {
  if (a.B * a.H == 0) return hipSuccess;
  if (slot_chunk_form(a, io_bf16)) return launch_slot_chunks(a, s);
  if (a.T > kSlotBlock && !a.tape) return launch_slot_runs(a, io_bf16, s);
  return io_bf16 ? launch_dims<bf16>(a, s) : launch_dims<float>(a, s);
}

}  // namespace pdn
