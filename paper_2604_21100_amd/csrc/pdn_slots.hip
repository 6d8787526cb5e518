// The gated delta rule over packed sequences whose states live in slots of a
// pool: decoding, prompts, and drafted tokens that are scored without moving
// the state.  Per sequence and value head, with S^T the state and G the
// inclusive prefix of the log-decay over a block of up to eight tokens
// (lam = exp(G)):
//   L[t][s] = beta_t k_t Lam_t/Lam_s . kt_s  (s < t)    P[t][s] = q_t Lam_t/Lam_s . kt_s  (s <= t)
//   X = Diag(beta) (V - Diag(lam) K S^T)                E = (I + L)^{-1} X
//   O = scale (Diag(lam) Q S^T + P E)                   S'^T = lam_C S^T + Kt^T Diag(lam_C / lam) E
// All of it in fp32: states, operands and products (the fp32 matrix
// instruction), so a state comes out as exact as a token-by-token one.
//
// A workgroup holds one head's state in registers: a wave 32 columns of it, a
// lane the rows 16 m + 4 (l / 16) + i of the columns 2 (l % 16) and the next.
// That is at once the accumulator layout of the update (16 x 16 tiles of S^T)
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

namespace pdn {

namespace {

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

constexpr int kBlk = 8;   // tokens of a block

// TB: tokens of a block, 1 (one-token calls: the products on the vector unit)
// or kBlk.
template <typename T, int DK, int DV, bool CH, int TB, bool DRAFT>
__global__ __launch_bounds__(DV * 2, TB == 1 && !DRAFT ? 4 : 1) void slot_tokens(SlotArgs a) {
  constexpr int NTHR = DV * 2, NW = DV / 32, MB = DK / 16, LD = DK + 4;
  __shared__ __attribute__((aligned(16))) float sKQ[2 * TB][LD], sKt[TB][LD], sKw[kBlk][LD];
  __shared__ __attribute__((aligned(16))) float sPart[NW][16][kBlk], sLP[16][kBlk + 4], sE[NW][kBlk][32];
  __shared__ __attribute__((aligned(16))) float sLam[DK], sSum[NW][TB];
  // of each token: log-decay, its sum from the first token, the decay to and from
  // the token within the block as factors (1 with a per-channel gate), write strength
  __shared__ __attribute__((aligned(16))) float sG[TB], sGp[TB], sTo[TB], sOn[TB], sB[TB];
  const int64_t seq = blockIdx.x / a.H, h = blockIdx.x % a.H, hk = h / (a.H / a.Hk);
  const int64_t src = a.slot ? a.slot[seq] : seq, dst = a.slot_out ? a.slot_out[seq] : src;
  if (src < 0 || src >= a.slots || dst < 0 || dst >= a.slots) return;
  const SlotRows rows = slot_rows(a, seq);
  const bool fresh = a.fresh && a.fresh[seq] != 0;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, lr = l & 15, lg = l >> 4;
  const int v0 = 32 * w + 2 * lr;
  const bool key = tid < DK, qry = NTHR >= 2 * DK ? tid / DK == 1 : key;
  const int c = tid % DK;
  const int prec = a.precond;
  const bool gram = has_gram(prec);

  // ---- the state
  floatx4 S[MB][2];
  {
    const float* sp = a.S + (src * a.H + h) * (DK * DV) + 4 * lg * DV + v0;
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const floatx2 x = fresh ? floatx2{0.f, 0.f} : *reinterpret_cast<const floatx2*>(sp + (16 * m + i) * DV);
        S[m][0][i] = x[0];
        S[m][1][i] = x[1];
      }
  }
  float A = gram && key && !fresh ? a.A[(src * a.H + h) * DK + c] : 0.f;
  auto store_state = [&]() {
    float* sp = a.S + (dst * a.H + h) * (DK * DV) + 4 * lg * DV + v0;
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<floatx2*>(sp + (16 * m + i) * DV) = floatx2{S[m][0][i], S[m][1][i]};
    if (gram && key) a.A[(dst * a.H + h) * DK + c] = A;
  };

  // ---- drafts: the accepted tokens of the tape
  const int64_t R = DK + DV + (CH ? DK : 4) + (gram ? DK : 0);
  if constexpr (DRAFT) {
    int cnt = 0;
    if (a.accepted && !fresh) {
      const int pend = min(a.pending[src * a.H + h], a.tape_tokens);
      cnt = max(min(a.accepted[seq], pend), 0);
    }
    if (cnt > 0) {
      const float* rec = a.tape + (src * a.tape_tokens * a.H + h) * R;
      const int64_t rs = a.H * R;   // to the next token's record
      const float* last = rec + (cnt - 1) * rs;
      const float Gn = CH ? 0.f : last[DK + DV];
      if (gram && key) A = last[DK + DV + (CH ? DK : 4) + c];
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        floatx4 lam;
        if (CH) {
          const floatx4 g = *reinterpret_cast<const floatx4*>(last + DK + DV + 16 * m + 4 * lg);
#pragma unroll
          for (int i = 0; i < 4; ++i) lam[i] = fast_exp(g[i]);
        } else {
          lam = fast_exp(Gn);
        }
        S[m][0] *= lam;
        S[m][1] *= lam;
      }
      for (int b0 = 0; b0 < cnt; b0 += kBlk) {
        for (int x = tid; x < kBlk * DK / 4; x += NTHR) {
          const int t = x / (DK / 4), cc = 4 * (x % (DK / 4));
          floatx4 kt = {0.f, 0.f, 0.f, 0.f};
          if (b0 + t < cnt) {
            const float* r = rec + (b0 + t) * rs;
            kt = *reinterpret_cast<const floatx4*>(r + cc);
            if (CH) {
              const floatx4 g = *reinterpret_cast<const floatx4*>(r + DK + DV + cc);
              const floatx4 gn = *reinterpret_cast<const floatx4*>(last + DK + DV + cc);
#pragma unroll
              for (int i = 0; i < 4; ++i) kt[i] *= fast_exp(gn[i] - g[i]);
            } else {
              kt *= fast_exp(Gn - r[DK + DV]);
            }
          }
          *reinterpret_cast<floatx4*>(&sKw[t][cc]) = kt;
        }
        floatx2 e[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int t = b0 + 4 * j + lg;
          e[j] = t < cnt ? *reinterpret_cast<const floatx2*>(rec + t * rs + DK + v0) : floatx2{0.f, 0.f};
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (b0 + 4 * j >= cnt) break;
#pragma unroll
          for (int m = 0; m < MB; ++m) {
            const float x = sKw[4 * j + lg][16 * m + lr];
            mma4(S[m][0], x, e[j][0]);
            mma4(S[m][1], x, e[j][1]);
          }
        }
        __syncthreads();
      }
    }
    if (cnt > 0 || fresh || src != dst) store_state();
    __syncthreads();   // (the count it overwrites may be the one just read)
    if (tid == 0) a.pending[dst * a.H + h] = static_cast<int>(rows.n);
  }

  // ---- the tokens, in blocks
  const T* qb = static_cast<const T*>(a.q) + hk * DK + c;
  const T* kb = static_cast<const T*>(a.k) + hk * DK + c;
  const T* xb = prec == kExternal ? static_cast<const T*>(a.ktilde) + hk * DK + c : nullptr;
  const T* vb = static_cast<const T*>(a.v) + h * DV + v0;
  T* ob = static_cast<T*>(a.o) + h * DV + v0;
  const float mu = prec == kSquash ? fast_exp(a.log_a_scale[h]) : 0.f;
  float gacc = 0.f;   // log-decay summed over the blocks before (of the channel, or the scalar)
  for (int64_t t0 = 0; t0 < rows.n; t0 += TB) {
    const int nt = static_cast<int>(min<int64_t>(TB, rows.n - t0));
    const int64_t row0 = rows.lo + t0;
    // ---- key, query and write-key rows (a token past the end: zeros)
    float kv[TB], qv[TB], kt[TB], gg[TB], bp[TB], gp[TB];
    const bool both = prec == kATQ;   // the query depends on A: the key's thread forms it
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      const int64_t row = row0 + min(t, nt - 1), sc = row * a.H + h;
      kv[t] = key ? to_f(kb[row * a.k_stride]) : 0.f;
      qv[t] = qry || (both && key) ? to_f(qb[row * a.q_stride]) : 0.f;
      kt[t] = prec == kExternal && key ? to_f(xb[row * a.Hk * DK]) : 0.f;
      gg[t] = CH ? a.g[sc * DK + c] : 0.f;
      bp[t] = gram ? a.beta_p[sc] : 0.f;
      gp[t] = gram && a.g_p ? a.g_p[sc] : 0.f;
      if (t >= nt) kv[t] = qv[t] = kt[t] = gg[t] = bp[t] = gp[t] = 0.f;
    }
    floatx2 vv[4];
#pragma unroll
    for (int i = 0; i < (TB == 1 ? 1 : 4); ++i) {
      const int t = TB == 1 ? 0 : 4 * (lg & 1) + i;
      vv[i] = ld2<T>(vb + (row0 + min(t, nt - 1)) * a.v_stride);
    }
    if (tid < TB) {
      const int64_t sc = (row0 + min(tid, nt - 1)) * a.H + h;
      sB[tid] = tid < nt ? a.beta[sc] : 0.f;
      const float g = a.gate == kGateScalar && tid < nt ? a.g[sc] : 0.f;
      const float nx = __shfl_down(g, 1, TB);
      float to = g, on = tid + 1 < TB ? nx : 0.f;
#pragma unroll
      for (int off = 1; off < TB; off <<= 1) {
        const float y = __shfl_up(to, off, TB), z = __shfl_down(on, off, TB);
        if (tid >= off) to += y;
        if (tid + off < TB) on += z;
      }
      sG[tid] = g;
      sGp[tid] = gacc + to;
      gacc += __shfl(to, TB - 1, TB);
      sTo[tid] = fast_exp(to);
      sOn[tid] = fast_exp(on);
    }
    float At[TB], rs[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      const float Ap = A;
      if (gram && t < nt) A = fast_exp(gp[t]) * A + bp[t] * kv[t] * kv[t];
      At[t] = A;
      if (prec == kSquash) kt[t] = squash_gain(A, mu, a.lnx) * kv[t];
      if (prec == kIdentity || prec == kATQ) kt[t] = kv[t];
      if (prec == kDiagSM) kt[t] = kv[t] / (Ap + a.ridge);
      if (prec == kATQ) qv[t] = qv[t] / (A + a.ridge);
    }
    if (prec == kDiagSM || a.knorm != kKnormNone) {   // the write key's row sums
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        rs[t] = wave_sum(key ? kv[t] * kt[t] : 0.f);
        if (l == 0) sSum[w][t] = rs[t];
      }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) m += sSum[i][t];
        float f;
        if (prec == kDiagSM) f = 1.f / (1.f + m);
        else if (a.knorm == kKnormM) f = 1.f / m;
        else if (a.knorm == kKnorm1pm) f = 1.f / (1.f + m);
        else {
          const float alpha = a.gate == kGateScalar ? fast_exp(sG[t]) : 1.f;
          f = sB[t] / (alpha + sB[t] * m);
        }
        kt[t] = t < nt ? f * kt[t] : 0.f;
      }
    }
    // a linear-attention update has no correction by the state: no key rows
    const bool la = prec == kATQ;
    {
      float G = 0.f, lam[TB], Gt[TB];
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        G += gg[t];
        Gt[t] = G;
        lam[t] = CH ? fast_exp(G) : 1.f;
      }
      float* rec = DRAFT && key ? a.tape + ((dst * a.tape_tokens + t0) * a.H + h) * R : nullptr;
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const float f = TB == 1 ? 1.f : lam[t];
        if (key) {
          sKQ[t][c] = la ? 0.f : f * kv[t];
          sKt[t][c] = CH && TB > 1 ? kt[t] * fast_exp(-Gt[t]) : kt[t];
          if (CH && TB > 1) sKw[t][c] = kt[t] * fast_exp(G - Gt[t]);
          if (rec && t < nt) {
            float* r = rec + t * a.H * R;
            r[c] = kt[t];
            if (CH) r[DK + DV + c] = gacc + Gt[t];
            if (gram) r[DK + DV + (CH ? DK : 4) + c] = At[t];
          }
        }
        if (both ? key : qry) sKQ[TB + t][c] = f * qv[t];
      }
      if (CH) {
        if (key) sLam[c] = lam[TB - 1];
        gacc += G;
      }
    }
    __syncthreads();
    if (DRAFT && !CH && tid < 4 * nt)
      a.tape[((dst * a.tape_tokens + t0 + tid / 4) * a.H + h) * R + DK + DV + tid % 4] = sGp[tid / 4];

    if constexpr (TB == 1) {
      const float lam0 = sTo[0], beta = sB[0];
      floatx2 y = {0.f, 0.f}, z = y;
      float kq = 0.f;
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const floatx4 k4 = *reinterpret_cast<const floatx4*>(&sKQ[0][16 * m + 4 * lg]);
        const floatx4 q4 = *reinterpret_cast<const floatx4*>(&sKQ[1][16 * m + 4 * lg]);
        const floatx4 t4 = *reinterpret_cast<const floatx4*>(&sKt[0][16 * m + 4 * lg]);
        if (CH) {
          const floatx4 f = *reinterpret_cast<const floatx4*>(&sLam[16 * m + 4 * lg]);
          S[m][0] *= f;
          S[m][1] *= f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[0] += k4[i] * S[m][0][i];
          y[1] += k4[i] * S[m][1][i];
          z[0] += q4[i] * S[m][0][i];
          z[1] += q4[i] * S[m][1][i];
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
      const floatx2 e = beta * (vv[0] - lam0 * y), o = a.scale * (lam0 * z + kq * e);
      if (lg == 0) st2<T>(ob + row0 * a.H * DV, o[0], o[1]);
      if (DRAFT) {
        if (lg == 0) *reinterpret_cast<floatx2*>(a.tape + ((dst * a.tape_tokens + t0) * a.H + h) * R + DK + v0) = e;
      } else {
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          const floatx4 t4 = *reinterpret_cast<const floatx4*>(&sKt[0][16 * m + 4 * lg]);
          S[m][0] = lam0 * S[m][0] + t4 * e[0];
          S[m][1] = lam0 * S[m][1] + t4 * e[1];
        }
      }
    } else {
      // ---- (rows of K over rows of Q) times Kt^T, this wave's share of the channels, and times S^T
      floatx4 g4 = {0.f, 0.f, 0.f, 0.f}, yz[2] = {g4, g4};
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const floatx4 r4 = *reinterpret_cast<const floatx4*>(&sKQ[lr][16 * m + 4 * lg]);
        if (m % NW == w) {
          const floatx4 t4 = *reinterpret_cast<const floatx4*>(&sKt[lr & 7][16 * m + 4 * lg]);
#pragma unroll
          for (int i = 0; i < 4; ++i) mma4(g4, r4[i], t4[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mma4(yz[0], r4[i], S[m][0][i]);
          mma4(yz[1], r4[i], S[m][1][i]);
        }
      }
      if (lr < kBlk)
#pragma unroll
        for (int i = 0; i < 4; ++i) sPart[w][4 * lg + i][lr] = g4[i];
      __syncthreads();
      if (tid < 16 * kBlk) {
        const int r = tid / kBlk, s = tid % kBlk, t = r % kBlk;
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) x += sPart[i][r][s];
        if (!CH) {   // (summed token by token: a difference of two long sums would lose a short one)
          float g = 0.f;
#pragma unroll
          for (int j = 1; j < kBlk; ++j) g += j > s && j <= t ? sG[j] : 0.f;
          x *= fast_exp(g);
        }
        sLP[r][s] = r < kBlk ? (s < t ? sB[t] * x : 0.f) : (s <= t ? x : 0.f);
      }
      __syncthreads();
      // ---- E: tokens 0-3 in the first 16 lanes, 4-7 in the next
      const int tb = 4 * (lg & 1);
      floatx4 ld[4], lx[4], e[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ld[i] = *reinterpret_cast<const floatx4*>(&sLP[tb + i][tb]);
        lx[i] = *reinterpret_cast<const floatx4*>(&sLP[4 + i][0]);
      }
      const floatx4 be = *reinterpret_cast<const floatx4*>(&sB[tb]), lam = *reinterpret_cast<const floatx4*>(&sTo[tb]),
                    wt = *reinterpret_cast<const floatx4*>(&sOn[tb]);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        floatx4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = be[i] * (vv[i][b] - lam[i] * yz[b][i]);
        auto solve = [&](floatx4 y) {
          y[1] -= ld[1][0] * y[0];
          y[2] -= ld[2][0] * y[0] + ld[2][1] * y[1];
          y[3] -= ld[3][0] * y[0] + ld[3][1] * y[1] + ld[3][2] * y[2];
          return y;
        };
        floatx4 y = solve(x);
        if (nt > 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float f = __shfl(y[j], lr, 64);   // e of token j
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] -= lx[i][j] * f;
          }
          const floatx4 y1 = solve(x);
          if (lg == 1) y = y1;
        }
        e[b] = lg < 2 ? y : floatx4{0.f, 0.f, 0.f, 0.f};
      }
      // ---- O: rows 8-15 of the products, plus P E
      {
        floatx4 p4 = *reinterpret_cast<const floatx4*>(&sLP[lr][tb]);
        if (lr < kBlk || lg >= 2) p4 = floatx4{0.f, 0.f, 0.f, 0.f};
        floatx4 o[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          o[b] = lam * yz[b];
#pragma unroll
          for (int i = 0; i < 4; ++i) mma4(o[b], p4[i], e[b][i]);
        }
        if (lg >= 2)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (tb + i < nt) st2<T>(ob + (row0 + tb + i) * a.H * DV, a.scale * o[0][i], a.scale * o[1][i]);
      }
      if (DRAFT) {
        if (lg < 2)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (tb + i < nt)
              *reinterpret_cast<floatx2*>(a.tape + ((dst * a.tape_tokens + t0 + tb + i) * a.H + h) * R + DK + v0) =
                  floatx2{e[0][i], e[1][i]};
      }
      // ---- the state after the block (drafts: only for the block after it)
      if (!DRAFT || t0 + TB < rows.n) {
        if (lg < 2)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<floatx2*>(&sE[w][tb + i][2 * lr]) = floatx2{wt[i] * e[0][i], wt[i] * e[1][i]};
        __syncthreads();
        const float lc = sTo[TB - 1];
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          floatx4 f = {lc, lc, lc, lc};
          if (CH) f = *reinterpret_cast<const floatx4*>(&sLam[16 * m + 4 * lg]);
          S[m][0] *= f;
          S[m][1] *= f;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (4 * j >= nt) break;
          const floatx2 ej = *reinterpret_cast<const floatx2*>(&sE[w][4 * j + lg][2 * lr]);
#pragma unroll
          for (int m = 0; m < MB; ++m) {
            const float x = CH ? sKw[4 * j + lg][16 * m + lr] : sKt[4 * j + lg][16 * m + lr];
            mma4(S[m][0], x, ej[0]);
            mma4(S[m][1], x, ej[1]);
          }
        }
      }
    }
    __syncthreads();
  }
  if (!DRAFT) store_state();
}

template <typename T, int DK, int DV, bool CH, bool DRAFT>
hipError_t launch_tb(const SlotArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.B * a.H));
  if (a.T <= 1) hipLaunchKernelGGL((slot_tokens<T, DK, DV, CH, 1, DRAFT>), grid, dim3(DV * 2), 0, s, a);
  else hipLaunchKernelGGL((slot_tokens<T, DK, DV, CH, kBlk, DRAFT>), grid, dim3(DV * 2), 0, s, a);
  return hipGetLastError();
}
template <typename T, int DK, int DV, bool CH>
hipError_t launch_draft(const SlotArgs& a, hipStream_t s) {
  return a.tape ? launch_tb<T, DK, DV, CH, true>(a, s) : launch_tb<T, DK, DV, CH, false>(a, s);
}

template <typename T, int DK, int DV>
hipError_t launch_gate(const SlotArgs& a, hipStream_t s) {
  return a.gate == kGateChannel ? launch_draft<T, DK, DV, true>(a, s) : launch_draft<T, DK, DV, false>(a, s);
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
  return io_bf16 ? launch_dims<bf16>(a, s) : launch_dims<float>(a, s);
}

}  // namespace pdn
