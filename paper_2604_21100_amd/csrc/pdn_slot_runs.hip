// pdn_slot_fwd over more than a block of tokens in the modes whose operands are not
// bf16 numbers (fp32 tensors, per-channel decays, write keys that need a sum over their
// channels, preconditioned queries): the blocks of eight of pdn_slots.hip, one after
// the other, in fp32 throughout, with the work split over two kinds of waves.
//
// Consumer waves hold the head's state, 16 columns each, and do what depends on it:
//   X = Diag(beta) (V - Diag(lam) K S^T)   E = (I + L)^{-1} X   O = scale (Diag(lam) Q S^T + P E)
//   S'^T = lam_C S^T + Kt^T Diag(lam_C / lam) E
// Four producer waves form the operands of the blocks after it: key, query and write-
// key rows, a channel a lane; their products, a share of the channels a wave.  A step
// has two barriers; block n's operands are formed in one step, its L and P are
// summed and it is consumed in the next.
//
// What bounds it: the step's chain, 1.8 us at 64 x 64 and 3.7 at 128 x 128, of which the
// fp32 matrix instructions are a fifth and two fifths (the products with the state fill
// the matrix unit while nothing else gets on; then the producers' write keys, decays
// and rows; then solve, update and output).  3 fp32 prompts of up to 333 tokens x 4
// heads of 64: 76 us; 12 per-channel ones of up to 700 x 16 heads of 128: 327 us (one
// after the other, without producers, 135 and, with products a quarter cheaper, 479).
// Producers at a higher priority made it 5 and 4 % slower.
#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_slots.hpp"
#include "pdn_tile.hpp"

namespace pdn {

namespace {

template <typename T, int DK, int W, bool CH>
struct Run {
  static constexpr int LD = DK + 4, NW = W / 16, LC = CH ? kSlotBlock : 1;
  alignas(16) T raw[3][kSlotBlock][DK];              // keys, queries, the caller's write keys
  alignas(16) float g[LC][LD];                       // CH: log-decays
  // operands, of the block in use and the one after it: keys over queries; write
  // keys, with CH as they are and decayed to the block's end; CH: the decay over it
  alignas(16) float KQ[2][2 * kSlotBlock][LD], Kt[2][kSlotBlock][LD], Kw[2][LC][LD], lam[2][CH ? DK : 4];
  // CH: operands of the products of channel_rows (the columns of the second are Kt)
  alignas(16) float R1[CH ? 16 : 1][LD], R2[CH ? 16 : 1][LD], C1[CH ? kPairCols : 1][LD];
  alignas(16) float part[4][16][kSlotBlock], LP[16][kSlotBlock + 4], E[NW][kSlotBlock][16], sum[4][kSlotBlock];
  // of each token: log-decay, the decay to it and from it within the block, write
  // strength, preconditioner gain and decay
  alignas(16) float tok[4][6][kSlotBlock];
};

// W: the head's columns that a workgroup holds (half of them: without a preconditioner
// state, which in place is one workgroup's to read and write)
template <typename T, int DK, int DV, bool CH, int W>
__global__ __launch_bounds__(W * 4 + 256) void slot_runs(SlotArgs a) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  using R = Run<T, DK, W, CH>;
  constexpr int B = kSlotBlock, NW = R::NW, MB = DK / 16;
  __shared__ R s;
  const SlotWhere where = slot_where(a, DV / W);
  const int64_t seq = where.seq, h = where.h, hk = where.hk;
  const int64_t src = a.slot ? a.slot[seq] : seq, dst = a.slot_out ? a.slot_out[seq] : src;
  if (src < 0 || src >= a.slots || dst < 0 || dst >= a.slots) return;
  const SlotRows rows = slot_rows(a, seq);
  const bool fresh = a.fresh && a.fresh[seq] != 0;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, lr = l & 15, lg = l >> 4;
  const int nb = static_cast<int>((rows.n + B - 1) / B);
  const bool sums = slot_needs_sum(a);
  // A tensor's rows block by block: a buffer that ends with the sequence (past it reads
  // are zeros and writes are dropped; of a tensor that is not there, all), moved on by
  // a block each time (its place as a product would take tens of instructions).
  struct Rows {
    const char* base;
    uint32_t step, width;   // bytes
  };
  auto rows_of = [&](const void* p, int64_t stride, int64_t first, int width, int esz) {
    return Rows{static_cast<const char*>(p) + (rows.lo * stride + first) * esz, p ? static_cast<uint32_t>(stride * esz) : 0,
                p ? static_cast<uint32_t>(width * esz) : 0};
  };
  auto next = [&](Rows& r, int n) {   // n: rows left
    const __amdgpu_buffer_rsrc_t v = buf_rsrc(r.base, n > 0 ? (min(n, B) - 1) * r.step + r.width : 0);
    r.base += static_cast<uint64_t>(r.step) * B;
    return v;
  };

  if (w < NW) {
    // ------------------------------------------------------------ consumers
    const int v0 = where.part * W + 16 * w + lr, tb = 4 * (lg & 1), at = 4 * lg * DV + v0;
    SlotColumns<DK, DV> S;
    if (fresh) S.zero();
    else S.load(slot_head<DK, DV>(a, src, h), at);
    float vn[4];
    Rows rv = rows_of(a.v, a.v_stride, h * DV, DV, sizeof(T)), ro = rows_of(a.o, a.H * DV, h * DV, DV, sizeof(T));
    int left = static_cast<int>(rows.n), left_v = left;   // rows from the block in use, and from the next values
    auto load_v = [&]() {
      const __amdgpu_buffer_rsrc_t r = next(rv, left_v);
      left_v -= B;
#pragma unroll
      for (int i = 0; i < 4; ++i) vn[i] = buf_get<T>(r, static_cast<int>((tb + i) * rv.step + v0 * sizeof(T)));
    };
    if (nb > 0) {
      load_v();
      lds_sync();
    }
    for (int it = 0; it <= nb && nb > 0; ++it) {
      const int blk = it - 1, u = blk & 1;
      if (sums) lds_sync();
      floatx4 yz = {0.f, 0.f, 0.f, 0.f}, yz1 = yz;
      if (blk >= 0) {
        // ---- (rows of K over rows of Q) times S^T
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          const floatx4 r4 = *reinterpret_cast<const floatx4*>(&s.KQ[u][lr][16 * m + 4 * lg]);
#pragma unroll
          for (int i = 0; i < 4; ++i) mma4(i & 1 ? yz1 : yz, r4[i], S.t[m][i]);
        }
        settled(yz, yz1);
        yz += yz1;
      }
      lds_sync();   // A
      if (blk >= 0) {
        const float(*tok)[B] = s.tok[blk & 3];
        // ---- E: tokens 0-3 in the first 16 lanes, 4-7 in the next
        floatx4 ld[4], lx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ld[i] = *reinterpret_cast<const floatx4*>(&s.LP[tb + i][tb]);
          lx[i] = *reinterpret_cast<const floatx4*>(&s.LP[4 + i][0]);
        }
        const floatx4 be = *reinterpret_cast<const floatx4*>(&tok[3][tb]), lam = *reinterpret_cast<const floatx4*>(&tok[1][tb]),
                      wt = *reinterpret_cast<const floatx4*>(&tok[2][tb]);
        floatx4 p4 = *reinterpret_cast<const floatx4*>(&s.LP[lr][tb]);
        const float lc = tok[1][B - 1];
        reads_done();
        floatx4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = be[i] * (vn[i] - lam[i] * yz[i]);
        yz *= lam;
        load_v();
        floatx4 e = slot_solve4(ld, x);
        {
          floatx4 f;   // e of tokens 0-3
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = __shfl(e[j], lr, 64);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] -= (lx[i][0] * f[0] + lx[i][1] * f[1]) + (lx[i][2] * f[2] + lx[i][3] * f[3]);
          x = slot_solve4(ld, x);
          if (lg == 1) e = x;
        }
        if (lg >= 2) e = floatx4{0.f, 0.f, 0.f, 0.f};
        if (lg < 2)
#pragma unroll
          for (int i = 0; i < 4; ++i) s.E[w][tb + i][lr] = wt[i] * e[i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // ---- the state after the block
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          floatx4 f = {lc, lc, lc, lc};
          if (CH) f = *reinterpret_cast<const floatx4*>(&s.lam[u][16 * m + 4 * lg]);
          S.t[m] *= f;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float ej = s.E[w][4 * j + lg][lr];
#pragma unroll
          for (int m = 0; m < MB; ++m) mma4(S.t[m], (CH ? s.Kw[u] : s.Kt[u])[4 * j + lg][16 * m + lr], ej);
        }
        // ---- O: rows 8-15 of the products, plus P E
        if (lr < B || lg >= 2) p4 = floatx4{0.f, 0.f, 0.f, 0.f};
        floatx4 pe = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) mma4(pe, p4[i], e[i]);
        // (the state's products are behind it too: its next use is a step away)
#pragma unroll
        for (int m = 0; m < MB; ++m) asm volatile("" : "+v"(S.t[m]));
        settled(pe);
        if (__any(!all_numbers(e))) {   // (once more, without them)
          const int first = first_of(take_out(e, tb, B));
          pe = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; ++i) mma4(pe, p4[i], e[i]);
          settled(pe);
          put_from(pe, tb, first, __builtin_nanf(""));
        }
        yz += pe;
        const __amdgpu_buffer_rsrc_t r = next(ro, left);
        left -= B;
        if (lg >= 2)
#pragma unroll
          for (int i = 0; i < 4; ++i) buf_put<T>(r, static_cast<int>((tb + i) * ro.step + v0 * sizeof(T)), a.scale * yz[i]);
      }
      lds_sync();   // B
    }
    S.store(slot_head<DK, DV>(a, dst, h), at);
  } else {
    // ------------------------------------------------------------ producers
    const int pw = w - NW, pt = pw * 64 + l, c = pt % DK;
    const bool key = pt < DK, qry = !key && pt < 2 * DK;
    const int prec = a.precond;
    const bool gram = has_gram(prec), both = prec == kATQ, scalar = a.gate == kGateScalar;
    const float mu = prec == kSquash ? fast_exp(a.log_a_scale[h]) : 0.f;
    float A = gram && !fresh ? a.A[(src * a.H + h) * DK + c] : 0.f;   // (query threads follow it too)
    constexpr int RP = B * DK * sizeof(T) / 16, NRP = (RP + 255) / 256, GP = B * DK * 4 / 16, NGP = (GP + 255) / 256;
    u32x4 rk[NRP], rq[NRP], rx[NRP], rg[NGP];
    float s_b, s_g, s_bp, s_gp;
    // (each read whether it is used or not: a branch would wait for the loads)
    Rows vk = rows_of(a.k, a.k_stride, hk * DK, DK, sizeof(T)), vq = rows_of(a.q, a.q_stride, hk * DK, DK, sizeof(T)),
         vx = rows_of(prec == kExternal ? a.ktilde : nullptr, a.Hk * DK, hk * DK, DK, sizeof(T)),
         vg = rows_of(CH ? a.g : nullptr, a.H * DK, h * DK, DK, 4),
         nbe = rows_of(a.beta, a.H, h, 1, 4), ng = rows_of(scalar ? a.g : nullptr, a.H, h, 1, 4),
         nbp = rows_of(gram ? a.beta_p : nullptr, a.H, h, 1, 4), ngp = rows_of(gram ? a.g_p : nullptr, a.H, h, 1, 4);
    int left = static_cast<int>(rows.n);
    auto load_rows = [&]() {
      auto piece = [&](__amdgpu_buffer_rsrc_t r, uint32_t step, int row_bytes, int x) {
        const uint32_t at = x * 256 + pt, t = at * 16 / row_bytes, o = at * 16 % row_bytes;
        return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, static_cast<int>(t * step + o), 0, 0));
      };
      auto rows_in = [&](Rows& v, auto& to, int row_bytes) {
        const __amdgpu_buffer_rsrc_t r = next(v, left);
#pragma unroll
        for (int x = 0; x < static_cast<int>(sizeof(to) / 16); ++x) to[x] = piece(r, v.step, row_bytes, x);
      };
      rows_in(vk, rk, DK * sizeof(T));
      rows_in(vq, rq, DK * sizeof(T));
      rows_in(vx, rx, DK * sizeof(T));
      if (CH) rows_in(vg, rg, DK * 4);
      auto number = [&](Rows& v) { return buf_get<float>(next(v, left), static_cast<int>((l & 7) * v.step)); };
      s_b = number(nbe);
      s_g = number(ng);
      s_bp = number(nbp);
      s_gp = number(ngp);
      left -= B;
    };
    auto put_rows = [&](int blk) {
      auto put = [&](void* p, const u32x4& v, int x, int pieces, int row_bytes, int ld_bytes) {
        const int at = x * 256 + pt;
        if (at < pieces)
          *reinterpret_cast<u32x4*>(static_cast<char*>(p) + at * 16 / row_bytes * ld_bytes + at * 16 % row_bytes) = v;
      };
#pragma unroll
      for (int x = 0; x < NRP; ++x) {
        put(s.raw[0], rk[x], x, RP, DK * sizeof(T), DK * sizeof(T));
        put(s.raw[1], rq[x], x, RP, DK * sizeof(T), DK * sizeof(T));
        put(s.raw[2], rx[x], x, RP, DK * sizeof(T), DK * sizeof(T));
      }
      if (CH)
#pragma unroll
        for (int x = 0; x < NGP; ++x) put(s.g, rg[x], x, GP, DK * 4, R::LD * 4);
      if (pw == 3) {
        const int t = l & 7;
        const float g = sum_decay(s_g);   // (zero where there is none)
        float to, on;
        block_sums(g, l, &to, &on);
        if (l < B) {
          float(*tok)[B] = s.tok[blk & 3];
          tok[0][t] = g;
          tok[1][t] = fast_exp(to);
          tok[2][t] = fast_exp(on);
          tok[3][t] = s_b;
          tok[4][t] = s_bp;
          tok[5][t] = fast_exp(s_gp);
        }
      }
    };
    // key, query and write-key rows
    auto put_operands = [&](int blk) {
      const int u = blk & 1;
      const float(*tok)[B] = s.tok[blk & 3];
      const int nt = static_cast<int>(min<int64_t>(B, rows.n - static_cast<int64_t>(blk) * B));
      float kt[B], kv[B], At[B];
      float ex[B], up[B], lam = 1.f;   // CH: a token's decay, that from the block's start
      const float Ab = A;
#pragma unroll
      for (int t = 0; t < B; ++t) {
        kv[t] = to_f(s.raw[0][t][c]);
        if (CH) {
          ex[t] = fast_exp(s.g[t][c]);
          lam *= ex[t];
          up[t] = lam;
        }
      }
      if (gram)   // (a token past the end leaves A: no gain, no decay)
#pragma unroll
        for (int t = 0; t < B; ++t) {
          A = tok[5][t] * A + tok[4][t] * kv[t] * kv[t];
          At[t] = A;
        }
      if (qry) {
        float q[B];
#pragma unroll
        for (int t = 0; t < B; ++t) {
          q[t] = to_f(s.raw[1][t][c]);
          if (both) q[t] /= At[t] + a.ridge;
          if (!CH) s.KQ[u][B + t][c] = q[t];
        }
        if constexpr (CH) channel_rows(q, ex, up, 1, c, s.KQ[u], s.R1, s.R2);
      }
      if (key) {
        if (prec == kSquash) {
#pragma unroll
          for (int t = 0; t < B; ++t) kt[t] = squash_gain(At[t], mu, a.lnx) * kv[t];
        } else if (prec == kDiagSM) {
#pragma unroll
          for (int t = 0; t < B; ++t) kt[t] = kv[t] / ((t ? At[t - 1] : Ab) + a.ridge);
        } else {
#pragma unroll
          for (int t = 0; t < B; ++t) kt[t] = prec == kExternal ? to_f(s.raw[2][t][c]) : kv[t];
        }
      }
      if (sums) {   // the write key's row sums
#pragma unroll
        for (int t = 0; t < B; ++t) {
          float x = key ? kv[t] * kt[t] : 0.f;
#pragma unroll
          for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
          if (l == 0) s.sum[pw][t] = x;
        }
        lds_sync();
        if (key)
#pragma unroll
          for (int t = 0; t < B; ++t) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < DK / 64; ++i) m += s.sum[i][t];
            kt[t] = t < nt ? slot_sum_factor(a, m, tok[3][t], tok[0][t]) * kt[t] : 0.f;
          }
      }
      if (key) {
        // (a linear-attention update has no correction by the state: no key rows)
        if (both)
#pragma unroll
          for (int t = 0; t < B; ++t) kv[t] = 0.f;
        if constexpr (CH) {
          channel_rows(kv, ex, up, 0, c, s.KQ[u], s.R1, s.R2);
          channel_cols(kt, ex, c, s.C1, s.Kt[u], s.Kw[u]);
          s.lam[u][c] = lam;
        } else {
#pragma unroll
          for (int t = 0; t < B; ++t) {
            s.KQ[u][t][c] = kv[t];
            s.Kt[u][t][c] = kt[t];
          }
        }
      }
    };
    // (rows of K over rows of Q) times Kt^T, a share of the channels a wave; CH: two waves
    // each of the two products
    constexpr int NP = CH ? 2 : 4;
    auto put_products = [&](int blk) {
      const int u = blk & 1, pass = pw / NP;
      const float(*const rows16)[R::LD] = !CH ? s.KQ[u] : pass ? s.R2 : s.R1;
      const float(*const cols8)[R::LD] = !CH || pass ? s.Kt[u] : s.C1;
      floatx4 g4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < MB / NP; ++x) {
        const int m = NP * x + pw % NP;
        const floatx4 r4 = *reinterpret_cast<const floatx4*>(&rows16[lr][16 * m + 4 * lg]);
        const floatx4 t4 = *reinterpret_cast<const floatx4*>(&cols8[lr & 7][16 * m + 4 * lg]);
#pragma unroll
        for (int i = 0; i < 4; ++i) mma4(g4, r4[i], t4[i]);
      }
      settled(g4);
      if (lr < B)
#pragma unroll
        for (int i = 0; i < 4; ++i) s.part[pw][4 * lg + i][lr] = g4[i];
    };
    auto put_lp = [&](int blk) {   // (by the last two waves, which have no write keys to form)
      const int r = (pt - 128) / B, x = pt % B, t = r % B;
      const float(*tok)[B] = s.tok[blk & 3];
      float v;
      if (CH) {
        int col;
        const int row = channel_pair(r, x, &col), p = row / 16 * NP;
        v = s.part[p][row % 16][col] + s.part[p + 1][row % 16][col];
      } else {
        v = (s.part[0][r][x] + s.part[1][r][x]) + (s.part[2][r][x] + s.part[3][r][x]);
      }
      if (!CH) {   // (summed token by token: a difference of two long sums would lose a short one)
        float g = 0.f;
#pragma unroll
        for (int j = 1; j < B; ++j) g += j > x && j <= t ? tok[0][j] : 0.f;
        v *= fast_exp(g);
      }
      s.LP[r][x] = r < B ? (x < t ? tok[3][t] * v : 0.f) : (x <= t ? v : 0.f);
    };
    auto store_A = [&]() {
      if (gram && key) a.A[(dst * a.H + h) * DK + c] = A;
    };
    if (nb == 0) {   // (by itself: see below)
      store_A();
      return;
    }
    load_rows();
    put_rows(0);
    // A has been loaded too.  Said outright (vmcnt 0), and on every way into the loop, or
    // the compiler waits for it, and with it for the loads just issued, each time round.
    __builtin_amdgcn_s_waitcnt(0x0f70);
    load_rows();
    lds_sync();
    for (int it = 0; it <= nb; ++it) {
      if (it > 0 && pw >= 2) put_lp(it - 1);
      if (it < nb) put_operands(it);
      else if (sums) lds_sync();
      lds_sync();   // A
      if (it < nb) put_products(it);
      put_rows(it + 1);
      load_rows();
      lds_sync();   // B
    }
    store_A();
  }
}

template <typename T, int DK, int DV, bool CH>
hipError_t launch(const SlotArgs& a, hipStream_t s) {
  const unsigned heads = static_cast<unsigned>(a.B * a.H);
  if constexpr (DV == 128) {
    if (slot_halves(a)) {
      hipLaunchKernelGGL((slot_runs<T, DK, DV, CH, 64>), dim3(2 * heads), dim3(64 * 4 + 256), 0, s, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((slot_runs<T, DK, DV, CH, DV>), dim3(heads), dim3(DV * 4 + 256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DK, int DV>
hipError_t launch_gate(const SlotArgs& a, hipStream_t s) {
  return a.gate == kGateChannel ? launch<T, DK, DV, true>(a, s) : launch<T, DK, DV, false>(a, s);
}

template <typename T>
hipError_t launch_dims(const SlotArgs& a, hipStream_t s) {
  if (a.dk == 64) return a.dv == 64 ? launch_gate<T, 64, 64>(a, s) : launch_gate<T, 64, 128>(a, s);
  return a.dv == 64 ? launch_gate<T, 128, 64>(a, s) : launch_gate<T, 128, 128>(a, s);
}

}  // namespace

hipError_t launch_slot_runs(const SlotArgs& a, int io_bf16, hipStream_t s) {
  return io_bf16 ? launch_dims<bf16>(a, s) : launch_dims<float>(a, s);
}

}  // namespace pdn
