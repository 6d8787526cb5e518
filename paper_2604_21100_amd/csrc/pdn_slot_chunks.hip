// pdn_slot_fwd over prompts: the rule in chunks of 32 tokens, one launch, fp32
// results from bf16 matrix products.  Per chunk, from the state S^T at its start
// (lam_t the decay from the chunk's start, w_t that to its end):
//   X = Diag(beta) (V - Diag(lam) K S^T)     E = M X,  M = (I + L)^{-1}
//   O = scale (Diag(lam) Q S^T + P E)        S'^T = lam_C S^T + Kt^T Diag(w) E
//   L[t][s] = beta_t lam_t/lam_s k_t . kt_s (s < t)   P[t][s] = lam_t/lam_s q_t . kt_s (s <= t)
//
// Precision.  An fp32 operand goes into the bf16 matrix instruction as the sum of
// three bf16 numbers, which hold all its 24 bits, and of a product of two such
// sums the six terms down to 2^-16 are taken: what is dropped is 2^-24 of the
// product.  Queries and keys in bf16 are exact as they are.  The instruction adds
// in fp32, and the state stays fp32 in its accumulators.  That goes for o as well: its
// terms may cancel, and two parts (2^-16) would show in it after its own rounding (they
// took 158 and 220 us where three take 164 and 238).
//
// A workgroup holds one head's state for all of its sequence.  Its consumer waves
// own 16 columns each: a lane has rows 32 kk + 8 g + 4 u + i (g = lane / 16) of
// column lane % 16, the rows of an accumulator tile (kk, u) being so chosen that
// two tiles are the eight contraction elements of the next product, so S, X and E
// never leave registers.  Four producer waves meanwhile form the next chunk's
// operands in LDS: write keys and preconditioner state, two channels and an
// eighth or a quarter of the chunk a lane; L and P by matrix products; M from two
// 16 x 16 inverses by substitution and M21 = -M22 L21 M11.
//
// What bounds it: a chunk's chain on one compute unit, which a workgroup has to itself
// (its LDS), 5.3 us with SQUASH and 3.8 without.  The vector unit issues in about two
// thirds of the cycles (splitting operands, a third of it; write keys and their
// logarithms), the matrix unit in a third.  16 ragged prompts of up to 1000 tokens x 16
// heads, SQUASH: 168 us; 8 of up to 2048 x 32 heads, k~ = k: 242 us; on the fp32 matrix
// instruction the operations alone would be 100 and 171 us, were lengths equal.
// Measured and not kept: 32 columns a wave (217 against 178 us: too few waves hide
// the chain), tokens shared unevenly among the producers to even out their time (171
// to 172 us), the remainders x - p[0] by the bf16 dot product (no faster).
#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_slots.hpp"
#include "pdn_tile.hpp"

namespace pdn {

namespace {

constexpr int kC = 32;

// two bf16 numbers in a register
__device__ __forceinline__ floatx2 pair_f(uint32_t x) {
  return floatx2{__builtin_bit_cast(float, x << 16), __builtin_bit_cast(float, x & 0xffff0000u)};
}
// The parts of two fp32 numbers: x = p[0] + p[1] + .., each bf16, in the halves of
// a register (the conversion takes two at a time; said so, or it is made twice).
template <int N>
__device__ __forceinline__ void parts(floatx2 x, uint32_t (&p)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    p[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, typename Vec2<bf16>::type));
    if (j + 1 < N) x -= pair_f(p[j]);
  }
}
// two accumulator tiles as the right operand of a slab
template <int N>
__device__ __forceinline__ void parts8(const floatx4& a, const floatx4& b, bf16x8 (&f)[N]) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 r[N];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t p[N];
    parts<N>(i < 2 ? floatx2{a[2 * i], a[2 * i + 1]} : floatx2{b[2 * i - 4], b[2 * i - 3]}, p);
#pragma unroll
    for (int j = 0; j < N; ++j) r[j][i] = p[j];
  }
#pragma unroll
  for (int j = 0; j < N; ++j) f[j] = __builtin_bit_cast(bf16x8, r[j]);
}
// acc += (a[0] + a[1] + ..) (b[0] + b[1] + ..), small terms first, those of
// part numbers past `most` left out
template <int NA, int NB>
__device__ __forceinline__ void mma_parts(floatx4& acc, const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], int most) {
#pragma unroll
  for (int s = NA + NB - 2; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s <= most && s - i >= 0 && s - i < NB) acc = mfma(a[i], b[s - i], acc);
}

// LDS, byte offsets.  K and Q tiles and per-token numbers four times (the chunk in
// use, and those one, two and three after it), what is formed from them twice.
template <int DK, int NP>
struct Lay {
  static constexpr int kTile = kC * DK * 2, kMat = kC * kC * 2;
  static constexpr int oK = 0, oQ = oK + 4 * kTile, oX = oQ + 4 * kTile;            // oX: external write keys
  static constexpr int oT = oX + (NP == 0 ? 4 * kTile : 0);                         // write keys' parts
  static constexpr int oM = oT + (NP == 3 ? 2 * 3 * kTile : 0), oP = oM + 3 * kMat;
  static constexpr int oL = oP + 2 * 3 * kMat, kL = kC * (kC + 4) * 4, oF = oL + kL;   // L, M in fp32
  static constexpr int oA = oF + kL;                                                // per segment and channel, sums of bp k^2
  static constexpr int oS = oA + (NP == 3 ? 512 * 4 : 0), kS = 8 * kC * 4;          // see load_scalars
  static constexpr int total = oS + 4 * kS;
};

// NP: the write keys' parts, 3 (SQUASH); 1: they are the keys; 0: the caller's.
// W: the head's columns that a workgroup holds.
template <int DK, int DV, int NP, int W>
__global__ __launch_bounds__(W * 4 + 256) void slot_chunks(SlotArgs a) {
  using L = Lay<DK, NP>;
  static_assert(W == DV || NP != 3, "a preconditioner state in place is one workgroup's to read and write");
  constexpr int NC = W / 16, KK = DK / 32, NCH = DK / 8, RK = DK * 2, NT = NP == 3 ? 3 : 1;
  __shared__ __attribute__((aligned(1024))) char smem[L::total];
  lds_char* const sm = (lds_char*)smem;
  const SlotWhere where = slot_where(a, DV / W);
  const int64_t seq = where.seq, h = where.h, hk = where.hk;
  const int64_t src = a.slot ? a.slot[seq] : seq, dst = a.slot_out ? a.slot_out[seq] : src;
  if (src < 0 || src >= a.slots || dst < 0 || dst >= a.slots) return;
  const SlotRows rows = slot_rows(a, seq);
  const bool fresh = a.fresh && a.fresh[seq] != 0;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, m = l & 15, g = l >> 4;
  const int r0 = 8 * (m >> 2) + (m & 3);   // left-operand row of this lane, then + 4 u
  const int nch = static_cast<int>((rows.n + kC - 1) / kC);
  auto kt_tile = [&](int it, int p) {   // part p of chunk it's write keys
    return sm + (NP == 3 ? L::oT + ((it & 1) * 3 + p) * L::kTile : (NP == 1 ? L::oK : L::oX) + (it & 3) * L::kTile);
  };
  auto mat_m = [&](int p) { return sm + L::oM + p * L::kMat; };
  auto mat_p = [&](int it, int p) { return sm + L::oP + ((it & 1) * 3 + p) * L::kMat; };
  auto scal = [&](int it, int x) { return sm + L::oS + (it & 3) * L::kS + x * kC * 4; };
  // the first row of chunk it's L that is not all numbers (the inverse is formed without
  // what is none, and its rows from that one on are made NaN)
  typedef __attribute__((address_space(3))) int lds_int;
  auto first_row = [&](int it) { return reinterpret_cast<lds_int*>(scal(it, 5) + 8 * 4); };

  if (w < NC) {
    // ------------------------------------------------------------ consumers
    const int v0 = where.part * W + 16 * w + m;
    floatx4 S[KK][2];
    {
      const float* sp = a.S + (src * a.H + h) * (DK * DV) + 8 * g * DV + v0;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int r = 0; r < 8; ++r) S[kk][r / 4][r % 4] = fresh ? 0.f : sp[(32 * kk + r) * DV];
    }
    // A chunk's rows of v and o, this lane's eight of a column (two bytes a lane: 32
    // adjacent ones a row and wave, and the waves of a row run together).  Past the
    // sequence's end nothing is read, or written.
    auto view = [&](const void* p, int64_t stride, int ch) {
      const int64_t t0 = static_cast<int64_t>(ch) * kC, n = min<int64_t>(kC, rows.n - t0);
      return buf_rsrc(static_cast<const char*>(p) + ((rows.lo + t0) * stride + h * DV) * 2,
                      n > 0 ? static_cast<uint32_t>(((n - 1) * stride + DV) * 2) : 0);
    };
    float vn[8];
    auto load_v = [&](int ch) {
      const __amdgpu_buffer_rsrc_t r = view(a.v, a.v_stride, ch);
      const uint32_t step = static_cast<uint32_t>(a.v_stride * 2), at = 8 * g * step + v0 * 2;
#pragma unroll
      for (int i = 0; i < 8; ++i) vn[i] = buf_get<bf16>(r, static_cast<int>(at + i * step));
    };
    load_v(0);
    lds_sync();
    lds_sync();
    lds_sync();   // (the first chunk is being formed)
    lds_sync();
    for (int ch = 0; ch < nch; ++ch) {
      // ---- K S^T and Q S^T (operands are read one slab ahead of their use)
      floatx4 y[2], z[2], e[2], be[2], lam[2];
      bf16x8 kq[2][2][2][1];
      auto load_kq = [&](int kk) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int off = (ch & 3) * L::kTile + tile_off<NCH>(r0, 4 * kk + g) + 4 * u * RK;
          kq[kk & 1][0][u][0] = lds_frag(sm + L::oK + off);
          kq[kk & 1][1][u][0] = lds_frag(sm + L::oQ + off);
        }
      };
      load_kq(0);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        y[u] = z[u] = e[u] = floatx4{0.f, 0.f, 0.f, 0.f};
        be[u] = lds_f4(scal(ch, 0) + (8 * g + 4 * u) * 4);
        lam[u] = lds_f4(scal(ch, 1) + (8 * g + 4 * u) * 4);
      }
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (kk + 1 < KK) load_kq(kk + 1);
        reads_done();
        bf16x8 sp[3];
        parts8<3>(S[kk][0], S[kk][1], sp);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          mma_parts(y[u], kq[kk & 1][0][u], sp, 2);
          mma_parts(z[u], kq[kk & 1][1][u], sp, 2);
        }
      }
      // ---- X
      bf16x8 tp[2][NT];
      auto load_t = [&](int x) {   // the write keys' columns of tile x = 2 kk + u
#pragma unroll
        for (int p = 0; p < NT; ++p)
          tp[x & 1][p] = lds_frag_t(kt_tile(ch, p) + tile_off<NCH>(8 * g + (m >> 2), 4 * (x >> 1) + (m & 3)) + (x & 1) * 8, 4 * RK);
      };
      load_t(0);
      reads_done();
      bf16x8 xp[3];
      floatx4 x[2];
      {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i)   // (a row past the end has no strength, and no value that could spoil that)
            x[u][i] = be[u][i] * (vn[4 * u + i] - lam[u][i] * y[u][i]);
          z[u] *= lam[u];
        }
        load_v(ch + 1);
        parts8<3>(x[0], x[1], xp);
      }
      lds_sync();   // A
      // ---- E = M X, the state after the chunk
      bf16x8 ep[3], wp[3], mp[2][3];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int p = 0; p < 3; ++p) mp[u][p] = lds_frag(mat_m(p) + tile_off<4>(r0, g) + 4 * u * (kC * 2));
      const floatx4 w0 = lds_f4(scal(ch, 2) + 8 * g * 4), w1 = lds_f4(scal(ch, 2) + (8 * g + 4) * 4);
      const float lc = lds_f4(scal(ch, 1) + (kC - 4) * 4)[3];
      reads_done();
#pragma unroll
      for (int u = 0; u < 2; ++u) mma_parts(e[u], mp[u], xp, 2);
      parts8<3>(w0 * e[0], w1 * e[1], wp);
      bf16x8 pp[2][3];
#pragma unroll
      for (int x = 0; x < 2 * KK; ++x) {
        if (x + 1 < 2 * KK) {
          load_t(x + 1);
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int p = 0; p < 3; ++p) pp[u][p] = lds_frag(mat_p(ch, p) + tile_off<4>(r0, g) + 4 * u * (kC * 2));
        }
        reads_done();
        floatx4& t = S[x >> 1][x & 1];
        t *= lc;
        mma_parts(t, tp[x & 1], wp, 2);
      }
      parts8<3>(e[0], e[1], ep);
      // ---- O
      const __amdgpu_buffer_rsrc_t ro = view(a.o, a.H * DV, ch);
      const uint32_t step = static_cast<uint32_t>(a.H * DV * 2), at = 8 * g * step + v0 * 2;
      floatx4 pe[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        pe[u] = floatx4{0.f, 0.f, 0.f, 0.f};
        mma_parts(pe[u], pp[u], ep, 2);
      }
      if (__any(!all_numbers(e[0]) || !all_numbers(e[1]))) {   // (both once more, without them)
        const int first = min(first_of(take_out(x[0], 8 * g, take_out(x[1], 8 * g + 4, kC))), *first_row(ch));
        parts8<3>(x[0], x[1], xp);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bf16x8 m3[3];
#pragma unroll
          for (int p = 0; p < 3; ++p) m3[p] = lds_frag(mat_m(p) + tile_off<4>(r0, g) + 4 * u * (kC * 2));
          e[u] = floatx4{0.f, 0.f, 0.f, 0.f};
          mma_parts(e[u], m3, xp, 2);
        }
        settled(e[0], e[1]);
        put_from(e[0], 8 * g, first, 0.f);
        put_from(e[1], 8 * g + 4, first, 0.f);
        parts8<3>(e[0], e[1], ep);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          pe[u] = floatx4{0.f, 0.f, 0.f, 0.f};
          mma_parts(pe[u], pp[u], ep, 2);
        }
        settled(pe[0], pe[1]);
        put_from(pe[0], 8 * g, first, __builtin_nanf(""));
        put_from(pe[1], 8 * g + 4, first, __builtin_nanf(""));
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        z[u] += pe[u];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, static_cast<bf16>(a.scale * z[u][i])), ro,
                                                static_cast<int>(at + (4 * u + i) * step), 0, 0);
      }
      lds_sync();   // B
    }
    int at = 8 * g * DV + v0;
    asm volatile("" : "+v"(at));   // (or these addresses are formed at the start and held throughout)
    float* sp = a.S + (dst * a.H + h) * (DK * DV) + at;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int r = 0; r < 8; ++r) sp[(32 * kk + r) * DV] = S[kk][r / 4][r % 4];
  } else {
    // ------------------------------------------------------------ producers
    constexpr int PAIRS = DK / 2, SEGS = 256 / PAIRS, TOK = kC / SEGS;   // channel pairs; tokens a lane forms keys of
    typedef __attribute__((address_space(3))) floatx2 lds_floatx2;
    typedef __attribute__((address_space(3))) double lds_double;
    typedef __attribute__((address_space(3))) uint32_t lds_u32;
    typedef __attribute__((address_space(3))) uint16_t lds_u16;
    const int pw = w - NC, pt0 = pw * 64 + l;
    // The lane's number, made anew for each phase: what is formed from it, LDS
    // addresses above all, is then formed where it is used (held throughout, all of
    // them together take more registers than there are).
    int ll = l;
    __builtin_amdgcn_s_setprio(3);   // (a step ends with the slowest producer)
    auto anew = [&]() { asm volatile("" : "+v"(ll)); };
    const bool gram = NP == 3;
    const float mu = gram ? fast_exp(a.log_a_scale[h]) : 0.f;
    floatx2 A = {0.f, 0.f};
    float* const ap = gram ? a.A + h * DK + 2 * (pt0 % PAIRS) : nullptr;
    if (gram && !fresh) A = *reinterpret_cast<const floatx2*>(ap + src * a.H * DK);
    // A chunk's rows, through registers (16 bytes a lane and piece of a tile) into
    // LDS; those past the sequence's end read as zeros.
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    auto load_tile = [&](int ch, const void* p, int64_t stride, int64_t first, u32x4* to) {
      const int64_t row = rows.lo + static_cast<int64_t>(ch) * kC;
      const int n = static_cast<int>(min<int64_t>(kC, rows.n - static_cast<int64_t>(ch) * kC));
      const __amdgpu_buffer_rsrc_t r = buf_rsrc(static_cast<const char*>(p) + (row * stride + first) * 2,
                                                static_cast<uint32_t>(((n - 1) * stride + DK) * 2));
#pragma unroll
      for (int x = 0; x < kC * NCH / 256; ++x) {
        const uint32_t at = pw * 64 + ll + 256 * x;
        to[x] = __builtin_amdgcn_raw_buffer_load_b128(r, static_cast<int>(at / NCH * static_cast<uint32_t>(stride * 2) + at % NCH * 16), 0, 0);
      }
    };
    auto put_tile = [&](const u32x4* from, int o) {
#pragma unroll
      for (int x = 0; x < kC * NCH / 256; ++x) {
        const uint32_t at = pw * 64 + ll + 256 * x;
        lds_put(sm + o + tile_off<NCH>(at / NCH, at % NCH), __builtin_bit_cast(bf16x8, from[x]));
      }
    };
    u32x4 rk[DK / 64], rq[DK / 64], rx[DK / 64];
    auto load_keys = [&](int ch) {
      load_tile(ch, a.k, a.k_stride, hk * DK, rk);
      load_tile(ch, a.q, a.q_stride, hk * DK, rq);
      if (NP == 0) load_tile(ch, a.ktilde, a.Hk * DK, hk * DK, rx);
    };
    auto put_keys = [&](int ch) {
      const int buf = (ch & 3) * L::kTile;
      put_tile(rk, L::oK + buf);
      put_tile(rq, L::oQ + buf);
      if (NP == 0) put_tile(rx, L::oX + buf);
    };
    // Its per-token numbers, a lane a token: 0 write strength, 1 lam, 2 w, 3 gain
    // and 4 decay of the preconditioner, 5 that decay over a segment, 6 log-decay
    // from the chunk's start (64 bits: the decay between two tokens is a difference
    // of two of these)
    // (each read whether it is used or not: a branch here would wait for the loads)
    const float *const gb = a.gate == kGateScalar ? a.g : a.beta, *const bpb = gram ? a.beta_p : a.beta,
                *const gpb = gram && a.g_p ? a.g_p : a.beta;
    float s_be = 0.f, s_g = 0.f, s_bp = 0.f, s_gp = 0.f;
    auto load_scalars = [&](int ch) {
      const int64_t sc = (rows.lo + min(static_cast<int64_t>(ch) * kC + (ll & 31), rows.n - 1)) * a.H + h;
      s_be = a.beta[sc];
      s_g = gb[sc];
      s_bp = bpb[sc];
      s_gp = gpb[sc];
    };
    auto put_scalars = [&](int ch) {
      const int t = ll & 31;
      const bool in = static_cast<int64_t>(ch) * kC + t < rows.n;
      const float be = in ? s_be : 0.f, bp = in ? s_bp : 0.f, gp = in && a.g_p ? s_gp : 0.f;
      double to = in && a.gate == kGateScalar ? sum_decay(s_g) : 0.f;
#pragma unroll
      for (int off = 1; off < kC; off <<= 1) {
        const double x = __shfl_up(to, off, kC);
        if (t >= off) to += x;
      }
      const double end = __shfl(to, kC - 1, kC);
      const float dp = fast_exp(gp);
      float ds = dp;
#pragma unroll
      for (int off = 1; off < TOK; off <<= 1) ds *= __shfl_xor(ds, off, kC);
      if (ll < kC) {
        auto put = [&](int x, float v) { *reinterpret_cast<lds_float*>(scal(ch, x) + t * 4) = v; };
        put(0, be);
        put(1, fast_exp(static_cast<float>(to)));
        put(2, fast_exp(static_cast<float>(end - to)));
        put(3, bp);
        put(4, dp);
        if (t % TOK == 0) *reinterpret_cast<lds_float*>(scal(ch, 5) + t / TOK * 4) = ds;   // (eight at most)
        if (t == 0) *first_row(ch) = kC;
        *reinterpret_cast<lds_double*>(scal(ch, 6) + t * 8) = to;
      }
    };
    auto fl = [&](int o, int t, int x) { return reinterpret_cast<lds_float*>(sm + o + (t * (kC + 4) + x) * 4); };
    auto seg_sum = [&](int sg, int cp) { return reinterpret_cast<lds_floatx2*>(sm + L::oA + (sg * DK + 2 * cp) * 4); };
    // what this lane's tokens add to the preconditioner state of its two channels
    auto put_sums = [&](int ch) {
      const int pt = pw * 64 + ll, cp = pt % PAIRS, seg = pt / PAIRS;
      const lds_char* kp = sm + L::oK + (ch & 3) * L::kTile + (cp % 4) * 4;
      uint32_t x[TOK];
      floatx4 bp[TOK / 4], dp[TOK / 4];
#pragma unroll
      for (int j = 0; j < TOK; ++j) x[j] = *reinterpret_cast<const lds_u32*>(kp + tile_off<NCH>(seg * TOK + j, cp / 4));
#pragma unroll
      for (int j = 0; j < TOK / 4; ++j) {
        bp[j] = lds_f4(scal(ch, 3) + (seg * TOK + 4 * j) * 4);
        dp[j] = lds_f4(scal(ch, 4) + (seg * TOK + 4 * j) * 4);
      }
      reads_done();
      floatx2 sum = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < TOK; ++j) {
        const floatx2 k = pair_f(x[j]);
        sum = dp[j / 4][j % 4] * sum + bp[j / 4][j % 4] * k * k;
      }
      *seg_sum(seg, cp) = sum;
    };
    // its tokens' write keys; A: to the chunk's end
    auto put_write_keys = [&](int ch) {
      const int pt = pw * 64 + ll, cp = pt % PAIRS, seg = pt / PAIRS;
      const lds_char* kp = sm + L::oK + (ch & 3) * L::kTile + (cp % 4) * 4;
      uint32_t x[TOK];
      floatx4 bp[TOK / 4], dp[TOK / 4], ds[SEGS / 4];
      floatx2 sum[SEGS];
#pragma unroll
      for (int j = 0; j < SEGS; ++j) sum[j] = *seg_sum(j, cp);
#pragma unroll
      for (int j = 0; j < SEGS / 4; ++j) ds[j] = lds_f4(scal(ch, 5) + 16 * j);
#pragma unroll
      for (int j = 0; j < TOK / 4; ++j) {
        bp[j] = lds_f4(scal(ch, 3) + (seg * TOK + 4 * j) * 4);
        dp[j] = lds_f4(scal(ch, 4) + (seg * TOK + 4 * j) * 4);
      }
#pragma unroll
      for (int j = 0; j < TOK; ++j) x[j] = *reinterpret_cast<const lds_u32*>(kp + tile_off<NCH>(seg * TOK + j, cp / 4));
      reads_done();
      floatx2 s = A;
#pragma unroll
      for (int j = 0; j < SEGS; ++j) {
        if (j == seg) s = A;
        A = ds[j / 4][j % 4] * A + sum[j];
      }
#pragma unroll
      for (int j = 0; j < TOK; ++j) {
        const floatx2 k = pair_f(x[j]);
        s = dp[j / 4][j % 4] * s + bp[j / 4][j % 4] * k * k;
        uint32_t p[3];
        parts<3>(floatx2{squash_gain(s[0], mu, a.lnx) * k[0], squash_gain(s[1], mu, a.lnx) * k[1]}, p);
#pragma unroll
        for (int q = 0; q < 3; ++q)
          *reinterpret_cast<lds_u32*>(kt_tile(ch, q) + tile_off<NCH>(seg * TOK + j, cp / 4) + (cp % 4) * 4) = p[q];
      }
    };
    // L and P: a wave the rows 8 g + 4 u + i and columns r0 + 4 c of K Kt^T and Q Kt^T
    auto put_products = [&](int ch) {
      const int u = pw >> 1, c = pw & 1, m = ll & 15, g = ll >> 4, r0 = 8 * (m >> 2) + (m & 3);
      floatx4 kk4 = {0.f, 0.f, 0.f, 0.f}, qk4 = kk4;
      const int tile = (ch & 3) * L::kTile, s = r0 + 4 * c;
      const double Gs = *reinterpret_cast<const lds_double*>(scal(ch, 6) + s * 8);
      double Gt[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) Gt[i] = *reinterpret_cast<const lds_double*>(scal(ch, 6) + (8 * g + 4 * u + i) * 8);
      const floatx4 be = lds_f4(scal(ch, 0) + (8 * g + 4 * u) * 4);
#pragma unroll
      for (int k2 = 0; k2 < KK; k2 += 2) {
        bf16x8 k1[2][1], q1[2][1], tp[2][NT];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int off = tile_off<NCH>(r0, 4 * (k2 + x) + g);
          k1[x][0] = lds_frag(sm + L::oK + tile + off + 4 * u * RK);
          q1[x][0] = lds_frag(sm + L::oQ + tile + off + 4 * u * RK);
#pragma unroll
          for (int p = 0; p < NT; ++p) tp[x][p] = lds_frag(kt_tile(ch, p) + off + 4 * c * RK);
        }
        reads_done();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          mma_parts(kk4, k1[x], tp[x], 2);
          mma_parts(qk4, q1[x], tp[x], 2);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = 8 * g + 4 * u + i;
        const float d = fast_exp(static_cast<float>(Gt[i] - Gs));
        kk4[i] = s < t ? be[i] * d * kk4[i] : 0.f;
        qk4[i] = s <= t ? d * qk4[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const floatx2 pr = {qk4[i], qk4[i + 1]};
#pragma unroll
        for (int b = 0; b < 2; ++b) *fl(L::oL, 8 * g + 4 * u + i + b, s) = kk4[i + b];
        uint32_t p[3];
        parts<3>(pr, p);
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
          for (int b = 0; b < 2; ++b)
            *reinterpret_cast<lds_u16*>(mat_p(ch, q) + tile_off<4>(8 * g + 4 * u + i + b, s >> 3) + (s & 7) * 2) =
                static_cast<uint16_t>(b ? p[q] >> 16 : p[q]);
      }
      if (__any(!all_numbers(kk4))) {
        const int t = take_out(kk4, 8 * g + 4 * u, kC);
        if (t < kC) __hip_atomic_fetch_min(first_row(ch), t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
#pragma unroll
        for (int i = 0; i < 4; ++i) *fl(L::oL, 8 * g + 4 * u + i, s) = kk4[i];
      }
    };
    // M, by two waves: a lane a row of a 16 x 16 block, from M (I + L) = I, column
    // after column from the last, in both; then one puts the blocks into place, the
    // other forms M21.
    auto put_inverse = [&](int ch) {
      const int m = ll & 15, g = ll >> 4, b0 = ll & 16;   // lanes 0-15 the first block, 16-31 the second
      float x[16];
#pragma unroll
      for (int c = 0; c < 16; ++c) x[c] = m == c ? 1.f : 0.f;
      // (rows of L two at a time, two such groups ahead of their use)
      floatx4 lt[8][2][4];
      auto load_l = [&](int j2) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int c = 0; c <= j2 / 2; ++c) lt[j2][j][c] = *reinterpret_cast<lds_floatx4*>(fl(L::oL, b0 + 2 * j2 + j, b0 + 4 * c));
        reads_done();
      };
      load_l(7);
      load_l(6);
#pragma unroll
      for (int j2 = 7; j2 >= 0; --j2) {
        if (j2 >= 2) load_l(j2 - 2);
#pragma unroll
        for (int j = 2 * j2 + 1; j >= 2 * j2; --j)
#pragma unroll
          for (int c = 0; c < j; ++c) x[c] -= x[j] * lt[j2][j & 1][c / 4][c % 4];
      }
      if (pw == 0) {
        const int first = *first_row(ch);
        if (__any(first < kC))
#pragma unroll
          for (int c = 0; c < 16; ++c) x[c] = b0 + m >= first ? __builtin_nanf("") : x[c];
        if (ll < 32)
#pragma unroll
          for (int c = 0; c < 16; c += 8) {
            bf16x8 f8[3];
            parts8<3>(floatx4{x[c], x[c + 1], x[c + 2], x[c + 3]}, floatx4{x[c + 4], x[c + 5], x[c + 6], x[c + 7]}, f8);
#pragma unroll
            for (int q = 0; q < 3; ++q) lds_put(mat_m(q) + tile_off<4>(b0 + m, (b0 + c) / 8), f8[q]);
          }
        return;
      }
      if (ll < 32)
#pragma unroll
        for (int c = 0; c < 16; c += 4)
          *reinterpret_cast<lds_floatx4*>(fl(L::oF, b0 + m, b0 + c)) = floatx4{x[c], x[c + 1], x[c + 2], x[c + 3]};
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      // M21 transposed, a lane four columns of a row: M11^T ((M22 L21)^T)
      floatx4 t1 = {0.f, 0.f, 0.f, 0.f}, m21 = t1;
#pragma unroll
      for (int j = 0; j < 4; ++j) mma4(t1, *fl(L::oL, 16 + 4 * j + g, m), *fl(L::oF, 16 + m, 16 + 4 * j + g));
#pragma unroll
      for (int i = 0; i < 4; ++i) mma4(m21, *fl(L::oF, 4 * g + i, m), t1[i]);
      uint32_t p[2][3];
#pragma unroll
      for (int i = 0; i < 2; ++i) parts<3>(floatx2{-m21[2 * i], -m21[2 * i + 1]}, p[i]);
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
#pragma unroll
      for (int q = 0; q < 3; ++q)
        *reinterpret_cast<lds_u32x2*>(mat_m(q) + tile_off<4>(16 + m, g >> 1) + (g & 1) * 8) = u32x2{p[0][q], p[1][q]};
    };
    // (M's upper right block stays zero)
    for (int x = pt0; x < 3 * L::kMat / 16; x += 256) lds_put(sm + L::oM + x * 16, bf16x8{});
    for (int ch = 0; ch < min(nch, 2); ++ch) {
      load_keys(ch);
      put_keys(ch);
      if (pw == 3) {
        load_scalars(ch);
        put_scalars(ch);
      }
    }
    lds_sync();
    if (gram && nch > 0) put_sums(0);
    lds_sync();
    // A step of two phases: the write keys of chunk it beside M of the one before,
    // which the consumers hold already; then the L and P of chunk it.  Loads are
    // issued when a step begins and waited for when it ends.
    for (int it = 0; it <= nch; ++it) {
      const bool live = it < nch;
      anew();
      if (it > 0 && pw < 2) put_inverse(it - 1);
      anew();
      if (it > 0 && it + 1 < nch && pw == 3) put_scalars(it + 1);
      if (it + 2 < nch) {
        load_keys(it + 2);
        if (pw == 3) load_scalars(it + 2);
      }
      anew();
      if (gram && live) put_write_keys(it);
      lds_sync();   // A
      anew();
      if (live) put_products(it);
      anew();
      if (gram && it + 1 < nch) put_sums(it + 1);
      anew();
      if (it + 2 < nch) put_keys(it + 2);
      // No load is under way any more.  Said outright (vmcnt 0), or the compiler,
      // which does not see that a load's branch and its use's go together, waits
      // for loads just issued before it reuses a register in the next step.
      __builtin_amdgcn_s_waitcnt(0x0f70);
      lds_sync();   // B
    }
    if (gram && pt0 < PAIRS) *reinterpret_cast<floatx2*>(ap + dst * a.H * DK) = A;
  }
}

template <int DK, int DV, int NP, int W>
hipError_t launch_parts(const SlotArgs& a, hipStream_t st) {
  static_assert(Lay<DK, NP>::total <= 160 * 1024, "a chunk's operands must fit the LDS of a compute unit");
  hipLaunchKernelGGL((slot_chunks<DK, DV, NP, W>), dim3(static_cast<unsigned>(a.B * a.H * (DV / W))), dim3(W * 4 + 256), 0, st, a);
  return hipGetLastError();
}

template <int DK, int DV, int NP>
hipError_t launch(const SlotArgs& a, hipStream_t st) {
  if constexpr (DV == 128 && NP != 3)
    if (slot_halves(a)) return launch_parts<DK, DV, NP, 64>(a, st);
  return launch_parts<DK, DV, NP, DV>(a, st);
}

template <int NP>
hipError_t launch_dims(const SlotArgs& a, hipStream_t s) {
  if (a.dk == 64) return a.dv == 64 ? launch<64, 64, NP>(a, s) : launch<64, 128, NP>(a, s);
  return a.dv == 64 ? launch<128, 64, NP>(a, s) : launch<128, 128, NP>(a, s);
}

}  // namespace

hipError_t launch_slot_chunks(const SlotArgs& a, hipStream_t s) {
  if (a.precond == kSquash) return launch_dims<3>(a, s);
  return a.precond == kIdentity ? launch_dims<1>(a, s) : launch_dims<0>(a, s);
}

}  // namespace pdn
