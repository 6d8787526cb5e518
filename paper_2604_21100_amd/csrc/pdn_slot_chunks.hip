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
// in fp32, and the state stays fp32 in its accumulators.  What only goes into o,
// which is rounded to bf16, is taken as two numbers (2^-16).
//
// A workgroup holds one head's state for all of its sequence.  Its consumer waves
// own 32 columns each: a lane has rows 32 kk + 8 g + 4 u + i (g = lane / 16) of
// columns 2 (lane % 16) and the next, the rows of an accumulator tile (kk, u) being
// so chosen that two tiles are the eight contraction elements of the next
// product, so S, X and E never leave registers.  Four producer waves meanwhile
// form the next chunk's operands in LDS: write keys and preconditioner state,
// two channels a lane; L and P by matrix products; M from two 16 x 16 inverses by
// substitution and M21 = -M22 L21 M11.
#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_slots.hpp"
#include "pdn_tile.hpp"

namespace pdn {

namespace {

constexpr int kC = 32;

// the parts of an fp32 number: x = p[0] + p[1] + .., each bf16
template <int N>
__device__ __forceinline__ void parts(float x, bf16 (&p)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    p[j] = static_cast<bf16>(x);
    x -= static_cast<float>(p[j]);
  }
}
// two accumulator tiles as the right operand of a slab
template <int N>
__device__ __forceinline__ void parts8(const floatx4& a, const floatx4& b, bf16x8 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    bf16 p[N];
    parts<N>(i < 4 ? a[i] : b[i - 4], p);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j][i] = p[j];
  }
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

// LDS, byte offsets.  K and Q tiles three times (one in use, one that operands are
// formed from, one on its way), what is formed from them twice; per-token
// numbers three times.
template <int DK, int NP>
struct Lay {
  static constexpr int kTile = kC * DK * 2, kMat = kC * kC * 2;
  static constexpr int oK = 0, oQ = oK + 3 * kTile, oX = oQ + 3 * kTile;            // oX: external write keys
  static constexpr int oT = oX + (NP == 0 ? 3 * kTile : 0);                         // write keys' parts
  static constexpr int oM = oT + (NP == 3 ? 2 * 3 * kTile : 0), oP = oM + 2 * 3 * kMat;
  static constexpr int oL = oP + 2 * 2 * kMat, kL = kC * (kC + 4) * 4, oF = oL + kL;   // L, M in fp32
  static constexpr int oS = oF + kL, kS = 7 * kC * 4;   // beta, lam, w, gain, decay, G (64 bits)
  static constexpr int total = oS + 3 * kS;
};

// NP: the write keys' parts, 3 (SQUASH); 1: they are the keys; 0: the caller's
template <int DK, int DV, int NP>
__global__ __launch_bounds__(DV * 2 + 256) void slot_chunks(SlotArgs a) {
  using L = Lay<DK, NP>;
  constexpr int NC = DV / 32, KK = DK / 32, NCH = DK / 8, RK = DK * 2, NT = NP == 3 ? 3 : 1;
  constexpr int UNITS = kC * NCH / 64;   // 1 KB copies of a tile
  __shared__ __attribute__((aligned(1024))) char smem[L::total];
  lds_char* const sm = (lds_char*)smem;
  const int64_t seq = blockIdx.x / a.H, h = blockIdx.x % a.H, hk = h / (a.H / a.Hk);
  const int64_t src = a.slot ? a.slot[seq] : seq, dst = a.slot_out ? a.slot_out[seq] : src;
  if (src < 0 || src >= a.slots || dst < 0 || dst >= a.slots) return;
  const SlotRows rows = slot_rows(a, seq);
  const bool fresh = a.fresh && a.fresh[seq] != 0;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, m = l & 15, g = l >> 4;
  const int r0 = 8 * (m >> 2) + (m & 3);   // left-operand row of this lane, then + 4 u
  const int nch = static_cast<int>((rows.n + kC - 1) / kC);
  auto kt_tile = [&](int it, int p) {   // part p of chunk it's write keys
    return sm + (NP == 3 ? L::oT + ((it & 1) * 3 + p) * L::kTile : (NP == 1 ? L::oK : L::oX) + (it % 3) * L::kTile);
  };
  auto mat = [&](int o, int n, int it, int p) { return sm + o + ((it & 1) * n + p) * L::kMat; };
  auto scal = [&](int it, int x) { return sm + L::oS + (it % 3) * L::kS + x * kC * 4; };

  if (w < NC) {
    // ------------------------------------------------------------ consumers
    const int v0 = 32 * w + 2 * m;
    floatx4 S[KK][2][2];
    {
      const float* sp = a.S + (src * a.H + h) * (DK * DV) + 8 * g * DV + v0;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const floatx2 x = fresh ? floatx2{0.f, 0.f} : *reinterpret_cast<const floatx2*>(sp + (32 * kk + r) * DV);
          S[kk][r / 4][0][r % 4] = x[0];
          S[kk][r / 4][1][r % 4] = x[1];
        }
    }
    const bf16* vb = static_cast<const bf16*>(a.v) + h * DV + v0;
    bf16* ob = static_cast<bf16*>(a.o) + h * DV + v0;
    uint32_t vv[8];
    auto load_v = [&](int ch) {
      const int64_t t0 = static_cast<int64_t>(ch) * kC;
#pragma unroll
      for (int r = 0; r < 8; ++r)
        vv[r] = *reinterpret_cast<const uint32_t*>(vb + (rows.lo + min(t0 + 8 * g + r, rows.n - 1)) * a.v_stride);
    };
    if (nch > 0) load_v(0);
    lds_sync();
    for (int it = 0; it <= nch; ++it) {
      const int ch = it - 1;
      if (ch < 0) {
        lds_sync();
        lds_sync();
        lds_sync();
        continue;
      }
      const int64_t t0 = static_cast<int64_t>(ch) * kC;
      const int n = static_cast<int>(min<int64_t>(kC, rows.n - t0));
      // ---- K S^T and Q S^T
      floatx4 y[2][2], z[2][2], e[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int b = 0; b < 2; ++b) y[u][b] = z[u][b] = e[u][b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        bf16x8 k1[2][1], q1[2][1], sp[2][3];
        reads_done();   // (a slab at a time: all slabs' parts at once do not fit the registers)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int off = (ch % 3) * L::kTile + tile_off<NCH>(r0, 4 * kk + g) + 4 * u * RK;
          k1[u][0] = lds_frag(sm + L::oK + off);
          q1[u][0] = lds_frag(sm + L::oQ + off);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) parts8<3>(S[kk][0][b], S[kk][1][b], sp[b]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            mma_parts(y[u][b], k1[u], sp[b], 2);
            mma_parts(z[u][b], q1[u], sp[b], 1);
          }
      }
      lds_sync();   // A
      // ---- X, E = M X
      {
        floatx4 x[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const floatx4 be = lds_f4(scal(ch, 0) + (8 * g + 4 * u) * 4), lam = lds_f4(scal(ch, 1) + (8 * g + 4 * u) * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t v = vv[4 * u + i];
            const float v2[2] = {__builtin_bit_cast(float, v << 16), __builtin_bit_cast(float, v & 0xffff0000u)};
#pragma unroll
            for (int b = 0; b < 2; ++b)
              x[u][b][i] = 8 * g + 4 * u + i < n ? be[i] * (v2[b] - lam[i] * y[u][b][i]) : 0.f;
          }
          z[u][0] *= lam;
          z[u][1] *= lam;
        }
        if (ch + 1 < nch) load_v(ch + 1);
        bf16x8 mp[2][3], xp[2][3];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int p = 0; p < 3; ++p) mp[u][p] = lds_frag(mat(L::oM, 3, ch, p) + tile_off<4>(r0, g) + 4 * u * (kC * 2));
#pragma unroll
        for (int b = 0; b < 2; ++b) parts8<3>(x[0][b], x[1][b], xp[b]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b = 0; b < 2; ++b) mma_parts(e[u][b], mp[u], xp[b], 2);
      }
      lds_sync();   // B
      // ---- the state after the chunk, and O
      {
        bf16x8 ep[2][2], wp[2][3];
        const floatx4 w0 = lds_f4(scal(ch, 2) + 8 * g * 4), w1 = lds_f4(scal(ch, 2) + (8 * g + 4) * 4);
        const float lc = lds_f4(scal(ch, 1) + (kC - 4) * 4)[3];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          parts8<3>(w0 * e[0][b], w1 * e[1][b], wp[b]);
          parts8<2>(e[0][b], e[1][b], ep[b]);
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            bf16x8 tp[NT];
            reads_done();
#pragma unroll
            for (int p = 0; p < NT; ++p)
              tp[p] = lds_frag_t(kt_tile(ch, p) + tile_off<NCH>(8 * g + (m >> 2), 4 * kk + (m & 3)) + u * 8, 4 * RK);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              S[kk][u][b] *= lc;
              mma_parts(S[kk][u][b], tp, wp[b], 2);
            }
          }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bf16x8 pp[2];
#pragma unroll
          for (int p = 0; p < 2; ++p) pp[p] = lds_frag(mat(L::oP, 2, ch, p) + tile_off<4>(r0, g) + 4 * u * (kC * 2));
#pragma unroll
          for (int b = 0; b < 2; ++b) mma_parts(z[u][b], pp, ep[b], 1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = 8 * g + 4 * u + i;
            if (t < n) st2<bf16>(ob + (rows.lo + t0 + t) * a.H * DV, a.scale * z[u][0][i], a.scale * z[u][1][i]);
          }
        }
      }
      lds_sync();   // C
    }
    float* sp = a.S + (dst * a.H + h) * (DK * DV) + 8 * g * DV + v0;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int r = 0; r < 8; ++r)
        *reinterpret_cast<floatx2*>(sp + (32 * kk + r) * DV) = floatx2{S[kk][r / 4][0][r % 4], S[kk][r / 4][1][r % 4]};
  } else {
    // ------------------------------------------------------------ producers
    constexpr int PAIRS = DK / 2, SEGS = 256 / PAIRS, TOK = kC / SEGS;   // channel pairs; tokens a lane forms keys of
    const int pw = w - NC, pt = pw * 64 + l;
    const int cp = pt % PAIRS, seg = pt / PAIRS;
    const bool gram = NP == 3;
    const float mu = gram ? fast_exp(a.log_a_scale[h]) : 0.f;
    floatx2 A = {0.f, 0.f};
    float* const ap = gram ? a.A + h * DK + 2 * cp : nullptr;
    if (gram && !fresh) A = *reinterpret_cast<const floatx2*>(ap + src * a.H * DK);
    // a chunk's rows into LDS; those past the sequence's end read as zeros
    auto copy_rows = [&](int ch) {
      const int64_t row = rows.lo + static_cast<int64_t>(ch) * kC;
      const int n = static_cast<int>(min<int64_t>(kC, rows.n - static_cast<int64_t>(ch) * kC));
      const int buf = (ch % 3) * L::kTile;
      auto tile = [&](const void* p, int64_t stride, int o) {
        const __amdgpu_buffer_rsrc_t r =
            buf_rsrc(static_cast<const char*>(p) + (row * stride + hk * DK) * 2, static_cast<uint32_t>(((n - 1) * stride + DK) * 2));
#pragma unroll
        for (int x = 0; x < UNITS / 4; ++x) {
          const int unit = UNITS / 4 * pw + x;
          unit_copy(r, unit_src<NCH>(unit, l, static_cast<uint32_t>(stride * 2)), sm + o + buf + unit * 1024);
        }
      };
      tile(a.k, a.k_stride, L::oK);
      tile(a.q, a.q_stride, L::oQ);
      if (NP == 0) tile(a.ktilde, a.Hk * DK, L::oX);
    };
    // its per-token numbers, a lane a token
    auto load_scalars = [&](int ch) {
      const int64_t t0 = static_cast<int64_t>(ch) * kC;
      const int n = static_cast<int>(min<int64_t>(kC, rows.n - t0)), t = l & 31;
      const int64_t sc = (rows.lo + t0 + min(t, n - 1)) * a.H + h;
      const float be = a.beta[sc], gt = a.gate == kGateScalar && t < n ? a.g[sc] : 0.f;
      const float bp = gram ? a.beta_p[sc] : 0.f, gp = gram && a.g_p ? a.g_p[sc] : 0.f;
      double to = gt;   // (64 bits: the decay between two tokens is a difference of two of these)
#pragma unroll
      for (int off = 1; off < kC; off <<= 1) {
        const double x = __shfl_up(to, off, kC);
        if (t >= off) to += x;
      }
      const double end = __shfl(to, kC - 1, kC);
      if (l < kC) {
        auto put = [&](int x, float v) { *reinterpret_cast<lds_float*>(scal(ch, x) + t * 4) = v; };
        put(0, t < n ? be : 0.f);
        put(1, fast_exp(static_cast<float>(to)));
        put(2, fast_exp(static_cast<float>(end - to)));
        put(3, t < n ? bp : 0.f);
        put(4, t < n ? fast_exp(gp) : 1.f);
        *reinterpret_cast<__attribute__((address_space(3))) double*>(scal(ch, 5) + t * 8) = to;
      }
    };
    auto fl = [&](int o, int t, int x) { return reinterpret_cast<lds_float*>(sm + o + (t * (kC + 4) + x) * 4); };
    auto put16 = [&](lds_char* tile, int t, int x, bf16 v) {
      *reinterpret_cast<__attribute__((address_space(3))) bf16*>(tile + tile_off<4>(t, x >> 3) + (x & 7) * 2) = v;
    };
    // (M's upper right block stays zero)
    for (int x = pt; x < 2 * 3 * L::kMat / 16; x += 256) lds_put(sm + L::oM + x * 16, bf16x8{});
    if (nch > 0) {
      copy_rows(0);
      if (pw == 3) load_scalars(0);
    }
    wait_loads<0>();
    lds_sync();
    for (int it = 0; it <= nch; ++it) {
      const bool live = it < nch;
      if (it + 1 < nch) copy_rows(it + 1);
      if (gram && live) {
        // ---- preconditioner state of two channels over the chunk, and this lane's tokens' write keys
        const lds_char* kp = sm + L::oK + (it % 3) * L::kTile;
        floatx2 At[TOK], kt[TOK];
#pragma unroll
        for (int t4 = 0; t4 < kC; t4 += 4) {
          const floatx4 bp = lds_f4(scal(it, 3) + t4 * 4), dp = lds_f4(scal(it, 4) + t4 * 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = t4 + j;
            const uint32_t x = *reinterpret_cast<const __attribute__((address_space(3))) uint32_t*>(
                kp + tile_off<NCH>(t, cp / 4) + (cp % 4) * 4);
            const floatx2 k = {__builtin_bit_cast(float, x << 16), __builtin_bit_cast(float, x & 0xffff0000u)};
            A = dp[j] * A + bp[j] * k * k;
            if (seg == t / TOK) {
              At[t % TOK] = A;
              kt[t % TOK] = k;
            }
          }
        }
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
          bf16 p[2][3];
#pragma unroll
          for (int b = 0; b < 2; ++b) parts<3>(squash_gain(At[j][b], mu, a.lnx) * kt[j][b], p[b]);
#pragma unroll
          for (int q = 0; q < 3; ++q) {
            typename Vec2<bf16>::type v;
            v[0] = p[0][q];
            v[1] = p[1][q];
            *reinterpret_cast<__attribute__((address_space(3))) typename Vec2<bf16>::type*>(
                kt_tile(it, q) + tile_off<NCH>(seg * TOK + j, cp / 4) + (cp % 4) * 4) = v;
          }
        }
      }
      lds_sync();   // A
      if (live) {
        // ---- a wave the rows 8 g + 4 u + i and columns r0 + 4 c of K Kt^T and Q Kt^T
        const int u = pw >> 1, c = pw & 1;
        floatx4 kk4 = {0.f, 0.f, 0.f, 0.f}, qk4 = kk4;
        const int tile = (it % 3) * L::kTile;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const int off = tile_off<NCH>(r0, 4 * kk + g);
          bf16x8 k1[1], q1[1], tp[NT];
          k1[0] = lds_frag(sm + L::oK + tile + off + 4 * u * RK);
          q1[0] = lds_frag(sm + L::oQ + tile + off + 4 * u * RK);
#pragma unroll
          for (int p = 0; p < NT; ++p) tp[p] = lds_frag(kt_tile(it, p) + off + 4 * c * RK);
          mma_parts(kk4, k1, tp, 2);
          mma_parts(qk4, q1, tp, 1);
        }
        const int s = r0 + 4 * c;
        typedef __attribute__((address_space(3))) double lds_double;
        const double Gs = *reinterpret_cast<const lds_double*>(scal(it, 5) + s * 8);
        const floatx4 be = lds_f4(scal(it, 0) + (8 * g + 4 * u) * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = 8 * g + 4 * u + i;
          const float d = fast_exp(static_cast<float>(*reinterpret_cast<const lds_double*>(scal(it, 5) + t * 8) - Gs));
          *fl(L::oL, t, s) = s < t ? be[i] * d * kk4[i] : 0.f;
          bf16 p[2];
          parts<2>(s <= t ? d * qk4[i] : 0.f, p);
          put16(mat(L::oP, 2, it, 0), t, s, p[0]);
          put16(mat(L::oP, 2, it, 1), t, s, p[1]);
        }
      }
      lds_sync();   // B
      if (live && pw == 0) {
        // ---- M: a lane a column of a 16 x 16 block, row after row
        const int b0 = l & 16;   // lanes 0-15 the first block, 16-31 the second
        float x[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          x[t] = t == m ? 1.f : 0.f;
#pragma unroll
          for (int j = 0; j < t; j += 4) {
            const floatx4 f = *reinterpret_cast<lds_floatx4*>(fl(L::oL, b0 + t, b0 + j));
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (j + i < t) x[t] -= f[i] * x[j + i];
          }
        }
        if (l < 32)
#pragma unroll
          for (int t = 0; t < 16; ++t) *fl(L::oF, b0 + t, b0 + m) = x[t];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        floatx4 t1 = {0.f, 0.f, 0.f, 0.f}, m21 = t1;
#pragma unroll
        for (int j = 0; j < 4; ++j) mma4(t1, *fl(L::oL, 16 + m, 4 * j + g), *fl(L::oF, 4 * j + g, m));   // L21 M11
        const floatx4 m22 = *reinterpret_cast<lds_floatx4*>(fl(L::oF, 16 + m, 16 + 4 * g));
#pragma unroll
        for (int i = 0; i < 4; ++i) mma4(m21, m22[i], t1[i]);
        bf16 p[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          parts<3>(-m21[i], p);
#pragma unroll
          for (int q = 0; q < 3; ++q) put16(mat(L::oM, 3, it, q), 16 + 4 * g + i, m, p[q]);
        }
        if (l < 32)
#pragma unroll
          for (int t = 0; t < 16; ++t) {
            parts<3>(x[t], p);
#pragma unroll
            for (int q = 0; q < 3; ++q) put16(mat(L::oM, 3, it, q), b0 + t, b0 + m, p[q]);
          }
      }
      if (it + 1 < nch && pw == 3) load_scalars(it + 1);
      wait_loads<0>();
      lds_sync();   // C
    }
    if (gram && seg == 0) *reinterpret_cast<floatx2*>(ap + dst * a.H * DK) = A;
  }
}

template <int DK, int DV, int NP>
hipError_t launch(const SlotArgs& a, hipStream_t st) {
  static_assert(Lay<DK, NP>::total <= 160 * 1024, "a chunk's operands must fit the LDS of a compute unit");
  hipLaunchKernelGGL((slot_chunks<DK, DV, NP>), dim3(static_cast<unsigned>(a.B * a.H)), dim3(DV * 2 + 256), 0, st, a);
  return hipGetLastError();
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
