// What the kernels on a pool of states share (pdn_slots.hip, pdn_slot_chunks.hip,
// pdn_slot_runs.hip).
#pragma once

#include <type_traits>

#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_tile.hpp"

namespace pdn {

// two consecutive elements, as fp32
template <typename T> struct Vec2;
template <> struct Vec2<float> { typedef floatx2 type; };
template <> struct Vec2<bf16> { typedef __bf16 type __attribute__((ext_vector_type(2))); };
template <typename T>
__device__ __forceinline__ floatx2 ld2(const T* p) {
  const auto v = *reinterpret_cast<const typename Vec2<T>::type*>(p);
  return floatx2{to_f(v[0]), to_f(v[1])};
}
template <typename T>
__device__ __forceinline__ void st2(T* p, float x, float y) {
  typename Vec2<T>::type v;
  v[0] = from_f<T>(x);
  v[1] = from_f<T>(y);
  *reinterpret_cast<typename Vec2<T>::type*>(p) = v;
}

// A workgroup's sequence, value head, key head and which of the head's `parts` of
// the columns (B H is below 2^22; divided in 32 bits, as 64 take hundreds of
// instructions).
struct SlotWhere {
  int64_t seq, h, hk;
  int part;
};
__device__ __forceinline__ SlotWhere slot_where(const SlotArgs& a, uint32_t parts = 1) {
  const uint32_t at = blockIdx.x / parts, H = static_cast<uint32_t>(a.H), seq = at / H, h = at - seq * H;
  return SlotWhere{seq, h, h / (H / static_cast<uint32_t>(a.Hk)), static_cast<int>(blockIdx.x - at * parts)};
}

// The rows of a sequence: n of the packed tensors, from lo.  What `starts`
// holds is device data: whatever it is, the rows stay inside the tensors.
struct SlotRows {
  int64_t lo, n;
};
__device__ __forceinline__ SlotRows slot_rows(const SlotArgs& a, int64_t seq) {
  int64_t lo = seq * a.T, hi = lo + a.T;
  if (a.starts) {
    lo = a.starts[seq];
    hi = a.starts[seq + 1];
  }
  lo = min(max(lo, (int64_t)0), a.tokens);
  hi = min(min(hi, a.tokens), lo + a.T);
  return SlotRows{lo, max(hi - lo, (int64_t)0)};
}

constexpr int kSlotBlock = 8;   // tokens of a block

// A token's log-decay where those of several tokens are added up.  e^-128 is zero
// in fp32, and so is every decay over such a token; a sum that held a value far
// below, an infinity above all, would have lost the tokens after it.  (NaN stays.)
__device__ __forceinline__ float sum_decay(float g) { return g < -128.f ? -128.f : g; }

// Of a block's log-decays, one in each of the first eight lanes: the sum up to a lane's
// own, and of those after it.
__device__ __forceinline__ void block_sums(float g, int l, float* to, float* on) {
  auto moved = [](float x, auto ctrl) {   // from another of 16 lanes, past their ends zero
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  auto down = [&](float x, auto n) { return moved(x, std::integral_constant<int, 0x100 + decltype(n)::value>{}); };   // lane + n
  auto up = [&](float x, auto n) { return moved(x, std::integral_constant<int, 0x110 + decltype(n)::value>{}); };     // lane - n
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  constexpr std::integral_constant<int, 4> four;
  const float x = l < kSlotBlock ? g : 0.f;
  float p = x, s = down(x, one);
  p += up(p, one);
  s += down(s, one);
  p += up(p, two);
  s += down(s, two);
  *to = p + up(p, four);
  *on = s + down(s, four);
}

// With a per-channel gate the products of a block's eight tokens,
//   sum over c of x_t[c] (e_s+1 .. e_t)[c] kt_s[c],   x a key or query, e_t = exp(g_t),
// take the decays between two tokens apart at a token r between them, s <= r < t, so that
// both factors, x_t e_r+1 .. e_t and kt_s e_s+1 .. e_r, are of decays that a channel goes through and
// none is ever divided by, however little a channel keeps.  With r the last
// token of the half, pair or token of the block that s is in and t is not, each
// pair of tokens is in one of two products of sixteen rows:
//   the first     rows  keys 4-7, queries 4-7 (r = 3), keys and queries 2, 3 (r = 1) and 6, 7 (r = 5)
//                 columns  write keys 0-3 (r = 3), 0, 1 (r = 1), 4, 5 (r = 5)
//   the second    rows  keys 1, 3, 5, 7 and queries 1, 3, 5, 7 (r = t - 1), queries as they are
//                 columns  write keys as they are
// (One product, of rows with the decay from the block's start and write keys
// divided by it, overflows where a block's log-decays add up to less than -87 and
// its write keys are not small; it took 299 and 61 us where the two take 324 and 65: 12 per-
// channel prompts of up to 700 tokens x 16 heads, 96 x 16 drafts of four.)
constexpr int kPairCols = 8;   // columns of either
// a channel's keys (q 0) or queries (q 1), x: rows for the products with the state
// (decayed from the block's start: up[t]), and of both products
template <int LD>
__device__ __forceinline__ void channel_rows(const float (&x)[kSlotBlock], const float (&e)[kSlotBlock],
                                             const float (&up)[kSlotBlock], int q, int c, float (*kq)[LD], float (*r1)[LD],
                                             float (*r2)[LD]) {
  float d = 1.f;
#pragma unroll
  for (int t = 0; t < kSlotBlock; ++t) {
    kq[kSlotBlock * q + t][c] = up[t] * x[t];
    if (t >= 4) {
      d *= e[t];
      r1[4 * q + t - 4][c] = d * x[t];
    }
    if (t & 2) r1[8 + 4 * q + (t >> 2) * 2 + (t & 1)][c] = (t & 1 ? e[t - 1] * e[t] : e[t]) * x[t];
    if (t & 1) r2[4 * q + t / 2][c] = e[t] * x[t];
    if (q) r2[8 + t][c] = x[t];
  }
}
// its write keys: columns of both, and decayed to the block's end
template <int LD>
__device__ __forceinline__ void channel_cols(const float (&kt)[kSlotBlock], const float (&e)[kSlotBlock], int c,
                                             float (*c1)[LD], float (*c2)[LD], float (*to_end)[LD]) {
  float on = 1.f, d = 1.f;
#pragma unroll
  for (int s = kSlotBlock - 1; s >= 0; --s) {
    c2[s][c] = kt[s];
    to_end[s][c] = on * kt[s];
    on *= e[s];
    if (s < 4) {
      c1[s][c] = d * kt[s];
      d *= e[s];
    }
    if (!(s & 2)) c1[4 + (s >> 2) * 2 + (s & 1)][c] = (s & 1 ? 1.f : e[s + 1]) * kt[s];
  }
}
// where of the two products (32 rows) row r of K over Q with token s <= t is
__device__ __forceinline__ int channel_pair(int r, int s, int* col) {
  const int t = r % kSlotBlock, q = r / kSlotBlock, x = t ^ s;
  *col = s;
  if (x >= 4) return 4 * q + (t & 3);
  if (x >= 2) {
    *col = 4 + (t >> 2) * 2 + (s & 1);
    return 8 + 4 * q + (t >> 2) * 2 + (t & 1);
  }
  return 16 + (x ? 4 * q + t / 2 : 8 + t);
}

// A head's state, seen through a buffer: a lane's rows are then one offset and
// constants, where pointers to them would take two registers each.
template <int DK, int DV>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t slot_head(const SlotArgs& a, int64_t slot, int64_t h) {
  return buf_rsrc(reinterpret_cast<const char*>(a.S + (slot * a.H + h) * (DK * DV)), DK * DV * 4);
}
// a wave's 16 columns of it, one a lane (from element `at` of the head)
template <int DK, int DV>
struct SlotColumns {
  static constexpr int MB = DK / 16;
  floatx4 t[MB];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int m = 0; m < MB; ++m) t[m] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int at) {
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        t[m][i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, 4 * at, (16 * m + i) * DV * 4, 0));
  }
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, int at) const {
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = t[m][i];   // (the bits of t[m][i] itself would be those of t[m][0])
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), r, 4 * at, (16 * m + i) * DV * 4, 0);
      }
  }
};
// A matrix product's result may be read ten or eleven issue slots after it at the
// earliest.  The compiler counts them, but has been seen to count along one side of a
// branch only and to read the last of a result's registers too early on the other.
// Where code that branches follows a product, its results go through here.
__device__ __forceinline__ void settled(floatx4& a) { asm volatile("s_nop 7\n\ts_nop 7" : "+v"(a)); }
__device__ __forceinline__ void settled(floatx4& a, floatx4& b) {
  asm volatile("s_nop 7\n\ts_nop 7" : "+v"(a), "+v"(b));
}
template <int N>
__device__ __forceinline__ void settled(floatx4 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4)
    asm volatile("s_nop 7\n\ts_nop 7" : "+v"(t[i]), "+v"(t[i + 1]), "+v"(t[i + 2]), "+v"(t[i + 3]));
}
// one element of a buffer, as fp32
template <typename T>
__device__ __forceinline__ float buf_get(__amdgpu_buffer_rsrc_t r, int off) {
  if constexpr (sizeof(T) == 2)
    return __builtin_bit_cast(float, static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0)) << 16);
  else
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
}

template <typename T>
__device__ __forceinline__ void buf_put(__amdgpu_buffer_rsrc_t r, int off, float x) {
  if constexpr (sizeof(T) == 2)
    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, from_f<T>(x)), r, off, 0, 0);
  else
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), r, off, 0, 0);
}

// whether a write key takes a factor that the sum m = k . kt gives, and that factor
__device__ __forceinline__ bool slot_needs_sum(const SlotArgs& a) {
  return a.precond == kDiagSM || a.knorm != kKnormNone;
}
__device__ __forceinline__ float slot_sum_factor(const SlotArgs& a, float m, float beta, float g) {
  if (a.precond == kDiagSM || a.knorm == kKnorm1pm) return 1.f / (1.f + m);
  if (a.knorm == kKnormM) return 1.f / m;
  return beta / ((a.gate == kGateScalar ? fast_exp(g) : 1.f) + beta * m);
}

// A matrix product with P or M, whose upper halves are zeros, multiplies a later token's
// correction by zero, and that is NaN where the correction is no number.  So where one
// is not, products go without it, and what comes from that token on, which it is
// part of, is made NaN afterwards: tokens before it keep their outputs.  (Looking for
// them takes 1 to 3 % of the long runs' time, nothing of the drafts'.)
__device__ __forceinline__ bool all_numbers(const floatx4& x) {
  return __builtin_isfinite(x[0]) && __builtin_isfinite(x[1]) && __builtin_isfinite(x[2]) && __builtin_isfinite(x[3]);
}
// takes what is no number out of tokens t0 .. t0 + 3 of a column; the first of these, or `first`
__device__ __forceinline__ int take_out(floatx4& x, int t0, int first) {
#pragma unroll
  for (int i = 3; i >= 0; --i)
    if (!__builtin_isfinite(x[i])) {
      first = t0 + i;
      x[i] = 0.f;
    }
  return first;
}
// the first of a column, from the four lanes that hold it
__device__ __forceinline__ int first_of(int first) {
  first = min(first, __shfl_xor(first, 16, 64));
  return min(first, __shfl_xor(first, 32, 64));
}
__device__ __forceinline__ void put_from(floatx4& x, int t0, int first, float value) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t0 + i >= first) x[i] = value;
}

// (I + L)^{-1} y for four rows, L's rows in l
__device__ __forceinline__ floatx4 slot_solve4(const floatx4 (&l)[4], floatx4 y) {
  y[1] -= l[1][0] * y[0];
  y[2] -= l[2][0] * y[0] + l[2][1] * y[1];
  y[3] -= l[3][0] * y[0] + l[3][1] * y[1] + l[3][2] * y[2];
  return y;
}

}  // namespace pdn
