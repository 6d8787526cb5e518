// Reductions over a wave's lanes on data-parallel primitives: they run at the rate of the
// VALU, where a shuffle goes through LDS (the residual norm's backward with everything on, four sums a row,
// 16384 x 2048 rows: of bf16 as long with shuffles, of fp32 4 % longer).
#pragma once

#include <hip/hip_runtime.h>

namespace pdn {

// x of another lane: CTRL a control of the primitive; `none` in lanes of the rows that MASK leaves out
template <int CTRL, int MASK = 0xf>
__device__ __forceinline__ float lane_of(float x, float none) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), CTRL, MASK, 0xf, false));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140, kBcast15 = 0x142, kBcast31 = 0x143;

__device__ __forceinline__ float read_lane(float x, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// over all 64 lanes, on each of them
__device__ __forceinline__ float wave_sum(float x) {
  x += lane_of<kXor1>(x, 0.f);
  x += lane_of<kXor2>(x, 0.f);
  x += lane_of<kHalfMirror>(x, 0.f);
  x += lane_of<kMirror>(x, 0.f);
  x += lane_of<kBcast15, 0xa>(x, 0.f);
  x += lane_of<kBcast31, 0xc>(x, 0.f);
  return read_lane(x, 63);
}
__device__ __forceinline__ float wave_max(float x) {   // (a NaN does not count)
  x = fmaxf(x, lane_of<kXor1>(x, x));
  x = fmaxf(x, lane_of<kXor2>(x, x));
  x = fmaxf(x, lane_of<kHalfMirror>(x, x));
  x = fmaxf(x, lane_of<kMirror>(x, x));
  x = fmaxf(x, lane_of<kBcast15, 0xa>(x, x));
  x = fmaxf(x, lane_of<kBcast31, 0xc>(x, x));
  return read_lane(x, 63);
}
// over groups of L lanes, a power of two
__device__ __forceinline__ float lanes_sum(float x, int L) {
  if (L > 1) x += lane_of<kXor1>(x, 0.f);
  if (L > 2) x += lane_of<kXor2>(x, 0.f);
  if (L > 4) x += lane_of<kHalfMirror>(x, 0.f);
  if (L > 8) x += lane_of<kMirror>(x, 0.f);
  for (int off = 16; off < L; off <<= 1) x += __shfl_xor(x, off, 64);
  return x;
}

}  // namespace pdn
