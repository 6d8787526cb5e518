// What the kernels on a pool of states share (pdn_slots.hip, pdn_slot_chunks.hip).
#pragma once

#include "pdn_device.hpp"
#include "pdn_internal.hpp"

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

}  // namespace pdn
