// Checks that the entry points share: sizes, alignment, overlapping buffers.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/pdn.h"

namespace pdn {

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
};

inline bool overlap(const Range& a, const Range& b) {
  return a.lo < b.hi && b.lo < a.hi;
}

// checked multiply of non-negative sizes
inline bool mul_ok(int64_t a, int64_t b, int64_t* out) {
  if (a < 0 || b < 0) return false;
  if (a != 0 && b > INT64_MAX / a) return false;
  *out = a * b;
  return true;
}

inline Range rng(const void* p, int64_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return Range{a, a + static_cast<uintptr_t>(bytes)};
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Buf {
  const void* p;
  int64_t bytes;
};

// outputs must not overlap inputs, each other or the workspace; the workspace
// must not overlap inputs
// (Bufs: a vector or an array)
template <typename Ins, typename Outs>
pdn_status check_aliasing(const Ins& ins, const Outs& outs, Buf ws) {
  for (size_t i = 0; i < outs.size(); ++i) {
    if (!outs[i].p || outs[i].bytes == 0) continue;
    const Range ro = rng(outs[i].p, outs[i].bytes);
    for (const Buf& in : ins)
      if (in.p && in.bytes && overlap(ro, rng(in.p, in.bytes))) return PDN_ERR_ALIAS;
    for (size_t j = i + 1; j < outs.size(); ++j)
      if (outs[j].p && outs[j].bytes && overlap(ro, rng(outs[j].p, outs[j].bytes))) return PDN_ERR_ALIAS;
    if (ws.p && ws.bytes && overlap(ro, rng(ws.p, ws.bytes))) return PDN_ERR_ALIAS;
  }
  if (ws.p && ws.bytes)
    for (const Buf& in : ins)
      if (in.p && in.bytes && overlap(rng(ws.p, ws.bytes), rng(in.p, in.bytes))) return PDN_ERR_ALIAS;
  return PDN_OK;
}

}  // namespace pdn
