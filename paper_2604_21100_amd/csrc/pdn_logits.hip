// From logits to the probabilities of a row's tokens, and the table of tokens that a sequence
// has had.  Token j of a row, c its count, l its logit (each step rounded to fp32):
//   l = l > 0 ? l / repetition : l * repetition    if c > 0 or the prompt has it
//   l = (l - frequency c) - presence               if c > 0
//   l = l + bias;  -inf where the mask forbids it
//   p = e / sum(e), e = exp((l - max l) / temperature), 1 where l is the largest
//
// Two launches: of every segment of a row the largest l, the sum of e under it, and where
// the temperature is zero its first place; then each segment again with those of all.
// A row's counts come from the table (read along with the logits) and from the few tokens
// of its own sequence's rows.
//
// What bounds it: reading the logits twice and writing p.
#include <algorithm>
#include <cmath>

#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_lanes.hpp"

namespace pdn {

namespace {

constexpr int kThreads = 256, kVec = 8, kWaveSpan = kWave * kVec, kSeg = kThreads * kVec;
constexpr float kInf = __builtin_inff();

struct Part {
  float top, sum;   // largest l, sum of e under it
  int32_t first;    // first token at the largest (temperature 0)
  int32_t unused;
};

__device__ __forceinline__ int64_t clamp_row(int64_t x, int64_t rows) { return min(max(x, (int64_t)0), rows); }
__device__ __forceinline__ int lane_int(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// a row's sequence and what it has of it
struct RowOf {
  bool out;             // left out
  int64_t first;        // its sequence's first row
  const int32_t* counts;
  const uint8_t* mask;
  float temperature, repetition, presence, frequency;
  int64_t bias_lo, bias_hi;
};
__device__ __forceinline__ RowOf row_of(const LogitsArgs& a, int64_t row) {
  RowOf r{};
  const int l = threadIdx.x & 63;
  int64_t n, slot = 0;
  const int64_t m = a.mask ? a.mask_rows ? a.mask_rows[row] : row : -1;
  const bool told = a.starts && a.N < kWave;   // a lane a sequence: all there is of each is read at once
  if (told) {
    const int at = min(l, static_cast<int>(a.N)), of = max(min(l, static_cast<int>(a.N) - 1), 0);
    const int32_t start = a.starts[at], from = a.counts && a.slot ? a.slot[of] : of, bias = a.bias_starts ? a.bias_starts[at] : 0;
    const float t = a.temperature ? a.temperature[of] : 1.f, p = a.repetition ? a.repetition[of] : 1.f;
    const float q = a.presence ? a.presence[of] : 0.f, f = a.frequency ? a.frequency[of] : 0.f;
    const unsigned long long before = __ballot(l < a.N && clamp_row(start, a.rows) <= row);
    const int s = before ? 63 - __clzll(before) : -1;
    r.out = s < 0 || clamp_row(lane_int(start, max(s, 0) + 1), a.rows) <= row;
    n = max(s, 0);
    r.first = clamp_row(lane_int(start, static_cast<int>(n)), a.rows);
    slot = lane_int(from, static_cast<int>(n));
    r.temperature = read_lane(t, static_cast<int>(n));
    r.repetition = read_lane(p, static_cast<int>(n));
    r.presence = read_lane(q, static_cast<int>(n));
    r.frequency = read_lane(f, static_cast<int>(n));
    r.bias_lo = clamp_row(lane_int(bias, static_cast<int>(n)), a.biases);
    r.bias_hi = clamp_row(lane_int(bias, static_cast<int>(n) + 1), a.biases);
  } else {
    if (a.starts) {   // the last sequence that starts at the row or before: 64 of them at a time
      int64_t upto = 0;
      for (int64_t n0 = 0; n0 < a.N; n0 += kWave) {
        const unsigned long long before = __ballot(n0 + l < a.N && clamp_row(a.starts[min(n0 + l, a.N)], a.rows) <= row);
        if (before) upto = n0 + 64 - __clzll(before);
      }
      n = max(upto - 1, (int64_t)0);
      r.first = clamp_row(a.starts[n], a.rows);
      r.out = upto == 0 || clamp_row(a.starts[n + 1], a.rows) <= row;
    } else {
      const uint32_t each = static_cast<uint32_t>(a.rows) / static_cast<uint32_t>(a.N);
      n = static_cast<uint32_t>(row) / each;
      r.first = n * each;
      r.out = false;
    }
    if (a.counts) slot = a.slot ? a.slot[n] : n;
    r.temperature = a.temperature ? a.temperature[n] : 1.f;
    r.repetition = a.repetition ? a.repetition[n] : 1.f;
    r.presence = a.presence ? a.presence[n] : 0.f;
    r.frequency = a.frequency ? a.frequency[n] : 0.f;
    if (a.bias_starts) {
      r.bias_lo = clamp_row(a.bias_starts[n], a.biases);
      r.bias_hi = clamp_row(a.bias_starts[n + 1], a.biases);
    }
  }
  if (a.counts) {
    if (slot < 0 || slot >= a.slots) r.out = true;
    else r.counts = a.counts + slot * a.V;
  }
  if (m >= 0 && m < a.masks) r.mask = reinterpret_cast<const uint8_t*>(a.mask + m * ((a.V + 31) / 32));
  return r;
}

// Lists that change a few of a row's tokens: the tokens fed in the sequence's rows up to this one, and
// its biases, from the last entry on (of a token listed twice the last holds).  A lane an entry, 64 at a
// time; a wave then goes through those of them that are among its own tokens.
struct Lists {
  int64_t fed, biases;   // entries
  const int32_t* ids;
  const int32_t* bias_ids;     // the last entry
  const float* bias_values;
  int32_t id, bias_id;   // the first 64 of each (-1: none)
  float bias_value;
  __device__ __forceinline__ void load(int64_t from) {
    const int64_t l = from + (threadIdx.x & 63);
    id = bias_id = -1;
    if (from < fed) {
      id = ids[min(l, fed - 1)];
      id = l < fed ? id : -1;
    }
    if (from < biases) {
      bias_id = bias_ids[-min(l, biases - 1)];
      bias_value = bias_values[-min(l, biases - 1)];
      bias_id = l < biases ? bias_id : -1;
    }
  }
  __device__ __forceinline__ Lists(const LogitsArgs& a, const RowOf& r, int64_t row) {
    fed = a.ids ? row + 1 - r.first : 0;
    biases = max(r.bias_hi - r.bias_lo, (int64_t)0);
    ids = a.ids + r.first;
    bias_ids = a.bias_ids + (r.bias_hi - 1);
    bias_values = a.bias_values + (r.bias_hi - 1);
    load(0);
  }
};

// A thread's eight tokens.  Loads do not branch (a wait for each would follow): a last thread with fewer
// than eight takes the row's last eight, one without any too, and `keep` says which are its own.  TINY: rows
// of fewer than eight.
template <typename T, bool TINY>
struct Piece {
  int at;
  uint32_t keep, bits;   // bits: what the mask allows
  T raw[kVec];
  int32_t count[kVec];
  __device__ __forceinline__ void load_logits(const LogitsArgs& a, int64_t row, int64_t j) {
    const T* const p = static_cast<const T*>(a.logits) + row * a.stride;
    if constexpr (TINY) {
      const int n = static_cast<int>(a.V);
      at = 0;
      keep = j == 0 ? (1u << n) - 1 : 0;
#pragma unroll
      for (int i = 0; i < kVec; ++i) raw[i] = p[min(i, n - 1)];
    } else {
      at = static_cast<int>(min(j, a.V - kVec));
      keep = j < a.V ? (0xffu << (j - at)) & 0xff : 0;
      __builtin_memcpy(raw, p + at, sizeof raw);
    }
  }
  __device__ __forceinline__ void load_rest(const LogitsArgs& a, const RowOf& r) {
    bits = keep;
    if (r.mask) {
      const uint32_t lo = r.mask[at >> 3], hi = r.mask[min(at + kVec - 1, static_cast<int>(a.V) - 1) >> 3];
      bits &= (lo | hi << 8) >> (at & 7);
    }
    if (r.counts) {
      if constexpr (TINY) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) count[i] = r.counts[min(i, static_cast<int>(a.V) - 1)];
      } else {
        __builtin_memcpy(count, r.counts + at, sizeof count);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i) count[i] = 0;
    }
  }
  // the changed logits; base: the wave's first token
  __device__ __forceinline__ void changed(const RowOf& r, const Lists& first, int64_t base, float (&l)[kVec]) {
#pragma clang fp contract(off)
    for (int64_t from = 0; from < first.fed; from += kWave) {
      Lists s = first;
      if (from) s.load(from);
      for (unsigned long long here = __ballot(static_cast<uint64_t>(s.id - base) < kWaveSpan); here; here &= here - 1) {
        const int d = lane_int(s.id, __ffsll(here) - 1) - at;
#pragma unroll
        for (int i = 0; i < kVec; ++i) count[i] += d == i;
      }
    }
    int32_t any = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      l[i] = to_f(raw[i]);
      any |= count[i];
    }
    if (any) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const int32_t c = count[i] & 0x7fffffff;
        const float x = count[i] ? l[i] > 0.f ? l[i] / r.repetition : l[i] * r.repetition : l[i];
        const float y = x - r.frequency * static_cast<float>(c);
        l[i] = c ? y - r.presence : x;
      }
    }
    uint32_t done = 0;
    for (int64_t from = 0; from < first.biases; from += kWave) {
      Lists s = first;
      if (from) s.load(from);
      for (unsigned long long here = __ballot(static_cast<uint64_t>(s.bias_id - base) < kWaveSpan); here; here &= here - 1) {
        const int k = __ffsll(here) - 1, d = lane_int(s.bias_id, k) - at;
        const float value = read_lane(s.bias_value, k);
        const uint32_t one = d >= 0 && d < kVec ? (1u << d) & ~done : 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) l[i] = one >> i & 1 ? l[i] + value : l[i];
        done |= one;
      }
    }
    if (bits != 0xff) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) l[i] = bits >> i & 1 ? l[i] : -kInf;
    }
  }
  template <typename TO>
  __device__ __forceinline__ void store(TO* out, const float (&v)[kVec]) const {
    TO x[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) x[i] = from_f<TO>(v[i]);
    if (!TINY && keep == 0xff) {
      __builtin_memcpy(out + at, x, sizeof x);
    } else if (keep) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (keep >> i & 1) out[at + i] = x[i];
    }
  }
};

// 1 / temperature as a factor of the base-2 exponential's argument; any temperature gives a
// number (so that zero times it is zero); not above 0: 1 (the sum only shows NaN then)
__device__ __forceinline__ float sharpness(float t) {
  if (!(t > 0.f)) return 1.f;
  return fminf(fmaxf(kLog2e / t, 1e-30f), 3e38f);
}
// e of l under the largest, and of -inf where nothing is left (`level`: that, or 0)
__device__ __forceinline__ float under(float l, float top, float level, float k) {
  return l == top ? (top > -kInf ? 1.f : 0.f) : exp2_hw((l - level) * k);
}
__device__ __forceinline__ float level_of(float top) { return top > -kInf ? top : 0.f; }

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = min(x, __shfl_xor(x, off, 64));
  return x;
}

// of a segment: CH times eight tokens a thread, a wave's in a row
template <typename T, int CH, bool TINY>
__global__ __launch_bounds__(kThreads) void logits_parts(LogitsArgs a, uint32_t segs) {
  __shared__ float sF[2][kThreads / kWave];
  __shared__ int sI[kThreads / kWave];
  const uint32_t row = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t base = (static_cast<int64_t>(seg) * (kThreads / kWave) + w) * (CH * kWaveSpan);
  Piece<T, TINY> piece[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) piece[c].load_logits(a, row, base + c * kWaveSpan + lane * kVec);
  const RowOf r = row_of(a, row);
  if (r.out) return;
#pragma unroll
  for (int c = 0; c < CH; ++c) piece[c].load_rest(a, r);
  const Lists lists(a, r, row);
  float l[CH][kVec], top = -kInf, sum = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    piece[c].changed(r, lists, base + c * kWaveSpan, l[c]);
#pragma unroll
    for (int i = 0; i < kVec; ++i) top = fmaxf(top, l[c][i]);
  }
  top = wave_max(top);
  if (lane == 0) sF[0][w] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sF[0][0], sF[0][1]), fmaxf(sF[0][2], sF[0][3]));
  const float k = sharpness(r.temperature), level = level_of(top);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum += under(l[c][i], top, level, k);
  sum = wave_sum(sum);
  if (lane == 0) sF[1][w] = sum;
  if (!(r.temperature > 0.f)) {
    int first = INT32_MAX;
#pragma unroll
    for (int c = CH - 1; c >= 0; --c)
#pragma unroll
      for (int i = kVec - 1; i >= 0; --i)
        if (l[c][i] == top) first = piece[c].at + i;
    first = wave_min(first);
    if (lane == 0) sI[w] = first;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Part p;
    p.top = top;
    p.sum = (sF[1][0] + sF[1][1]) + (sF[1][2] + sF[1][3]);
    p.first = !(r.temperature > 0.f) ? min(min(sI[0], sI[1]), min(sI[2], sI[3])) : 0;
    p.unused = 0;
    static_cast<Part*>(a.parts)[blockIdx.x] = p;
  }
}

// p of a segment from the parts of all, or the changed logits themselves
template <typename T, typename TO, int CH, bool TINY, bool PROBS>
__global__ __launch_bounds__(kThreads) void logits_out(LogitsArgs a, uint32_t segs) {
  const uint32_t row = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t base = (static_cast<int64_t>(seg) * (kThreads / kWave) + w) * (CH * kWaveSpan);
  Piece<T, TINY> piece[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) piece[c].load_logits(a, row, base + c * kWaveSpan + lane * kVec);
  const Part* const parts = static_cast<const Part*>(a.parts) + static_cast<int64_t>(row) * segs;
  Part p{-kInf, 0.f, INT32_MAX, 0};
  if constexpr (PROBS) {
    const Part x = parts[min(static_cast<uint32_t>(lane), segs - 1)];
    if (static_cast<uint32_t>(lane) < segs) p = x;
  }
  const RowOf r = row_of(a, row);
  if (r.out) return;
#pragma unroll
  for (int c = 0; c < CH; ++c) piece[c].load_rest(a, r);
  const Lists lists(a, r, row);
  float top = 0.f, level = 0.f, sum = 0.f, f = 0.f, k = 0.f;
  int first = INT32_MAX;
  if constexpr (PROBS) {
    k = sharpness(r.temperature);
    top = p.top;
    for (uint32_t s = kWave + lane; s < segs; s += kWave) top = fmaxf(top, parts[s].top);
    top = wave_max(top);
    level = level_of(top);
    auto add = [&](const Part& x) {
      // (a NaN in a segment that weighs nothing shows too)
      sum += x.sum == x.sum ? x.sum * under(x.top, top, level, k) : x.sum;
      if (x.top == top) first = min(first, x.first);
    };
    add(p);
    for (uint32_t s = kWave + lane; s < segs; s += kWave) add(parts[s]);
    sum = wave_sum(sum);
    f = sum == 0.f ? 0.f : 1.f / sum;
    if (!(r.temperature > 0.f)) first = wave_min(first);
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float l[kVec];
    piece[c].changed(r, lists, base + c * kWaveSpan, l);
    if constexpr (PROBS) {
      if (r.temperature > 0.f) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) l[i] = under(l[i], top, level, k) * f;
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) l[i] = sum != sum ? sum : top > -kInf && piece[c].at + i == first ? 1.f : 0.f;
      }
    }
    piece[c].store(static_cast<TO*>(a.out) + row * a.V, l);
  }
}

template <typename T, typename TO, int CH, bool TINY>
hipError_t logits_at(const LogitsArgs& a, hipStream_t s) {
  const int64_t segs = (a.V + CH * kSeg - 1) / (CH * kSeg);
  const dim3 grid(static_cast<unsigned>(a.rows * segs)), block(kThreads);
  if (!a.probs) {
    hipLaunchKernelGGL((logits_out<T, TO, CH, TINY, false>), grid, block, 0, s, a, static_cast<uint32_t>(segs));
    return hipGetLastError();
  }
  hipLaunchKernelGGL((logits_parts<T, CH, TINY>), grid, block, 0, s, a, static_cast<uint32_t>(segs));
  hipLaunchKernelGGL((logits_out<T, TO, CH, TINY, true>), grid, block, 0, s, a, static_cast<uint32_t>(segs));
  return hipGetLastError();
}
template <typename T, typename TO>
hipError_t logits_of(const LogitsArgs& a, hipStream_t s) {
  if (a.V < kVec) return logits_at<T, TO, 1, true>(a, s);
  if (a.rows * ((a.V + 4 * kSeg - 1) / (4 * kSeg)) >= 1024) return logits_at<T, TO, 4, false>(a, s);
  return logits_at<T, TO, 1, false>(a, s);
}

constexpr int32_t kPromptBit = INT32_MIN;

// a sequence's tokens and slots; from < 0: left out
struct SeqOf {
  int64_t lo, n, from, to;
  bool fresh;
};
__device__ __forceinline__ SeqOf seq_of(const CountArgs& a, int64_t seq) {
  SeqOf s{};
  int64_t hi;
  if (a.starts) {
    s.lo = clamp_row(a.starts[seq], a.rows);
    hi = clamp_row(a.starts[seq + 1], a.rows);
  } else {
    const int64_t each = a.rows / a.N;
    s.lo = seq * each;
    hi = s.lo + each;
  }
  s.n = max(hi - s.lo, (int64_t)0);
  if (a.accepted) s.n = min(s.n, max((int64_t)a.accepted[seq], (int64_t)0));
  s.from = a.slot ? a.slot[seq] : seq;
  s.to = a.slot_out ? a.slot_out[seq] : s.from;
  s.fresh = a.fresh && a.fresh[seq];
  if (s.from < 0 || s.from >= a.slots || s.to < 0 || s.to >= a.slots) s.from = -1;
  return s;
}

// tokens added in place: a workgroup a sequence (whole-number atomics, so any order gives the same)
__global__ __launch_bounds__(kThreads) void counts_add(CountArgs a) {
  const SeqOf s = seq_of(a, blockIdx.x);
  if (s.from < 0) return;
  int32_t* const row = a.counts + s.to * a.V;
  for (int64_t i = threadIdx.x; i < s.n; i += kThreads) {
    const int64_t j = a.ids[s.lo + i];
    if (j < 0 || j >= a.V) continue;
    if (a.prompt) atomicOr(&row[j], kPromptBit);
    else atomicAdd(&row[j], 1);
  }
}

// a whole row written: a workgroup a segment, its tokens counted in shared memory
__global__ __launch_bounds__(kThreads) void counts_write(CountArgs a) {
  __shared__ int32_t had[kSeg];
  const int64_t segs = count_segments(a.V), seq = blockIdx.x / segs, j0 = blockIdx.x % segs * kSeg;
  const SeqOf s = seq_of(a, seq);
  if (s.from < 0) return;
  const int64_t n = min((int64_t)kSeg, a.V - j0);
  for (int j = threadIdx.x; j < kSeg; j += kThreads) had[j] = 0;
  __syncthreads();
  for (int64_t i = threadIdx.x; i < s.n; i += kThreads) {
    const int64_t j = a.ids[s.lo + i] - j0;
    if (j >= 0 && j < n) atomicAdd(&had[j], 1);
  }
  __syncthreads();
  const int32_t* const from = a.counts + s.from * a.V + j0;
  int32_t* const to = a.counts + s.to * a.V + j0;
  for (int64_t j = threadIdx.x; j < n; j += kThreads) {
    const int32_t old = s.fresh ? 0 : from[j], c = had[j];
    to[j] = a.prompt ? (c ? old | kPromptBit : old) : old + c;
  }
}

}  // namespace

__host__ __device__ int64_t logits_segments(int64_t V) { return (V + kSeg - 1) / kSeg; }
__host__ __device__ int64_t count_segments(int64_t V) { return (V + kSeg - 1) / kSeg; }

hipError_t launch_logits(const LogitsArgs& a, int in_bf16, int out_bf16, hipStream_t s) {
  if (in_bf16) return out_bf16 ? logits_of<bf16, bf16>(a, s) : logits_of<bf16, float>(a, s);
  return out_bf16 ? logits_of<float, bf16>(a, s) : logits_of<float, float>(a, s);
}

hipError_t launch_counts(const CountArgs& a, hipStream_t s) {
  if (a.slot_out || a.fresh)
    hipLaunchKernelGGL(counts_write, dim3(static_cast<unsigned>(a.N * count_segments(a.V))), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(counts_add, dim3(static_cast<unsigned>(a.N)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace pdn
