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
// of its own sequence's rows, which the segment's workgroup counts in shared memory, as it
// marks there which entry of the bias list a token has.
//
// What bounds it: reading the logits twice and writing p.
#include <algorithm>
#include <cmath>

#include "pdn_device.hpp"
#include "pdn_internal.hpp"

namespace pdn {

namespace {

constexpr int kThreads = 256, kVec = 8, kSeg = kThreads * kVec;
constexpr float kInf = __builtin_inff();

struct Part {
  float top, sum;   // largest l, sum of e under it
  int32_t first;    // first token at the largest (temperature 0)
  int32_t unused;
};

__device__ __forceinline__ int64_t clamp_row(int64_t x, int64_t rows) { return min(max(x, (int64_t)0), rows); }

// a row's sequence and what it has of it
struct RowOf {
  int64_t seq, first;   // its first row; seq < 0: left out
  const int32_t* counts;
  float temperature, repetition, presence, frequency;
  const uint8_t* mask;
  int64_t bias_lo, bias_hi;
};
__device__ __forceinline__ RowOf row_of(const LogitsArgs& a, int64_t row) {
  RowOf r{};
  const int l = threadIdx.x & 63;
  if (a.starts) {   // the last sequence that starts at the row or before: 64 of them at a time
    int64_t upto = 0;
    for (int64_t n0 = 0; n0 < a.N; n0 += kWave) {
      const bool before = n0 + l < a.N && clamp_row(a.starts[n0 + l], a.rows) <= row;
      const unsigned long long m = __ballot(before);
      if (m) upto = n0 + 64 - __clzll(m);
    }
    r.seq = upto - 1;
    if (r.seq < 0 || clamp_row(a.starts[r.seq + 1], a.rows) <= row) {
      r.seq = -1;
      return r;
    }
    r.first = clamp_row(a.starts[r.seq], a.rows);
  } else {
    const int64_t each = a.rows / a.N;
    r.seq = row / each;
    r.first = r.seq * each;
  }
  const int64_t n = r.seq;
  if (a.counts) {
    const int64_t slot = a.slot ? a.slot[n] : n;
    if (slot < 0 || slot >= a.slots) {
      r.seq = -1;
      return r;
    }
    r.counts = a.counts + slot * a.V;
  }
  r.temperature = a.temperature ? a.temperature[n] : 1.f;
  r.repetition = a.repetition ? a.repetition[n] : 1.f;
  r.presence = a.presence ? a.presence[n] : 0.f;
  r.frequency = a.frequency ? a.frequency[n] : 0.f;
  if (a.mask) {
    const int64_t m = a.mask_rows ? a.mask_rows[row] : row;
    if (m >= 0 && m < a.masks) r.mask = reinterpret_cast<const uint8_t*>(a.mask + m * ((a.V + 31) / 32));
  }
  if (a.bias_starts) {
    r.bias_lo = clamp_row(a.bias_starts[n], a.biases);
    r.bias_hi = clamp_row(a.bias_starts[n + 1], a.biases);
  }
  return r;
}

// Counts of the segment's tokens from the sequence's rows up to this one, and the number (from
// one) of the entry of the bias list that each has.
struct Marks {
  int32_t fed[kSeg];
  int32_t bias[kSeg];
};
__device__ __forceinline__ void mark(const LogitsArgs& a, const RowOf& r, int64_t row, int64_t j0, Marks& m) {
  if (!a.ids && !a.bias_starts) return;
  for (int j = threadIdx.x; j < kSeg; j += kThreads) m.fed[j] = m.bias[j] = 0;
  __syncthreads();
  const int64_t end = min(j0 + kSeg, a.V);
  if (a.ids)
    for (int64_t i = r.first + threadIdx.x; i <= row; i += kThreads) {
      const int64_t j = a.ids[i];
      if (j >= j0 && j < end) atomicAdd(&m.fed[j - j0], 1);
    }
  for (int64_t i = r.bias_lo + threadIdx.x; i < r.bias_hi; i += kThreads) {
    const int64_t j = a.bias_ids[i];
    if (j >= j0 && j < end) atomicMax(&m.bias[j - j0], static_cast<int32_t>(i - r.bias_lo + 1));
  }
  __syncthreads();
}

// Eight tokens' changed logits from token j (-inf past the row)
template <typename T>
__device__ __forceinline__ void changed(const LogitsArgs& a, const RowOf& r, int64_t row, int64_t j, const Marks& m, float (&l)[kVec]) {
#pragma clang fp contract(off)
  const T* const p = static_cast<const T*>(a.logits) + row * a.stride;
  const bool whole = j + kVec <= a.V;
  T raw[kVec];
  int32_t t[kVec] = {};
  uint32_t bits = 0xff;
  if (whole) {
    __builtin_memcpy(raw, p + j, sizeof raw);
    if (r.counts) __builtin_memcpy(t, r.counts + j, sizeof t);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      raw[i] = j + i < a.V ? p[j + i] : from_f<T>(-kInf);
      if (r.counts) t[i] = j + i < a.V ? r.counts[j + i] : 0;
    }
  }
  if (r.mask && j < a.V) bits = r.mask[j >> 3];
  const int at = threadIdx.x * kVec;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    float x = to_f(raw[i]);
    const int32_t c = (t[i] & 0x7fffffff) + (a.ids ? m.fed[at + i] : 0);
    if (c | t[i]) {
      x = x > 0.f ? x / r.repetition : x * r.repetition;
      if (c) {
        x = x - r.frequency * static_cast<float>(c);
        x = x - r.presence;
      }
    }
    if (a.bias_starts) {
      const int32_t b = m.bias[at + i];
      if (b) x = x + a.bias_values[r.bias_lo + b - 1];
    }
    l[i] = (bits >> i) & 1 ? x : -kInf;
  }
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
  return x;
}
__device__ __forceinline__ float wave_add(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = min(x, __shfl_xor(x, off, 64));
  return x;
}

// 1 / temperature as a factor of the base-2 exponential's argument; any temperature gives a
// number (so that zero times it is zero); not above 0: 1 (the sum only shows NaN then)
__device__ __forceinline__ float sharpness(float t) {
  if (!(t > 0.f)) return 1.f;
  return fminf(fmaxf(kLog2e / t, 1e-30f), 3e38f);
}
// e of l under the largest (which is -inf where nothing is left: l is then -inf too, or NaN)
__device__ __forceinline__ float under(float l, float top, float k) {
  return l == top ? (top > -kInf ? 1.f : 0.f) : exp2_hw((l - (top > -kInf ? top : 0.f)) * k);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logits_parts(LogitsArgs a) {
  __shared__ Marks marks;
  __shared__ float sF[2][kThreads / kWave];
  __shared__ int sI[kThreads / kWave];
  const int64_t segs = logits_segments(a.V), row = blockIdx.x / segs, seg = blockIdx.x % segs;
  const RowOf r = row_of(a, row);
  if (r.seq < 0) return;
  mark(a, r, row, seg * kSeg, marks);
  const int64_t j = seg * kSeg + threadIdx.x * kVec;
  float l[kVec];
  changed<T>(a, r, row, j, marks, l);
  const int w = threadIdx.x >> 6;
  float top = l[0];
#pragma unroll
  for (int i = 1; i < kVec; ++i) top = fmaxf(top, l[i]);
  top = wave_max(top == top ? top : -kInf);
  if ((threadIdx.x & 63) == 0) sF[0][w] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sF[0][0], sF[0][1]), fmaxf(sF[0][2], sF[0][3]));
  const float k = sharpness(r.temperature);
  float sum = 0.f;
  int first = INT32_MAX;
#pragma unroll
  for (int i = kVec - 1; i >= 0; --i) {
    sum += under(l[i], top, k);
    if (l[i] == top) first = static_cast<int>(j) + i;
  }
  sum = wave_add(sum);
  first = wave_min(first);
  if ((threadIdx.x & 63) == 0) {
    sF[1][w] = sum;
    sI[w] = first;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Part p;
    p.top = top;
    p.sum = (sF[1][0] + sF[1][1]) + (sF[1][2] + sF[1][3]);
    p.first = min(min(sI[0], sI[1]), min(sI[2], sI[3]));
    p.unused = 0;
    static_cast<Part*>(a.parts)[blockIdx.x] = p;
  }
}

// p of a segment from the parts of all, or the changed logits themselves
template <typename T, typename TO, bool PROBS>
__global__ __launch_bounds__(kThreads) void logits_out(LogitsArgs a) {
  __shared__ Marks marks;
  const int64_t segs = logits_segments(a.V), row = blockIdx.x / segs, seg = blockIdx.x % segs;
  const RowOf r = row_of(a, row);
  if (r.seq < 0) return;
  mark(a, r, row, seg * kSeg, marks);
  const int64_t j = seg * kSeg + threadIdx.x * kVec;
  float l[kVec];
  changed<T>(a, r, row, j, marks, l);
  if constexpr (PROBS) {
    const Part* const parts = static_cast<const Part*>(a.parts) + row * segs;
    const int lane = threadIdx.x & 63;
    const float k = sharpness(r.temperature);
    float top = -kInf, sum = 0.f;
    int first = INT32_MAX;
    for (int64_t s = lane; s < segs; s += kWave) top = fmaxf(top, parts[s].top);
    top = wave_max(top);
    for (int64_t s = lane; s < segs; s += kWave) {
      const Part p = parts[s];
      sum += p.sum * under(p.top, top, k);
      if (p.sum != p.sum) sum = p.sum;   // (a NaN in a segment that weighs nothing)
      if (p.top == top) first = min(first, p.first);
    }
    sum = wave_add(sum);
    first = wave_min(first);
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    if (r.temperature > 0.f) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) l[i] = under(l[i], top, k) * f;
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i) l[i] = sum != sum ? sum : top > -kInf && j + i == first ? 1.f : 0.f;
    }
  }
  TO* const out = static_cast<TO*>(a.out) + row * a.V;
  TO raw[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) raw[i] = from_f<TO>(l[i]);
  if (j + kVec <= a.V) {
    __builtin_memcpy(out + j, raw, sizeof raw);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (j + i < a.V) out[j + i] = raw[i];
  }
}

template <typename T, typename TO>
hipError_t logits_of(const LogitsArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.rows * logits_segments(a.V))), block(kThreads);
  if (!a.probs) {
    hipLaunchKernelGGL((logits_out<T, TO, false>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((logits_parts<T>), grid, block, 0, s, a);
  hipLaunchKernelGGL((logits_out<T, TO, true>), grid, block, 0, s, a);
  return hipGetLastError();
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
