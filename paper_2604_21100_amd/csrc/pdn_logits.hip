// From logits to the probabilities of a row's tokens, and the table of tokens that a sequence
// has had.  Token j of a row, c its count, l its logit (each step rounded to fp32):
//   l = l > 0 ? l / repetition : l * repetition    if c > 0 or the prompt has it
//   l = (l - frequency c) - presence               if c > 0
//   l = l + bias;  -inf where the mask forbids it
//   p = e / sum(e), e = exp((l - max l) / temperature), 1 where l is the largest
//
// One launch with a row in registers, or two: of every segment of a row the largest l, the sum of e under
// it, and where the temperature is zero its first place; then each token again with those of all.
// A row's counts come from the table (read along with the logits) and from the few tokens
// of its own sequence's rows.
//
// What bounds it: reading the logits twice and writing p, for 314 rows of 131072 fp32 logits with penalties and masks
// 44 us (198 MB, 4.5 TB/s) and 58 us (363 MB, 6.3 TB/s), the vector units 0.75 of the time; for a few rows latency, 4.5 and 4.3 us for one of 50257.
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
// What a wave reads of all sequences at once, if there are less than 64: a lane a sequence (the loads
// that a row's others wait for come first, as loads are waited for in their order).
struct Told {
  bool all;
  int32_t start, slot, bias;
  float temperature, repetition, presence, frequency;
  __device__ __forceinline__ explicit Told(const LogitsArgs& a) {
    const int l = threadIdx.x & 63, n = static_cast<int>(min(a.N, (int64_t)kWave)), at = min(l, n), of = min(l, n - 1);
    all = a.starts && n < kWave;
    if (!all) return;
    start = a.starts[at];
    slot = a.counts && a.slot ? a.slot[of] : of;
    bias = a.bias_starts ? a.bias_starts[at] : 0;
    temperature = a.temperature ? a.temperature[of] : 1.f;
    repetition = a.repetition ? a.repetition[of] : 1.f;
    presence = a.presence ? a.presence[of] : 0.f;
    frequency = a.frequency ? a.frequency[of] : 0.f;
  }
};
__device__ __forceinline__ RowOf row_of(const LogitsArgs& a, int64_t row, const Told& told) {
  RowOf r{};
  const int l = threadIdx.x & 63;
  int64_t slot = 0;
  if (told.all) {
    const unsigned long long before = __ballot(l < a.N && clamp_row(told.start, a.rows) <= row);
    const int n = before ? 63 - __clzll(before) : 0;   // the last sequence that starts at the row or before
    r.first = clamp_row(lane_int(told.start, n), a.rows);
    r.out = !before || clamp_row(lane_int(told.start, n + 1), a.rows) <= row;
    slot = lane_int(told.slot, n);
    r.temperature = read_lane(told.temperature, n);
    r.repetition = read_lane(told.repetition, n);
    r.presence = read_lane(told.presence, n);
    r.frequency = read_lane(told.frequency, n);
    r.bias_lo = clamp_row(lane_int(told.bias, n), a.biases);
    r.bias_hi = clamp_row(lane_int(told.bias, n + 1), a.biases);
  } else {
    int64_t n;
    if (a.starts) {   // the same, of every 64^k-th sequence first (all of them 64 at a time: 16384 rows of 1000, one a sequence, 503 us, so 35)
      int shift = 0;
      while ((int64_t)kWave << shift < a.N) shift += 6;
      n = 0;
      bool any = true;
      for (; shift >= 0; shift -= 6) {
        const int64_t at = n + ((int64_t)l << shift);
        const unsigned long long before = __ballot(at < a.N && clamp_row(a.starts[min(at, a.N)], a.rows) <= row);
        any = any && before;
        if (before) n += (int64_t)(63 - __clzll(before)) << shift;
      }
      r.first = clamp_row(a.starts[n], a.rows);
      r.out = !any || clamp_row(a.starts[n + 1], a.rows) <= row;
    } else {
      const uint32_t each = static_cast<uint32_t>(a.rows) / static_cast<uint32_t>(a.N);
      n = static_cast<uint32_t>(row) / each;
      r.first = n * each;
      r.out = false;
    }
    slot = a.counts && a.slot ? a.slot[n] : n;
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
  const int64_t m = a.mask ? a.mask_rows ? a.mask_rows[row] : row : -1;
  if (m >= 0 && m < a.masks) r.mask = reinterpret_cast<const uint8_t*>(a.mask + m * ((a.V + 31) / 32));
  return r;
}

// Lists that change a few of a row's tokens: the tokens fed in the sequence's rows up to this one, and
// its biases, from the last entry on (of a token listed twice the last holds).  A lane an entry, 64 at a
// time (-1: none); a wave then goes through those of them that are among its own tokens.
struct Lists {
  int64_t fed, biases;   // entries
  const int32_t* ids;
  const int32_t* bias_ids;   // the last entry
  const float* bias_values;
  int32_t id, bias_id;       // of the first 64
  float bias_value;
  __device__ __forceinline__ int32_t fed_id(int64_t from) const {
    const int64_t l = from + (threadIdx.x & 63);
    const int32_t x = ids[min(l, fed - 1)];
    return l < fed ? x : -1;
  }
  __device__ __forceinline__ void bias(int64_t from, int32_t& x, float& value) const {
    const int64_t l = from + (threadIdx.x & 63);
    x = bias_ids[-min(l, biases - 1)];
    value = bias_values[-min(l, biases - 1)];
    x = l < biases ? x : -1;
  }
  __device__ __forceinline__ Lists(const LogitsArgs& a, const RowOf& r, uint32_t row) {
    fed = a.ids ? row + 1 - r.first : 0;
    biases = max(r.bias_hi - r.bias_lo, (int64_t)0);
    ids = a.ids + r.first;
    bias_ids = a.bias_ids + (r.bias_hi - 1);
    bias_values = a.bias_values + (r.bias_hi - 1);
    if (fed > 0) id = fed_id(0);
    if (biases > 0) bias(0, bias_id, bias_value);
  }
};

// Probabilities are written, and logits read for the last time, past the caches, where rows are aligned to the
// 16 bytes of an access (else an access ends in the next one's line): what is in the caches then is the
// logits that the second launch still has to read, and the verification reads a row or two of each sequence's
// only.  With and without, fp32 rows with penalties and masks, the call | with its verification, us: 314 of 131072
// 100 | 119 and 112 | 132, 64 of them 35 | 50 and 37 | 52; one launch, 314 of 16000 13.5 | 23 and 16.4 | 26.  Unaligned rows took 1.2
// times as long with it.
typedef uint32_t Sixteen __attribute__((ext_vector_type(4), aligned(2), may_alias));

// A thread's eight tokens from j on.  Loads do not branch (a wait for each would follow): a last thread with
// fewer than eight takes the row's last eight, one without any too, and `keep` says which are its own.  TINY:
// rows of fewer than eight.
template <bool TINY>
struct Place {
  int at, n;
  uint32_t keep;
  __device__ __forceinline__ Place(const LogitsArgs& a, uint32_t j) : n(static_cast<int>(a.V)) {
    if constexpr (TINY) {
      at = 0;
      keep = j == 0 ? (1u << n) - 1 : 0;
    } else {
      at = static_cast<int>(min(j, static_cast<uint32_t>(n - kVec)));
      keep = j < static_cast<uint32_t>(n) ? (0xffu << (j - at)) & 0xff : 0;
    }
  }
  template <bool PASSING = false, typename T>
  __device__ __forceinline__ void load(const T* row, T (&x)[kVec]) const {
    if constexpr (TINY) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) x[i] = row[min(i, n - 1)];
    } else if constexpr (PASSING) {
      Sixteen q[sizeof x / 16];
#pragma unroll
      for (unsigned i = 0; i < sizeof x / 16; ++i) q[i] = __builtin_nontemporal_load(reinterpret_cast<const Sixteen*>(row + at) + i);
      __builtin_memcpy(x, q, sizeof x);
    } else {
      __builtin_memcpy(x, row + at, sizeof x);
    }
  }
  template <bool PASSING, typename TO>
  __device__ __forceinline__ void store(TO* row, const float (&v)[kVec]) const {
    TO x[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) x[i] = from_f<TO>(v[i]);
    if (!TINY && keep == 0xff) {
      if constexpr (PASSING) {
        Sixteen q[sizeof x / 16];
        __builtin_memcpy(q, x, sizeof x);
#pragma unroll
        for (unsigned i = 0; i < sizeof x / 16; ++i) __builtin_nontemporal_store(q[i], reinterpret_cast<Sixteen*>(row + at) + i);
      } else {
        __builtin_memcpy(row + at, x, sizeof x);
      }
    } else if (keep) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (keep >> i & 1) row[at + i] = x[i];
    }
  }
};

// Eight tokens of a row with what changes them.
template <typename T, bool TINY, bool LAST = false>   // LAST: the logits are not read again
struct Tokens {
  Place<TINY> place;
  T raw[kVec];
  int32_t count[kVec];
  uint32_t bits[2];   // the mask's bytes at the first and the last of them
  __device__ __forceinline__ Tokens(const LogitsArgs& a, uint32_t row, uint32_t j) : place(a, j) {
    place.template load<LAST>(static_cast<const T*>(a.logits) + row * a.stride, raw);
  }
  __device__ __forceinline__ void load_rest(const RowOf& r) {
    if (r.counts) {
      place.load(r.counts, count);
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i) count[i] = 0;
    }
    if (r.mask) {
      bits[0] = r.mask[place.at >> 3];
      bits[1] = r.mask[(min(place.at + kVec, place.n) - 1) >> 3];
    }
  }
  // the changed logits; base: the wave's first token
  __device__ __forceinline__ void changed(const RowOf& r, const Lists& lists, uint32_t base, float (&l)[kVec]) {
#pragma clang fp contract(off)
    for (int64_t from = 0; from < lists.fed; from += kWave) {
      const int32_t id = from ? lists.fed_id(from) : lists.id;
      for (unsigned long long here = __ballot(static_cast<uint32_t>(id) - base < kWaveSpan); here; here &= here - 1) {
        const int d = lane_int(id, __ffsll(here) - 1) - place.at;
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
      for (int i = 0; i < kVec; ++i)
        if (count[i]) {
          const int32_t c = count[i] & 0x7fffffff;
          const float y = l[i] > 0.f ? l[i] / r.repetition : l[i] * r.repetition;
          const float z = y - r.frequency * static_cast<float>(c);
          l[i] = c ? z - r.presence : y;
        }
    }
    uint32_t done = 0;
    for (int64_t from = 0; from < lists.biases; from += kWave) {
      int32_t id = lists.bias_id;
      float value = lists.bias_value;
      if (from) lists.bias(from, id, value);
      for (unsigned long long here = __ballot(static_cast<uint32_t>(id) - base < kWaveSpan); here; here &= here - 1) {
        const int k = __ffsll(here) - 1, d = lane_int(id, k) - place.at;
        const float more = read_lane(value, k);
        const uint32_t one = d >= 0 && d < kVec ? (1u << d) & ~done : 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) l[i] = one >> i & 1 ? l[i] + more : l[i];
        done |= one;
      }
    }
    const uint32_t on = r.mask ? place.keep & (bits[0] | bits[1] << 8) >> (place.at & 7) : place.keep;
    if (on != 0xff) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) l[i] = on >> i & 1 ? l[i] : -kInf;
    }
  }
};

// log2(e) / temperature, the factor of the base-2 exponential's argument, from below (k), and the rest of it; both
// above 0, so that -inf times them is -inf, and numbers, so that zero times them is zero.  A temperature not above 0: 1
// (the sum only shows NaN then)
struct Sharpness {
  float k, rest;
};
__device__ __forceinline__ Sharpness sharpness(float t) {
  constexpr float kTiny = 1.4e-45f;   // (the smallest: an infinite temperature moves the lowest number by 1e-6)
  if (!(t > 0.f)) return Sharpness{1.f, kTiny};
  float k = kLog2e / t;
  if (k < 1e-30f || k > 1e30f) return Sharpness{fminf(fmaxf(k, kTiny), 3e38f), kTiny};   // (such a t may have no reciprocal)
  k = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, k) - 1u);   // (the quotient was rounded)
  const float rest = (fmaf(-k, t, kLog2e) + 1.925963033e-8f) * fast_rcp(t);   // (log2(e) = kLog2e + 1.93e-8)
  return Sharpness{read_lane(k, 0), read_lane(rest, 0)};   // (a row's, so a wave's)
}
// e^(d / temperature), d <= 0: the argument is rounded once, to 2^-24 of itself (with a rounded k alone 2.2 times that)
__device__ __forceinline__ float exp_of(float d, const Sharpness& s) { return exp2_hw(fmaf(d, s.k, d * s.rest)); }
// e of eight l under the largest, `top`.  Where nothing is left that is -inf, and so is every l (or NaN).
__device__ __forceinline__ float under(float l, float top, const Sharpness& s) {
  return l == top ? (top > -kInf ? 1.f : 0.f) : exp_of(l - (top > -kInf ? top : 0.f), s);
}
__device__ __forceinline__ void under(const float (&l)[kVec], float top, const Sharpness& s, float (&e)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) e[i] = l[i];
  float level = top > -kInf ? top : 0.f;
  if (top == kInf) {   // (as if those at infinity were at zero, the others, but for a NaN, below everything)
    level = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) e[i] = e[i] == kInf ? 0.f : e[i] - kInf;
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) e[i] = exp_of(e[i] - level, s);   // (zero times the factor is zero)
}

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = min(x, __shfl_xor(x, off, 64));
  return x;
}

// The first launch: a workgroup a segment of a row, `steps` times kSeg tokens, the next of them loaded ahead.
template <typename T>
__global__ __launch_bounds__(kThreads) void logits_parts(LogitsArgs a, uint32_t segs, uint32_t steps) {
  __shared__ Part waves[kThreads / kWave];
  const uint32_t row = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint32_t base = seg * steps * kSeg + w * kWaveSpan;
  const Told told(a);
  Tokens<T, false> next(a, row, base + lane * kVec);
  const RowOf r = row_of(a, row, told);
  if (r.out) return;
  next.load_rest(r);
  const Lists lists(a, r, row);
  const Sharpness k = sharpness(r.temperature);
  const bool greedy = !(r.temperature > 0.f);
  Part mine{-kInf, 0.f, INT32_MAX, 0};   // the thread's
  for (uint32_t s = 0; s < steps; ++s, base += kSeg) {
    Tokens<T, false> now = next;
    // (behind the segment: the row's end, which is not used)
    next = Tokens<T, false>(a, row, s + 1 < steps ? base + kSeg + lane * kVec : static_cast<uint32_t>(a.V));
    next.load_rest(r);
    float l[kVec], e[kVec], top = mine.top;
    now.changed(r, lists, base, l);
#pragma unroll
    for (int i = 0; i < kVec; ++i) top = fmaxf(top, l[i]);
    if (greedy && top > mine.top) {
#pragma unroll
      for (int i = kVec - 1; i >= 0; --i)
        if (l[i] == top) mine.first = now.place.at + i;
    }
    mine.sum *= under(mine.top, top, k);
    under(l, top, k, e);
#pragma unroll
    for (int i = 0; i < kVec; ++i) mine.sum += e[i];
    mine.top = top;
  }
  const float most = wave_max(mine.top);
  const float sum = wave_sum(mine.sum == mine.sum ? mine.sum * under(mine.top, most, k) : mine.sum);   // (a NaN shows, whatever it weighs)
  const int first = greedy ? wave_min(mine.top == most ? mine.first : INT32_MAX) : 0;
  if (lane == 0) waves[w] = Part{most, sum, first, 0};
  __syncthreads();
  if (threadIdx.x == 0) {
    Part p{fmaxf(fmaxf(waves[0].top, waves[1].top), fmaxf(waves[2].top, waves[3].top)), 0.f, INT32_MAX, 0};
    for (int i = 0; i < kThreads / kWave; ++i) {
      p.sum += waves[i].sum == waves[i].sum ? waves[i].sum * under(waves[i].top, p.top, k) : waves[i].sum;
      if (waves[i].top == p.top) p.first = min(p.first, waves[i].first);
    }
    static_cast<Part*>(a.parts)[blockIdx.x] = p;
  }
}

// a row's whole from its parts, on every lane of a wave; x: the part of the lane's number
__device__ __forceinline__ Part whole_of(const Part* parts, const Part& x, uint32_t segs, const Sharpness& k, bool greedy) {
  const uint32_t lane = threadIdx.x & 63;
  float top = lane < segs ? x.top : -kInf;
  for (uint32_t s = kWave + lane; s < segs; s += kWave) top = fmaxf(top, parts[s].top);
  Part all{wave_max(top), 0.f, INT32_MAX, 0};
  auto add = [&](const Part& p) {
    all.sum += p.sum == p.sum ? p.sum * under(p.top, all.top, k) : p.sum;   // (a NaN shows, whatever it weighs)
    if (p.top == all.top) all.first = min(all.first, p.first);
  };
  if (lane < segs) add(x);
  for (uint32_t s = kWave + lane; s < segs; s += kWave) add(parts[s]);
  all.sum = wave_sum(all.sum);
  if (greedy) all.first = wave_min(all.first);
  return all;
}

// The second launch: p of a window of kSeg tokens from the parts of all, or the changed logits themselves. No loop
// (two windows a workgroup: 58.3 us for 314 rows of 131072, so 57.5).
template <typename T, typename TO, bool TINY, bool PROBS, bool PASSING>
__global__ __launch_bounds__(kThreads) void logits_out(LogitsArgs a, uint32_t windows, uint32_t segs) {
  const uint32_t row = blockIdx.x / windows, base = blockIdx.x % windows * kSeg + (threadIdx.x >> 6) * kWaveSpan;
  const uint32_t lane = threadIdx.x & 63;
  const Told told(a);
  const Part* const parts = static_cast<const Part*>(a.parts) + static_cast<int64_t>(row) * segs;
  Part part{};
  if constexpr (PROBS) part = parts[min(lane, segs - 1)];
  Tokens<T, TINY, PASSING> now(a, row, base + lane * kVec);
  const RowOf r = row_of(a, row, told);
  if (r.out) return;
  now.load_rest(r);
  const Lists lists(a, r, row);
  const Sharpness k = sharpness(r.temperature);
  const bool greedy = !(r.temperature > 0.f);
  Part whole{};
  if constexpr (PROBS) whole = whole_of(parts, part, segs, k, greedy);
  float l[kVec];
  now.changed(r, lists, base, l);
  if constexpr (PROBS) {
    if (greedy) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        l[i] = whole.sum != whole.sum ? whole.sum : whole.top > -kInf && now.place.at + i == whole.first ? 1.f : 0.f;
    } else {
      const float f = whole.sum == 0.f ? 0.f : 1.f / whole.sum;
      under(l, whole.top, k, l);
#pragma unroll
      for (int i = 0; i < kVec; ++i) l[i] *= f;
    }
  }
  now.place.template store<PASSING>(static_cast<TO*>(a.out) + row * a.V, l);
}

// Both at once: a workgroup a row of up to CH windows of its threads, the changed logits kept in registers.
template <typename T, typename TO, int THREADS, int CH, bool TINY, bool PASSING>
__global__ __launch_bounds__(THREADS) void logits_one(LogitsArgs a) {
  constexpr int kOneWaves = THREADS / kWave, kOneSeg = THREADS * kVec;
  __shared__ float tops[kOneWaves], sums[kOneWaves];
  __shared__ int firsts[kOneWaves];
  const uint32_t row = blockIdx.x;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t base = w * kWaveSpan;
  const Told told(a);
  Tokens<T, TINY> next(a, row, base + lane * kVec);
  const RowOf r = row_of(a, row, told);
  if (r.out) return;
  next.load_rest(r);
  const Lists lists(a, r, row);
  const Sharpness k = sharpness(r.temperature);
  const bool greedy = !(r.temperature > 0.f);
  float l[CH][kVec], top = -kInf, sum = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    Tokens<T, TINY> now = next;
    if (c + 1 < CH) {
      next = Tokens<T, TINY>(a, row, base + (c + 1) * kOneSeg + lane * kVec);
      next.load_rest(r);
    }
    now.changed(r, lists, base + c * kOneSeg, l[c]);
#pragma unroll
    for (int i = 0; i < kVec; ++i) top = fmaxf(top, l[c][i]);
  }
  top = wave_max(top);
  if (lane == 0) tops[w] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOneWaves; ++i) top = fmaxf(top, tops[i]);
  if (greedy) {
    int first = INT32_MAX;
#pragma unroll
    for (int c = CH - 1; c >= 0; --c) {
      const Place<TINY> place(a, base + c * kOneSeg + lane * kVec);
#pragma unroll
      for (int i = kVec - 1; i >= 0; --i) {
        if (l[c][i] == top) first = place.at + i;
        sum += l[c][i] != l[c][i] ? l[c][i] : 0.f;   // (a NaN shows)
      }
    }
    first = wave_min(first);
    if (lane == 0) firsts[w] = first;
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      under(l[c], top, k, l[c]);
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum += l[c][i];
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) sums[w] = sum;
  __syncthreads();
  sum = 0.f;
  int first = INT32_MAX;
#pragma unroll
  for (int i = 0; i < kOneWaves; ++i) {
    sum += sums[i];
    if (greedy) first = min(first, firsts[i]);
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const Place<TINY> place(a, base + c * kOneSeg + lane * kVec);
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      l[c][i] = !greedy ? l[c][i] * f : sum != sum ? sum : top > -kInf && place.at + i == first ? 1.f : 0.f;
    place.template store<PASSING>(static_cast<TO*>(a.out) + row * a.V, l[c]);
  }
}

// A row's segments in the first of two launches: about so many workgroups in all, eight to a row or a multiple of it,
// as workgroups go to the eight L2s in turn: the rows of a sequence then find its counts in one. (314 rows of
// 131072: 8 segments 43.3 us, 16 44.2, 32 51.4, 13 51.6.)
constexpr int64_t kManyBlocks = 4096;
template <typename T, typename TO, bool TINY>
hipError_t logits_at(const LogitsArgs& a, hipStream_t s) {
  const int64_t windows = logits_segments(a.V);
  const dim3 block(kThreads), all(static_cast<unsigned>(a.rows * windows));
  if (TINY || !a.probs) {
    hipLaunchKernelGGL((logits_out<T, TO, TINY, false, false>), all, block, 0, s, a, static_cast<uint32_t>(windows), 0u);
    return hipGetLastError();
  }
  const int64_t most = (kManyBlocks / 8 + a.rows - 1) / a.rows * 8;
  const uint32_t segs = static_cast<uint32_t>(std::min(windows, most)), steps = static_cast<uint32_t>((windows + segs - 1) / segs);
  hipLaunchKernelGGL((logits_parts<T>), dim3(static_cast<unsigned>(a.rows * segs)), block, 0, s, a, segs, steps);
  if (a.passing) hipLaunchKernelGGL((logits_out<T, TO, false, true, true>), all, block, 0, s, a, static_cast<uint32_t>(windows), segs);
  else hipLaunchKernelGGL((logits_out<T, TO, false, true, false>), all, block, 0, s, a, static_cast<uint32_t>(windows), segs);
  return hipGetLastError();
}
// Whether one launch: it reads the logits once, but a row is one compute unit's.
// - Up to 16384 tokens always; to 32768 where no lists change the logits, else from 80 rows on (their work is then more than a
//   launch).
// - To 57344, seven windows a thread (which spill 10 to 23 registers), from 128 rows on; past 36000 not for 257 to 1535 aligned rows:
//   at most 256 are a compute unit's each, some more wait for a second turn of them, and the caches still hold what two launches
//   read twice, if p is written past them.
// Two launches | one, us a call (of small ones the host's time), bf16 with everything on, then fp32 logits alone:
//   rows                1            8           64           96          128          256          512         1024         2048
//    2000    10.0    6.1  10.5    6.3  11.0    6.2  11.1    6.2  11.3    6.3  12.2    6.4  13.8    7.6  18.1    9.2  27.3   13.0
//    8000     9.9    6.7  10.8    6.9  10.6    7.3  11.1    7.5  11.4    7.6  15.2    9.0  21.6   11.7  36.0   23.9  70.0   42.4
//   16000    10.0    8.5  10.5    9.0  11.1    9.8  12.4   10.0  13.6   10.3  20.3   13.0  32.4   19.3  60.6   36.6   123   64.8
//   32000     9.6   12.4   9.8   12.7  12.9   14.2  15.8   14.4  18.6   15.4  30.9   24.9  52.3   44.2  94.5   82.0   191    148
//   40000                                           18.1   20.1  21.6   21.8  42.2   34.4  61.2   61.5   116    114   234    202
//   49152     9.3   18.2   9.9   18.3  15.5   19.8  19.6   21.2  23.2   23.1  44.0   38.7  65.6   71.7   125    128   256    239
//   57344                                           21.1   22.5  25.8   24.1  47.3   43.3  76.4   80.0   145    143   303    278
//    2000     8.9    5.8   8.6    5.6   8.3    5.5   8.4    5.5   8.6    5.8   8.9    5.9   8.8    5.7  10.4    6.0  15.2    7.6
//    8000     8.0    5.7   8.3    5.9   8.5    6.0   8.9    6.0   8.7    5.8   9.8    6.2  13.1    8.3  22.2   15.1  48.4   31.6
//   16000     8.5    6.0   8.6    5.9   8.9    6.3   8.8    6.5   9.3    7.0  13.3   10.0  20.9   16.5  41.8   32.2  88.8   53.3
//   32000     9.2    7.2   8.7    7.4   9.7    8.5  10.9    8.9  12.6    9.6  20.2   18.8  39.1   35.3  70.1   61.2   143    112
//   40000                                           12.3   12.9  14.0   14.1  30.4   29.2  45.8   52.6  85.0   89.5   180    181
//   49152     8.6   11.1   8.6   11.6  11.3   12.8  13.4   14.6  15.6   15.7  33.2   33.6  52.2   60.8  96.7    107   214    211
//   57344                                           14.6   14.3  17.2   16.5  35.7   37.0  60.2   69.9   112    121   253    243
// 512 and 1024 rows of 49152, the other two kinds: bf16 alone 43.7 54.2 and 81.3 93.1, fp32 with everything on 71.1 74.8 and 133 139.
// Unaligned, 512 rows of 50257: bf16 with everything on 80.5 63.6, fp32 alone 57.8 53.9.
bool in_one_launch(const LogitsArgs& a) {
  const bool lists = a.counts || a.ids || a.bias_starts;
  if (a.V > 2048 && a.rows >= 1 << 22) return false;   // (a launch holds fewer than 2^32 work items)
  if (a.V <= 16384) return true;
  if (a.V <= 32768) return !lists || a.rows >= 80;
  return a.V <= 57344 && a.rows >= 128 && (a.V <= 36000 || a.rows <= 256 || a.rows >= 1536 || !a.passing);
}
template <typename T, typename TO, bool PASSING>
hipError_t one_launch(const LogitsArgs& a, hipStream_t s) {
  const dim3 rows(static_cast<unsigned>(a.rows));
  if (a.V <= 2048) hipLaunchKernelGGL((logits_one<T, TO, 256, 1, false, PASSING>), rows, dim3(256), 0, s, a);
  else if (a.V <= 8192) hipLaunchKernelGGL((logits_one<T, TO, 1024, 1, false, PASSING>), rows, dim3(1024), 0, s, a);
  else if (a.V <= 16384) hipLaunchKernelGGL((logits_one<T, TO, 1024, 2, false, PASSING>), rows, dim3(1024), 0, s, a);
  else if (a.V <= 32768) hipLaunchKernelGGL((logits_one<T, TO, 1024, 4, false, PASSING>), rows, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((logits_one<T, TO, 1024, 7, false, PASSING>), rows, dim3(1024), 0, s, a);
  return hipGetLastError();
}
template <typename T, typename TO>
hipError_t logits_of(const LogitsArgs& a, hipStream_t s) {
  if (a.probs && a.V < kVec) {
    hipLaunchKernelGGL((logits_one<T, TO, 256, 1, true, false>), dim3(static_cast<unsigned>(a.rows)), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (a.probs && in_one_launch(a)) return a.passing ? one_launch<T, TO, true>(a, s) : one_launch<T, TO, false>(a, s);
  if (a.V < kVec) return logits_at<T, TO, true>(a, s);   // (changed logits)
  return logits_at<T, TO, false>(a, s);
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

// tokens added in place: a workgroup a sequence (whole-number atomics, so any order gives the same); 64 sequences of up to
// eight tokens 2.4 us, a launch and two dependent reads.
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

// a whole row written: a workgroup a segment, its tokens counted in shared memory; 16 prompts of up to
// 2000 tokens into rows of 50257 5.2 us: a few rounds of reads of the prompt, which every segment makes.
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

hipError_t launch_logits(const LogitsArgs& args, int in_bf16, int out_bf16, hipStream_t s) {
  LogitsArgs a = args;
  const int in = in_bf16 ? 2 : 4, out = out_bf16 ? 2 : 4;
  a.passing = ((reinterpret_cast<uintptr_t>(a.logits) | a.stride * in | reinterpret_cast<uintptr_t>(a.out) | a.V * out) & 15) == 0;
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
