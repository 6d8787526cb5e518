// Verification of drafted tokens against the target's probabilities, from
// given random numbers.  Row t of a sequence is the target's distribution
// after its token t; token t + 1 was drafted from row t + 1 of q:
//   token t + 1 holds iff those before it do and u_t q_{t+1}(x) < p_t(x)
//   w = max(p_n - q_{n+1}, 0) where draft n + 1 is refused (p_n where that is
//   zero everywhere), p_n after the last draft
//   the next token: the first j with w_0 + .. + w_j > r (w_0 + .. + w_{V-1})
// Products, differences and sums in 64 bits: a product of two of the inputs'
// numbers is exact, and a running sum over a large vocabulary has to be finer
// than the steps between its tokens, which 32 bits are not.
//
// Two launches (one for smaller vocabularies: verify_one): the row the sequence stops at is
// summed in segments of 2048 tokens, a workgroup each (every one finds the row for
// itself: a few reads), then one wave a sequence finds the segment, and in it the token.
// Segment sums are added in one order, so the token does not depend on which
// workgroup was first.
//
// What bounds it: the row's (or two rows') reading in the first launch, 12 us for 64
// sequences of 131072 (56 MB, 4.5 TB/s), and two launches' latency: the second is one
// wave's chain of dependent reads, 5 to 8 us.  One sequence of 50257: 9.2 us in a graph
// (9.8 to 10.4 called one by one, the host's time), 64 of 131072: 18.1 us.  A whole workgroup a sequence in the second, with barriers between
// its levels, took 16 and 30 us in all.
#include "pdn_device.hpp"
#include "pdn_internal.hpp"

namespace pdn {

namespace {

constexpr int kThreads = 256, kVec = 8, kSeg = kThreads * kVec;

inline __host__ __device__ int64_t segments(int64_t V) { return (V + kSeg - 1) / kSeg; }

struct Span {
  int64_t lo, n;   // first row, rows
};
__device__ __forceinline__ Span seq_span(const VerifyArgs& a, int64_t seq) {
  int64_t lo = seq * (a.rows / a.N), hi = lo + a.rows / a.N;
  if (a.starts) {
    lo = a.starts[seq];
    hi = a.starts[seq + 1];
  }
  lo = min(max(lo, (int64_t)0), a.rows);
  return Span{lo, max(min(hi, a.rows) - lo, (int64_t)0)};
}

// drafts that hold, found by one wave (every lane returns it)
template <typename T>
__device__ __forceinline__ int64_t held(const VerifyArgs& a, const Span& s, int l) {
  const T* p = static_cast<const T*>(a.p);
  const T* q = static_cast<const T*>(a.q);
  for (int64_t t0 = 0; t0 + 1 < s.n; t0 += kWave) {
    const int64_t row = s.lo + t0 + l;
    const bool draft = t0 + l + 1 < s.n;
    bool ok = false;
    if (draft) {
      const int64_t x = a.ids[row + 1];
      if (x >= 0 && x < a.V) {
        const double px = to_f(p[row * a.V + x]), qx = q ? to_f(q[(row + 1) * a.V + x]) : 1.f;
        ok = a.u[row] * qx < px;
      }
    }
    const unsigned long long bad = __ballot(draft && !ok);
    if (bad) return t0 + __ffsll(bad) - 1;
  }
  return max(s.n - 1, (int64_t)0);
}

// Eight tokens' weights from j0: p (kind 1), or what is left of it over q or
// without the drafted token x (kind 0; x < 0 and q NULL: p).  No token past V,
// no NaN, nothing below zero.
template <typename T>
struct Row {
  const T* p;
  const T* q;   // NULL: without the one token x
  int64_t x;
};
template <typename T>
__device__ __forceinline__ void ld_row(const T* p, int64_t j0, int64_t V, float (&v)[kVec]) {
  T raw[kVec];
  if (j0 + kVec <= V) {
    __builtin_memcpy(raw, p + j0, sizeof raw);   // (rows of an odd V are aligned to an element only)
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) raw[i] = j0 + i < V ? p[j0 + i] : from_f<T>(0.f);
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = to_f(raw[i]);
}
template <typename T>
__device__ __forceinline__ void weights(const Row<T>& r, int64_t j0, int64_t V, double (&w0)[kVec], double (&w1)[kVec]) {
  float p[kVec], q[kVec];
  ld_row(r.p, j0, V, p);
  if (r.q) ld_row(r.q, j0, V, q);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const double x = p[i], y = r.q ? x - q[i] : (j0 + i == r.x ? 0.0 : x);
    w1[i] = x > 0.0 ? x : 0.0;
    w0[i] = y > 0.0 ? y : 0.0;
  }
}
template <typename T>
__device__ __forceinline__ Row<T> stop_row(const VerifyArgs& a, const Span& s, int64_t n) {
  const int64_t row = s.lo + n;
  Row<T> r{static_cast<const T*>(a.p) + row * a.V, nullptr, -1};
  if (n + 1 < s.n) {   // a draft was refused
    if (a.q) r.q = static_cast<const T*>(a.q) + (row + 1) * a.V;
    else r.x = a.ids[row + 1];
  }
  return r;
}

__device__ __forceinline__ double wave_add(double x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_sums(VerifyArgs a) {
  __shared__ double sW[2][kThreads / kWave];
  const int64_t segs = segments(a.V), seq = blockIdx.x / segs, seg = blockIdx.x % segs;
  const Span s = seq_span(a, seq);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  if (s.n == 0) return;
  const int64_t n = held<T>(a, s, l);
  if (seg == 0 && tid == 0) a.accepted[seq] = static_cast<int>(n + 1);
  double w0[kVec], w1[kVec], x0 = 0.0, x1 = 0.0;
  weights(stop_row<T>(a, s, n), seg * kSeg + tid * kVec, a.V, w0, w1);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    x0 += w0[i];
    x1 += w1[i];
  }
  x0 = wave_add(x0);
  x1 = wave_add(x1);
  if (l == 0) {
    sW[0][w] = x0;
    sW[1][w] = x1;
  }
  __syncthreads();
  if (tid < 2) a.sums[blockIdx.x * 2 + tid] = ((sW[tid][0] + sW[tid][1]) + sW[tid][2]) + sW[tid][3];
}

// inclusive sums over the wave's lanes, in order
__device__ __forceinline__ double wave_scan(double x, int l) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double y = __shfl_up(x, off, 64);
    if (l >= off) x += y;
  }
  return x;
}

// The first place of the wave's 64 (lane l's: its inclusive sum cum, its own share
// x) whose sum is over the target: the lane, or -1; `last` keeps the last place
// that has a share.
__device__ __forceinline__ int first_over(double cum, double x, double target, int* last) {
  const unsigned long long some = __ballot(x > 0.0), over = __ballot(x > 0.0 && cum > target);
  *last = some ? 63 - __clzll(some) : -1;
  return over ? __ffsll(over) - 1 : -1;
}

// The token, by one wave: the segment (of PER tokens a lane), 64 at a time, then in it
// the token.  load_sums(b, x): the sums of segment b + l, of both kinds; x holds
// those of the first 64.
template <typename T, int PER, typename Load>
__device__ __forceinline__ void pick(const VerifyArgs& a, int64_t seq, const Span& s, int64_t n, double r, int64_t segs,
                                     int l, const Load& load_sums, double (&x)[2]) {
  double cum[2];
  // running sums of 64 segments, of both kinds
  auto sum_segments = [&](int64_t b, const double (&base)[2]) {
    if (segs > kWave) load_sums(b, x);   // (else they are at hand)
#pragma unroll
    for (int k = 0; k < 2; ++k) cum[k] = base[k] + wave_scan(x[k], l);
  };
  double tot[2] = {0.0, 0.0};
  for (int64_t b = 0; b < segs; b += kWave) {
    sum_segments(b, tot);
#pragma unroll
    for (int k = 0; k < 2; ++k) tot[k] = __shfl(cum[k], 63, 64);
  }
  const int kind = tot[0] > 0.0 ? 0 : 1;   // nothing left over q: p itself
  const double target = r * tot[kind];
  // the first segment whose running sum is over the target, else the last that has a weight
  int64_t seg = -1;
  double base[2] = {0.0, 0.0}, before = 0.0;
  bool found = false;
  for (int64_t b = 0; b < segs && !found; b += kWave) {
    if (segs > kWave) sum_segments(b, base);   // (else they are at hand)
    const double c = kind ? cum[1] : cum[0], w = kind ? x[1] : x[0];
    int last;
    const int f = first_over(c, w, target, &last);
    found = f >= 0;
    const int at = found ? f : last;
    if (at >= 0) {
      seg = b + at;
      before = __shfl(c - w, at, 64);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) base[k] = __shfl(cum[k], 63, 64);
  }
  if (seg < 0) {   // no token has a weight
    if (l == 0) a.token[seq] = -1;
    return;
  }
  const Row<T> row = stop_row<T>(a, s, n);
  const int64_t j0 = (seg * kWave + l) * PER;
  double v[PER / kVec][kVec], mine = 0.0;
#pragma unroll
  for (int c = 0; c < PER / kVec; ++c) {
    double w0[kVec], w1[kVec];
    weights(row, j0 + c * kVec, a.V, w0, w1);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      v[c][i] = kind ? w1[i] : w0[i];
      mine += v[c][i];
    }
  }
  const double upto = wave_scan(mine, l);
  double sum = before + (upto - mine);
  int last, f = first_over(before + upto, mine, target, &last);
  if (f < 0 || !found) f = last;   // (rounding at a segment's very end, or no segment is over the target)
  int first = -1, final = -1;
#pragma unroll
  for (int c = 0; c < PER / kVec; ++c)
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      sum += v[c][i];
      if (v[c][i] > 0.0) {
        final = c * kVec + i;
        if (first < 0 && found && sum > target) first = c * kVec + i;
      }
    }
  if (l == f) a.token[seq] = static_cast<int>(j0 + (first >= 0 ? first : final));
}

template <typename T>
__global__ __launch_bounds__(kWave) void verify_pick(VerifyArgs a) {
  const int64_t segs = segments(a.V), seq = blockIdx.x;
  const int l = threadIdx.x;
  // Everything that can be read at once is, before the first of it is waited for (a
  // sequence without rows has no sums, and does not use what is read here).
  const double* const sums = a.sums + seq * segs * 2;
  int64_t n = 0;
  double r = 0.0, x[2];
  auto load_sums = [&](int64_t b, double (&x)[2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) x[k] = b + l < segs ? sums[2 * (b + l) + k] : 0.0;
  };
  if (a.rows > 0) {
    n = a.accepted[seq] - 1;
    r = a.r[seq];
    load_sums(0, x);
  }
  const Span s = seq_span(a, seq);
  if (s.n == 0) {   // no rows
    if (l == 0) {
      a.accepted[seq] = 0;
      a.token[seq] = -1;
    }
    return;
  }
  pick<T, kSeg / kWave>(a, seq, s, n, r, segs, l, load_sums, x);
}

// Smaller vocabularies in one launch: a workgroup a sequence, a wave a segment of 512
// tokens in turn; sums in LDS, the token by the first wave.  A step of 8192
// tokens takes 1.5 us of one compute unit, where the other form's first launch has them
// all and its second costs 4 to 5 us.  The more sequences there are the fewer compute units
// that leaves idle (fp32 with q, us, two launches | one; less with bf16 or without q, the
// line between them the same within 1 us):
//               1000       8000       16000      24576      32000      40000      50257      65536
//   1 sequence  10.2  5.4   9.3  6.1   9.3  7.6   9.1  8.8   9.3 10.4   9.1 12.1   9.2 13.7   9.2 16.4
//   16                               10.2  8.0   9.9  9.2  10.2 10.8  10.7 12.8  10.4 14.5  10.1 17.1
//   64          11.6  6.0  11.4  6.7  11.6  8.1  10.8  9.4  12.6 11.1  12.6 14.3  14.1 16.2  14.1 19.8
//   128                              13.1  8.5  12.8 10.7  15.0 12.9  17.2 15.5  18.0 17.0  18.9 20.2
//   256         12.0  6.3  13.4  7.2  15.9  9.8  17.3 11.9  20.0 14.4  21.9 16.9  24.5 18.6  26.8 21.9
//   512                              20.6 14.5  22.8 17.7  28.2 20.9  31.9 24.9  37.7 29.2  47.8 38.3
// (A wave's segments all loaded first: 8.3 us at 1000 tokens, 10.2 at 32000.)
constexpr int kOneWaves = 16, kOneSeg = kWave * kVec, kOneMost = 8 * kOneWaves * kOneSeg;
bool one_launch(int64_t N, int64_t V) {
  if (N >= 1 << 22) return false;   // (a launch holds fewer than 2^32 work items)
  return V <= 24576 || (V <= kOneMost && V <= 24576 + 192 * N);
}
template <typename T>
__global__ __launch_bounds__(kOneWaves * kWave) void verify_one(VerifyArgs a) {
  __shared__ double sums[kOneMost / kOneSeg][2];
  const int64_t seq = blockIdx.x;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, segs = static_cast<int>((a.V + kOneSeg - 1) / kOneSeg);
  const Span s = a.rows > 0 ? seq_span(a, seq) : Span{0, 0};
  if (s.n == 0) {   // no rows
    if (threadIdx.x == 0) {
      a.accepted[seq] = 0;
      a.token[seq] = -1;
    }
    return;
  }
  const double r = a.r[seq];
  const int64_t n = held<T>(a, s, l);
  if (threadIdx.x == 0) a.accepted[seq] = static_cast<int>(n + 1);
  const Row<T> row = stop_row<T>(a, s, n);
#pragma unroll 2
  for (int seg = w; seg < segs; seg += kOneWaves) {
    double w0[kVec], w1[kVec], x0 = 0.0, x1 = 0.0;
    weights(row, seg * static_cast<int64_t>(kOneSeg) + l * kVec, a.V, w0, w1);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      x0 += w0[i];
      x1 += w1[i];
    }
    x0 = wave_add(x0);
    x1 = wave_add(x1);
    if (l == 0) {
      sums[seg][0] = x0;
      sums[seg][1] = x1;
    }
  }
  __syncthreads();
  if (w > 0) return;
  double x[2];
  auto load_sums = [&](int64_t b, double (&x)[2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) x[k] = b + l < segs ? sums[b + l][k] : 0.0;
  };
  load_sums(0, x);
  pick<T, kVec>(a, seq, s, n, r, segs, l, load_sums, x);
}

template <typename T>
hipError_t launch(const VerifyArgs& a, hipStream_t s) {
  if (one_launch(a.N, a.V)) {
    hipLaunchKernelGGL((verify_one<T>), dim3(static_cast<unsigned>(a.N)), dim3(kOneWaves * kWave), 0, s, a);
    return hipGetLastError();
  }
  if (a.rows > 0)
    hipLaunchKernelGGL((verify_sums<T>), dim3(static_cast<unsigned>(a.N * segments(a.V))), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL((verify_pick<T>), dim3(static_cast<unsigned>(a.N)), dim3(kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int64_t verify_blocks(int64_t V) { return segments(V); }

hipError_t launch_verify(const VerifyArgs& a, int io_bf16, hipStream_t s) {
  return io_bf16 ? launch<bf16>(a, s) : launch<float>(a, s);
}

}  // namespace pdn
