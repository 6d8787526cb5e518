// Norms around the rule in a block.  Rows are independent; what bounds every call is
// the reading and writing of its tensors, so each kernel holds a row in registers, reads every
// tensor once and writes every output once.  bf16, of 5.15 TB/s that a copy has: the residual norm of 16384 x 2048
// rows on an fp32 stream 73 us (5.5 TB/s), its backward with both norms and a scale 77 and 5 for the sums
// (4.9); norms of 16384 x 16 heads of 128 24 us (5.7), the gated one's backward 70 and 5 (4.5).
//
// Residual norm, rows of D channels (r: 1 / sqrt(mean of squares + eps)):
//   a = y or y r_y w_post     h = residual + alpha s a      u = h r_h w
// backward, with g = du w and t the gradient of h:
//   t = dh + r_h g - h r_h^3 mean(g h)        dresidual = t     dw = sum_rows du h r_h
//   b = alpha s t                             ds = sum_rows alpha t a
//   dy = b, or with e = b w_post  r_y e - y r_y^3 mean(e y)     dw_post = sum_rows b y r_y
//
// Head norm, rows of d channels (r over the mean or the sum of squares, c = 1 / d or 1):
//   y = x r w act(z)
// backward, with g = dy w act(z):
//   dx = r g - x r^3 c sum(g x)    dz = dy w x r act'(z)    dw = sum_rows dy act(z) x r
#include <algorithm>

#include "pdn_device.hpp"
#include "pdn_internal.hpp"
#include "pdn_lanes.hpp"

namespace pdn {

namespace {

constexpr int kVec = 8;

// The eight columns of a thread: from `col` on in a row of n.  Loads must not branch (a wait for
// each would follow it, which took the backward of 16384 x 2048 rows 1.3 times as long), so every thread loads eight columns of the row that are there,
// and `keep` says which of them are its own: a last thread with fewer than eight takes the row's
// last eight, one without any the first.  By the row: a multiple of eight columns, more than
// eight, or fewer (its only thread then loads element by element).
enum RowKind { kEights, kMore, kFewer };
inline RowKind row_kind(int64_t n) { return n % 8 == 0 ? kEights : n > 8 ? kMore : kFewer; }
template <RowKind KIND>
struct Cols {
  int at, n;
  uint32_t keep;   // bit i: column at + i
  __device__ __forceinline__ Cols(int col, int n, bool whole = false) : n(n) {   // whole: eight of them are there for sure
    const bool on = col < n;
    if (whole) {
      at = col;
      keep = 0xff;
    } else if constexpr (KIND == kEights) {
      at = on ? col : 0;
      keep = on ? 0xff : 0;
    } else if constexpr (KIND == kMore) {
      at = on ? min(col, n - kVec) : 0;
      keep = on ? (0xffu << (col - at)) & 0xff : 0;
    } else {
      at = 0;
      keep = on ? (1u << n) - 1 : 0;
    }
  }
};

// Eight elements as they are in memory (aligned to an element only).
template <typename T>
struct Raw {
  static constexpr int kWords = kVec * sizeof(T) / 4;
  uint32_t w[kWords];
  template <RowKind KIND>
  __device__ __forceinline__ void load(const T* p, const Cols<KIND>& c) {
    if constexpr (KIND != kFewer) {
      __builtin_memcpy(w, p + c.at, sizeof w);
    } else {
      T x[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) x[i] = p[min(i, c.n - 1)];
      __builtin_memcpy(w, x, sizeof w);
    }
  }
  // zero in the columns that are not its own (apart from the load, as it waits for it)
  template <RowKind KIND>
  __device__ __forceinline__ void settle(const Cols<KIND>& c) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (KIND == kEights) w[i] = c.keep ? w[i] : 0;
      else if constexpr (sizeof(T) == 4) w[i] = c.keep >> i & 1 ? w[i] : 0;
      else w[i] &= (c.keep >> (2 * i) & 1 ? 0xffffu : 0) | (c.keep >> (2 * i + 1) & 1 ? 0xffff0000u : 0);
    }
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
    else return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};
template <typename T, RowKind KIND>
__device__ __forceinline__ void store(T* p, const Cols<KIND>& c, const float (&v)[kVec]) {
  T x[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) x[i] = from_f<T>(v[i]);
  if (c.keep == 0xff) {
    __builtin_memcpy(p + c.at, x, sizeof x);
  } else if constexpr (KIND != kEights) {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (c.keep >> i & 1) p[c.at + i] = x[i];
  }
}
// x, or zero in a column that is not its own: what enters a row's sum with a vector in it, since the zero
// of a row there times another column's infinite entry would be a NaN in the whole row.
template <RowKind KIND>
__device__ __forceinline__ float own(const Cols<KIND>& c, int i, float x) {
  return (KIND == kEights ? c.keep : c.keep >> i & 1) ? x : 0.f;
}
template <RowKind KIND>
__device__ __forceinline__ void settle(const Cols<KIND>& c, float (&v)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = own(c, i, v[i]);
}
// of a vector that may be NULL (= 1)
template <RowKind KIND>
__device__ __forceinline__ void ld_weight(const float* p, const Cols<KIND>& c, float (&v)[kVec]) {
  if (p) {
    Raw<float> r;
    r.load(p, c);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = r[i];
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = 1.f;
  }
}

__device__ __forceinline__ float factor(float squares, float c, float eps) { return 1.f / sqrtf(squares * c + eps); }
// in a backward pass: a row whose squares left fp32 has no gradient (a factor of zero would make it zeros)
__device__ __forceinline__ float factor_back(float squares, float c, float eps) {
  return squares == __builtin_inff() ? __builtin_nanf("") : factor(squares, c, eps);
}

// Sums over the workgroup's threads, the same on each of them.  Two buffers in turn: one barrier a sum.
template <int N>
__device__ __forceinline__ void block_sum(float (&x)[N], float (*buf)[16][4], int& turn) {
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = wave_sum(x[k]);
  const int waves = blockDim.x >> 6;   // (two at least)
  float(*const b)[4] = buf[turn & 1];
  ++turn;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) b[threadIdx.x >> 6][k] = x[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = 0.f;
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] += b[w][k];
}

// A workgroup's part of a vector's gradient from its groups of L lanes: a wave's by shuffles, then the waves'
// (columns of a lane that are another's are zero).
template <RowKind KIND>
__device__ __forceinline__ void group_part(float (&v)[kVec], const Cols<KIND>& o, int L, float (*sum)[kWave * kVec], float* part) {
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    for (int off = L; off < kWave; off <<= 1) v[i] += __shfl_xor(v[i], off, 64);
  const int wave = threadIdx.x / kWave, l = threadIdx.x & 63;
  __syncthreads();   // (of the last vector's)
  if (l < L)
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (o.keep >> i & 1) sum[wave][o.at + i] = v[i];
  __syncthreads();
  for (int j = threadIdx.x; j < o.n; j += blockDim.x) part[j] = (sum[0][j] + sum[1][j]) + (sum[2][j] + sum[3][j]);
}

// The threads of a row: a workgroup, or GROUP: L lanes of one (a power of two) where a row has not
// more than eight columns for each lane of a wave.
constexpr int kGroupThreads = 256;
template <bool GROUP>
struct Team {
  int lane, size, L;
  int64_t first, step;   // rows
  float (*buf)[16][4];
  int turn = 0;
  __device__ __forceinline__ Team(int L, float (*buf)[16][4]) : L(L), buf(buf) {
    const int groups = GROUP ? kGroupThreads / L : 1;
    lane = GROUP ? threadIdx.x & (L - 1) : threadIdx.x;
    size = GROUP ? L : blockDim.x;
    first = blockIdx.x * static_cast<int64_t>(groups) + (GROUP ? threadIdx.x / L : 0);
    step = gridDim.x * static_cast<int64_t>(groups);
  }
  template <int N>
  __device__ __forceinline__ void sum(float (&x)[N]) {
    if constexpr (GROUP) {
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = lanes_sum(x[k], L);
    } else {
      block_sum(x, buf, turn);
    }
  }
  // the k-th eight columns of a thread, of CH (of several all but the last are whole: row_threads)
  template <RowKind KIND, int CH>
  __device__ __forceinline__ Cols<KIND> cols(int k, int D) const {
    return Cols<KIND>((k * size + lane) * kVec, D, k + 1 < CH);
  }
};

template <typename TI, typename TS, int CH, bool POST, bool GROUP, RowKind KIND>
__global__ __launch_bounds__(GROUP ? kGroupThreads : 1024) void rnorm_fwd(RnormArgs a, int L) {
  __shared__ float buf[2][16][4];
  Team<GROUP> team(L, buf);
  const int D = static_cast<int>(a.D);
  const float c = 1.f / a.D;
  for (int64_t row = team.first; row < a.rows; row += team.step) {
    const int64_t at = row * a.D;
    Raw<TI> y[CH];
    Raw<TS> x[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, D);
      y[k].load(static_cast<const TI*>(a.y) + at, o);
      if (a.residual) x[k].load(static_cast<const TS*>(a.residual) + at, o);
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) y[k].settle(team.template cols<KIND, CH>(k, D));
    float h[CH][kVec], q[1] = {0.f}, ry = 1.f;
    if constexpr (POST) {
#pragma unroll
      for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < kVec; ++i) q[0] += y[k][i] * y[k][i];
      team.sum(q);
      ry = factor(q[0], c, a.eps);
      q[0] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, D);
      float v[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) h[k][i] = y[k][i];
      if constexpr (POST) {
        ld_weight(a.post_weight, o, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] *= ry * v[i];
      }
      if (a.scale) {
        ld_weight(a.scale, o, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] *= v[i];
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) h[k][i] *= a.alpha;
      if (a.residual) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] += x[k][i];
      }
      settle(o, h[k]);
      if (a.h) store(static_cast<TS*>(a.h) + at, o, h[k]);
#pragma unroll
      for (int i = 0; i < kVec; ++i) q[0] += h[k][i] * h[k][i];
    }
    team.sum(q);
    const float rh = factor(q[0], c, a.eps);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, D);
      float v[kVec];
      ld_weight(a.weight, o, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] *= h[k][i] * rh;
      store(static_cast<TI*>(a.u) + at, o, v);
    }
  }
}

// The backward: a team takes every so many-th row and keeps the vectors' gradients of its columns in
// registers, of D > 8192 two of them in shared memory; the workgroups' (rnorm_parts) are summed by sum_parts.
// Up to 8192 columns the next row is loaded while this one waits for its sums, and the vectors are
// in registers, or where a row takes more than 256 threads (and a thread has 128 of those) in shared memory.
template <typename TI, typename TS, int CH, bool Y, RowKind KIND>
struct BackRows {   // what a row's step reads
  Raw<TI> du[CH], y[Y ? CH : 1];
  Raw<TS> h[CH], dh[CH];
  template <typename TEAM>
  __device__ __forceinline__ void load(const RnormArgs& a, const TEAM& team, int64_t row) {
    const int64_t at = row * a.D;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, static_cast<int>(a.D));
      du[k].load(static_cast<const TI*>(a.du) + at, o);
      h[k].load(static_cast<const TS*>(a.h_in) + at, o);
      if constexpr (Y) {
        if (a.y) y[k].load(static_cast<const TI*>(a.y) + at, o);
      }
      if (a.dh) dh[k].load(static_cast<const TS*>(a.dh) + at, o);
    }
  }
  template <typename TEAM>
  __device__ __forceinline__ void settle(const RnormArgs& a, const TEAM& team) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, static_cast<int>(a.D));
      du[k].settle(o);
      h[k].settle(o);
      if constexpr (Y) y[k].settle(o);
      dh[k].settle(o);
    }
  }
};
constexpr int kBackWaves = 3;   // a SIMD's, where a workgroup has up to 256 threads
template <typename TI, typename TS, int CH, bool POST, bool SCALE, bool GROUP, int THREADS, RowKind KIND>
__global__ __launch_bounds__(THREADS, THREADS > 256 ? 4 : kBackWaves) void rnorm_bwd(RnormArgs a, int L) {
  constexpr bool kAhead = CH == 1, kShared = kAhead && THREADS > 256;
  constexpr int kVectors = 1 + POST + SCALE;
  // Where other columns' entries are made zero: once, or in rows of two times eight columns for each, in their products or as they
  // are loaded (what spills less: 2048 x 16384 with both norms and a scale 186 | 196 us, without the scale 188 | 156).
  constexpr bool kProducts = !kAhead && SCALE;
  __shared__ float buf[2][16][4];
  __shared__ float kept[CH > 1 && POST ? CH * kVec * THREADS : 1], kept2[CH > 1 && SCALE ? CH * kVec * THREADS : 1];
  __shared__ floatx4 vectors[kShared ? kVectors * 2 * THREADS : 1];   // (a thread's own places, THREADS apart)
  Team<GROUP> team(L, buf);
  const int D = static_cast<int>(a.D);
  const float c = 1.f / a.D;
  constexpr bool kRegs = CH == 1;   // (all three gradients in registers)
  float dw[CH][kVec] = {}, dp[POST && kRegs ? CH : 1][kVec] = {}, ds[SCALE && kRegs ? CH : 1][kVec] = {};
  float w[kVec], wp[kVec], sc[kVec];
  // weight (0), post_weight (1), scale (2) at the thread's columns
  auto of_memory = [&](int which, int k, float (&v)[kVec]) {
    ld_weight(which == 0 ? a.weight : which == 1 ? a.post_weight : a.scale, team.template cols<KIND, CH>(k, D), v);
  };
  auto place = [&](int which, int half) -> floatx4& {
    return vectors[((which == 2 && !POST ? 1 : which) * 2 + half) * THREADS + threadIdx.x];
  };
  auto get = [&](int which, int k, float (&v)[kVec]) {
    if constexpr (kShared) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = place(which, i / 4)[i % 4];
    } else if constexpr (!kAhead) {
      of_memory(which, k, v);
      if constexpr (!kProducts) settle(team.template cols<KIND, CH>(k, D), v);
    }
  };
  if constexpr (kAhead) {
    const auto o = team.template cols<KIND, CH>(0, D);
    of_memory(0, 0, w);
    settle(o, w);
    if constexpr (POST) {
      of_memory(1, 0, wp);
      settle(o, wp);
    }
    if constexpr (SCALE) {
      of_memory(2, 0, sc);
      settle(o, sc);
    }
    if constexpr (kShared) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        place(0, h) = floatx4{w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
        if constexpr (POST) place(1, h) = floatx4{wp[4 * h], wp[4 * h + 1], wp[4 * h + 2], wp[4 * h + 3]};
        if constexpr (SCALE) place(2, h) = floatx4{sc[4 * h], sc[4 * h + 1], sc[4 * h + 2], sc[4 * h + 3]};
      }
    }
  } else {   // (likewise)
#pragma unroll
    for (int i = 0; i < CH * kVec; ++i) {
      if constexpr (POST) kept[i * THREADS + threadIdx.x] = 0.f;
      if constexpr (SCALE) kept2[i * THREADS + threadIdx.x] = 0.f;
    }
  }
  BackRows<TI, TS, CH, POST || SCALE, KIND> r;
  if (team.first < a.rows) r.load(a, team, team.first);
  for (int64_t row = team.first; row < a.rows; row += team.step) {
    BackRows<TI, TS, CH, POST || SCALE, KIND> next;
    if constexpr (kAhead) {
      r.settle(a, team);
      if (row + team.step < a.rows) next.load(a, team, row + team.step);
    } else {
      if (row != team.first) r.load(a, team, row);
      r.settle(a, team);
    }
    const int64_t at = row * a.D;
    float e[POST ? CH : 1][kVec], q[POST ? 3 : 2] = {};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, D);
      get(0, k, w);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float g = r.du[k][i] * w[i];
        q[0] += r.h[k][i] * r.h[k][i];
        q[1] += (kProducts ? own(o, i, g) : g) * r.h[k][i];
        if constexpr (POST) q[2] += r.y[k][i] * r.y[k][i];
      }
    }
    team.sum(q);
    const float rh = factor_back(q[0], c, a.eps), mh = (rh * q[1] * c) * rh * rh;
    const float ry = POST ? factor_back(q[POST ? 2 : 0], c, a.eps) : 1.f;
    float p[1] = {0.f};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, D);
      get(0, k, w);
      if constexpr (POST) get(1, k, wp);
      if constexpr (SCALE) get(2, k, sc);
      float t[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        t[i] = rh * (r.du[k][i] * w[i]) - r.h[k][i] * mh;
        dw[k][i] += r.du[k][i] * (r.h[k][i] * rh);
        if (a.dh) t[i] += r.dh[k][i];
      }
      if (a.dresidual) store(static_cast<TS*>(a.dresidual) + at, o, t);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        t[i] *= a.alpha;
        if constexpr (SCALE) {
          if (a.y) {
            const float x = t[i] * (POST ? r.y[k][i] * ry * wp[i] : r.y[k][i]);
            if constexpr (kRegs) ds[k][i] += x;
            else kept2[(k * kVec + i) * THREADS + threadIdx.x] += x;
          }
          t[i] *= sc[i];
        }
        if constexpr (POST) {
          const float x = t[i] * (r.y[k][i] * ry);
          if constexpr (kRegs) dp[k][i] += x;
          else kept[(k * kVec + i) * THREADS + threadIdx.x] += x;
          e[k][i] = t[i] * wp[i];
          if constexpr (!kAhead) p[0] += (kProducts ? own(o, i, e[k][i]) : e[k][i]) * r.y[k][i];
        }
      }
      if constexpr (POST && kAhead) {   // (apart, as it spills less: fp32 8192 x 4096, everything on, 180 us, else 205)
#pragma unroll
        for (int i = 0; i < kVec; ++i) p[0] += e[k][i] * r.y[k][i];
      }
      if constexpr (!POST) store(static_cast<TI*>(a.dy) + at, o, t);
    }
    if constexpr (POST) {
      team.sum(p);
      const float my = (ry * p[0] * c) * ry * ry;
#pragma unroll
      for (int k = 0; k < CH; ++k) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) e[k][i] = ry * e[k][i] - r.y[k][i] * my;
        store(static_cast<TI*>(a.dy) + at, team.template cols<KIND, CH>(k, D), e[k]);
      }
    }
    if constexpr (kAhead) r = next;
  }
  float* const part = a.part + blockIdx.x * a.D;
  const int64_t each = gridDim.x * a.D;
  if constexpr (GROUP) {
    __shared__ float sum[kGroupThreads / kWave][kWave * kVec];
    const auto o = team.template cols<KIND, CH>(0, D);
    if (a.dweight) group_part(dw[0], o, L, sum, part);
    if constexpr (POST) {
      if (a.dpost_weight) group_part(dp[0], o, L, sum, part + each);
    }
    if constexpr (SCALE) {
      if (a.dscale) group_part(ds[0], o, L, sum, part + 2 * each);
    }
  } else {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const auto o = team.template cols<KIND, CH>(k, D);
      if constexpr (!kRegs) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if constexpr (POST) dp[0][i] = kept[(k * kVec + i) * THREADS + threadIdx.x];
          if constexpr (SCALE) ds[0][i] = kept2[(k * kVec + i) * THREADS + threadIdx.x];
        }
      }
      if (a.dweight) store(part, o, dw[k]);
      if constexpr (POST) {
        if (a.dpost_weight) store(part + each, o, dp[0]);
      }
      if constexpr (SCALE) {
        if (a.dscale) store(part + 2 * each, o, ds[0]);
      }
    }
  }
}

// out[j] = sum over p of part[p][j], for up to three vectors: COLS columns a workgroup, every
// kSumRows-th part a thread, in 64 bits and always in the same order.  What bounds it is
// latency: eight parts are loaded at a time.  Columns, 16 | 32, us: 745 parts of 3 x 2048
// 7.7 | 5.0, 500 of 1001 3.6 | 4.2, 1024 of 128 4.7 | 5.6.
struct SumArgs {
  const float* part[3];
  float* out[3];
  int64_t parts, width;
};
constexpr int kSumDeep = 8;
template <int kSumCols>
__global__ __launch_bounds__(1024) void sum_parts(SumArgs a) {
  constexpr int kSumRows = 1024 / kSumCols;
  __shared__ double sum[kSumRows][kSumCols + 1];
  const int c = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
  const int64_t j = blockIdx.x * static_cast<int64_t>(kSumCols) + c;
  const float* const part = a.part[blockIdx.y] + min(j, a.width - 1);
  double x = 0.0;
  for (int64_t p = g; p < a.parts; p += kSumRows * kSumDeep) {
    float v[kSumDeep];
#pragma unroll
    for (int k = 0; k < kSumDeep; ++k) v[k] = part[min(p + k * kSumRows, a.parts - 1) * a.width];   // (no branch, so no wait)
#pragma unroll
    for (int k = 0; k < kSumDeep; ++k) x += p + k * kSumRows < a.parts ? v[k] : 0.f;
  }
  sum[g][c] = x;
  __syncthreads();
  if (g < 8) {
    for (int k = 8; k < kSumRows; k += 8) x += sum[g + k][c];
    sum[g][c] = x;   // (rows past the eighth are read above, these below)
  }
  __syncthreads();
  if (g == 0 && j < a.width) {
    for (int k = 1; k < 8; ++k) x += sum[k][c];
    a.out[blockIdx.y][j] = static_cast<float>(x);
  }
}
hipError_t launch_sums(const SumArgs& a, int vectors, hipStream_t s) {
  if (vectors == 0) return hipSuccess;
  const bool wide = vectors * a.width >= 4096;
  const int64_t cols = wide ? 32 : 16;
  const dim3 grid(static_cast<unsigned>((a.width + cols - 1) / cols), vectors), block(1024);
  if (wide) hipLaunchKernelGGL(sum_parts<32>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(sum_parts<16>, grid, block, 0, s, a);
  return hipGetLastError();
}

// lanes for n columns, eight each: a power of two
int lanes_for(int64_t n) {
  int L = 1;
  while (L * kVec < n) L *= 2;
  return L;
}
// (D up to 512: rows are groups of a workgroup's lanes, else of 65536 x 512 the backward takes 110 us, of 524288 x 64 654)
bool grouped(int64_t D) { return D <= kWave * kVec; }
// a row's threads else: whole waves of eight columns a thread, or twice eight past 8192
int row_threads(int64_t D) {
  const int64_t each = D > 1024 * kVec ? 2 * kVec : kVec;
  return static_cast<int>((D + each * kWave - 1) / (each * kWave) * kWave);
}

template <typename TI, typename TS, int CH, bool GROUP, RowKind KIND>
hipError_t rnorm_fwd_ch(const RnormArgs& a, hipStream_t s) {
  const int L = GROUP ? lanes_for(a.D) : 0, rows = GROUP ? kGroupThreads / L : 1;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.rows + rows - 1) / rows, 1 << 20))), block(GROUP ? kGroupThreads : row_threads(a.D));
  if (a.post_norm) hipLaunchKernelGGL((rnorm_fwd<TI, TS, CH, true, GROUP, KIND>), grid, block, 0, s, a, L);
  else hipLaunchKernelGGL((rnorm_fwd<TI, TS, CH, false, GROUP, KIND>), grid, block, 0, s, a, L);
  return hipGetLastError();
}
template <typename TI, typename TS, RowKind KIND>
hipError_t rnorm_fwd_at(const RnormArgs& a, hipStream_t s) {
  if constexpr (KIND != kFewer) {
    if (a.D > 1024 * kVec) return rnorm_fwd_ch<TI, TS, 2, false, KIND>(a, s);
    if (!grouped(a.D)) return rnorm_fwd_ch<TI, TS, 1, false, KIND>(a, s);
  }
  return rnorm_fwd_ch<TI, TS, 1, true, KIND>(a, s);
}
template <typename TI, typename TS>
hipError_t rnorm_fwd_of(const RnormArgs& a, hipStream_t s) {
  const RowKind kind = row_kind(a.D);
  return kind == kEights ? rnorm_fwd_at<TI, TS, kEights>(a, s) : kind == kMore ? rnorm_fwd_at<TI, TS, kMore>(a, s)
                                                                              : rnorm_fwd_at<TI, TS, kFewer>(a, s);
}

template <typename TI, typename TS, int CH, bool GROUP, int THREADS, RowKind KIND>
hipError_t rnorm_bwd_ch(const RnormArgs& a, hipStream_t s) {
  const int L = GROUP ? lanes_for(a.D) : 0;
  const dim3 grid(static_cast<unsigned>(rnorm_parts(a.rows, a.D))), block(GROUP ? kGroupThreads : row_threads(a.D));
  const bool scale = a.scale || a.dscale;
  if (a.post_norm && scale) hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, true, true, GROUP, THREADS, KIND>), grid, block, 0, s, a, L);
  else if (a.post_norm) hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, true, false, GROUP, THREADS, KIND>), grid, block, 0, s, a, L);
  else if (scale) hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, false, true, GROUP, THREADS, KIND>), grid, block, 0, s, a, L);
  else hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, false, false, GROUP, THREADS, KIND>), grid, block, 0, s, a, L);
  return hipGetLastError();
}
template <typename TI, typename TS, RowKind KIND>
hipError_t rnorm_bwd_at(const RnormArgs& a, hipStream_t s) {
  if constexpr (KIND != kFewer) {
    if (a.D > 1024 * kVec) return rnorm_bwd_ch<TI, TS, 2, false, 1024, KIND>(a, s);
    if (a.D > 512 * kVec) return rnorm_bwd_ch<TI, TS, 1, false, 1024, KIND>(a, s);
    if (a.D > 256 * kVec) return rnorm_bwd_ch<TI, TS, 1, false, 512, KIND>(a, s);
    if (!grouped(a.D)) return rnorm_bwd_ch<TI, TS, 1, false, 256, KIND>(a, s);
  }
  return rnorm_bwd_ch<TI, TS, 1, true, 256, KIND>(a, s);
}
template <typename TI, typename TS>
hipError_t rnorm_bwd_of(const RnormArgs& a, hipStream_t s) {
  const RowKind kind = row_kind(a.D);
  return kind == kEights ? rnorm_bwd_at<TI, TS, kEights>(a, s) : kind == kMore ? rnorm_bwd_at<TI, TS, kMore>(a, s)
                                                                              : rnorm_bwd_at<TI, TS, kFewer>(a, s);
}

// act(z) and its derivative, from e = exp(-|z|) (no overflow at either end).  FULL: what the exponential's argument rounds
// off is put back; without, e is off by up to 1.3 |z| 2^-24 of itself, which no bf16 output shows.  The backward is FULL for
// rows of either type, as a weight's gradient is fp32: silu of bf16 z up to 80, 2^-24s, without | with: largest 57 | 3.2, root of mean
// square 15 | 0.62, mean -4.7 | -0.02 (16384 x 16 heads of 128 69.4 | 70.4 us, of 80 channels 73.6 | 79.8).  fp32 rows: the
// reciprocal's too (0.80 | 0.79).
template <typename T, bool FULL, int ACT>
__device__ __forceinline__ void gate(float z, float& act, float& slope) {
  if constexpr (ACT == kActNone) {
    act = 1.f;
    slope = 0.f;
  } else {
    float e, r;
    if constexpr (FULL) {
      e = -fabsf(z) * kLog2e;
      float lo = fmaf(-fabsf(z), 1.925963033e-8f, fmaf(-fabsf(z), kLog2e, -e));   // log2(e) = kLog2e + 1.93e-8
      lo = fminf(fmaxf(lo, -1.f), 1.f);   // (far from 0 e is zero and lo may be anything; a NaN stays in e)
      e = exp2_hw(e);
      e = fmaf(e, lo * kLn2, e);
      r = fast_rcp(1.f + e);
      if constexpr (sizeof(T) == 4) r = fmaf(fmaf(-(1.f + e), r, 1.f), r, r);
    } else {
      e = exp2_hw(-fabsf(z) * kLog2e);
      r = fast_rcp(1.f + e);
    }
    const float s = z >= 0.f ? r : e * r, rest = z >= 0.f ? e * r : r;   // sigmoid(z), 1 - sigmoid(z)
    act = ACT == kActSilu ? z * s : s;
    slope = ACT == kActSilu ? s + act * rest : s * rest;
  }
}

// A group of L lanes (a power of two, eight channels a lane) takes a head's row.  Neighbouring groups take
// neighbouring heads, so that a workgroup reads whole tokens (one head a workgroup: 16 heads of 8, 33, 64 and 128
// channels, gated backward of 2^25 elements, 304, 171, 82, 74 us; so 76, 113, 73, 71); with a weight for each head a workgroup
// stays with one, whose gradient it can sum.
constexpr int kThreads = 256;
struct Walk {   // a group's step: so many tokens and heads on
  int64_t tokens;
  int32_t heads;
};
Walk walk_of(const HnormArgs& a, int64_t blocks) {
  if (a.head_weight) return Walk{blocks / a.H * (kThreads / lanes_for(a.d)), 0};
  const int64_t rows = blocks * (kThreads / lanes_for(a.d));
  return Walk{rows / a.H, static_cast<int32_t>(rows % a.H)};
}
struct HeadRow {
  int64_t t;
  int32_t head;
  __device__ __forceinline__ HeadRow(const HnormArgs& a, int L) {
    const uint32_t group = threadIdx.x / L, groups = kThreads / L, H = static_cast<uint32_t>(a.H);
    if (a.head_weight) {
      t = static_cast<int64_t>(blockIdx.x / H) * groups + group;
      head = blockIdx.x % H;
    } else {   // (fewer than 2^32 work items, so fewer rows at first)
      const uint32_t row = blockIdx.x * groups + group;
      t = row / H;
      head = row % H;
    }
  }
  __device__ __forceinline__ void next(const HnormArgs& a, const Walk& by) {
    t += by.tokens;
    head += by.heads;
    if (head >= a.H) {
      head -= static_cast<int32_t>(a.H);
      ++t;
    }
  }
};

template <typename T, int ACT, RowKind KIND>
__global__ __launch_bounds__(kThreads) void hnorm_fwd(HnormArgs a, int L, Walk by) {
  const Cols<KIND> o((threadIdx.x & (L - 1)) * kVec, a.d);
  HeadRow at(a, L);
  float w[kVec];
  ld_weight(a.weight ? a.weight + (a.head_weight ? at.head * a.d : 0) : nullptr, o, w);
  for (; at.t < a.M; at.next(a, by)) {
    Raw<T> x, z;
    const int64_t h = static_cast<int64_t>(at.head) * a.d;
    x.load(static_cast<const T*>(a.x) + at.t * a.sx + h, o);
    if constexpr (ACT != kActNone) z.load(static_cast<const T*>(a.z) + at.t * a.sz + h, o);
    x.settle(o);
    float v[kVec], q = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) q += x[i] * x[i];
    const float r = factor(lanes_sum(q, L), a.l2 ? 1.f : 1.f / a.d, a.eps);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float act, slope;
      gate<T, sizeof(T) == 4, ACT>(ACT == kActNone ? 0.f : z[i], act, slope);
      v[i] = x[i] * r * w[i];
      if constexpr (ACT != kActNone) v[i] *= act;
    }
    store(static_cast<T*>(a.y) + at.t * a.sy + h, o, v);
  }
}

template <typename T, int ACT, RowKind KIND>
__global__ __launch_bounds__(kThreads) void hnorm_bwd(HnormArgs a, int L, Walk by) {
  __shared__ float sum[kThreads / kWave][kWave * kVec];
  const Cols<KIND> o((threadIdx.x & (L - 1)) * kVec, a.d);
  const float c = a.l2 ? 1.f : 1.f / a.d;
  HeadRow at(a, L);
  float w[kVec], dw[kVec] = {};
  ld_weight(a.weight ? a.weight + (a.head_weight ? at.head * a.d : 0) : nullptr, o, w);
  if (a.weight) settle(o, w);
  Raw<T> next[3];   // the next row's
  auto load = [&](const HeadRow& r) {
    const int64_t t = min(r.t, a.M - 1), h = static_cast<int64_t>(r.head) * a.d;   // (behind the last: not used)
    next[0].load(static_cast<const T*>(a.x) + t * a.sx + h, o);
    next[1].load(static_cast<const T*>(a.dy) + t * a.sdy + h, o);
    if constexpr (ACT != kActNone) next[2].load(static_cast<const T*>(a.z) + t * a.sz + h, o);
  };
  load(at);
  while (at.t < a.M) {
    const int64_t t = at.t, h = static_cast<int64_t>(at.head) * a.d;
    Raw<T> x = next[0], dy = next[1], z = next[2];
    at.next(a, by);
    load(at);
    x.settle(o);
    dy.settle(o);
    if constexpr (ACT != kActNone) z.settle(o);
    float g[kVec], v[kVec], slope[kVec], q = 0.f, p = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float act;
      q += x[i] * x[i];
      gate<T, true, ACT>(ACT == kActNone ? 0.f : z[i], act, slope[i]);
      slope[i] *= dy[i] * w[i];
      g[i] = ACT == kActNone ? dy[i] : dy[i] * act;
      p += g[i] * w[i] * x[i];
    }
    const float r = factor_back(lanes_sum(q, L), c, a.eps), m = (r * lanes_sum(p, L) * c) * r * r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      slope[i] *= x[i] * r;
      dw[i] += g[i] * (x[i] * r);
      v[i] = r * (g[i] * w[i]) - x[i] * m;
    }
    store(static_cast<T*>(a.dx) + t * a.sdx + h, o, v);
    if constexpr (ACT != kActNone) store(static_cast<T*>(a.dz) + t * a.sdz + h, o, slope);
  }
  if (a.dweight) group_part(dw, o, L, sum, a.part + blockIdx.x * static_cast<int64_t>(a.d));
}

// workgroups: at most so many, with a weight for each head as many for each
int64_t hnorm_blocks(const HnormArgs& a, int64_t most) {
  const int groups = kThreads / lanes_for(a.d);
  if (a.head_weight) return a.H * std::max<int64_t>(std::min<int64_t>((a.M + groups - 1) / groups, most / a.H), 1);
  return std::min<int64_t>((a.M * a.H + groups - 1) / groups, most);
}
template <typename T, RowKind KIND>
hipError_t hnorm_fwd_at(const HnormArgs& a, hipStream_t s) {
  const int L = lanes_for(a.d);
  const int64_t blocks = hnorm_blocks(a, 1 << 20);
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  const Walk by = walk_of(a, blocks);
  if (a.act == kActSilu) hipLaunchKernelGGL((hnorm_fwd<T, kActSilu, KIND>), grid, block, 0, s, a, L, by);
  else if (a.act == kActSigmoid) hipLaunchKernelGGL((hnorm_fwd<T, kActSigmoid, KIND>), grid, block, 0, s, a, L, by);
  else hipLaunchKernelGGL((hnorm_fwd<T, kActNone, KIND>), grid, block, 0, s, a, L, by);
  return hipGetLastError();
}
template <typename T, RowKind KIND>
hipError_t hnorm_bwd_at(const HnormArgs& a, hipStream_t s) {
  const int L = lanes_for(a.d);
  const int64_t blocks = hnorm_parts(a);
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  const Walk by = walk_of(a, blocks);
  if (a.act == kActSilu) hipLaunchKernelGGL((hnorm_bwd<T, kActSilu, KIND>), grid, block, 0, s, a, L, by);
  else if (a.act == kActSigmoid) hipLaunchKernelGGL((hnorm_bwd<T, kActSigmoid, KIND>), grid, block, 0, s, a, L, by);
  else hipLaunchKernelGGL((hnorm_bwd<T, kActNone, KIND>), grid, block, 0, s, a, L, by);
  return hipGetLastError();
}

template <typename T>
hipError_t hnorm_fwd_of(const HnormArgs& a, hipStream_t s) {
  const RowKind kind = row_kind(a.d);
  return kind == kEights ? hnorm_fwd_at<T, kEights>(a, s) : kind == kMore ? hnorm_fwd_at<T, kMore>(a, s) : hnorm_fwd_at<T, kFewer>(a, s);
}
template <typename T>
hipError_t hnorm_bwd_of(const HnormArgs& a, hipStream_t s) {
  const RowKind kind = row_kind(a.d);
  return kind == kEights ? hnorm_bwd_at<T, kEights>(a, s) : kind == kMore ? hnorm_bwd_at<T, kMore>(a, s) : hnorm_bwd_at<T, kFewer>(a, s);
}

// at most so many parts, of as nearly the same number of rows as can be
int64_t balanced_parts(int64_t rows, int64_t most) {
  const int64_t each = std::max<int64_t>((rows + most - 1) / most, rows > 512 ? 2 : 1);   // (1048 rows of 1000, everything on: 18.6 us with one each, 14.7)
  return (rows + each - 1) / each;
}

}  // namespace

int64_t rnorm_parts(int64_t rows, int64_t D) {
  const int64_t at_once = grouped(D) ? kGroupThreads / lanes_for(D) : 1;
  // the workgroups that 256 compute units hold by their registers: 12 waves each up to 256 threads, else 16.  Aligned rows
  // in which hardly a lane is without columns wait for memory alone, and ten waves ask for enough.  Twelve | ten, us, everything
  // on: bf16 16384 x 2048 88 | 81, fp32 161 | 153, bf16 33554 x 1000 90 | 88; else 55924 x 600 96 | 104, 111848 x 300 114 | 142, bf16 on an
  // fp32 stream 32784 x 2047 255 | 274; without norm and scale 20971 x 1600 66 | 76.
  const int threads = grouped(D) ? kGroupThreads : row_threads(D);
  const bool full = D % kVec == 0 && D > (kVec - 1) * (grouped(D) ? lanes_for(D) : threads);
  const int waves = threads > 256 ? 16 : full ? 10 : 4 * kBackWaves;
  return balanced_parts((rows + at_once - 1) / at_once, 256 * (waves / (threads / kWave)));
}

hipError_t launch_rnorm_fwd(const RnormArgs& a, int io_bf16, int stream_bf16, hipStream_t s) {
  if (io_bf16) return stream_bf16 ? rnorm_fwd_of<bf16, bf16>(a, s) : rnorm_fwd_of<bf16, float>(a, s);
  return stream_bf16 ? rnorm_fwd_of<float, bf16>(a, s) : rnorm_fwd_of<float, float>(a, s);
}
hipError_t launch_rnorm_bwd(const RnormArgs& a, int io_bf16, int stream_bf16, hipStream_t s) {
  if (a.rows > 0) {
    hipError_t e;
    if (io_bf16) e = stream_bf16 ? rnorm_bwd_of<bf16, bf16>(a, s) : rnorm_bwd_of<bf16, float>(a, s);
    else e = stream_bf16 ? rnorm_bwd_of<float, bf16>(a, s) : rnorm_bwd_of<float, float>(a, s);
    if (e != hipSuccess) return e;
  }
  SumArgs sums{};
  sums.parts = rnorm_parts(a.rows, a.D);
  sums.width = a.D;
  float* const outs[3] = {a.dweight, a.dpost_weight, a.dscale};
  int n = 0;
  for (int k = 0; k < 3; ++k)
    if (outs[k]) {
      sums.part[n] = a.part + k * sums.parts * a.D;
      sums.out[n++] = outs[k];
    }
  return launch_sums(sums, n, s);
}

int64_t hnorm_parts(const HnormArgs& a) { return a.M == 0 || a.H == 0 ? 0 : hnorm_blocks(a, 1024); }

hipError_t launch_hnorm_fwd(const HnormArgs& a, int io_bf16, hipStream_t s) {
  return io_bf16 ? hnorm_fwd_of<bf16>(a, s) : hnorm_fwd_of<float>(a, s);
}
hipError_t launch_hnorm_bwd(const HnormArgs& a, int io_bf16, hipStream_t s) {
  const int64_t parts = hnorm_parts(a);
  if (parts > 0) {
    const hipError_t e = io_bf16 ? hnorm_bwd_of<bf16>(a, s) : hnorm_bwd_of<float>(a, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dweight) return hipSuccess;
  SumArgs sums{};
  sums.part[0] = a.part;
  sums.out[0] = a.dweight;
  sums.parts = a.head_weight ? parts / a.H : parts;
  sums.width = a.head_weight ? a.H * a.d : a.d;
  return launch_sums(sums, 1, s);
}

}  // namespace pdn
