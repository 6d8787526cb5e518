// Norms around the rule in a block.  Rows are independent; what bounds every call is
// the reading and writing of its tensors, so each kernel holds a row in registers, reads every
// tensor once and writes every output once.
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

namespace pdn {

namespace {

constexpr int kVec = 8;

// Eight elements from column c of a row of n (aligned to an element only; past the
// row: zero), or back.
template <typename T>
__device__ __forceinline__ void ld_row(const T* p, int c, int n, float (&v)[kVec]) {
  T raw[kVec];
  if (c + kVec <= n) {
    __builtin_memcpy(raw, p + c, sizeof raw);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) raw[i] = c + i < n ? p[c + i] : from_f<T>(0.f);
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = to_f(raw[i]);
}
template <typename T>
__device__ __forceinline__ void st_row(T* p, int c, int n, const float (&v)[kVec]) {
  T raw[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) raw[i] = from_f<T>(v[i]);
  if (c + kVec <= n) {
    __builtin_memcpy(p + c, raw, sizeof raw);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (c + i < n) p[c + i] = raw[i];
  }
}
// of a vector that may be NULL (= 1)
__device__ __forceinline__ void ld_weight(const float* p, int c, int n, float (&v)[kVec]) {
  if (p) {
    ld_row(p, c, n, v);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = 1.f;
  }
}

__device__ __forceinline__ float factor(float squares, float c, float eps) { return 1.f / sqrtf(squares * c + eps); }

// Sums over the workgroup's threads, the same on each of them.  Two buffers in turn: one barrier a sum.
template <int N>
__device__ __forceinline__ void block_sum(float (&x)[N], float (*buf)[16][4], int& turn) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x[k] += __shfl_xor(x[k], off, 64);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return;
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

template <typename TI, typename TS, int CH, bool POST>
__global__ void rnorm_fwd(RnormArgs a) {
  __shared__ float buf[2][16][4];
  int turn = 0;
  const int D = static_cast<int>(a.D);
  const float c = 1.f / a.D;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float h[CH][kVec], q[1];
    const TI* const y = static_cast<const TI*>(a.y) + row * D;
    float ry = 1.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) ld_row(y, (k * blockDim.x + threadIdx.x) * kVec, D, h[k]);
    if constexpr (POST) {
      q[0] = 0.f;
#pragma unroll
      for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < kVec; ++i) q[0] += h[k][i] * h[k][i];
      block_sum(q, buf, turn);
      ry = factor(q[0], c, a.eps);
    }
    q[0] = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * kVec;
      float v[kVec];
      if constexpr (POST) {
        ld_weight(a.post_weight, col, D, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] *= ry * v[i];
      }
      if (a.scale) {
        ld_row(a.scale, col, D, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] *= v[i];
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) h[k][i] *= a.alpha;
      if (a.residual) {
        ld_row(static_cast<const TS*>(a.residual) + row * D, col, D, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[k][i] += v[i];
      }
      if (a.h) st_row(static_cast<TS*>(a.h) + row * D, col, D, h[k]);
#pragma unroll
      for (int i = 0; i < kVec; ++i) q[0] += h[k][i] * h[k][i];
    }
    block_sum(q, buf, turn);
    const float rh = factor(q[0], c, a.eps);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * kVec;
      float v[kVec];
      ld_weight(a.weight, col, D, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] *= h[k][i] * rh;
      st_row(static_cast<TI*>(a.u) + row * D, col, D, v);
    }
  }
}

// A workgroup takes every gridDim-th row and keeps the vectors' gradients of its columns in
// registers; rnorm_parts of them are summed by sum_parts.
template <typename TI, typename TS, int CH, bool POST, bool SCALE>
__global__ void rnorm_bwd(RnormArgs a) {
  __shared__ float buf[2][16][4];
  int turn = 0;
  const int D = static_cast<int>(a.D);
  const float c = 1.f / a.D;
  float dw[CH][kVec] = {}, dp[POST ? CH : 1][kVec] = {}, ds[SCALE ? CH : 1][kVec] = {};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float du[CH][kVec], h[CH][kVec], y[POST || SCALE ? CH : 1][kVec], q[POST ? 3 : 2] = {};
    const int64_t at = row * D;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * kVec;
      float w[kVec];
      ld_row(static_cast<const TI*>(a.du) + at, col, D, du[k]);
      ld_row(static_cast<const TS*>(a.h_in) + at, col, D, h[k]);
      if constexpr (POST || SCALE) {
        if (a.y) ld_row(static_cast<const TI*>(a.y) + at, col, D, y[k]);
      }
      ld_weight(a.weight, col, D, w);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        q[0] += h[k][i] * h[k][i];
        q[1] += du[k][i] * w[i] * h[k][i];
        if constexpr (POST) q[2] += y[k][i] * y[k][i];
      }
    }
    block_sum(q, buf, turn);
    const float rh = factor(q[0], c, a.eps), mh = (rh * q[1] * c) * rh * rh;
    const float ry = POST ? factor(q[POST ? 2 : 0], c, a.eps) : 1.f;
    float p[1] = {0.f};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int col = (k * blockDim.x + threadIdx.x) * kVec;
      float t[kVec], v[kVec];
      ld_weight(a.weight, col, D, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        t[i] = rh * (du[k][i] * v[i]) - h[k][i] * mh;
        dw[k][i] += du[k][i] * (h[k][i] * rh);
      }
      if (a.dh) {
        ld_row(static_cast<const TS*>(a.dh) + at, col, D, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) t[i] += v[i];
      }
      if (a.dresidual) st_row(static_cast<TS*>(a.dresidual) + at, col, D, t);
#pragma unroll
      for (int i = 0; i < kVec; ++i) t[i] *= a.alpha;
      float wp[kVec];
      if constexpr (POST) ld_weight(a.post_weight, col, D, wp);
      if constexpr (SCALE) {
        ld_weight(a.scale, col, D, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if (a.y) ds[k][i] += t[i] * (POST ? y[k][i] * ry * wp[i] : y[k][i]);
          t[i] *= v[i];
        }
      }
      if constexpr (POST) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          dp[k][i] += t[i] * (y[k][i] * ry);
          t[i] *= wp[i];
          p[0] += t[i] * y[k][i];
          du[k][i] = t[i];
        }
      } else {
        st_row(static_cast<TI*>(a.dy) + at, col, D, t);
      }
    }
    if constexpr (POST) {
      block_sum(p, buf, turn);
      const float my = (ry * p[0] * c) * ry * ry;
#pragma unroll
      for (int k = 0; k < CH; ++k) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) du[k][i] = ry * du[k][i] - y[k][i] * my;
        st_row(static_cast<TI*>(a.dy) + at, (k * blockDim.x + threadIdx.x) * kVec, D, du[k]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int col = (k * blockDim.x + threadIdx.x) * kVec;
    float* const part = a.part + blockIdx.x * a.D;
    const int64_t each = gridDim.x * a.D;
    if (a.dweight) st_row(part, col, D, dw[k]);
    if constexpr (POST) {
      if (a.dpost_weight) st_row(part + each, col, D, dp[k]);
    }
    if constexpr (SCALE) {
      if (a.dscale) st_row(part + 2 * each, col, D, ds[k]);
    }
  }
}

// out[j] = sum over p of part[p][j], for up to three vectors: 64 columns a workgroup, a
// sixteenth of the parts a wave, in 64 bits and always in the same order.
struct SumArgs {
  const float* part[3];
  float* out[3];
  int64_t parts, width;
};
__global__ __launch_bounds__(1024) void sum_parts(SumArgs a) {
  __shared__ double sum[16][kWave];
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int64_t j = blockIdx.x * static_cast<int64_t>(kWave) + l;
  const float* const part = a.part[blockIdx.y];
  double x = 0.0;
  if (j < a.width)
    for (int64_t p = w; p < a.parts; p += 16) x += part[p * a.width + j];
  sum[w][l] = x;
  __syncthreads();
  if (w == 0 && j < a.width) {
    for (int k = 1; k < 16; ++k) x += sum[k][l];
    a.out[blockIdx.y][j] = static_cast<float>(x);
  }
}
hipError_t launch_sums(const SumArgs& a, int vectors, hipStream_t s) {
  if (vectors == 0) return hipSuccess;
  const unsigned blocks = static_cast<unsigned>((a.width + kWave - 1) / kWave);
  hipLaunchKernelGGL(sum_parts, dim3(blocks, vectors), dim3(1024), 0, s, a);
  return hipGetLastError();
}

// threads a row: eight columns each, CH times
int row_threads(int64_t D) {
  int t = kWave;
  while (t < 1024 && t * kVec < D) t *= 2;
  return t;
}

template <typename TI, typename TS, int CH>
hipError_t rnorm_fwd_ch(const RnormArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.rows, 1 << 20))), block(row_threads(a.D));
  if (a.post_norm) hipLaunchKernelGGL((rnorm_fwd<TI, TS, CH, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rnorm_fwd<TI, TS, CH, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <typename TI, typename TS>
hipError_t rnorm_fwd_of(const RnormArgs& a, hipStream_t s) {
  return a.D > 1024 * kVec ? rnorm_fwd_ch<TI, TS, 2>(a, s) : rnorm_fwd_ch<TI, TS, 1>(a, s);
}

template <typename TI, typename TS, int CH>
hipError_t rnorm_bwd_ch(const RnormArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(rnorm_parts(a.rows, a.D))), block(row_threads(a.D));
  const bool scale = a.scale || a.dscale;
  if (a.post_norm && scale) hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, true, true>), grid, block, 0, s, a);
  else if (a.post_norm) hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, true, false>), grid, block, 0, s, a);
  else if (scale) hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, false, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rnorm_bwd<TI, TS, CH, false, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <typename TI, typename TS>
hipError_t rnorm_bwd_of(const RnormArgs& a, hipStream_t s) {
  return a.D > 1024 * kVec ? rnorm_bwd_ch<TI, TS, 2>(a, s) : rnorm_bwd_ch<TI, TS, 1>(a, s);
}

// act(z) and its derivative, from e = exp(-|z|) (no overflow at either end)
template <typename T, int ACT>
__device__ __forceinline__ void gate(float z, float& act, float& slope) {
  if constexpr (ACT == kActNone) {
    act = 1.f;
    slope = 0.f;
  } else {
    const float x = fabsf(z) > 200.f ? -200.f : -fabsf(z);
    float e = x * kLog2e;
    if constexpr (sizeof(T) == 4) {   // (the product's rounding put back: fp32 outputs show it)
      const float lo = fmaf(x, kLog2e, -e) + x * 1.925963033e-8f;   // log2(e) = kLog2e + 1.93e-8
      e = exp2_hw(e);
      e = fmaf(e, lo * kLn2, e);
    } else {
      e = exp2_hw(e);
    }
    float r = fast_rcp(1.f + e);
    r = fmaf(fmaf(-(1.f + e), r, 1.f), r, r);
    const float s = z >= 0.f ? r : e * r, rest = z >= 0.f ? e * r : r;   // sigmoid(z), 1 - sigmoid(z)
    act = ACT == kActSilu ? z * s : s;
    slope = ACT == kActSilu ? s + act * rest : s * rest;
  }
}

// A group of L lanes (a power of two, eight channels a lane) takes a head's row, a workgroup
// one head of kThreads / L tokens at a time.
constexpr int kThreads = 256;
int head_lanes(int d) {
  int L = 1;
  while (L * kVec < d) L *= 2;
  return L;
}
__device__ __forceinline__ float lanes_sum(float x, int L) {
  for (int off = L >> 1; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void hnorm_fwd(HnormArgs a, int L) {
  const int col = (threadIdx.x & (L - 1)) * kVec, group = threadIdx.x / L, groups = kThreads / L;
  const int64_t head = blockIdx.x % a.H, first = blockIdx.x / a.H, each = gridDim.x / a.H;
  float w[kVec];
  ld_weight(a.weight ? a.weight + (a.head_weight ? head * a.d : 0) : nullptr, col, a.d, w);
  for (int64_t t = first * groups + group; t < a.M; t += each * groups) {
    float x[kVec], z[kVec], q = 0.f;
    ld_row(static_cast<const T*>(a.x) + t * a.sx + head * a.d, col, a.d, x);
    if constexpr (ACT != kActNone) ld_row(static_cast<const T*>(a.z) + t * a.sz + head * a.d, col, a.d, z);
#pragma unroll
    for (int i = 0; i < kVec; ++i) q += x[i] * x[i];
    const float r = factor(lanes_sum(q, L), a.l2 ? 1.f : 1.f / a.d, a.eps);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float act, slope;
      gate<T, ACT>(ACT == kActNone ? 0.f : z[i], act, slope);
      x[i] = x[i] * r * w[i];
      if constexpr (ACT != kActNone) x[i] *= act;
    }
    st_row(static_cast<T*>(a.y) + t * a.sy + head * a.d, col, a.d, x);
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void hnorm_bwd(HnormArgs a, int L) {
  __shared__ float sum[kThreads / kWave][kWave * kVec];
  const int col = (threadIdx.x & (L - 1)) * kVec, group = threadIdx.x / L, groups = kThreads / L;
  const int64_t head = blockIdx.x % a.H, first = blockIdx.x / a.H, each = gridDim.x / a.H;
  const float c = a.l2 ? 1.f : 1.f / a.d;
  float w[kVec], dw[kVec] = {};
  ld_weight(a.weight ? a.weight + (a.head_weight ? head * a.d : 0) : nullptr, col, a.d, w);
  for (int64_t t = first * groups + group; t < a.M; t += each * groups) {
    float x[kVec], z[kVec], dy[kVec], slope[kVec], q = 0.f, p = 0.f;
    ld_row(static_cast<const T*>(a.x) + t * a.sx + head * a.d, col, a.d, x);
    ld_row(static_cast<const T*>(a.dy) + t * a.sdy + head * a.d, col, a.d, dy);
    if constexpr (ACT != kActNone) ld_row(static_cast<const T*>(a.z) + t * a.sz + head * a.d, col, a.d, z);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      q += x[i] * x[i];
      float act;
      gate<T, ACT>(ACT == kActNone ? 0.f : z[i], act, slope[i]);
      slope[i] *= dy[i] * w[i];
      if constexpr (ACT != kActNone) dy[i] *= act;
      p += dy[i] * w[i] * x[i];
    }
    const float r = factor(lanes_sum(q, L), c, a.eps), m = (r * lanes_sum(p, L) * c) * r * r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      slope[i] *= x[i] * r;
      dw[i] += dy[i] * (x[i] * r);
      x[i] = r * (dy[i] * w[i]) - x[i] * m;
    }
    st_row(static_cast<T*>(a.dx) + t * a.sdx + head * a.d, col, a.d, x);
    if constexpr (ACT != kActNone) st_row(static_cast<T*>(a.dz) + t * a.sdz + head * a.d, col, a.d, slope);
  }
  if (!a.dweight) return;
  // the groups' sums: over a wave's by shuffles, then over the waves
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    for (int off = L; off < kWave; off <<= 1) dw[i] += __shfl_xor(dw[i], off, 64);
  const int wave = threadIdx.x / kWave, l = threadIdx.x & 63;
  if (l < L)
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum[wave][l * kVec + i] = dw[i];
  __syncthreads();
  for (int j = threadIdx.x; j < a.d; j += kThreads)
    a.part[blockIdx.x * static_cast<int64_t>(a.d) + j] = (sum[0][j] + sum[1][j]) + (sum[2][j] + sum[3][j]);
}

template <typename T>
hipError_t hnorm_fwd_of(const HnormArgs& a, hipStream_t s) {
  const int L = head_lanes(a.d), groups = kThreads / L;
  const int64_t each = std::max<int64_t>(std::min<int64_t>((a.M + groups - 1) / groups, (1 << 20) / a.H), 1);
  const dim3 grid(static_cast<unsigned>(each * a.H)), block(kThreads);
  if (a.act == kActSilu) hipLaunchKernelGGL((hnorm_fwd<T, kActSilu>), grid, block, 0, s, a, L);
  else if (a.act == kActSigmoid) hipLaunchKernelGGL((hnorm_fwd<T, kActSigmoid>), grid, block, 0, s, a, L);
  else hipLaunchKernelGGL((hnorm_fwd<T, kActNone>), grid, block, 0, s, a, L);
  return hipGetLastError();
}
template <typename T>
hipError_t hnorm_bwd_of(const HnormArgs& a, hipStream_t s) {
  const int L = head_lanes(a.d);
  const dim3 grid(static_cast<unsigned>(hnorm_parts(a.M, a.H, a.d))), block(kThreads);
  if (a.act == kActSilu) hipLaunchKernelGGL((hnorm_bwd<T, kActSilu>), grid, block, 0, s, a, L);
  else if (a.act == kActSigmoid) hipLaunchKernelGGL((hnorm_bwd<T, kActSigmoid>), grid, block, 0, s, a, L);
  else hipLaunchKernelGGL((hnorm_bwd<T, kActNone>), grid, block, 0, s, a, L);
  return hipGetLastError();
}

}  // namespace

int64_t rnorm_parts(int64_t rows, int64_t) { return std::min<int64_t>(rows, 1024); }

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

// a head's tokens in at most so many parts that all heads' are 2048 (H where there are more heads)
int64_t hnorm_parts(int64_t M, int64_t H, int d) {
  if (M == 0 || H == 0) return 0;
  const int groups = kThreads / head_lanes(d);
  return H * std::max<int64_t>(std::min<int64_t>((M + groups - 1) / groups, 2048 / H), 1);
}

hipError_t launch_hnorm_fwd(const HnormArgs& a, int io_bf16, hipStream_t s) {
  return io_bf16 ? hnorm_fwd_of<bf16>(a, s) : hnorm_fwd_of<float>(a, s);
}
hipError_t launch_hnorm_bwd(const HnormArgs& a, int io_bf16, hipStream_t s) {
  const int64_t parts = hnorm_parts(a.M, a.H, a.d);
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
