// Layer norm: forward pass, and backward pass with the reduction of the parameters' gradients.
#pragma once
#include "op_common.h"

namespace accop {

// Sum over the THREADS lanes that share a row (16 lanes, one wave, or a whole workgroup: then every thread calls this),
// the same value in all of them.
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* red) {
  if (THREADS == 16) return row16_sum(v);
  v = wave_sum(v);
  if (THREADS == kWave) return v;
  constexpr int waves = THREADS / kWave;
  __syncthreads();                       // red may still be read from the sum before
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = red[0];
#pragma unroll
  for (int i = 1; i < waves; ++i) s += red[i];
  return s;
}
template <int THREADS>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* red) {
  if (THREADS == 16) {
    a = row16_sum(a);
    b = row16_sum(b);
    return;
  }
  a = wave_sum(a);
  b = wave_sum(b);
  if (THREADS == kWave) return;
  constexpr int waves = THREADS / kWave;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    red[2 * (threadIdx.x >> 6)] = a;
    red[2 * (threadIdx.x >> 6) + 1] = b;
  }
  __syncthreads();
  a = red[0];
  b = red[1];
#pragma unroll
  for (int i = 1; i < waves; ++i) {
    a += red[2 * i];
    b += red[2 * i + 1];
  }
}

template <int N>
__device__ __forceinline__ float sum_of(const F32<N>& v) {
  float s = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) s += v[i];
  return s;
}

// ---- forward ----------------------------------------------------------------------------------------------
// THREADS lanes hold a row in registers (K requests of N elements each): one read, one write, bound by memory; the deviations are
// summed from the registers, after the mean.  65536 x 2048 bf16 103 us (5.2 TB/s), 4096 x 8192 bf16 24, 131072 x 64 fp32 13 (a wave per
// row 33), 700 x 672 fp32 4.4; plain stores 107, 35.  Rows of odd length end in accesses of single elements, which the whole wave goes
// through: 20000 x 1021 bf16 18.5 and x 1024 15.3, fp32 29.6 and 26.9.
template <typename T, int N, int THREADS, int K, int BLOCK>
__global__ __launch_bounds__(BLOCK) void layernorm_forward_kernel(const T* __restrict__ x, const float* __restrict__ weight,
                                                                const float* __restrict__ bias, T* __restrict__ y,
                                                                float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                                int64_t rows, int dim, int64_t x_stride, int64_t y_stride, float eps) {
  __shared__ float red[2 * BLOCK / kWave];
  const int64_t row = (int64_t)blockIdx.x * (BLOCK / THREADS) + threadIdx.x / THREADS;
  if (row >= rows) return;               // THREADS == BLOCK: the whole workgroup
  const int c = (threadIdx.x % THREADS) * N;
  const T* from = x + row * x_stride;
  F32<N> v[K];
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int at = c + k * THREADS * N;
    v[k] = widen<T, N>(load_some<N>(from + at, dim - at));
    s += sum_of<N>(v[k]);
  }
  const float mean = row_sum<THREADS>(s, red) / (float)dim;
  float q = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int at = c + k * THREADS * N;
    v[k] -= mean;
#pragma unroll
    for (int i = 0; i < N; ++i) q += at + i < dim ? v[k][i] * v[k][i] : 0.f;
  }
  const float rstd = 1.0f / sqrtf(row_sum<THREADS>(q, red) / (float)dim + eps);
  if (mean_out && c == 0) {
    mean_out[row] = mean;
    rstd_out[row] = rstd;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int at = c + k * THREADS * N;
    if (at >= dim) continue;
    F32<N> r = v[k] * rstd * widen<float, N>(load_some<N>(weight + at, dim - at));
    if (bias) r += widen<float, N>(load_some<N>(bias + at, dim - at));
    store_some_stream<T, N>(y + row * y_stride + at, r, dim - at);
  }
}

// Rows too long for the registers of a workgroup (beyond 16384 fp32 or 32768 bf16 columns): read three times (the second and third time
// from a cache, as far as it holds them).  2000 x 20000 fp32 97 us for 58 at the rate of a copy, 4000 x 40000 bf16 237 for 115.
template <typename T, int N>
__global__ __launch_bounds__(256) void layernorm_forward_long_kernel(const T* __restrict__ x, const float* __restrict__ weight,
                                                                     const float* __restrict__ bias, T* __restrict__ y,
                                                                     float* __restrict__ mean_out, float* __restrict__ rstd_out,
                                                                     int dim, int64_t x_stride, int64_t y_stride, float eps) {
  __shared__ float red[8];
  const int64_t row = blockIdx.x;
  const T* from = x + row * x_stride;
  float s = 0.f;
  for (int at = threadIdx.x * N; at < dim; at += 256 * N) s += sum_of<N>(widen<T, N>(load_some<N>(from + at, dim - at)));
  const float mean = row_sum<256>(s, red) / (float)dim;
  float q = 0.f;
  for (int at = threadIdx.x * N; at < dim; at += 256 * N) {
    const F32<N> v = widen<T, N>(load_some<N>(from + at, dim - at)) - mean;
#pragma unroll
    for (int i = 0; i < N; ++i) q += at + i < dim ? v[i] * v[i] : 0.f;
  }
  const float rstd = 1.0f / sqrtf(row_sum<256>(q, red) / (float)dim + eps);
  if (mean_out && threadIdx.x == 0) {
    mean_out[row] = mean;
    rstd_out[row] = rstd;
  }
  for (int at = threadIdx.x * N; at < dim; at += 256 * N) {
    F32<N> r = (widen<T, N>(load_some<N>(from + at, dim - at)) - mean) * rstd * widen<float, N>(load_some<N>(weight + at, dim - at));
    if (bias) r += widen<float, N>(load_some<N>(bias + at, dim - at));
    store_some<T, N>(y + row * y_stride + at, r, dim - at);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------
// A group of THREADS lanes takes every gridDim.x * groups-th row, holds it in registers (one read of x and grad_y)
// and keeps its columns' sums of grad_y xh and grad_y over its rows in registers as well.  A workgroup adds its
// groups' sums and leaves them in parts (two rows of dim per workgroup); layernorm_join_kernel adds the workgroups'.
// Bound by memory: 65536 x 2048 bf16 148 us (5.4 TB/s); by the rows' latency where a wave has few: 5003 x 1001 fp32 14.2 (4.2);
// by instructions where rows are narrow (100000 x 56 bf16 22 us for 6 at the rate of a copy) and, as forward, by the ends of odd rows (x 53 28 us;
// 20000 x 1021 bf16 33, x 1024 27.5).  fp32 rows of 8193 to 16384 columns spill 4 registers of a lane: 2000 x 16384 78 us for 71.
template <typename T, int N, int THREADS, int K, int BLOCK>
__global__ __launch_bounds__(BLOCK) void layernorm_backward_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                                   const float* __restrict__ weight, const float* __restrict__ mean_in,
                                                                   const float* __restrict__ rstd_in, T* __restrict__ dx, int64_t rows,
                                                                   int dim, int64_t dy_stride, int64_t x_stride, int64_t dx_stride,
                                                                   float* __restrict__ parts) {
  constexpr int groups = BLOCK / THREADS;
  __shared__ float red[2 * BLOCK / kWave];
  __shared__ F32<N> fold[groups > 1 ? (groups - 1) * THREADS : 1];
  const int c = (threadIdx.x % THREADS) * N, group = threadIdx.x / THREADS;
  F32<N> dw[K], db[K], w[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int at = c + k * THREADS * N;
    dw[k] = db[k] = F32<N>{};
    w[k] = widen<float, N>(load_some<N>(weight + at, dim - at));
  }
  for (int64_t row = (int64_t)blockIdx.x * groups + group; row < rows; row += (int64_t)gridDim.x * groups) {
    const float mean = mean_in[row], rstd = rstd_in[row];
    F32<N> g[K], xh[K];
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int at = c + k * THREADS * N;
      g[k] = widen<T, N>(load_some<N>(dy + row * dy_stride + at, dim - at));
      xh[k] = widen<T, N>(load_some<N>(x + row * x_stride + at, dim - at));
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xh[k] = (xh[k] - mean) * rstd;     // beyond the row g is zero
      dw[k] += g[k] * xh[k];
      db[k] += g[k];
      g[k] *= w[k];
      sg += sum_of<N>(g[k]);
      sgx += sum_of<N>(g[k] * xh[k]);
    }
    row_sum2<THREADS>(sg, sgx, red);
    sg /= (float)dim;
    sgx /= (float)dim;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int at = c + k * THREADS * N;
      if (at < dim) store_some_stream<T, N>(dx + row * dx_stride + at, (g[k] - sg - xh[k] * sgx) * rstd, dim - at);
    }
  }
  float* to = parts + 2 * (int64_t)blockIdx.x * dim;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int at = c + k * THREADS * N;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      F32<N> v = which ? db[k] : dw[k];
      if (groups > 1) {
        __syncthreads();
        if (group > 0) fold[(group - 1) * THREADS + threadIdx.x % THREADS] = v;
        __syncthreads();
        if (group == 0)
          for (int o = 0; o < groups - 1; ++o) v += fold[o * THREADS + threadIdx.x];
      }
      if (group == 0 && at < dim) store_some<float, N>(to + which * (int64_t)dim + at, v, dim - at);
    }
  }
}

// Rows too long for registers (beyond 16384 columns): x and grad_y are read twice (the second time from a cache), and the columns' sums
// are formed by layernorm_columns_kernel in a pass of its own.  2000 x 20000 fp32 214 us for 87 at the rate of a copy, 4000 x 40000 bf16 452
// for 173.
template <typename T, int N>
__global__ __launch_bounds__(256) void layernorm_backward_long_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                                      const float* __restrict__ weight, const float* __restrict__ mean_in,
                                                                      const float* __restrict__ rstd_in, T* __restrict__ dx, int dim,
                                                                      int64_t dy_stride, int64_t x_stride, int64_t dx_stride) {
  __shared__ float red[8];
  const int64_t row = blockIdx.x;
  const float mean = mean_in[row], rstd = rstd_in[row];
  float sg = 0.f, sgx = 0.f;
  for (int at = threadIdx.x * N; at < dim; at += 256 * N) {
    const F32<N> g = widen<T, N>(load_some<N>(dy + row * dy_stride + at, dim - at)) * widen<float, N>(load_some<N>(weight + at, dim - at));
    const F32<N> xh = (widen<T, N>(load_some<N>(x + row * x_stride + at, dim - at)) - mean) * rstd;
    sg += sum_of<N>(g);
    sgx += sum_of<N>(g * xh);
  }
  row_sum2<256>(sg, sgx, red);
  sg /= (float)dim;
  sgx /= (float)dim;
  for (int at = threadIdx.x * N; at < dim; at += 256 * N) {
    const F32<N> g = widen<T, N>(load_some<N>(dy + row * dy_stride + at, dim - at)) * widen<float, N>(load_some<N>(weight + at, dim - at));
    const F32<N> xh = (widen<T, N>(load_some<N>(x + row * x_stride + at, dim - at)) - mean) * rstd;
    store_some<T, N>(dx + row * dx_stride + at, (g - sg - xh * sgx) * rstd, dim - at);
  }
}

template <typename T, int N>
__global__ __launch_bounds__(256) void layernorm_columns_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                                const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                                int64_t rows, int dim, int64_t dy_stride, int64_t x_stride,
                                                                float* __restrict__ parts) {
  const int at = (blockIdx.y * 256 + threadIdx.x) * N;
  if (at >= dim) return;
  F32<N> dw = {}, db = {};
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const F32<N> g = widen<T, N>(load_some<N>(dy + row * dy_stride + at, dim - at));
    const F32<N> xh = (widen<T, N>(load_some<N>(x + row * x_stride + at, dim - at)) - mean_in[row]) * rstd_in[row];
    dw += g * xh;
    db += g;
  }
  float* to = parts + 2 * (int64_t)blockIdx.x * dim + at;
  store_some<float, N>(to, dw, dim - at);
  store_some<float, N>(to + dim, db, dim - at);
}

// Adds the workgroups' sums per column, in order: a workgroup takes 64 columns of one of the two gradients, each
// of its 16 waves a run of consecutive parts.  Bound by latency: 512 parts of 2048 columns 4.8 us (one part under way at a time: 11.4).
constexpr int kJoinAhead = 16;   // parts under way
__global__ __launch_bounds__(1024) void layernorm_join_kernel(const float* __restrict__ parts, int count, int dim,
                                                              float* __restrict__ grad_weight, float* __restrict__ grad_bias,
                                                              int accumulate) {
  __shared__ float fold[16][kWave];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * kWave + l;
  float* to = blockIdx.y ? grad_bias : grad_weight;
  if (!to) return;
  const int share = (count + 15) / 16, lo = w * share, hi = min(count, lo + share);
  float s = 0.f;
  if (c < dim)
    for (int i = lo; i < hi; i += kJoinAhead) {
      float v[kJoinAhead];
#pragma unroll
      for (int k = 0; k < kJoinAhead; ++k) v[k] = i + k < hi ? parts[(2 * (int64_t)(i + k) + blockIdx.y) * dim + c] : 0.f;
#pragma unroll
      for (int k = 0; k < kJoinAhead; ++k) s += v[k];
    }
  fold[w][l] = s;
  __syncthreads();
  if (w == 0 && c < dim) {
    s = 0.f;
    for (int i = 0; i < 16; ++i) s += fold[i][l];
    to[c] = accumulate ? to[c] + s : s;
  }
}

}  // namespace accop
