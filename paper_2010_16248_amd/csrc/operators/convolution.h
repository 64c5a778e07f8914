// Short causal convolution of every channel along a sequence: forward and backward pass.
#pragma once
#include "op_common.h"

namespace accop {

struct ConvolutionShape {
  int64_t batch, steps, channels;
  int64_t x_b, x_t, out_b, out_t, dx_b, dx_t;      // backward: out is grad_out
  int64_t run, runs;                               // steps of a run, runs of a sequence
  int lanes_log2;                                  // lanes that share a row
};

// W x N weights of N channels: of channel i, its W weights lie together.
template <int W, int N>
__device__ __forceinline__ void load_weights(const float* weight, int64_t c, int64_t left, F32<N> (&w)[W]) {
  float v[W * N];
  const float* from = weight + c * W;
#pragma unroll
  for (int k = 0; k < W * N; k += 4) {
    const F32<4> four = widen<float, 4>(load_some<4>(from + k, left * W - k));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[k + i] = four[i];
  }
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) w[j][i] = v[i * W + j];
}

// The W - 1 inputs in front of step t, which is within the sequence or its start (the last one in front[W - 2]); those in front of the sequence from the state.
template <typename T, int N, int W>
__device__ __forceinline__ void load_front(const T* x, int64_t x_t, const float* state, int64_t channels, int64_t t, int64_t left,
                                           F32<N>* front) {
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t at = t - (W - 1) + j;
    front[j] = F32<N>{};
    if (at >= 0) front[j] = widen<T, N>(load_some<N>(x + at * x_t, left));
    else if (state) front[j] = widen<float, N>(load_some<N>(state + (at + W - 1) * channels, left));
  }
}

// ---- forward ----------------------------------------------------------------------------------------------
// A lane takes N channels through a run of steps: the inputs slide through its registers, each is read once (the first W - 1 of a run
// twice).
constexpr int kConvolutionAhead = 4;   // steps under way

template <typename T, int N, int W, bool SILU>
__global__ __launch_bounds__(256) void convolution_forward_kernel(ConvolutionShape s, const T* __restrict__ x,
                                                                  const float* __restrict__ weight, const float* __restrict__ bias,
                                                                  const float* state, const int32_t* __restrict__ lengths,
                                                                  T* __restrict__ out, float* last) {
  constexpr int U = kConvolutionAhead;
  const int64_t lane = (int64_t)blockIdx.x * 256 + threadIdx.x, unit = lane >> s.lanes_log2;
  const int64_t b = unit / s.runs, run = unit - b * s.runs;
  const int64_t c = (((int64_t)blockIdx.y << s.lanes_log2) + (lane & ((1 << s.lanes_log2) - 1))) * N, left = s.channels - c;
  if (b >= s.batch || left <= 0) return;
  const int64_t len = steps_of(lengths, b, s.steps);
  const int64_t t0 = run * s.run, t1 = min(t0 + s.run, s.steps), end = min(t1, len);
  const T* from = x + b * s.x_b + c;
  T* to = out + b * s.out_b + c;
  const float* front = state ? state + b * (W - 1) * s.channels + c : nullptr;
  F32<N> w[W], bias_of = {}, v[W - 1 + U];
  load_weights<W, N>(weight, c, left, w);
  if (bias) bias_of = widen<float, N>(load_some<N>(bias + c, left));
  if (run == 0 || t0 < len) load_front<T, N, W>(from, s.x_t, front, s.channels, t0, left, v);
  F32<N> first[W];                     // what the sequence starts from
#pragma unroll
  for (int j = 0; j < W - 1; ++j) first[j] = v[j];
  for (int64_t t = t0; t < end; t += U) {
    Pack<T, N> raw[U];
#pragma unroll
    for (int j = 0; j < U; ++j) raw[j] = load_some<N>(from + min(t + j, end - 1) * s.x_t, left);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      v[W - 1 + j] = widen<T, N>(raw[j]);
      F32<N> u = bias_of;
#pragma unroll
      for (int k = 0; k < W; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = fmaf(w[k][i], v[j + k][i], u[i]);
      if (SILU)
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] *= sigmoid(u[i]).a;
      if (t + j < end) store_some<T, N>(to + (t + j) * s.out_t, u, left);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) v[j] = v[U + j];
  }
  for (int64_t t = max(t0, len); t < t1; ++t) store_some<T, N>(to + t * s.out_t, F32<N>{}, left);
  if (!last || run != 0) return;
  // (state may be last: this lane has read all of its part)
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t at = len - (W - 1) + j;
    F32<N> r = {};
    if (at >= 0) {
      r = widen<T, N>(load_some<N>(from + at * s.x_t, left));
    } else {
#pragma unroll
      for (int k = 0; k < W - 1; ++k)
        if (k == at + W - 1) r = first[k];
    }
    store_some<float, N>(last + (b * (W - 1) + j) * s.channels + c, r, left);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------
// A lane takes N channels through a run of steps and the W - 1 behind it, whose g it needs: inputs and g slide through its registers.
// The gradients of its weights stay in registers over the run; a workgroup adds its runs' and leaves them in parts (W + 1 rows of
// channels), which parts_join_kernel adds.
template <typename T, int N, int W, bool SILU>
__global__ __launch_bounds__(256) void convolution_backward_kernel(ConvolutionShape s, const T* __restrict__ x,
                                                                   const float* __restrict__ weight, const float* __restrict__ bias,
                                                                   const float* __restrict__ state, const int32_t* __restrict__ lengths,
                                                                   const T* __restrict__ dout, const float* __restrict__ dlast,
                                                                   T* __restrict__ dx, float* __restrict__ dstate,
                                                                   float* __restrict__ parts) {
  constexpr int U = kConvolutionAhead;
  __shared__ F32<N> fold[256];
  const int64_t lane = (int64_t)blockIdx.x * 256 + threadIdx.x, unit = lane >> s.lanes_log2;
  const int64_t b = unit / s.runs, run = unit - b * s.runs;
  const int64_t c = (((int64_t)blockIdx.y << s.lanes_log2) + (lane & ((1 << s.lanes_log2) - 1))) * N, left = s.channels - c;
  const bool mine = b < s.batch && left > 0;
  F32<N> dw[W], db = {};
#pragma unroll
  for (int k = 0; k < W; ++k) dw[k] = F32<N>{};
  if (mine) {
    const int64_t len = steps_of(lengths, b, s.steps);
    const int64_t t0 = run * s.run, t1 = min(t0 + s.run, s.steps), end = min(t1, len);
    const T* from = x + b * s.x_b + c;
    const T* grad = dout + b * s.out_b + c;
    T* to = dx + b * s.dx_b + c;
    F32<N> w[W], bias_of = {}, v[W - 1 + U], g[W - 1 + U];
    load_weights<W, N>(weight, c, left, w);
    if (bias) bias_of = widen<float, N>(load_some<N>(bias + c, left));
#pragma unroll
    for (int j = 0; j < W - 1; ++j) v[j] = g[j] = F32<N>{};
    if (t0 < len)
      load_front<T, N, W>(from, s.x_t, state ? state + b * (W - 1) * s.channels + c : nullptr, s.channels, t0, left, v);
    // the gradient of the input at step t, of which all products with g are in r
    auto put = [&](int64_t t, F32<N> r) {
      if (t < (run == 0 ? -(W - 1) : t0) || t >= t1) return;
      if (dlast && t >= len - (W - 1) && t < len)
        r += widen<float, N>(load_some<N>(dlast + (b * (W - 1) + t - len + W - 1) * s.channels + c, left));
      if (t >= 0) store_some<T, N>(to + t * s.dx_t, r, left);
      else if (dstate) store_some<float, N>(dstate + (b * (W - 1) + t + W - 1) * s.channels + c, r, left);
    };
    const int64_t seen = min(t1 + W - 1, len);      // steps whose g this run needs
    for (int64_t t = t0; t < t1 + W - 1; t += U) {
      if (t >= seen + W - 1) {                      // nothing but zeros from here on
        for (int64_t z = max(t - (W - 1), run == 0 ? -(int64_t)(W - 1) : t0); z < t1; ++z) put(z, F32<N>{});
        break;
      }
      Pack<T, N> raw[U], up[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        raw[j] = up[j] = Pack<T, N>{};
        if (t + j < seen) {
          raw[j] = load_some<N>(from + (t + j) * s.x_t, left);
          up[j] = load_some<N>(grad + (t + j) * s.out_t, left);
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        v[W - 1 + j] = widen<T, N>(raw[j]);
        F32<N> d = widen<T, N>(up[j]);
        if (SILU) {
          F32<N> u = bias_of;
#pragma unroll
          for (int k = 0; k < W; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = fmaf(w[k][i], v[j + k][i], u[i]);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const Gates z = sigmoid(u[i]);
            d[i] *= z.a * fmaf(u[i], z.z, 1.f);
          }
          if (t + j >= seen) d = F32<N>{};
        }
        g[W - 1 + j] = d;
        if (t + j < end) {
          db += d;
#pragma unroll
          for (int k = 0; k < W; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) dw[k][i] = fmaf(d[i], v[j + k][i], dw[k][i]);
        }
        F32<N> r = {};
#pragma unroll
        for (int k = 0; k < W; ++k)
#pragma unroll
          for (int i = 0; i < N; ++i) r[i] = fmaf(w[k][i], g[W - 1 + j - k][i], r[i]);
        put(t + j - (W - 1), r);
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        v[j] = v[U + j];
        g[j] = g[U + j];
      }
    }
  }
  const int row = 1 << s.lanes_log2;
  float* to = parts + (int64_t)blockIdx.x * (W + 1) * s.channels + c;
#pragma unroll
  for (int k = 0; k <= W; ++k) {
    F32<N> r = k < W ? dw[k < W ? k : 0] : db;
    __syncthreads();
    fold[threadIdx.x] = r;
    __syncthreads();
    if (threadIdx.x < row && left > 0) {
      for (int o = threadIdx.x + row; o < 256; o += row) r += fold[o];
      store_some<float, N>(to + (int64_t)k * s.channels, r, left);
    }
  }
}

}  // namespace accop
