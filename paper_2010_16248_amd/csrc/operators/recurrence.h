// Gated linear recurrence h_t = a_t h_{t-1} + z_t x_t, a = sigmoid(gate), z = sigmoid(-gate): forward and backward pass.
#pragma once
#include "op_common.h"

namespace accop {

struct RecurrenceShape {
  int64_t steps, channels;
  int64_t gate_b, gate_t, input_b, input_t, out_b, out_t;
  int64_t dgate_b, dgate_t, dinput_b, dinput_t, dout_b, dout_t;
};

// e^-x for x >= 0 (NaN for NaN): 2^t of the rounded product t = -x log2(e), corrected by what the rounding lost.
// From 104 on the result is below the smallest fp32 number.
__device__ __forceinline__ float exp_neg(float x) {
  x = x > 104.f ? 104.f : x;
  const float t = -1.44269502f * x;
  const float lost = fmaf(-1.44269502f, x, -t) + -1.92596303e-8f * x;
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, lost * 0.693147182f, e);
}

// sigmoid(f) and sigmoid(-f).  Neither is a difference from one: a gate near one keeps all digits of 1 - a.
__device__ __forceinline__ void gates(float f, float& a, float& z) {
  const float e = exp_neg(fabsf(f));
  const float d = 1.f + e;
  float big = __builtin_amdgcn_rcpf(d);
  big = fmaf(fmaf(-d, big, 1.f), big, big);
  const float small = e * big;
  a = f >= 0.f ? big : small;
  z = f >= 0.f ? small : big;
}

__device__ __forceinline__ int64_t steps_of(const int32_t* lengths, int64_t batch, int64_t steps) {
  if (!lengths) return steps;
  const int64_t n = lengths[batch];
  return n < 0 ? 0 : (n < steps ? n : steps);
}

// ---- a lane per N channels, step after step ---------------------------------------------------------------
constexpr int kWalkAhead = 8;   // steps under way

template <typename T, int N>
__global__ __launch_bounds__(256) void recurrence_forward_walk_kernel(RecurrenceShape s, const T* __restrict__ gate,
                                                                      const T* __restrict__ input, const float* h0,
                                                                      const int32_t* __restrict__ lengths, T* __restrict__ out,
                                                                      float* h_last) {
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N, b = blockIdx.y, left = s.channels - c;
  if (left <= 0) return;
  const int64_t len = steps_of(lengths, b, s.steps);
  const T* g = gate + b * s.gate_b + c;
  const T* x = input + b * s.input_b + c;
  T* o = out + b * s.out_b + c;
  F32<N> h = {};
  if (h0) h = widen<float, N>(load_some<N>(h0 + b * s.channels + c, left));
  for (int64_t t0 = 0; t0 < len; t0 += kWalkAhead) {
    Pack<T, N> f[kWalkAhead], v[kWalkAhead];
#pragma unroll
    for (int j = 0; j < kWalkAhead; ++j) {
      const int64_t t = min(t0 + j, len - 1);
      f[j] = load_some<N>(g + t * s.gate_t, left);
      v[j] = load_some<N>(x + t * s.input_t, left);
    }
#pragma unroll
    for (int j = 0; j < kWalkAhead; ++j) {
      if (t0 + j >= len) break;
      const F32<N> ff = widen<T, N>(f[j]), xx = widen<T, N>(v[j]);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float a, z;
        gates(ff[i], a, z);
        h[i] = a * h[i] + z * xx[i];
      }
      store_some<T, N>(o + (t0 + j) * s.out_t, h, left);
    }
  }
  for (int64_t t = len; t < s.steps; ++t) store_some<T, N>(o + t * s.out_t, F32<N>{}, left);
  if (h_last) store_some<float, N>(h_last + b * s.channels + c, h, left);
}

template <typename T, int N>
__global__ __launch_bounds__(256) void recurrence_backward_walk_kernel(RecurrenceShape s, const T* __restrict__ gate,
                                                                       const T* __restrict__ input, const T* __restrict__ out,
                                                                       const float* __restrict__ h0, const int32_t* __restrict__ lengths,
                                                                       const T* __restrict__ dout, const float* __restrict__ dlast,
                                                                       T* __restrict__ dgate, T* __restrict__ dinput,
                                                                       float* __restrict__ dh0) {
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N, b = blockIdx.y, left = s.channels - c;
  if (left <= 0) return;
  const int64_t len = steps_of(lengths, b, s.steps);
  F32<N> total = {}, first = {};
  if (dlast) total = widen<float, N>(load_some<N>(dlast + b * s.channels + c, left));
  if (h0) first = widen<float, N>(load_some<N>(h0 + b * s.channels + c, left));
  for (int64_t t = s.steps - 1; t >= len; --t) {
    store_some<T, N>(dgate + b * s.dgate_b + t * s.dgate_t + c, F32<N>{}, left);
    store_some<T, N>(dinput + b * s.dinput_b + t * s.dinput_t + c, F32<N>{}, left);
  }
  for (int64_t t0 = len - 1; t0 >= 0; t0 -= kWalkAhead) {
    Pack<T, N> f[kWalkAhead], x[kWalkAhead], h[kWalkAhead], d[kWalkAhead];
#pragma unroll
    for (int j = 0; j < kWalkAhead; ++j) {
      const int64_t t = max(t0 - j, (int64_t)0);
      f[j] = load_some<N>(gate + b * s.gate_b + t * s.gate_t + c, left);
      x[j] = load_some<N>(input + b * s.input_b + t * s.input_t + c, left);
      h[j] = load_some<N>(out + b * s.out_b + max(t - 1, (int64_t)0) * s.out_t + c, left);
      d[j] = load_some<N>(dout + b * s.dout_b + t * s.dout_t + c, left);
    }
#pragma unroll
    for (int j = 0; j < kWalkAhead; ++j) {
      const int64_t t = t0 - j;
      if (t < 0) break;
      total += widen<T, N>(d[j]);
      const F32<N> before = t > 0 ? widen<T, N>(h[j]) : first;
      const F32<N> ff = widen<T, N>(f[j]), xx = widen<T, N>(x[j]);
      F32<N> dg, dx;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float a, z;
        gates(ff[i], a, z);
        dx[i] = z * total[i];
        dg[i] = (before[i] - xx[i]) * a * dx[i];
        total[i] = a * total[i];
      }
      store_some<T, N>(dgate + b * s.dgate_b + t * s.dgate_t + c, dg, left);
      store_some<T, N>(dinput + b * s.dinput_b + t * s.dinput_t + c, dx, left);
    }
  }
  if (dh0) store_some<float, N>(dh0 + b * s.channels + c, total, left);
}

}  // namespace accop
