// Short causal convolution of every channel along a sequence: forward and backward pass.
#pragma once
#include "op_common.h"

namespace accop {

struct ConvolutionShape {
  int64_t batch, steps, channels;
  int64_t x_b, x_t, out_b, out_t, dx_b, dx_t;      // backward: out is grad_out
  int64_t run, runs;                               // steps of a run, runs of a sequence
  int lanes_log2;                                  // lanes that share a row
  bool whole;                                      // packs at the ends of rows are made whole
};

// N elements of a row; FULL: all of them are there.  (Wide accesses need no alignment beyond the element's.)
template <bool FULL, int N, typename T>
__device__ __forceinline__ Pack<T, N> row_request(const T* p, int64_t left) {
  return FULL ? load<N>(p) : load_some<N>(p, left);
}
template <bool FULL, int N, typename T>
__device__ __forceinline__ F32<N> row_load(const T* p, int64_t left) {
  return widen<T, N>(FULL ? load<N>(p) : load_some<N>(p, left));
}
template <bool FULL, int N, typename T>
__device__ __forceinline__ void row_store(T* p, const F32<N>& v, int64_t left) {
  if (FULL) store<T, N>(p, v);
  else store_some<T, N>(p, v, left);
}

// What a lane has: N channels of a run of steps of a sequence.  FULL: a wave has one run, so that all but the channel lies in its scalar
// registers, and every pack is whole, as it may be without: the last one of a row that is not a multiple of N starts among the channels of the
// one in front, whose results it makes once more, the same ones.  (Single elements there cost every wave of the row's end a second path:
// 55 x 3025 x 455 bf16 forward 177 us, backward 276, with whole packs 74 and 176; 55 x 3025 x 125 44 and 92, with whole ones 28 and 52.)
struct ConvolutionPlace {
  int64_t batch, run, channel, left;      // left: channels from its first one on
};
template <int N, bool FULL>
__device__ __forceinline__ ConvolutionPlace convolution_place(const ConvolutionShape& s) {
  ConvolutionPlace p;
  const int64_t lane = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t unit = FULL ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : lane >> s.lanes_log2;
  p.batch = unit / s.runs;
  p.run = unit - p.batch * s.runs;
  p.channel = (((int64_t)blockIdx.y << s.lanes_log2) + (lane & ((1 << s.lanes_log2) - 1))) * N;
  p.left = s.channels - p.channel;
  if ((FULL || s.whole) && p.left > 0 && p.left < N) {
    p.channel = s.channels - N;
    p.left = N;
  }
  return p;
}

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

// The W - 1 inputs in front of step t, which is within the sequence or its start (the last one in front[W - 2]); those in front of the
// sequence from the state.
template <typename T, int N, int W, bool FULL>
__device__ __forceinline__ void load_front(const T* x, int64_t x_t, const float* state, int64_t channels, int64_t t, int64_t left,
                                           F32<N>* front) {
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t at = t - (W - 1) + j;
    front[j] = F32<N>{};
    if (at >= 0) front[j] = row_load<FULL, N>(x + at * x_t, left);
    else if (state) front[j] = row_load<FULL, N>(state + (at + W - 1) * channels, left);
  }
}

template <int N, int W>
__device__ __forceinline__ F32<N> weighed(const F32<N> (&w)[W], const F32<N>* v, F32<N> u) {
#pragma unroll
  for (int k = 0; k < W; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = fmaf(w[k][i], v[k][i], u[i]);
  return u;
}

// ---- forward ----------------------------------------------------------------------------------------------
// A lane takes N channels through a run of steps: the inputs slide through its registers, each is read once (the first W - 1 of a run
// twice).  Bound by memory where there is work: width 4, SiLU, 8 x 4096 x 4096 bf16 106 us, 5.1 TB/s, the rate of a large copy; 7 x 1999 x 1001
// fp32, width 3, ragged 17.5 us, 4.8 TB/s where the inputs are still in the Infinity Cache.  A turn's inputs are not under way during the turn
// in front, which other waves have to cover.  One token of 64 x 1344 channels: 6.2 us, nearly all of it two waits, one for weights, state and
// input and one for the input that last takes once more.
constexpr int kConvolutionAhead = 4;   // steps under way

template <typename T, int N, int W, bool FULL>
__global__ __launch_bounds__(256) void convolution_forward_kernel(ConvolutionShape s, const T* __restrict__ x,
                                                                  const float* __restrict__ weight, const float* __restrict__ bias,
                                                                  const float* state, const int32_t* __restrict__ lengths,
                                                                  T* __restrict__ out, float* last, int silu) {
  constexpr int U = kConvolutionAhead;
  const ConvolutionPlace p = convolution_place<N, FULL>(s);
  const int64_t b = p.batch, c = p.channel, left = p.left;
  if (b >= s.batch || left <= 0) return;
  const int64_t len = steps_of(lengths, b, s.steps);
  const int64_t t0 = p.run * s.run, t1 = min(t0 + s.run, s.steps), end = min(t1, len);
  const T* const from = x + b * s.x_b + c;
  T* const to = out + b * s.out_b + c;
  F32<N> w[W], bias_of = {}, v[W - 1 + U];
  load_weights<W, N>(weight, c, left, w);
  if (bias) bias_of = row_load<FULL, N>(bias + c, left);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) v[j] = F32<N>{};
  if (p.run == 0 || t0 < len)
    load_front<T, N, W, FULL>(from, s.x_t, state ? state + b * (W - 1) * s.channels + c : nullptr, s.channels, t0, left, v);
  F32<N> first[W];                     // what the sequence starts from
#pragma unroll
  for (int j = 0; j < W - 1; ++j) first[j] = v[j];
  for (int64_t t = t0; t < end; t += U) {
#pragma unroll
    for (int j = 0; j < U; ++j) v[W - 1 + j] = row_load<FULL, N>(from + min(t + j, end - 1) * s.x_t, left);
    F32<N> u[U];
#pragma unroll
    for (int j = 0; j < U; ++j) u[j] = weighed<N, W>(w, v + j, bias_of);
    if (silu) {
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) u[j][i] *= sigmoid(u[j][i]).a;
    }
    if (t + U <= end) {
#pragma unroll
      for (int j = 0; j < U; ++j) row_store<FULL, N>(to + (t + j) * s.out_t, u[j], left);
    } else {
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (t + j < end) row_store<FULL, N>(to + (t + j) * s.out_t, u[j], left);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) v[j] = v[U + j];
  }
  for (int64_t t = max(t0, len); t < t1; ++t) row_store<FULL, N>(to + t * s.out_t, F32<N>{}, left);
  if (!last || p.run != 0) return;
  // (state may be last: this lane has read all of its part)
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int64_t at = len - (W - 1) + j;
    F32<N> r = {};
    if (at >= 0) {
      r = row_load<FULL, N>(from + at * s.x_t, left);
    } else {
#pragma unroll
      for (int k = 0; k < W - 1; ++k)
        if (k == at + W - 1) r = first[k];
    }
    row_store<FULL, N>(last + (b * (W - 1) + j) * s.channels + c, r, left);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------
// A lane takes N channels through a run of steps and the W - 1 behind it, whose g it needs: inputs and g slide through its registers.
// The gradients of its weights stay in registers over the run; a workgroup adds its runs' and leaves them in parts (W + 1 rows of
// channels), which parts_join_kernel adds.  Packs of 4 channels: 8 would need twice the registers of w, dw, v and g.  Width 4, SiLU, 8 x 4096 x 4096 bf16:
// 175 us with calls in a row, 4.6 TB/s: memory.
template <typename T, int N, int W, bool FULL>
__global__ __launch_bounds__(256) void convolution_backward_kernel(ConvolutionShape s, const T* __restrict__ x,
                                                                   const float* __restrict__ weight, const float* __restrict__ bias,
                                                                   const float* __restrict__ state, const int32_t* __restrict__ lengths,
                                                                   const T* __restrict__ dout, const float* __restrict__ dlast,
                                                                   T* __restrict__ dx, float* __restrict__ dstate,
                                                                   float* __restrict__ parts, int silu) {
  constexpr int U = kConvolutionAhead;
  __shared__ F32<N> fold[256];
  const ConvolutionPlace p = convolution_place<N, FULL>(s);
  const int64_t b = p.batch, c = p.channel, left = p.left;
  F32<N> dw[W], db = {};
#pragma unroll
  for (int k = 0; k < W; ++k) dw[k] = F32<N>{};
  if (b < s.batch && left > 0) {
    const int64_t len = steps_of(lengths, b, s.steps);
    const int64_t t0 = p.run * s.run, t1 = min(t0 + s.run, s.steps), end = min(t1, len);
    const T* const from = x + b * s.x_b + c;
    const T* const grad = dout + b * s.out_b + c;
    T* const to = dx + b * s.dx_b + c;
    F32<N> w[W], bias_of = {}, v[W - 1 + U], g[W - 1 + U];
    load_weights<W, N>(weight, c, left, w);
    if (bias) bias_of = row_load<FULL, N>(bias + c, left);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) v[j] = g[j] = F32<N>{};
    if (t0 < len)
      load_front<T, N, W, FULL>(from, s.x_t, state ? state + b * (W - 1) * s.channels + c : nullptr, s.channels, t0, left, v);
    const int64_t least = p.run == 0 ? -(int64_t)(W - 1) : t0;       // steps whose inputs' gradients are this run's
    // the gradient of the input at step t, of which all products with g are in r
    auto put = [&](int64_t t, F32<N> r) {
      if (t < least || t >= t1) return;
      if (dlast && t >= len - (W - 1) && t < len) r += row_load<FULL, N>(dlast + (b * (W - 1) + t - len + W - 1) * s.channels + c, left);
      if (t >= 0) row_store<FULL, N>(to + t * s.dx_t, r, left);
      else if (dstate) row_store<FULL, N>(dstate + (b * (W - 1) + t + W - 1) * s.channels + c, r, left);
    };
    // g of the steps in v[j .. j + W - 1], from the gradient of out
    auto through = [&](int j, F32<N> d) {
      const F32<N> u = weighed<N, W>(w, v + j, bias_of);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Gates z = sigmoid(u[i]);
        d[i] *= z.a * fmaf(u[i], z.z, 1.f);
      }
      return d;
    };
    auto count = [&](int j) {
      db += g[W - 1 + j];
#pragma unroll
      for (int k = 0; k < W; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) dw[k][i] = fmaf(g[W - 1 + j][i], v[j + k][i], dw[k][i]);
    };
    auto input = [&](int j) {
      F32<N> r = {};
#pragma unroll
      for (int k = 0; k < W; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = fmaf(w[k][i], g[W - 1 + j - k][i], r[i]);
      return r;
    };
    const int64_t seen = min(t1 + W - 1, len);      // steps whose g this run needs
    Pack<T, N> next_x[U], next_d[U];                // the steps behind those at work
    auto request = [&](int64_t t) {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        next_x[j] = row_request<FULL, N>(from + min(t + j, seen - 1) * s.x_t, left);
        next_d[j] = row_request<FULL, N>(grad + min(t + j, seen - 1) * s.out_t, left);
      }
    };
    if (t0 < seen) request(t0);
    for (int64_t t = t0; t < t1 + W - 1; t += U) {
      if (t >= seen + W - 1) {                      // nothing but zeros from here on
        for (int64_t z = max(t - (W - 1), least); z < t1; ++z) put(z, F32<N>{});
        break;
      }
      F32<N> d[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        v[W - 1 + j] = widen<T, N>(next_x[j]);
        d[j] = widen<T, N>(next_d[j]);
      }
      if (t + U < seen) request(t + U);
      if (t - (W - 1) >= t0 && t + U <= end) {      // every step is this run's own, with all its g
#pragma unroll
        for (int j = 0; j < U; ++j) g[W - 1 + j] = d[j];
        if (silu) {
#pragma unroll
          for (int j = 0; j < U; ++j) g[W - 1 + j] = through(j, d[j]);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
          count(j);
          row_store<FULL, N>(to + (t + j - (W - 1)) * s.dx_t, input(j), left);
        }
      } else {
#pragma unroll
        for (int j = 0; j < U; ++j) {
          if (t + j >= seen) v[W - 1 + j] = d[j] = F32<N>{};
          g[W - 1 + j] = d[j];
          if (silu && t + j < seen) g[W - 1 + j] = through(j, d[j]);
          if (t + j < end) count(j);
          put(t + j - (W - 1), input(j));
        }
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        v[j] = v[U + j];
        g[j] = g[U + j];
      }
    }
  }
  const int row = 1 << s.lanes_log2;
  float* const to = parts + (int64_t)blockIdx.x * (W + 1) * s.channels + c;
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
