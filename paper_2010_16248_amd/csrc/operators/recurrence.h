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
struct Gates {
  float a, z;
};
__device__ __forceinline__ Gates gates(float f) {
  const float e = exp_neg(fabsf(f));
  const float d = 1.f + e;
  float big = __builtin_amdgcn_rcpf(d);
  big = fmaf(fmaf(-d, big, 1.f), big, big);
  const float small = e * big;
  return f >= 0.f ? Gates{big, small} : Gates{small, big};
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
        const Gates k = gates(ff[i]);
        h[i] = fmaf(k.a, h[i], k.z * xx[i]);
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
        const Gates k = gates(ff[i]);
        dx[i] = k.z * total[i];
        dg[i] = (before[i] - xx[i]) * k.a * dx[i];
        total[i] = k.a * total[i];
      }
      store_some<T, N>(dgate + b * s.dgate_b + t * s.dgate_t + c, dg, left);
      store_some<T, N>(dinput + b * s.dinput_b + t * s.dinput_t + c, dx, left);
    }
  }
  if (dh0) store_some<float, N>(dh0 + b * s.channels + c, total, left);
}

// ---- a workgroup per chunk of steps ---------------------------------------------------------------------------
// The step maps of a chunk compose to one map h -> A h + H.  A wave takes S consecutive steps of 64 N channels and keeps
// their maps in registers, a workgroup as many waves as it has; so the inputs are read once.  Where a sequence has several
// chunks, a chunk leaves its map in the workspace, takes the state at its start from the chunks before it (look_back) and
// leaves the state at its end.  Whatever it finds there, the state it starts with is the fold of the maps in front of it,
// from the first one on, map after map: the bits do not depend on who was faster.
//
// Maps and the states between waves are fp64: composed maps meet in differences (A h against H) that the steps one by
// one do not have, and so a wave starts from the state that steps without rounding would have reached.
//
// Chunks are handed out by a counter in the order of the steps, so that all chunks a workgroup waits for have
// been taken by workgroups that run already.  A map is left without waiting for anything; of the chunks without
// a state at their end the first one always finds the one in front of it: every wait ends.
//
// A word of the workspace holds a value and the news that it is there at once (all ones: not yet); its accesses are
// atomic and go past the caches that compute units do not share.
constexpr int kChunkWaves = 16;       // most waves of a workgroup
constexpr int kLookBack = 8;          // chunks looked at in one go
constexpr unsigned long long kNotYet = ~0ull;

template <int N>
using F64 = double __attribute__((ext_vector_type(N)));

struct ChunkSlots {
  unsigned long long* map_a;          // per chain, chunk and channel
  unsigned long long* map_h;
  unsigned long long* state;          // the state at the chunk's end
  uint32_t* counter;                  // chunks handed out
  int64_t chains, channel_blocks;     // (sequence, block of 64 N channels)
  int chunks;
};

__global__ __launch_bounds__(256) void recurrence_clear_kernel(unsigned long long* words, int64_t n, uint32_t* counter) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i == 0) *counter = 0;
  if (i < n) words[i] = kNotYet;
}

// No result is the word that says "not yet": a NaN is given its common form.
__device__ __forceinline__ void leave(unsigned long long* p, double v) {
  const unsigned long long word = v == v ? (unsigned long long)__double_as_longlong(v) : 0x7ff8000000000000ull;
  __hip_atomic_store(p, word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long look(const unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The state at the start of chunk `chunk` > 0 of one channel per lane.  slot0: the channel's slot in chunk 0, pitch: slots
// per chunk.
__device__ __forceinline__ double look_back(const ChunkSlots& s, int64_t slot0, int64_t pitch, int chunk) {
  const int most = min(chunk, kLookBack);
  for (;;) {
    unsigned long long st[kLookBack];
#pragma unroll
    for (int q = 0; q < kLookBack; ++q) st[q] = look(s.state + slot0 + (int64_t)(chunk - 1 - min(q, most - 1)) * pitch);
    int at = -1;
    double h = 0.0;
#pragma unroll
    for (int q = kLookBack - 1; q >= 0; --q)
      if (q < most && __ballot(st[q] == kNotYet) == 0) {
        at = q;
        h = __longlong_as_double((long long)st[q]);
      }
    if (at == 0) return h;
    if (at > 0) {
      unsigned long long a[kLookBack - 1], b[kLookBack - 1];
#pragma unroll
      for (int q = 0; q < kLookBack - 1; ++q) {
        const int64_t slot = slot0 + (int64_t)(chunk - 1 - min(q, at - 1)) * pitch;
        a[q] = look(s.map_a + slot);
        b[q] = look(s.map_h + slot);
      }
      bool all = true;
#pragma unroll
      for (int q = kLookBack - 2; q >= 0; --q)
        if (q < at) {
          all = all && a[q] != kNotYet && b[q] != kNotYet;
          h = fma(__longlong_as_double((long long)a[q]), h, __longlong_as_double((long long)b[q]));
        }
      if (__ballot(!all) == 0) return h;
    }
    __builtin_amdgcn_s_sleep(1);
  }
}

// Where a workgroup works: which chunk of which chain.
struct ChunkPlace {
  int chunk;
  int64_t b, c, left;                 // sequence, the lane's first channel, channels from there on
  int64_t slot0;                      // the chain's first slot
};

template <int N>
__device__ __forceinline__ ChunkPlace chunk_place(const ChunkSlots& s, const RecurrenceShape& shape, uint32_t* shared_ticket) {
  uint32_t ticket = blockIdx.x;
  if (s.chunks > 1) {
    if (threadIdx.x == 0) *shared_ticket = atomicAdd(s.counter, 1u);
    __syncthreads();
    ticket = __builtin_amdgcn_readfirstlane(*shared_ticket);
  }
  ChunkPlace p;
  p.chunk = (int)(ticket / (uint32_t)s.chains);
  const uint32_t chain = ticket % (uint32_t)s.chains;
  p.b = chain / (uint32_t)s.channel_blocks;
  p.c = (int64_t)(chain % (uint32_t)s.channel_blocks) * (kWave * N) + (threadIdx.x & 63) * N;
  p.left = shape.channels - p.c;
  p.slot0 = (int64_t)chain * s.chunks * (kWave * N);
  return p;
}

// Maps of a workgroup's waves, per channel of its block.
template <int N>
struct ChunkFold {
  double a[kChunkWaves][kWave * N], h[kChunkWaves][kWave * N], start[kWave * N];
};

// From the waves' maps to the state at this wave's start.  first: the state at the chain's start (used in chunk 0 only).
template <int N>
__device__ __forceinline__ F32<N> chunk_state(const ChunkSlots& s, const ChunkPlace& p, const F64<N>& a_mine, const F64<N>& h_mine,
                                              const F32<N>& first, ChunkFold<N>& fold) {
  constexpr int pitch = kWave * N;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    fold.a[w][l * N + i] = a_mine[i];
    fold.h[w][l * N + i] = h_mine[i];
    if (w == 0) fold.start[l * N + i] = (double)first[i];
  }
  __syncthreads();
  if (s.chunks > 1) {
    if (w < N) {                       // a wave for every 64 channels
      const int ch = w * kWave + l;
      double A = fold.a[0][ch], H = fold.h[0][ch];
      for (int k = 1; k < waves; ++k) {
        const double ak = fold.a[k][ch];
        A *= ak;
        H = fma(ak, H, fold.h[k][ch]);
      }
      const int64_t slot = p.slot0 + (int64_t)p.chunk * pitch + ch;
      const bool last = p.chunk + 1 == s.chunks;
      double h = fold.start[ch];
      if (p.chunk > 0) {
        if (!last) {
          leave(s.map_a + slot, A);
          leave(s.map_h + slot, H);
        }
        h = look_back(s, p.slot0 + ch, pitch, p.chunk);
        fold.start[ch] = h;
      }
      if (!last) leave(s.state + slot, fma(A, h, H));
    }
    __syncthreads();
  }
  F64<N> h;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    h[i] = fold.start[l * N + i];
    for (int k = 0; k < w; ++k) h[i] = fma(fold.a[k][l * N + i], h[i], fold.h[k][l * N + i]);
  }
  return __builtin_convertvector(h, F32<N>);
}

// Rows of S steps, one every `pitch` elements, from p on; steps beyond the last-th (counted from zero) load that one again.
template <typename T, int N, int S>
__device__ __forceinline__ void load_steps(Pack<T, N> (&v)[S], const T* p, int64_t pitch, int last) {
#pragma unroll
  for (int j = 0; j < S; ++j) {
    v[j] = load<N>(p);
    p += j < last ? pitch : 0;
  }
}

// N divides the channels, so a lane has all of its N channels or none (it then works on the first ones and stores nothing).
template <typename T, int N, int S>
__global__ __launch_bounds__(kWave* kChunkWaves) void recurrence_forward_chunk_kernel(
    RecurrenceShape s, ChunkSlots slots, const T* __restrict__ gate, const T* __restrict__ input, const float* h0,
    const int32_t* __restrict__ lengths, T* __restrict__ out, float* h_last) {
  __shared__ ChunkFold<N> fold;
  __shared__ uint32_t ticket;
  const ChunkPlace p = chunk_place<N>(slots, s, &ticket);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const bool mine = p.left > 0;
  const int64_t c = mine ? p.c : 0, ends = p.b * s.channels + c;
  const int64_t t0 = ((int64_t)p.chunk * waves + w) * S;
  const int in = (int)min((int64_t)S, max(steps_of(lengths, p.b, s.steps) - t0, (int64_t)0));   // steps of the sequence
  const int here = (int)min((int64_t)S, max(s.steps - t0, (int64_t)0));                        // steps of the tensors
  F32<N> a[S], b[S], first = {};
  F64<N> A = F64<N>{} + 1.0, H = {};
  if (in > 0) {
    Pack<T, N> f[S], v[S];
    load_steps<T, N, S>(f, gate + p.b * s.gate_b + t0 * s.gate_t + c, s.gate_t, in - 1);
    load_steps<T, N, S>(v, input + p.b * s.input_b + t0 * s.input_t + c, s.input_t, in - 1);
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const F32<N> ff = widen<T, N>(f[j]), xx = widen<T, N>(v[j]);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Gates k = gates(ff[i]);
        a[j][i] = j < in ? k.a : 1.f;
        b[j][i] = j < in ? k.z * xx[i] : 0.f;
        A[i] *= (double)a[j][i];
        H[i] = fma((double)a[j][i], H[i], (double)b[j][i]);
      }
    }
  }
  if (h0 && p.chunk == 0) first = widen<float, N>(load<N>(h0 + ends));
  F32<N> h = chunk_state<N>(slots, p, A, H, first, fold);
  if (!mine) return;
  T* o = out + p.b * s.out_b + t0 * s.out_t + c;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    if (j < in) {
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = fmaf(a[j][i], h[i], b[j][i]);
      store<T, N>(o, h);
    } else if (j < here) {
      store<T, N>(o, F32<N>{});
    }
    o += s.out_t;
  }
  if (h_last && p.chunk == slots.chunks - 1 && w == waves - 1) store<float, N>(h_last + ends, h);
}

// Backward in time: the state is c_t = a_t G_t, the gradient of h_{t-1}; c_t = a_t c_{t+1} + a_t grad_out_t.  Steps are counted from
// the last one on.
template <typename T, int N, int S>
__global__ __launch_bounds__(kWave* kChunkWaves) void recurrence_backward_chunk_kernel(
    RecurrenceShape s, ChunkSlots slots, const T* __restrict__ gate, const T* __restrict__ input, const T* __restrict__ out,
    const float* __restrict__ h0, const int32_t* __restrict__ lengths, const T* __restrict__ dout, const float* __restrict__ dlast,
    T* __restrict__ dgate, T* __restrict__ dinput, float* __restrict__ dh0) {
  __shared__ ChunkFold<N> fold;
  __shared__ uint32_t ticket;
  const ChunkPlace p = chunk_place<N>(slots, s, &ticket);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const bool mine = p.left > 0;
  const int64_t c = mine ? p.c : 0, ends = p.b * s.channels + c;
  const int64_t t0 = s.steps - 1 - ((int64_t)p.chunk * waves + w) * S;                          // the wave's latest step
  const int here = (int)min((int64_t)S, max(t0 + 1, (int64_t)0));                               // steps of the tensors: j < here
  const int out_of = (int)min((int64_t)here, max(t0 + 1 - steps_of(lengths, p.b, s.steps), (int64_t)0));   // of the sequence: out_of <= j
  F32<N> a[S], z[S], first = {}, state;
  F64<N> A = F64<N>{} + 1.0, H = {};
  Pack<T, N> d[S], x[S], before[S];
  if (out_of < here) {
    // steps that do not belong to the sequence load its latest one, or its first one again
    Pack<T, N> f[S];
    const T* pf = gate + p.b * s.gate_b + (t0 - out_of) * s.gate_t + c;
    const T* pd = dout + p.b * s.dout_b + (t0 - out_of) * s.dout_t + c;
    const T* px = input + p.b * s.input_b + (t0 - out_of) * s.input_t + c;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const bool on = j >= out_of && j < here - 1;
      f[j] = load<N>(pf);
      d[j] = load<N>(pd);
      pf -= on ? s.gate_t : 0;
      pd -= on ? s.dout_t : 0;
    }
    const T* pb = out + p.b * s.out_b + max(t0 - out_of - 1, (int64_t)0) * s.out_t + c;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      x[j] = load<N>(px);
      before[j] = load<N>(pb);
      px -= j >= out_of && j < here - 1 ? s.input_t : 0;
      pb -= j >= out_of && j < here - 1 && t0 - j - 1 > 0 ? s.out_t : 0;
    }
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const bool on = j >= out_of && j < here;
      const F32<N> ff = widen<T, N>(f[j]), dd = widen<T, N>(d[j]);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Gates k = gates(ff[i]);
        a[j][i] = on ? k.a : 1.f;
        z[j][i] = k.z;
        A[i] *= (double)a[j][i];
        H[i] = (double)a[j][i] * (H[i] + (on ? (double)dd[i] : 0.0));
      }
    }
  }
  if (dlast && p.chunk == 0) first = widen<float, N>(load<N>(dlast + ends));
  state = chunk_state<N>(slots, p, A, H, first, fold);
  if (!mine) return;
  F32<N> h_first = {};
  if (h0 && here > 0 && t0 - here + 1 == 0) h_first = widen<float, N>(load<N>(h0 + ends));
  T* og = dgate + p.b * s.dgate_b + t0 * s.dgate_t + c;
  T* ox = dinput + p.b * s.dinput_b + t0 * s.dinput_t + c;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    if (j < here) {
      F32<N> dg = {}, dx = {};
      if (j >= out_of) {
        const F32<N> total = state + widen<T, N>(d[j]), xx = widen<T, N>(x[j]);
        const F32<N> h = t0 - j > 0 ? widen<T, N>(before[j]) : h_first;
        dx = z[j] * total;
        dg = (h - xx) * a[j] * dx;
        state = a[j] * total;
      }
      store<T, N>(og, dg);
      store<T, N>(ox, dx);
    }
    og -= s.dgate_t;
    ox -= s.dinput_t;
  }
  if (dh0 && p.chunk == slots.chunks - 1 && w == waves - 1) store<float, N>(dh0 + ends, state);
}

}  // namespace accop
