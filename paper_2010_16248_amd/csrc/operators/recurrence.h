// Gated linear recurrence h_t = a_t h_{t-1} + z_t x_t, a = sigmoid(gate), z = sigmoid(-gate): forward and backward pass.
#pragma once
#include "op_common.h"

namespace accop {

struct RecurrenceShape {
  int64_t steps, channels;
  int64_t gate_b, gate_t, input_b, input_t, out_b, out_t;
  int64_t dgate_b, dgate_t, dinput_b, dinput_t, dout_b, dout_t;
};

// e^-x for x >= 0 (NaN for NaN), times 2^32 where `far`: 2^t of the rounded t = -x log2(e), times e^d with d = -x - t ln 2, what the
// rounding lost (d is below 2^-16, so e^d = 1 + d; ln 2 rounded to fp32 is off by 1.9e-9, times t): within 4 units of 2^-24 up to
// x = 20, 7 beyond.  The power's instruction gives zero below 2^-126, so the last ones are taken 2^32 times as large.
__device__ __forceinline__ float exp_neg(float x, bool* far) {
  x = x > 104.f ? 104.f : x;              // below half the smallest fp32 number from there on
  const float t = -1.44269502f * x;
  *far = t < -125.f;
  const float d = fmaf(t, -0.693147182f, -x);
  const float e = __builtin_amdgcn_exp2f(*far ? t + 32.f : t);
  return fmaf(e, d, e);
}

// sigmoid(f) and sigmoid(-f).  Neither is a difference from one: a gate near one keeps all digits of 1 - a.
struct Gates {
  float a, z;
};
__device__ __forceinline__ Gates gates(float f) {
  bool far;
  const float e = exp_neg(fabsf(f), &far);
  const float d = 1.f + e;                // 1 where far, and so is big
  float big = __builtin_amdgcn_rcpf(d);
  big = fmaf(fmaf(-d, big, 1.f), big, big);
  const float small = e * (far ? 0x1p-32f : big);
  return f >= 0.f ? Gates{big, small} : Gates{small, big};
}

__device__ __forceinline__ int64_t steps_of(const int32_t* lengths, int64_t batch, int64_t steps) {
  if (!lengths) return steps;
  const int64_t n = lengths[batch];
  return n < 0 ? 0 : (n < steps ? n : steps);
}

// ---- a lane per N channels, step after step ---------------------------------------------------------------
// For sequences of up to 16 steps: bound by the launch (64 x 1 x 672 fp32 3.2 us) and the steps' latency (64 x 16 x 672 fp32 forward 6.4,
// backward 7.2).
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
// their maps in registers, a workgroup has up to kChunkWaves waves; so the inputs are read once.  Where a sequence has
// several chunks, they meet in the workspace, in groups of kChunkGroup:
//   a chunk leaves its map there and takes those of the chunks in front of it in its group,
//   the last one of a group also leaves the group's map, and the state at the group's end once it has its start,
//   the state at a group's start is the nearest state found in front of it, taken through the groups' maps in between.
// Whatever a chunk finds, it starts from the same fold of the same maps in the same order: the bits do not depend on who was
// faster.
//
// Maps and the states between waves are fp64: composed maps meet in differences (A h against H) that the steps one by
// one do not have, and so a wave starts from the state that steps without rounding would have reached.
//
// Chunks are handed out by a counter in the order of the steps, so that all chunks a workgroup waits for have
// been taken by workgroups that run already.  Chunks' maps wait for nothing, groups' maps for chunks' maps alone, and of the
// groups without a state at their end the first one finds the one in front of it: every wait ends.
//
// A word of the workspace holds a value and the news that it is there at once (all ones: not yet); its accesses are
// atomic and go past the caches that compute units do not share.
//
// Bound by memory with some 35 (forward) and 55 (backward) vector instructions per element beside it.  us: 1 x 65536 x 672 fp32 forward 111
// (4.7 TB/s), backward 217 (4.9); 8 x 4096 x 2048 bf16 forward 93 (4.3), backward 172 (4.7).  With sixteen waves 124, 215, 153, 198, with
// four 370, 331, 224, 296 (before the groups); steps per wave: as many as the registers hold.  Of these, keeping products of open gates above
// zero costs 1 %, gates below the normal numbers another 1 to 2.
constexpr int kChunkWaves = 8;        // most waves of a workgroup; all of them where there are several chunks
constexpr int kChunkGroup = 8;        // a wave for every chunk in front of the group's last one
constexpr int kLookBack = 4;          // groups looked at in one go
constexpr unsigned long long kNotYet = ~0ull;

template <int N>
using F64 = double __attribute__((ext_vector_type(N)));

// A product of gates must not become zero unless a gate is: an infinite state stays infinite through any number of gates above zero, and
// meets no 0 x infinity.  (Below 2^-1022 its size plays no other role.)
constexpr double kLeastGates = 0x1p-1022;
__device__ __forceinline__ double keep_gates(double product, bool shut) { return product == 0.0 && !shut ? kLeastGates : product; }

struct ChunkSlots {
  unsigned long long *map_a, *map_h;             // per chain, chunk and channel
  unsigned long long *group_a, *group_h, *state; // per chain, group and channel: the group's map, the state at its end
  uint32_t* counter;                             // chunks handed out
  int64_t chains, channel_blocks;                // (sequence, block of 64 N channels)
  int chunks, groups;
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
__device__ __forceinline__ double value(unsigned long long word) { return __longlong_as_double((long long)word); }

// The state at the start of group `group` > 0 of one channel per lane.  slot0: the channel's slot in group 0, pitch: slots per
// group.
__device__ __forceinline__ double look_back(const ChunkSlots& s, int64_t slot0, int64_t pitch, int group) {
  const int most = min(group, kLookBack);
  for (;;) {
    unsigned long long st[kLookBack];
#pragma unroll
    for (int q = 0; q < kLookBack; ++q) st[q] = look(s.state + slot0 + (int64_t)(group - 1 - min(q, most - 1)) * pitch);
    int at = -1;
    double h = 0.0;
#pragma unroll
    for (int q = kLookBack - 1; q >= 0; --q)
      if (q < most && __ballot(st[q] == kNotYet) == 0) {
        at = q;
        h = value(st[q]);
      }
    if (at == 0) return h;
    if (at > 0) {
      unsigned long long a[kLookBack - 1], b[kLookBack - 1];
#pragma unroll
      for (int q = 0; q < kLookBack - 1; ++q) {
        const int64_t slot = slot0 + (int64_t)(group - 1 - min(q, at - 1)) * pitch;
        a[q] = look(s.group_a + slot);
        b[q] = look(s.group_h + slot);
      }
      bool all = true;
#pragma unroll
      for (int q = kLookBack - 2; q >= 0; --q)
        if (q < at) {
          all = all && a[q] != kNotYet && b[q] != kNotYet;
          h = fma(value(a[q]), h, value(b[q]));
        }
      if (__ballot(!all) == 0) return h;
    }
    __builtin_amdgcn_s_sleep(1);
  }
}

// Where a workgroup works: which chunk of which chain.
struct ChunkPlace {
  int chunk;
  uint32_t chain;
  int64_t b, c, left;                 // sequence, the lane's first channel, channels from there on
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
  p.chain = ticket % (uint32_t)s.chains;
  p.b = p.chain / (uint32_t)s.channel_blocks;
  p.c = (int64_t)(p.chain % (uint32_t)s.channel_blocks) * (kWave * N) + (threadIdx.x & 63) * N;
  p.left = shape.channels - p.c;
  return p;
}

// Per channel of the workgroup's block: the maps of its waves, those of the chunks in front of it in its group, the state at its start.
template <int N>
struct ChunkFold {
  double a[kChunkWaves][kWave * N], h[kChunkWaves][kWave * N];
  double before_a[kChunkGroup - 1][kWave * N], before_h[kChunkGroup - 1][kWave * N];
  double start[kWave * N];
};

// From the waves' maps to the state at this wave's start.  first: the state at the chain's start (used in its first group only; wave 0
// has read it before the chunk leaves its map, so the last chunk may write over it).
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
    const int group = p.chunk / kChunkGroup, at = p.chunk % kChunkGroup, ch = w * kWave + l;
    const int64_t slot0 = (int64_t)p.chain * s.chunks * pitch, group0 = (int64_t)p.chain * s.groups * pitch;
    const bool ends = at == kChunkGroup - 1 && group + 1 < s.groups;   // other groups build on this chunk
    double A = 1.0, H = 0.0;
    if (w < N) {                       // a wave for every 64 channels
      bool shut = false;
#pragma unroll 2
      for (int k = 0; k < waves; ++k) {
        const double ak = fold.a[k][ch];
        A *= ak;
        shut |= ak == 0.0;
        H = fma(ak, H, fold.h[k][ch]);
      }
      A = keep_gates(A, shut);
      if (at < kChunkGroup - 1 && p.chunk + 1 < s.chunks) {
        leave(s.map_a + slot0 + (int64_t)p.chunk * pitch + ch, A);
        leave(s.map_h + slot0 + (int64_t)p.chunk * pitch + ch, H);
      }
    }
    if (w < at) {
      const int64_t slot = slot0 + (int64_t)(p.chunk - at + w) * pitch + l;
      for (;;) {
        unsigned long long a[N], b[N];
        bool all = true;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          a[i] = look(s.map_a + slot + i * kWave);
          b[i] = look(s.map_h + slot + i * kWave);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
          all = all && a[i] != kNotYet && b[i] != kNotYet;
          fold.before_a[w][l + i * kWave] = value(a[i]);
          fold.before_h[w][l + i * kWave] = value(b[i]);
        }
        if (__ballot(!all) == 0) break;
        __builtin_amdgcn_s_sleep(1);
      }
    }
    __syncthreads();
    if (w < N) {
      const int64_t slot = group0 + (int64_t)group * pitch + ch;
      if (ends) {
        double GA = 1.0, GH = 0.0;
        bool shut = A == 0.0;
#pragma unroll 2
        for (int k = 0; k < at; ++k) {
          GA *= fold.before_a[k][ch];
          shut |= fold.before_a[k][ch] == 0.0;
          GH = fma(fold.before_a[k][ch], GH, fold.before_h[k][ch]);
        }
        A = keep_gates(A * GA, shut);
        H = fma(fold.a[0][ch], GH, fold.h[0][ch]);
#pragma unroll 2
        for (int k = 1; k < waves; ++k) H = fma(fold.a[k][ch], H, fold.h[k][ch]);
        if (group > 0) {
          leave(s.group_a + slot, A);
          leave(s.group_h + slot, H);
        }
      }
      double h = group > 0 ? look_back(s, group0 + ch, pitch, group) : fold.start[ch];
      if (ends) leave(s.state + slot, fma(A, h, H));
#pragma unroll 2
      for (int k = 0; k < at; ++k) h = fma(fold.before_a[k][ch], h, fold.before_h[k][ch]);
      fold.start[ch] = h;
    }
    __syncthreads();
  }
  F64<N> h;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    h[i] = fold.start[l * N + i];
#pragma unroll 2
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

// A lane has all of its N channels or none (it then works on the first ones and stores nothing) -- or, of an odd number of channels
// (ODD, N = 2), the last one alone: it loads the one in front of it too, takes its own for both and stores one.
// (bf16, one channel per lane instead: 32 x 757 x 1717 backward 226 us, this way 163.)
template <typename T, int N, bool ODD>
__device__ __forceinline__ F32<N> lane_values(const Pack<T, N>& v, bool alone) {
  F32<N> f = widen<T, N>(v);
  if (ODD && alone) f[0] = f[N - 1];
  return f;
}
template <typename T, int N, bool ODD, bool STREAM>
__device__ __forceinline__ void store_lane(T* p, const F32<N>& v, bool alone) {
  if (ODD && alone) *p = (T)v[0];
  else if (STREAM) store_stream<T, N>(p, v);
  else store<T, N>(p, v);
}

// WHOLE: every step of the chunk belongs to the sequence.  STREAM: outputs go past the caches, where rows start on whole pieces of memory
// (64 x 512 x 1024 fp32 backward 160 -> 153 us; 35 x 5659 x 317 forward 213 -> 226, 32 x 757 x 1717 bf16 backward 151 -> 161: not there).
template <typename T, int N, int S, bool ODD, bool STREAM, bool WHOLE>
__device__ __forceinline__ void forward_chunk(const RecurrenceShape& s, const ChunkSlots& slots, const ChunkPlace& p, ChunkFold<N>& fold,
                                              const T* gate, const T* input, const float* h0, int64_t len, T* out, float* h_last) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const bool mine = p.left > 0, alone = ODD && p.left == 1;
  const int64_t c = mine ? p.c - (alone ? 1 : 0) : 0, ends = p.b * s.channels + c;
  const int64_t t0 = ((int64_t)p.chunk * waves + w) * S;
  const int in = WHOLE ? S : (int)min((int64_t)S, max(len - t0, (int64_t)0));          // steps of the sequence
  const int here = WHOLE ? S : (int)min((int64_t)S, max(s.steps - t0, (int64_t)0));    // steps of the tensors
  F32<N> a[S], b[S], first = {}, least = F32<N>{} + 1.f;
  F64<N> A = F64<N>{} + 1.0, H = {};
  if (in > 0) {
    Pack<T, N> f[S], v[S];
    load_steps<T, N, S>(f, gate + p.b * s.gate_b + t0 * s.gate_t + c, s.gate_t, in - 1);
    load_steps<T, N, S>(v, input + p.b * s.input_b + t0 * s.input_t + c, s.input_t, in - 1);
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const F32<N> ff = lane_values<T, N, ODD>(f[j], alone), xx = lane_values<T, N, ODD>(v[j], alone);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Gates k = gates(ff[i]);
        a[j][i] = j < in ? k.a : 1.f;
        b[j][i] = j < in ? k.z * xx[i] : 0.f;
        A[i] *= (double)a[j][i];
        least[i] = fminf(least[i], a[j][i]);
        H[i] = fma((double)a[j][i], H[i], (double)b[j][i]);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) A[i] = keep_gates(A[i], least[i] == 0.f);
  }
  if (h0 && p.chunk < kChunkGroup) first = lane_values<float, N, ODD>(load<N>(h0 + ends), alone);
  F32<N> h = chunk_state<N>(slots, p, A, H, first, fold);
  if (!mine) return;
  T* o = out + p.b * s.out_b + t0 * s.out_t + p.c;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    if (j < in) {
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = fmaf(a[j][i], h[i], b[j][i]);
      store_lane<T, N, ODD, STREAM>(o, h, alone);
    } else if (j < here) {
      store_lane<T, N, ODD, STREAM>(o, F32<N>{}, alone);
    }
    o += s.out_t;
  }
  if (h_last && p.chunk == slots.chunks - 1 && w == waves - 1) store_lane<float, N, ODD, false>(h_last + p.b * s.channels + p.c, h, alone);
}

template <typename T, int N, int S, bool ODD, bool STREAM>
__global__ __launch_bounds__(kWave* kChunkWaves, 3) void recurrence_forward_chunk_kernel(
    RecurrenceShape s, ChunkSlots slots, const T* __restrict__ gate, const T* __restrict__ input, const float* h0,
    const int32_t* __restrict__ lengths, T* __restrict__ out, float* h_last) {
  __shared__ ChunkFold<N> fold;
  __shared__ uint32_t ticket;
  const ChunkPlace p = chunk_place<N>(slots, s, &ticket);
  const int64_t len = steps_of(lengths, p.b, s.steps), per = (int64_t)(blockDim.x >> 6) * S;
  if ((p.chunk + 1) * per <= len) forward_chunk<T, N, S, ODD, STREAM, true>(s, slots, p, fold, gate, input, h0, len, out, h_last);
  else forward_chunk<T, N, S, ODD, STREAM, false>(s, slots, p, fold, gate, input, h0, len, out, h_last);
}

// Backward in time: the state is c_t = a_t G_t, the gradient of h_{t-1}; c_t = a_t c_{t+1} + a_t grad_out_t.  Steps are counted from
// the last one on.  WHOLE: every step of the chunk belongs to the sequence and none is its first.
template <typename T, int N, int S, bool ODD, bool STREAM, bool WHOLE>
__device__ __forceinline__ void backward_chunk(const RecurrenceShape& s, const ChunkSlots& slots, const ChunkPlace& p, ChunkFold<N>& fold,
                                               const T* gate, const T* input, const T* out, const float* h0, int64_t len, const T* dout,
                                               const float* dlast, T* dgate, T* dinput, float* dh0) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const bool mine = p.left > 0, alone = ODD && p.left == 1;
  const int64_t c = mine ? p.c - (alone ? 1 : 0) : 0, ends = p.b * s.channels + c;
  const int64_t t0 = s.steps - 1 - ((int64_t)p.chunk * waves + w) * S;                          // the wave's latest step
  const int here = WHOLE ? S : (int)min((int64_t)S, max(t0 + 1, (int64_t)0));                   // steps of the tensors: j < here
  const int out_of = WHOLE ? 0 : (int)min((int64_t)here, max(t0 + 1 - len, (int64_t)0));        // of the sequence: out_of <= j
  F32<N> a[S], z[S], first = {}, least = F32<N>{} + 1.f, state;
  F64<N> A = F64<N>{} + 1.0, H = {};
  Pack<T, N> d[S], x[S], before[S];
  if (out_of < here) {
    // steps that do not belong to the sequence load its latest one, or its first one again
    Pack<T, N> f[S];
    const T* pf = gate + p.b * s.gate_b + (t0 - out_of) * s.gate_t + c;
    const T* pd = dout + p.b * s.dout_b + (t0 - out_of) * s.dout_t + c;
    const T* px = input + p.b * s.input_b + (t0 - out_of) * s.input_t + c;
    const T* pb = out + p.b * s.out_b + (WHOLE ? t0 - 1 : max(t0 - out_of - 1, (int64_t)0)) * s.out_t + c;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const bool on = j >= out_of && j < here - 1;
      f[j] = load<N>(pf);
      d[j] = load<N>(pd);
      pf -= on ? s.gate_t : 0;
      pd -= on ? s.dout_t : 0;
    }
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const bool on = j >= out_of && j < here - 1;
      x[j] = load<N>(px);
      before[j] = load<N>(pb);
      px -= on ? s.input_t : 0;
      pb -= on && (WHOLE || t0 - j - 1 > 0) ? s.out_t : 0;
    }
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const bool on = j >= out_of && j < here;
      const F32<N> ff = lane_values<T, N, ODD>(f[j], alone), dd = lane_values<T, N, ODD>(d[j], alone);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Gates k = gates(ff[i]);
        a[j][i] = on ? k.a : 1.f;
        z[j][i] = k.z;
        A[i] *= (double)a[j][i];
        least[i] = fminf(least[i], a[j][i]);
        H[i] = (double)a[j][i] * (H[i] + (on ? (double)dd[i] : 0.0));
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) A[i] = keep_gates(A[i], least[i] == 0.f);
  }
  if (dlast && p.chunk < kChunkGroup) first = lane_values<float, N, ODD>(load<N>(dlast + ends), alone);
  state = chunk_state<N>(slots, p, A, H, first, fold);
  if (!mine) return;
  F32<N> h_first = {};
  if (!WHOLE && h0 && here > 0 && t0 - here + 1 == 0) h_first = lane_values<float, N, ODD>(load<N>(h0 + ends), alone);
  T* og = dgate + p.b * s.dgate_b + t0 * s.dgate_t + p.c;
  T* ox = dinput + p.b * s.dinput_b + t0 * s.dinput_t + p.c;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    if (j < here) {
      F32<N> dg = {}, dx = {};
      if (j >= out_of) {
        const F32<N> total = state + lane_values<T, N, ODD>(d[j], alone), xx = lane_values<T, N, ODD>(x[j], alone);
        const F32<N> h = WHOLE || t0 - j > 0 ? lane_values<T, N, ODD>(before[j], alone) : h_first;
        dx = z[j] * total;
        dg = (h - xx) * a[j] * dx;
        state = a[j] * total;
      }
      store_lane<T, N, ODD, STREAM>(og, dg, alone);
      store_lane<T, N, ODD, STREAM>(ox, dx, alone);
    }
    og -= s.dgate_t;
    ox -= s.dinput_t;
  }
  if (dh0 && p.chunk == slots.chunks - 1 && w == waves - 1) store_lane<float, N, ODD, false>(dh0 + p.b * s.channels + p.c, state, alone);
}

template <typename T, int N, int S, bool ODD, bool STREAM>
__global__ __launch_bounds__(kWave* kChunkWaves, 3) void recurrence_backward_chunk_kernel(
    RecurrenceShape s, ChunkSlots slots, const T* __restrict__ gate, const T* __restrict__ input, const T* __restrict__ out,
    const float* __restrict__ h0, const int32_t* __restrict__ lengths, const T* __restrict__ dout, const float* __restrict__ dlast,
    T* __restrict__ dgate, T* __restrict__ dinput, float* __restrict__ dh0) {
  __shared__ ChunkFold<N> fold;
  __shared__ uint32_t ticket;
  const ChunkPlace p = chunk_place<N>(slots, s, &ticket);
  const int64_t len = steps_of(lengths, p.b, s.steps), per = (int64_t)(blockDim.x >> 6) * S;
  const int64_t latest = s.steps - p.chunk * per, earliest = latest - per;     // steps [earliest, latest)
  if (latest <= len && earliest > 0)
    backward_chunk<T, N, S, ODD, STREAM, true>(s, slots, p, fold, gate, input, out, h0, len, dout, dlast, dgate, dinput, dh0);
  else
    backward_chunk<T, N, S, ODD, STREAM, false>(s, slots, p, fold, gate, input, out, h0, len, dout, dlast, dgate, dinput, dh0);
}

}  // namespace accop
