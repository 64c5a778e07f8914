// Selective state space scan h_t = exp(dt_t a) h_{t-1} + dt_t b_t x_t, y_t = c_t . h_t + d x_t: forward and backward pass.
#pragma once
#include "op_common.h"
#include "parts.h"

#include <type_traits>

namespace accop {

struct ScanShape {
  int64_t steps, channels;
  int64_t x_b, x_t, delta_b, delta_t, gate_b, gate_t, out_b, out_t;                  // backward: out is grad_out
  int64_t dx_b, dx_t, ddelta_b, ddelta_t, dgate_b, dgate_t;
  int64_t chunk, rows;      // steps of a chunk; rows of a sequence's b and c
  int chunks;
  int states, padded;       // states of a channel, and as many as are held of them
  int groups, group, blocks;// groups, channels of one, blocks of 64 channels of one
  int softplus;
};

// Constant memory: loads at an address that a wave has in common go to its scalar registers.
typedef const float __attribute__((address_space(4))) * Shared;
__device__ __forceinline__ Shared shared_at(const float* p) { return (Shared)(uintptr_t)p; }

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f, kMost = 3.40282347e38f;

// a log2(e), finite where a is: a step of dt = 0 keeps the state.
__device__ __forceinline__ float decay_of(float a) {
  const float v = a * kLog2e;
  return fabsf(v) > kMost ? copysignf(kMost, v) : v;
}

// 2^z h + v, for a power over many steps.  It may be beyond fp32 where its product with h is not: it is applied in two halves.  Zero stays zero, and infinity
// infinite, through steps whose powers are numbers above zero, as theirs all are.  (A z that is no number leaves none.)
__device__ __forceinline__ float carried(float z, float h, float v) {
  const float half = __builtin_amdgcn_exp2f(0.5f * z);
  return h + h == h && fabsf(z) < INFINITY ? h + v : fmaf(h * half, half, v);
}

// log(1 + e^r) = max(r, 0) + log(1 + e), e = e^-|r|, and its derivative, the sigmoid of r.  log(1 + e) = 2 atanh(s), s = e / (2 + e) <= 1/3;
// atanh(s) / s = 1 + z q(z), z = s^2, q of degree 3 with the least largest error (fitted: below 2^-27 of the whole).
struct Softplus {
  float value, slope;
};
__device__ __forceinline__ Softplus softplus(float r) {
  const float x = fminf(fabsf(r), 100.f);
  const float t = -1.44269502f * x;
  const float d = fmaf(t, -0.693147182f, -x);
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e, d, e);
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), z = s * s;
  float q = fmaf(0.140060782f, z, 0.140008867f);
  q = fmaf(q, z, 0.200107649f);
  q = fmaf(q, z, 0.333332092f);
  const float half = fmaf(q * z, s, s), big = __builtin_amdgcn_rcpf(1.f + e);
  return {fmaf(2.f, half, r < 0.f ? 0.f : r), r < 0.f ? e * big : big};
}

// ---- b and c as the scan reads them -----------------------------------------------------------------------
// [batch, group, step]: the states' b, then their c, in fp32, both filled up with zeros; zeros from the sequence's length on, up to whole turns
// of kScanAhead steps.
constexpr int kScanAhead = 8;    // steps of a turn: under way together

// A lane makes four numbers of a row.  65536 x 32 fp32: 5.4 us, of which a launch that does little takes 3.  (All counts are below 2^32: divisions
// of 64 bits took more than half of the time.)
template <typename T>
__global__ __launch_bounds__(256) void scan_pack_kernel(const T* __restrict__ b, const T* __restrict__ c, int64_t b_b, int64_t b_t,
                                                        int64_t c_b, int64_t c_t, unsigned all, int64_t steps, unsigned rows, unsigned groups,
                                                        int states, int padded, int fours_log2, const int32_t* __restrict__ lengths,
                                                        float* __restrict__ to) {
  const unsigned at = blockIdx.x * 256 + threadIdx.x, row = at >> fours_log2;
  if (row >= all) return;
  const int k = (int)(at & ((1u << fours_log2) - 1)) * 4, n = k < padded ? k : k - padded;
  const unsigned rest = row / rows, t = row - rest * rows;
  const int64_t batch = rest / groups, g = rest - (unsigned)batch * groups;
  F32<4> v = {};
  if (n < states && t < steps_of(lengths, batch, steps)) {
    const T* const from = (k < padded ? b + batch * b_b + t * b_t : c + batch * c_b + t * c_t) + g * states + n;
    v = widen<T, 4>(load_some<4>(from, states - n));
  }
  store<float, 4>(to + (int64_t)at * 4, v);
}

// ---- what the passes share --------------------------------------------------------------------------------
// A lane has one channel and NP of its states; a wave 64 channels of a group.  The WAVES waves of a workgroup have NP states each; what the states of
// a channel have in common (dt, dt x, the gradient through the gate) each works out for some of a turn's steps and leaves in LDS, and what they
// contribute to a sum over states they add there.  Steps of a turn that lie beyond the sequence have dt = 0: they change nothing.
// All kernels that walk steps are bound by the vector units: a step of a state takes a power of two (the time of two other instructions), its
// argument, the product with h and those of the pass, for 1 / 16 of the bytes of a step of a channel.  4 states a wave cost the least registers, so that
// other waves run while one waits: a wave of 16 states, which shares nothing, needs 126 registers in scan_ends_kernel backward, 4 waves a SIMD, and
// kept the vector units busy for 0.77 of the time; four waves of 4 states with 74 registers 0.96.

struct ScanPlace {
  int lane, part, group;
  unsigned block, channel;
  unsigned byte2, byte4;         // of the channel's element in a row of 2 and of 4 bytes each
  bool valid;
  int64_t batch, chunk;
  int64_t len, from, to, end;    // steps of the sequence, of the chunk, and where both end
};

__device__ __forceinline__ ScanPlace scan_place(const ScanShape& s, const int32_t* lengths) {
  ScanPlace p;
  p.lane = threadIdx.x & 63;
  p.part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.block = blockIdx.x;
  p.group = (int)(blockIdx.x / (unsigned)s.blocks);
  const int within = (int)(blockIdx.x - (unsigned)p.group * s.blocks) * kWave + p.lane;
  p.valid = within < s.group;
  p.channel = (unsigned)p.group * s.group + (p.valid ? within : s.group - 1);
  p.byte2 = 2 * p.channel;
  p.byte4 = 4 * p.channel;
  p.chunk = blockIdx.y;
  p.batch = blockIdx.z;
  p.len = steps_of(lengths, p.batch, s.steps);
  p.from = p.chunk * s.chunk;
  p.to = min(p.from + s.chunk, s.steps);
  p.end = min(p.to, p.len);
  return p;
}

// A lane's element of rows that the wave has in common: a base in scalar registers and 32 bits of a lane's, as one access takes them.  (The 32
// bits go through an empty statement where the accesses are, or the compiler widens them once for all and adds 64 bits for each.)
struct LaneOf {
  unsigned byte2, byte4;
  __device__ __forceinline__ explicit LaneOf(const ScanPlace& p) : byte2(p.byte2), byte4(p.byte4) {
    asm volatile("" : "+v"(byte2), "+v"(byte4));
  }
  template <typename T>
  __device__ __forceinline__ T& of(T* row) const {
    return *reinterpret_cast<T*>((char*)row + (sizeof(T) == 2 ? byte2 : byte4));
  }
};

// a log2(e) of a lane's states (zero beyond the last).
template <int NP>
__device__ __forceinline__ void load_decay(const ScanShape& s, const ScanPlace& p, const float* a, float (&decay)[NP]) {
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int at = p.part * NP + n;
    decay[n] = at < s.states ? decay_of(a[(int64_t)p.channel * s.states + at]) : 0.f;
  }
}

// States as callers hold them: batch x channels x states.
template <int NP>
__device__ __forceinline__ void load_states(const ScanShape& s, const ScanPlace& p, const float* from, float (&h)[NP]) {
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int at = p.part * NP + n;
    h[n] = from && at < s.states ? from[(p.batch * s.channels + p.channel) * s.states + at] : 0.f;
  }
}
template <int NP>
__device__ __forceinline__ void store_states(const ScanShape& s, const ScanPlace& p, float* to, const float (&h)[NP]) {
  if (!p.valid) return;
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    const int at = p.part * NP + n;
    if (at < s.states) to[(p.batch * s.channels + p.channel) * s.states + at] = h[n];
  }
}
// The workspace's: batch x chunks x states, filled up, x channels.
template <int NP, int WAVES>
__device__ __forceinline__ int64_t slot_of(const ScanShape& s, const ScanPlace& p) {
  return ((p.batch * s.chunks + p.chunk) * (NP * WAVES) + p.part * NP) * s.channels;
}
template <int NP, int WAVES>
__device__ __forceinline__ void load_slots(const ScanShape& s, const ScanPlace& p, const float* from, float (&h)[NP]) {
  const float* at = from + slot_of<NP, WAVES>(s, p);
  const LaneOf lane(p);
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = lane.of(at + n * s.channels);
}
template <int NP, int WAVES>
__device__ __forceinline__ void store_slots(const ScanShape& s, const ScanPlace& p, float* to, const float (&h)[NP]) {
  if (!p.valid) return;
  float* at = to + slot_of<NP, WAVES>(s, p);
  const LaneOf lane(p);
#pragma unroll
  for (int n = 0; n < NP; ++n) lane.of(at + n * s.channels) = h[n];
}

// What scan_ends_kernel leaves in front of the turn at step t.
template <int NP, int WAVES, typename F>
__device__ __forceinline__ F* marks_of(const ScanShape& s, const ScanPlace& p, F* marks, int64_t t) {
  return marks + ((p.batch * (s.rows / kScanAhead) + t / kScanAhead) * (NP * WAVES + 1) + p.part * NP) * s.channels;
}

// The values of one step that a wave reads: c, and b where the pass needs it.
template <int NP, int WAVES, bool B>
struct SharedRow {
  float b[B ? NP : 1], c[NP];
  __device__ __forceinline__ void load(Shared at) {
    if (B) {
#pragma unroll
      for (int n = 0; n < NP; ++n) b[n] = at[n];
    }
#pragma unroll
    for (int n = 0; n < NP; ++n) c[n] = at[NP * WAVES + n];
  }
};
// Where a wave's values of the sequence's first step lie.
template <int NP, int WAVES>
__device__ __forceinline__ int64_t rows_of(const ScanShape& s, const ScanPlace& p) {
  return (p.batch * s.groups + p.group) * s.rows * (2 * NP * WAVES) + p.part * NP;
}
template <int NP, int WAVES>
__device__ __forceinline__ Shared shared_rows(const ScanShape& s, const ScanPlace& p, const float* bc) {
  return shared_at(bc) + rows_of<NP, WAVES>(s, p);
}
// What products along the states take comes through scalar registers.  Rows are requested in groups of as many as 16 of them hold (at least
// one), a group ahead.  Scalar loads return in any order, so a wait for one is a wait for all: a group is awaited before the next one is
// requested, which the compiler's own waits, at first use, would not do.  The stops keep the scheduler from gathering more rows than the scalar
// registers hold.
__device__ __forceinline__ void stop() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ void await_shared() {
  stop();
  __builtin_amdgcn_s_waitcnt(0xc07f);        // lgkmcnt(0), the others as they are
  stop();
}
// Values are worked out here, not where they are used: a step that the compiler has moved behind a later branch finds its row gone from the
// scalar registers.
template <int N>
__device__ __forceinline__ void pin(float (&v)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) asm volatile("" : "+v"(v[n]));
}
__device__ __forceinline__ void pin(float& v) { asm volatile("" : "+v"(v)); }
// Whether there is a NaN among some values (or infinities of both signs).
template <int N>
__device__ __forceinline__ bool has_nan(const float (&v)[N]) {
  float sum = v[0];
#pragma unroll
  for (int n = 1; n < N; ++n) sum += v[n];
  return sum != sum;
}
template <int NP, int WAVES, bool B>
struct SharedGroup {
  static constexpr int kRow = 2 * NP * WAVES;
  static constexpr int kCount = NP * (B ? 2 : 1) >= 16 ? 1 : NP * (B ? 2 : 1) >= 8 ? 2 : 4;
  SharedRow<NP, WAVES, B> row[kCount];
  __device__ __forceinline__ void load(Shared at) {
#pragma unroll
    for (int k = 0; k < kCount; ++k) row[k].load(at + k * kRow);
  }
};

// Products of a step's b or c, which the channels share, with a value of each channel's: what a matrix instruction of 16 blocks of 4 states x 4
// channels makes of 4 numbers and 64, and adds to 4 states of 64 channels, a lane's own, at the issue of one vector instruction for 4.  The numbers
// of a turn lie with the lanes of one register: lane l has state l % NP of step l / NP.  The instruction takes those of the four lanes it names for
// all its blocks.  (8 x 4096 x 2048, 16 states, bf16: with products and sums by vector instructions the ends of the backward pass took 411 us, with these and
// nothing else changed 374.)
template <int NP>
struct HeldRows {
  static_assert(NP * kScanAhead <= kWave, "a turn's numbers in one register");
  float v;
  __device__ __forceinline__ void load(const float* rows, int row, int lane) {
    v = rows[(unsigned)min(lane / NP, kScanAhead - 1) * row + lane % NP];
  }
};
template <int FROM>
__device__ __forceinline__ F32<4> four_states(float held, float u, F32<4> add) {
  return __builtin_amdgcn_mfma_f32_4x4x1f32(held, u, add, 4, FROM, 0);
}
// add + (step j's numbers of the q-th four states) u.  (j and q are known when this is compiled.)
template <int NP>
__device__ __forceinline__ F32<4> add_products(const HeldRows<NP>& held, int j, int q, float u, F32<4> add) {
  const float v = held.v;
  switch (j * (NP / 4) + q) {
    case 0: return four_states<0>(v, u, add);
    case 1: return four_states<1>(v, u, add);
    case 2: return four_states<2>(v, u, add);
    case 3: return four_states<3>(v, u, add);
    case 4: return four_states<4>(v, u, add);
    case 5: return four_states<5>(v, u, add);
    case 6: return four_states<6>(v, u, add);
    case 7: return four_states<7>(v, u, add);
    case 8: return four_states<8>(v, u, add);
    case 9: return four_states<9>(v, u, add);
    case 10: return four_states<10>(v, u, add);
    case 11: return four_states<11>(v, u, add);
    case 12: return four_states<12>(v, u, add);
    case 13: return four_states<13>(v, u, add);
    case 14: return four_states<14>(v, u, add);
    default: return four_states<15>(v, u, add);
  }
}

// Runs f with the number of a wave's states that there are, `own` of NP (WHOLE: all waves have NP).  Those that fill up have no part in sums over states: what
// is zero beside finite numbers is not beside an infinite input or step.  (us with them in the sums and without, 4 x 2048 x 1024 bf16: forward 7 states 59.7, 61.3;
// 40 states 207, 200; backward 7 states 145.6, 144.6; 40 states 601, 539.)
template <int NP, bool WHOLE, int N = NP, typename F>
__device__ __forceinline__ void with_states(int own, F&& f) {
  if constexpr (WHOLE || N == 0) {
    f(std::integral_constant<int, N>());
  } else {
    if (own >= N) f(std::integral_constant<int, N>());
    else with_states<NP, WHOLE, N - 1>(own, f);
  }
}

// The last of a turn's steps that there is.
__device__ __forceinline__ int last_of(const ScanPlace& p, int64_t t) { return (int)min(p.end - 1 - t, (int64_t)kScanAhead - 1); }

// ---- chunks: what each does to a state --------------------------------------------------------------------
// The state behind a chunk that starts from zero, the sum of its dt (the state in front decays by exp(a sum)) and, for the backward pass,
// the gradient of the state in front of it if nothing came from behind, and in marks the state and the sum in front of each of its turns
// (batch x turns x (states, filled up, + 1) x channels).
// 8 x 4096 x 2048, 16 states, bf16: backward 351 us, vector units busy for 0.96 of them, 5 % of the time with matrix instructions beside; 65536 x 672 fp32:
// forward 150 us, 0.99.  (Minimum of four waves a SIMD: without one the matrix instructions' sums go to registers that vector instructions cannot take.)
template <typename T, int NP, int WAVES, bool BACKWARD>
__global__ __launch_bounds__(WAVES * kWave, 4) void scan_ends_kernel(ScanShape s, const T* __restrict__ x, const T* __restrict__ delta,
                                                                     const float* __restrict__ a, const float* __restrict__ bc,
                                                                     const T* __restrict__ gate, const float* __restrict__ delta_bias,
                                                                     const int32_t* __restrict__ lengths, const T* __restrict__ dout,
                                                                     float* __restrict__ ends, float* __restrict__ starts,
                                                                     float* __restrict__ sums, float* __restrict__ marks) {
  constexpr int U = kScanAhead, SHARE = U / WAVES, KINDS = BACKWARD ? 3 : 2;
  __shared__ float held[2 * KINDS * U * kWave];         // dt, u and dy of a turn's steps, for two turns
  const ScanPlace p = scan_place(s, lengths);
  float decay[NP], h[NP], g[NP], reach[NP];
  load_decay<NP>(s, p, a, decay);
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    h[n] = g[n] = 0.f;
    reach[n] = 1.f;
  }
  const float shift = delta_bias ? delta_bias[p.channel] : 0.f;
  const T* const xs = x + p.batch * s.x_b;
  const T* const ds = delta + p.batch * s.delta_b;
  const T* const gs = BACKWARD && gate ? gate + p.batch * s.gate_b : nullptr;
  const T* const os = BACKWARD ? dout + p.batch * s.out_b : nullptr;
  constexpr int kRow = 2 * NP * WAVES;
  const float* rows = bc + rows_of<NP, WAVES>(s, p) + p.from * kRow;
  float sum = 0.f;
  HeldRows<NP> next_b, next_c;
  next_b.load(rows, kRow, p.lane);
  if (BACKWARD) next_c.load(rows + NP * WAVES, kRow, p.lane);
  T xn[SHARE], dn[SHARE], gn[SHARE], on[SHARE];         // this wave's steps of the turn ahead
  auto request = [&](int64_t t) {
    const LaneOf lane(p);
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const int64_t at = min(t + p.part * SHARE + k, p.end - 1);
      xn[k] = lane.of(xs + at * s.x_t);
      dn[k] = lane.of(ds + at * s.delta_t);
      if (BACKWARD) on[k] = lane.of(os + at * s.out_t);
      if (gs) gn[k] = lane.of(gs + at * s.gate_t);
    }
  };
  if (p.from < p.end) request(p.from);
  int turn = 0;
  for (int64_t t = p.from; t < p.end; t += U) {
    const int last = last_of(p, t);
    float* const common = held + (turn & 1) * KINDS * U * kWave + p.lane;
    ++turn;
    float step[SHARE], dy_of[SHARE];
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      step[k] = (float)dn[k] + shift;
      if (BACKWARD) dy_of[k] = (float)on[k];
    }
    if (s.softplus) {
#pragma unroll
      for (int k = 0; k < SHARE; ++k) step[k] = softplus(step[k]).value;
    }
    if (gs) {
#pragma unroll
      for (int k = 0; k < SHARE; ++k) dy_of[k] *= (float)gn[k] * sigmoid((float)gn[k]).a;
    }
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const bool in = p.part * SHARE + k <= last;
      float* const to = common + (p.part * SHARE + k) * KINDS * kWave;
      to[0] = in ? step[k] : 0.f;
      to[kWave] = in ? step[k] * (float)xn[k] : 0.f;
      if (BACKWARD) to[2 * kWave] = in ? dy_of[k] : 0.f;
    }
    if (BACKWARD && p.valid && t > p.from) {
      float* to = marks_of<NP, WAVES>(s, p, marks, t);
      const LaneOf lane(p);
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        lane.of(to) = h[n];
        to += s.channels;
      }
      if (p.part == 0) lane.of(to + (WAVES - 1) * NP * s.channels) = sum;
    }
    if (t + U < p.end) request(t + U);
    if (WAVES > 1) __syncthreads();
    float dt[U], u[U], dy[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      dt[j] = common[j * KINDS * kWave];
      u[j] = common[(j * KINDS + 1) * kWave];
      if (BACKWARD) dy[j] = common[(j * KINDS + 2) * kWave];
    }
    const HeldRows<NP> b_of = next_b, c_of = next_c;
    rows += U * kRow;
    next_b.load(rows, kRow, p.lane);
    if (BACKWARD) next_c.load(rows + NP * WAVES, kRow, p.lane);
    if (p.part == 0) {
#pragma unroll
      for (int j = 0; j < U; ++j) sum += dt[j];
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
#pragma unroll
      for (int q = 0; q < NP / 4; ++q) {
        F32<4> h4, from = {};
        if (BACKWARD) from = add_products<NP>(c_of, j, q, dy[j], from);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = 4 * q + i;
          const float e = __builtin_amdgcn_exp2f(dt[j] * decay[n]);
          h4[i] = e * h[n];
          if (BACKWARD) {
            reach[n] *= e;
            g[n] = fmaf(reach[n], from[i], g[n]);
          }
        }
        h4 = add_products<NP>(b_of, j, q, u[j], h4);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[4 * q + i] = h4[i];
      }
    }
  }
  // (an infinite gradient may have met a power that the steps in front of it have taken below fp32: once more, power and gradient as they are carried)
  if (BACKWARD && has_nan(g)) {
    const float* row = bc + rows_of<NP, WAVES>(s, p) + p.from * kRow + NP * WAVES;
    const LaneOf lane(p);
    float passed = 0.f;
#pragma unroll
    for (int n = 0; n < NP; ++n) g[n] = 0.f;
    for (int64_t t = p.from; t < p.end; ++t, row += kRow) {
      const float raw = (float)lane.of(ds + t * s.delta_t) + shift;
      float dy = (float)lane.of(os + t * s.out_t);
      if (gs) {
        const float gt = (float)lane.of(gs + t * s.gate_t);
        dy *= gt * sigmoid(gt).a;
      }
      passed += s.softplus ? softplus(raw).value : raw;
#pragma unroll
      for (int n = 0; n < NP; ++n) g[n] = carried(passed * decay[n], row[n] * dy, g[n]);
    }
  }
  store_slots<NP, WAVES>(s, p, ends, h);
  if (BACKWARD) store_slots<NP, WAVES>(s, p, starts, g);
  if (p.valid && p.part == 0) sums[(p.batch * s.chunks + p.chunk) * s.channels + p.channel] = sum;
}

// The state in front of every chunk, in place of the one behind it, and the gradient of the state behind every chunk, in place of that in front.
// A lane has one state of one channel; the waves of a workgroup have runs of consecutive chunks.  Each folds its run, takes what comes out
// of those in front, and walks its run once more.  512 chunks of 672 channels x 16 states: 18.6 us for 70 MB; 16 chunks of 8 x 2048 x 16, both ways: 18 us
// for 67 MB.
constexpr int kCarryAhead = 8;
constexpr int kCarryWaves = 16;

// The state behind `count` chunks (all kCarryAhead at most), of which v are the states behind each from zero and d the sums of dt; put(j, h) takes the one in
// front of the j-th.  First as for any numbers; once more as carried() has it where that left none, or with a power beyond fp32.  (With carried() at once: 512
// chunks of 672 channels x 16 states 20.5 us for 18.6.)
template <typename F>
__device__ __forceinline__ float carry_over(const float (&v)[kCarryAhead], const float (&d)[kCarryAhead], int count, float decay, float h, F&& put) {
  const float front = h;
  float most = 0.f;
#pragma unroll
  for (int j = 0; j < kCarryAhead; ++j)
    if (j < count) {
      const float z = d[j] * decay;
      most = fmaxf(most, z);
      put(j, h);
      h = fmaf(__builtin_amdgcn_exp2f(z), h, v[j]);
    }
  if (h != h || most > 127.f) {
    h = front;
#pragma unroll
    for (int j = 0; j < kCarryAhead; ++j)
      if (j < count) {
        put(j, h);
        h = carried(d[j] * decay, h, v[j]);
      }
  }
  return h;
}

// values: of all chunks, in their order of walking, `step` apart, and so the sums `sum_step`.  Leaves the state in front of each in its place; what lies behind
// the last one is not needed, and in the forward pass not there.
__device__ __forceinline__ void carry_runs(float* values, int64_t step, const float* total, int64_t sum_step, int count, float decay, float h,
                                           bool valid, float (*fold)[2][kWave]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int steps = count - 1, share = (steps + waves - 1) / waves, lo = min(wave * share, steps), hi = min(lo + share, steps);
  if (waves > 1) {
    float end = 0.f, sum = 0.f;
    for (int k = lo; k < hi; k += kCarryAhead) {
      float v[kCarryAhead], d[kCarryAhead];
#pragma unroll
      for (int j = 0; j < kCarryAhead; ++j) {
        const int64_t i = min(k + j, hi - 1);
        v[j] = values[i * step];
        d[j] = total[i * sum_step];
      }
#pragma unroll
      for (int j = 0; j < kCarryAhead; ++j)
        if (k + j < hi) sum += d[j];
      end = carry_over(v, d, hi - k, decay, end, [](int, float) {});
    }
    __syncthreads();
    fold[wave][0][lane] = end;
    fold[wave][1][lane] = sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) h = carried(fold[w][1][lane] * decay, h, fold[w][0][lane]);
  }
  for (int k = lo; k < hi; k += kCarryAhead) {
    float v[kCarryAhead], d[kCarryAhead];
#pragma unroll
    for (int j = 0; j < kCarryAhead; ++j) {
      const int64_t i = min(k + j, hi - 1);
      v[j] = values[i * step];
      d[j] = total[i * sum_step];
    }
    h = carry_over(v, d, hi - k, decay, h, [&](int j, float front) {
      if (valid) values[(k + j) * step] = front;
    });
  }
  if (valid && lo < hi && hi == steps) values[steps * step] = h;
}

template <bool BACKWARD>
__global__ __launch_bounds__(kWave * kCarryWaves) void scan_carry_kernel(ScanShape s, const float* __restrict__ a, const float* __restrict__ h0,
                                                                         const float* __restrict__ dlast, float* ends, float* starts,
                                                                         const float* __restrict__ sums) {
  __shared__ float fold[kCarryWaves][2][kWave];
  const int64_t b = blockIdx.z, at = (int64_t)blockIdx.x * kWave + (threadIdx.x & 63), c = min(at, s.channels - 1);
  // (the gradients' workgroups lie behind the states')
  const bool back = BACKWARD && blockIdx.y >= (unsigned)s.padded;
  const int n = (int)blockIdx.y - (back ? s.padded : 0);
  const bool held = n < s.states, valid = at < s.channels;
  const float decay = held ? decay_of(a[c * s.states + n]) : 0.f;
  const int64_t own = (b * s.channels + c) * s.states + n, step = (int64_t)s.padded * s.channels;
  const int64_t first = (b * s.chunks * s.padded + n) * s.channels + c, last = first + (s.chunks - 1) * step;
  const float* const total = sums + b * s.chunks * s.channels + c;
  if (!back)
    carry_runs(ends + first, step, total, s.channels, s.chunks, decay, held && h0 ? h0[own] : 0.f, valid, fold);
  else
    carry_runs(starts + last, -step, total + (s.chunks - 1) * s.channels, -s.channels, s.chunks, decay, held && dlast ? dlast[own] : 0.f, valid,
               fold);
}

// ---- forward ----------------------------------------------------------------------------------------------
// Each wave finishes the outputs of its steps of a turn.  8 x 4096 x 2048, 16 states, bf16, ragged (0.63 of the steps): 187 us, vector units busy for 0.95
// of them.
template <typename T, int NP, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * kWave, 4) void scan_forward_kernel(
    ScanShape s, const T* __restrict__ x, const T* __restrict__ delta, const float* __restrict__ a, const float* __restrict__ bc,
    const float* __restrict__ d, const T* __restrict__ gate, const float* __restrict__ delta_bias, const int32_t* __restrict__ lengths,
    const float* h0, const float* __restrict__ ends, T* __restrict__ out, float* h_last) {
  constexpr int U = kScanAhead, SHARE = U / WAVES;
  __shared__ float held[(2 + WAVES) * U * kWave];
  const ScanPlace p = scan_place(s, lengths);
  float* const common = held + p.lane;                  // dt and u of a turn's steps
  float* const add = common + 2 * U * kWave;            // what the waves' states contribute to a turn's steps
  const int own = s.states - p.part * NP;
  float decay[NP], h[NP];
  load_decay<NP>(s, p, a, decay);
  if (s.chunks > 1) load_slots<NP, WAVES>(s, p, ends, h);
  else load_states<NP>(s, p, h0, h);
  const float shift = delta_bias ? delta_bias[p.channel] : 0.f, skip = d ? d[p.channel] : 0.f;
  const T* const xs = x + p.batch * s.x_b;
  const T* const ds = delta + p.batch * s.delta_b;
  const T* const gs = gate ? gate + p.batch * s.gate_b : nullptr;
  T* const os = out + p.batch * s.out_b;
  constexpr int kRow = 2 * NP * WAVES;
  Shared rows = shared_rows<NP, WAVES>(s, p, bc) + p.from * kRow;
  const float* held_rows = bc + rows_of<NP, WAVES>(s, p) + p.from * kRow;
  using Group = SharedGroup<NP, WAVES, false>;
  Group next;
  next.load(rows);
  HeldRows<NP> next_b;
  next_b.load(held_rows, kRow, p.lane);
  T xn[SHARE], dn[SHARE], gn[SHARE];                    // this wave's steps of the turn ahead
  auto request = [&](int64_t t) {
    const LaneOf lane(p);
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const int64_t at = min(t + p.part * SHARE + k, p.end - 1);
      xn[k] = lane.of(xs + at * s.x_t);
      dn[k] = lane.of(ds + at * s.delta_t);
      if (gs) gn[k] = lane.of(gs + at * s.gate_t);
    }
  };
  if (p.from < p.end) request(p.from);
  for (int64_t t = p.from; t < p.end; t += U) {
    const int last = last_of(p, t);
    T xv[SHARE], gv[SHARE];
    float step[SHARE];
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      xv[k] = xn[k];
      gv[k] = gn[k];
      step[k] = (float)dn[k] + shift;
    }
    if (s.softplus) {
#pragma unroll
      for (int k = 0; k < SHARE; ++k) step[k] = softplus(step[k]).value;
    }
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const bool in = p.part * SHARE + k <= last;
      float* const to = common + (p.part * SHARE + k) * 2 * kWave;
      to[0] = in ? step[k] : 0.f;
      to[kWave] = in ? step[k] * (float)xv[k] : 0.f;
    }
    if (WAVES > 1) __syncthreads();
    if (t + U < p.end) request(t + U);
    float dt[U], u[U], y[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      dt[j] = common[j * 2 * kWave];
      u[j] = common[(j * 2 + 1) * kWave];
    }
    const HeldRows<NP> b_of = next_b;
    held_rows += U * kRow;
    next_b.load(held_rows, kRow, p.lane);
    with_states<NP, WHOLE>(own, [&](auto count) {
      constexpr int N = decltype(count)::value;
#pragma unroll
      for (int first = 0; first < U; first += Group::kCount) {
        await_shared();
        const Group group = next;
        next.load(rows + (first + Group::kCount) * Group::kRow);
        stop();
#pragma unroll
        for (int k = 0; k < Group::kCount; ++k) {
          const int j = first + k;
          y[j] = 0.f;
#pragma unroll
          for (int q = 0; q < (N + 3) / 4; ++q) {
            F32<4> h4 = {};
#pragma unroll
            for (int i = 0; i < 4 && 4 * q + i < N; ++i) h4[i] = __builtin_amdgcn_exp2f(dt[j] * decay[4 * q + i]) * h[4 * q + i];
            h4 = add_products<NP>(b_of, j, q, u[j], h4);
#pragma unroll
            for (int i = 0; i < 4 && 4 * q + i < N; ++i) {
              h[4 * q + i] = h4[i];
              y[j] = fmaf(group.row[k].c[4 * q + i], h4[i], y[j]);
            }
          }
          pin(y[j]);
        }
        pin(h);
      }
    });
#pragma unroll
    for (int j = 0; j < U; ++j) add[(p.part * U + j) * kWave] = y[j];
    if (WAVES > 1) __syncthreads();
    float r[SHARE];
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      r[k] = 0.f;
#pragma unroll
      for (int o = 0; o < WAVES; ++o) r[k] += add[(o * U + p.part * SHARE + k) * kWave];
      r[k] = fmaf(skip, (float)xv[k], r[k]);
    }
    if (gs) {
#pragma unroll
      for (int k = 0; k < SHARE; ++k) r[k] *= (float)gv[k] * sigmoid((float)gv[k]).a;
    }
    if (p.valid) {
      const LaneOf lane(p);
#pragma unroll
      for (int k = 0; k < SHARE; ++k)
        if (p.part * SHARE + k <= last) lane.of(os + (t + p.part * SHARE + k) * s.out_t) = (T)r[k];
    }
    rows += U * (2 * NP * WAVES);
  }
  if (p.valid && p.part == 0) {
    const LaneOf lane(p);
    for (int64_t t = max(p.from, p.len); t < p.to; ++t) lane.of(os + t * s.out_t) = (T)0.f;
  }
  if (h_last && p.chunk == (p.len > 0 ? (p.len - 1) / s.chunk : 0)) store_states<NP>(s, p, h_last, h);
}

// ---- a few steps: lanes share a channel ----------------------------------------------------------------------
// L lanes have 4 states each of a channel: states come and go in whole pieces of memory.  One token of 64 x 1344 channels x 16 states: 5.1 us, of which
// 11 MB of states at the rate of a large copy are 2.2; a launch that does nothing takes 2.
template <typename T, int L>
__global__ __launch_bounds__(256) void scan_walk_kernel(ScanShape s, const T* __restrict__ x, const T* __restrict__ delta,
                                                        const float* __restrict__ a, const T* __restrict__ b, const T* __restrict__ c,
                                                        int64_t b_b, int64_t b_t, int64_t c_b, int64_t c_t, const float* __restrict__ d,
                                                        const T* __restrict__ gate, const float* __restrict__ delta_bias,
                                                        const int32_t* __restrict__ lengths, const float* h0, T* __restrict__ out,
                                                        float* h_last) {
  const int64_t channel = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L, batch = blockIdx.y;
  const int first = (threadIdx.x % L) * 4;
  if (channel >= s.channels) return;             // all lanes of a channel together
  const int64_t len = steps_of(lengths, batch, s.steps), left = s.states - first, group = channel / s.group;
  F32<4> decay = widen<float, 4>(load_some<4>(a + channel * s.states + first, left));
#pragma unroll
  for (int n = 0; n < 4; ++n) decay[n] = decay_of(decay[n]);
  const int64_t own = (batch * s.channels + channel) * s.states + first;
  F32<4> h = {};
  if (h0) h = widen<float, 4>(load_some<4>(h0 + own, left));
  const float shift = delta_bias ? delta_bias[channel] : 0.f, skip = d ? d[channel] : 0.f;
  for (int64_t t = 0; t < len; ++t) {
    const float xv = (float)x[batch * s.x_b + t * s.x_t + channel];
    const float raw = (float)delta[batch * s.delta_b + t * s.delta_t + channel] + shift;
    const F32<4> bv = widen<T, 4>(load_some<4>(b + batch * b_b + t * b_t + group * s.states + first, left));
    const F32<4> cv = widen<T, 4>(load_some<4>(c + batch * c_b + t * c_t + group * s.states + first, left));
    const float gt = gate ? (float)gate[batch * s.gate_b + t * s.gate_t + channel] : 0.f;
    const float dt = s.softplus ? softplus(raw).value : raw;
    const float u = dt * xv;
    float y = 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      h[n] = fmaf(__builtin_amdgcn_exp2f(dt * decay[n]), h[n], u * bv[n]);
      y = fmaf(cv[n], n < left ? h[n] : 0.f, y);
    }
    if (L > 1) y += dpp<0xB1>(y);
    if (L > 2) y += dpp<0x4E>(y);
    if (L > 4) y += dpp<0x141>(y);
    if (L > 8) y += dpp<0x140>(y);
    if (first == 0) {
      float r = fmaf(skip, xv, y);
      if (gate) r *= gt * sigmoid(gt).a;
      out[batch * s.out_b + t * s.out_t + channel] = (T)r;
    }
  }
  if (first == 0)
    for (int64_t t = len; t < s.steps; ++t) out[batch * s.out_b + t * s.out_t + channel] = (T)0.f;
  if (h_last) store_some<float, 4>(h_last + own, h, left);
}

// ---- backward ---------------------------------------------------------------------------------------------

// Sums over the 64 lanes of V values a lane (16 or 32), which the lanes have put into V rows of LDS, a wave's own: value i ends in the lanes l with
// l / (64 / V) = i.  A lane reads V lanes' of one value and adds them by pairs, the lanes of a value add theirs.  (Rows of 68 numbers: 16 lanes read 16
// pieces of different banks.)  Exchanges between the lanes' registers, half of the values less at every stage, take 35 vector instructions for 16 values where
// this takes 19: 4 x 1024 x 1536 fp32 backward 140 us and 133, 2 x 2048 x 768 with 64 states bf16 244 and 238, 8 x 4096 x 2048 1125 either way.
constexpr int kSumRow = kWave + 4;
// What the wave's lanes have put into LDS is there for its other lanes, and what these have read may be overwritten.  (A wave's accesses to LDS keep their order
// by themselves; this keeps the compiler from changing it, and is no instruction.)
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}
template <int V>
struct LanesSum {
  static_assert(V == 16 || V == 32, "two or four lanes add up a value");
  F32<4> part[V / 4];
  __device__ __forceinline__ void request(const float* room, int l) {
    const float* const from = room + l / (kWave / V) * kSumRow + l % (kWave / V) * V;
    wave_fence();
#pragma unroll
    for (int i = 0; i < V / 4; ++i) part[i] = *reinterpret_cast<const F32<4>*>(from + 4 * i);
    wave_fence();
  }
  __device__ __forceinline__ float sum() {
#pragma unroll
    for (int left = V / 8; left > 0; left /= 2)
#pragma unroll
      for (int i = 0; i < left; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) part[i][k] += part[i + left][k];
    float s = (part[0][0] + part[0][1]) + (part[0][2] + part[0][3]);
    s += dpp<0xB1>(s);
    return V == 16 ? s + dpp<0x4E>(s) : s;
  }
};

// A chunk, from its end: the states of kScanAhead steps at a time are computed from what scan_ends_kernel left in front of them and from the state
// in front of the chunk, kept in registers, and walked back.  (All states of a chunk in LDS would be 32 KB for 8 steps of 64 channels x 16 states.)  Each wave
// finishes the gradients of its steps of a turn.  8 x 4096 x 2048, 16 states, bf16: 820 us, vector units busy for 0.84 of them, at 2.1 GHz and less
// when it runs for long (2.4 where there is less to do at once): what it draws bounds it too.  With a turn's inputs and marks requested where it starts, and not a turn
// ahead, 977 for 858.
// parts: of a chunk, states + 2 rows of channels (grad_a, grad_d, grad_delta_bias); shared_parts: of a block of channels and a step, the
// sums of grad_b and grad_c over the block.
template <typename T, int NP, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * kWave, NP == 4 && WAVES > 2 ? 3 : 2) void scan_backward_kernel(
    ScanShape s, const T* __restrict__ x, const T* __restrict__ delta, const float* __restrict__ a, const float* __restrict__ bc,
    const float* __restrict__ d, const T* __restrict__ gate, const float* __restrict__ delta_bias, const int32_t* __restrict__ lengths,
    const T* __restrict__ dout, const float* __restrict__ h0, const float* __restrict__ dlast, const float* __restrict__ ends,
    const float* __restrict__ starts, const float* __restrict__ marks, T* __restrict__ dx, T* __restrict__ ddelta, T* __restrict__ dgate,
    float* __restrict__ dh0, float* __restrict__ parts, float* __restrict__ shared_parts) {
  constexpr int U = kScanAhead, SHARE = U / WAVES;    // steps of a turn that a wave finishes
  constexpr int row_size = 2 * NP * WAVES;
  const ScanPlace p = scan_place(s, lengths);
  constexpr int kRoom = 4 * NP * kSumRow;
  __shared__ alignas(16) float held[3 * U * kWave * (1 + WAVES) + WAVES * kRoom];
  float* const room = held + 3 * U * kWave * (1 + WAVES) + p.part * kRoom;
  float* const common = held + p.lane;              // dt, u, dy of a turn's steps
  float* const add = common + 3 * U * kWave;        // what the waves' states contribute to a turn's steps
  const int own = s.states - p.part * NP;
  float decay[NP], g[NP], da[NP];
  load_decay<NP>(s, p, a, decay);
  const float shift = delta_bias ? delta_bias[p.channel] : 0.f, skip = d ? d[p.channel] : 0.f;
  const T* const xs = x + p.batch * s.x_b;
  const T* const ds = delta + p.batch * s.delta_b;
  const Shared rows = shared_rows<NP, WAVES>(s, p, bc);
  const int turns = p.end > p.from ? (int)((p.end - p.from + U - 1) / U) : 0;
  const float* const held_rows = bc + rows_of<NP, WAVES>(s, p);
  using Both = SharedGroup<NP, WAVES, true>;
  HeldRows<NP> next_b, next_c;
  {
    const float* const of = held_rows + (p.from + max(turns - 1, 0) * U) * row_size;
    next_b.load(of, row_size, p.lane);
    next_c.load(of + NP * WAVES, row_size, p.lane);
  }
  if (s.chunks > 1) load_slots<NP, WAVES>(s, p, starts, g);
  else load_states<NP>(s, p, dlast, g);
  const T* const gs = gate ? gate + p.batch * s.gate_b : nullptr;
  const T* const os = dout + p.batch * s.out_b;
  float dskip = 0.f, dshift = 0.f;
#pragma unroll
  for (int n = 0; n < NP; ++n) da[n] = 0.f;
  // Where a lane puts what it adds to sums over channels.  Lanes without a channel put it behind the row, and zeros into their places: beside infinity their
  // products are not zero.
  const int column = p.valid ? p.lane : kWave;
  if (!p.valid) {
#pragma unroll
    for (int i = 0; i < 4 * NP; ++i) room[i * kSumRow + p.lane] = 0.f;
  }
  // where a lane's sum of two steps goes: the later one's come first
  const int sum_of = p.lane / (kWave / (4 * NP)), value = sum_of % (2 * NP);
  float* const shared_to = shared_parts + (p.batch * s.groups * s.blocks + p.block) * s.rows * row_size + (sum_of < 2 * NP ? row_size : 0) +
                           p.part * NP + (value < NP ? value : NP * WAVES + value - NP);
  float start[NP];                                  // the state in front of the chunk
  if (s.chunks > 1) load_slots<NP, WAVES>(s, p, ends, start);
  else load_states<NP>(s, p, h0, start);
  bool odd = false;                                 // zero or infinite for a lane of the wave
#pragma unroll
  for (int n = 0; n < NP; ++n) odd |= __any(start[n] + start[n] == start[n]);
  // this wave's steps of the turn ahead, and the marks in front of that
  T xn[SHARE], dn[SHARE], gn[SHARE], on[SHARE];
  float mark[NP], mark_sum = 0.f;
  auto request = [&](int i) {
    const int64_t t = p.from + i * U;
    const int last = last_of(p, t);
    const LaneOf lane(p);
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const int64_t step = t + min(p.part * SHARE + k, last);
      xn[k] = lane.of(xs + step * s.x_t);
      dn[k] = lane.of(ds + step * s.delta_t);
      on[k] = lane.of(os + step * s.out_t);
      if (gs) gn[k] = lane.of(gs + step * s.gate_t);
    }
    if (i > 0) {
      const float* from = marks_of<NP, WAVES>(s, p, marks, t);
      mark_sum = lane.of(from + (WAVES - p.part) * NP * s.channels);
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        mark[n] = lane.of(from);
        from += s.channels;
      }
    }
  };
  // A turn.  ENDS: the sequence ends in it, and steps beyond that leave everything as it is.  (Infinity times the zeros that stand for them would not.  It is the
  // first one walked, outside the loop: a branch around every step of every turn took 1170 us for 1140.)
  auto walk = [&](int i, auto ends) {
    constexpr bool ENDS = decltype(ends)::value;
    const int64_t t = p.from + i * U;
    const int last = ENDS ? last_of(p, t) : U - 1;
    const Shared at = rows + t * row_size;
    T xv[SHARE], dv[SHARE], gv[SHARE], ov[SHARE];
    float slope[SHARE], through[SHARE];
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      xv[k] = xn[k];
      dv[k] = dn[k];
      ov[k] = on[k];
      gv[k] = gn[k];
    }
    float own_dt[SHARE], own_dy[SHARE];
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      own_dt[k] = (float)dv[k] + shift;
      slope[k] = 1.f;
      own_dy[k] = (float)ov[k];
    }
    if (s.softplus) {
#pragma unroll
      for (int k = 0; k < SHARE; ++k) {
        const Softplus soft = softplus(own_dt[k]);
        own_dt[k] = soft.value;
        slope[k] = soft.slope;
      }
    }
    if (gs) {
#pragma unroll
      for (int k = 0; k < SHARE; ++k) {
        const float gt = (float)gv[k];
        const Gates z = sigmoid(gt);
        through[k] = own_dy[k] * (z.a * fmaf(gt, z.z, 1.f));
        own_dy[k] *= gt * z.a;
      }
    }
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const bool in = p.part * SHARE + k <= last;
      float* const to = common + (p.part * SHARE + k) * 3 * kWave;
      to[0] = in ? own_dt[k] : 0.f;
      to[kWave] = in ? own_dt[k] * (float)xv[k] : 0.f;
      to[2 * kWave] = in ? own_dy[k] : 0.f;
    }
    if (WAVES > 1) __syncthreads();
    float hs[U + 1][NP], e[U][NP], dt[U], u[U], dy[U];
#pragma unroll
    for (int n = 0; n < NP; ++n) hs[0][n] = i > 0 ? fmaf(__builtin_amdgcn_exp2f(mark_sum * decay[n]), start[n], mark[n]) : start[n];
    pin(hs[0]);
    if (odd && i > 0 && has_nan(hs[0])) {                  // (infinity and zero may have met)
#pragma unroll
      for (int n = 0; n < NP; ++n) hs[0][n] = carried(mark_sum * decay[n], start[n], mark[n]);
      pin(hs[0]);
    }
    if (i > 0) request(i - 1);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      dt[j] = common[j * 3 * kWave];
      u[j] = common[(j * 3 + 1) * kWave];
      dy[j] = common[(j * 3 + 2) * kWave];
    }
    const HeldRows<NP> b_of = next_b, c_of = next_c;
    {
      const float* const of = held_rows + max(t - U, p.from) * row_size;
      next_b.load(of, row_size, p.lane);
      next_c.load(of + NP * WAVES, row_size, p.lane);
    }
    with_states<NP, WHOLE>(own, [&](auto count) {
      constexpr int N = decltype(count)::value;
      Both both;
      both.load(at + (U - Both::kCount) * row_size);
#pragma unroll
      for (int j = 0; j < U; ++j) {
#pragma unroll
        for (int q = 0; q < (N + 3) / 4; ++q) {
          F32<4> h4 = {};
#pragma unroll
          for (int i = 0; i < 4 && 4 * q + i < N; ++i) {
            e[j][4 * q + i] = __builtin_amdgcn_exp2f(dt[j] * decay[4 * q + i]);
            h4[i] = e[j][4 * q + i] * hs[j][4 * q + i];
          }
          h4 = add_products<NP>(b_of, j, q, u[j], h4);
#pragma unroll
          for (int i = 0; i < 4 && 4 * q + i < N; ++i) hs[j + 1][4 * q + i] = h4[i];
        }
      }
      LanesSum<4 * NP> behind;       // what the two steps behind gave to grad_b and grad_c
#pragma unroll
      for (int first = U - Both::kCount; first >= 0; first -= Both::kCount) {
        await_shared();
        const Both group = both;
        stop();
        // (LDS and scalar loads share a counter, and the latter come in any order: a wait for sums from LDS would be one for them)
        auto ahead = [&](int k) {
          if (k == Both::kCount - 1 && first > 0) both.load(at + (first - Both::kCount) * row_size);
          stop();
        };
#pragma unroll
        for (int k = Both::kCount - 1; k >= 0; --k) {
          const int j = first + k;
          float* const pair = room + (j & 1 ? 0 : 2 * NP) * kSumRow + column;
          const bool sums = j % 2 == 1 && j < U - 1;
          if (sums) behind.request(room, p.lane);
          else ahead(k);
          if (!ENDS || j <= last) {
            float y = 0.f, along = 0.f, step = 0.f;
            float totals[NP];
#pragma unroll
            for (int q = 0; q < (N + 3) / 4; ++q) {
              F32<4> g4 = {};
#pragma unroll
              for (int i = 0; i < 4 && 4 * q + i < N; ++i) g4[i] = g[4 * q + i];
              g4 = add_products<NP>(c_of, j, q, dy[j], g4);
#pragma unroll
              for (int i = 0; i < 4 && 4 * q + i < N; ++i) totals[4 * q + i] = g4[i];
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
              const float total = totals[n];
              y = fmaf(group.row[k].c[n], hs[j + 1][n], y);
              pair[n * kSumRow] = total * u[j];
              pair[(NP + n) * kSumRow] = dy[j] * hs[j + 1][n];
              along = fmaf(total, group.row[k].b[n], along);
              g[n] = total * e[j][n];
              const float back = g[n] * hs[j][n];
              step = fmaf(back, decay[n], step);
              da[n] = fmaf(back, dt[j], da[n]);
            }
            float* const to = add + (p.part * U + j) * 3 * kWave;
            to[0] = y;
            to[kWave] = along;
            to[2 * kWave] = step;
          }
          if (sums) {
            shared_to[(t + j + 1) * row_size] = behind.sum();
            ahead(k);
          }
          stop();
        }
      }
      behind.request(room, p.lane);
      shared_to[t * row_size] = behind.sum();
    });
    if (WAVES > 1) __syncthreads();
    const LaneOf done(p);
#pragma unroll
    for (int k = 0; k < SHARE; ++k) {
      const int j = p.part * SHARE + k;
      float y = 0.f, along = 0.f, step = 0.f;
#pragma unroll
      for (int o = 0; o < WAVES; ++o) {
        const float* const from = add + (o * U + j) * 3 * kWave;
        y += from[0];
        along += from[kWave];
        step += from[2 * kWave];
      }
      if (j > last || !p.valid) continue;
      const float dt_of = common[j * 3 * kWave], dy_of = common[(j * 3 + 2) * kWave], xt = (float)xv[k];
      const float r = fmaf(along, xt, step * kLn2) * slope[k];
      done.of(dx + p.batch * s.dx_b + (t + j) * s.dx_t) = (T)fmaf(dt_of, along, skip * dy_of);
      done.of(ddelta + p.batch * s.ddelta_b + (t + j) * s.ddelta_t) = (T)r;
      dshift += r;
      dskip = fmaf(dy_of, xt, dskip);
      if (gs) done.of(dgate + p.batch * s.dgate_b + (t + j) * s.dgate_t) = (T)(fmaf(skip, xt, y) * through[k]);
    }
    if (WAVES > 1) __syncthreads();      // common and add are written again
  };
  if (turns > 0) request(turns - 1);
  const bool whole = (p.end - p.from) % U == 0;
  if (turns > 0 && !whole) walk(turns - 1, std::true_type());
  for (int i = turns - (whole ? 1 : 2); i >= 0; --i) walk(i, std::false_type());
  float* const to = parts + (p.batch * s.chunks + p.chunk) * (s.states + 2) * s.channels;
  const LaneOf lane(p);
  if (p.valid) {
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int at = p.part * NP + n;
      if (at < s.states) lane.of(to + at * s.channels) = da[n];
    }
    if (dh0 && p.chunk == 0) store_states<NP>(s, p, dh0, g);
  }
  if (WAVES > 1) {
    add[p.part * 2 * kWave] = dskip;
    add[(p.part * 2 + 1) * kWave] = dshift;
    __syncthreads();
    dskip = dshift = 0.f;
#pragma unroll
    for (int o = 0; o < WAVES; ++o) {
      dskip += add[o * 2 * kWave];
      dshift += add[(o * 2 + 1) * kWave];
    }
  }
  if (!p.valid || p.part != 0) return;
  lane.of(to + s.states * s.channels) = dskip;
  lane.of(to + (s.states + 1) * s.channels) = dshift;
  for (int64_t t = max(p.from, p.len); t < p.to; ++t) {
    lane.of(dx + p.batch * s.dx_b + t * s.dx_t) = (T)0.f;
    lane.of(ddelta + p.batch * s.ddelta_b + t * s.ddelta_t) = (T)0.f;
    if (gs) lane.of(dgate + p.batch * s.dgate_b + t * s.dgate_t) = (T)0.f;
  }
}

// grad_b and grad_c: the sums of a group's blocks of channels, in their order; and, in the workgroups behind `shared_blocks`, the sums of the
// chunks' parts.  8 x 4096 rows of 32 blocks x 32 numbers: 30 us for 134 MB, 4.5 TB/s.
template <typename T>
__global__ __launch_bounds__(kPartsThreads) void scan_join_kernel(const float* __restrict__ shared_parts, int64_t rows, int64_t steps,
                                                                  int64_t held, int groups, int blocks, int states, int padded,
                                                                  const int32_t* __restrict__ lengths, T* __restrict__ db, T* __restrict__ dc,
                                                                  int64_t db_b, int64_t db_t, int64_t dc_b, int64_t dc_t,
                                                                  unsigned shared_blocks, const float* __restrict__ parts, int64_t count,
                                                                  int64_t channels, PartsTo to, int accumulate) {
  __shared__ float fold[kPartsThreads];
  if (blockIdx.x >= shared_blocks) {
    const unsigned at = blockIdx.x - shared_blocks, across = (unsigned)((channels + kWave - 1) / kWave);
    parts_join(parts, count, states + 2, channels, to, accumulate, at % across, (int)(at / across), fold);
    return;
  }
  const int64_t at = (int64_t)blockIdx.x * kPartsThreads + threadIdx.x, row = at / (2 * padded);
  if (row >= rows) return;
  const int k = (int)(at - row * 2 * padded), n = k < padded ? k : k - padded;
  if (n >= states) return;
  const int64_t t = row % steps, g = row / steps % groups, batch = row / steps / groups;
  float s = 0.f;
  if (t < steps_of(lengths, batch, steps)) {
    const float* from = shared_parts + ((batch * groups + g) * blocks * held + t) * 2 * padded + k;
    for (int i = 0; i < blocks; i += kPartsAhead) {
      float v[kPartsAhead];
#pragma unroll
      for (int j = 0; j < kPartsAhead; ++j) v[j] = i + j < blocks ? from[(int64_t)(i + j) * held * 2 * padded] : 0.f;
#pragma unroll
      for (int j = 0; j < kPartsAhead; ++j) s += v[j];
    }
  }
  if (k < padded) db[batch * db_b + t * db_t + g * states + n] = (T)s;
  else dc[batch * dc_b + t * dc_t + g * states + n] = (T)s;
}

}  // namespace accop
