// Log probabilities of given tokens, entropies and most probable tokens of rows of logits; the gradient of the first two.
#pragma once
#include "op_common.h"

namespace accop {

// Running sums over some of a row's logits: the largest (at least -FLT_MAX, so that differences to it are numbers), the sum s of e^(l - top)
// and the sum of e^(l - top) (l - top).
struct RowSums {
  float top, s, t;
};
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2eRow = 1.44269504f;
constexpr float kFar = -200.f;           // e^kFar is zero in fp32; keeps (l - top) e^(l - top) from being infinity times zero

__device__ __forceinline__ RowSums no_sums() { return {kLowest, 0.f, 0.f}; }

// The same sums with a larger top.
__device__ __forceinline__ void raise(RowSums& r, float top) {
  const float d = fmaxf(r.top - top, kFar), f = __builtin_amdgcn_exp2f(d * kLog2eRow);
  r.t = f * fmaf(d, r.s, r.t);
  r.s *= f;
  r.top = top;
}
__device__ __forceinline__ RowSums joined(RowSums a, RowSums b) {
  const float top = fmaxf(a.top, b.top);
  raise(a, top);
  raise(b, top);
  return {top, a.s + b.s, a.t + b.t};
}
template <int N, bool ENTROPY>
__device__ __forceinline__ void add_pack(RowSums& r, const F32<N>& l) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = l[i] - r.top, e = __builtin_amdgcn_exp2f(d * kLog2eRow);
    r.s += e;
    if (ENTROPY) r.t = fmaf(e, fmaxf(d, kFar), r.t);
  }
}
template <int N>
__device__ __forceinline__ float top_of(const F32<N>& l) {
  float m = l[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, l[i]);
  return m;
}

// Over the threads of a workgroup, the same in all of them.
template <int THREADS>
__device__ __forceinline__ RowSums group_sums(RowSums r, RowSums* red) {
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) {
    RowSums o;
    o.top = __shfl_xor(r.top, k);
    o.s = __shfl_xor(r.s, k);
    o.t = __shfl_xor(r.t, k);
    r = threadIdx.x & k ? joined(o, r) : joined(r, o);
  }
  constexpr int waves = THREADS / kWave;
  if (waves == 1) return r;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = r;
  __syncthreads();
  r = red[0];
#pragma unroll
  for (int i = 1; i < waves; ++i) r = joined(r, red[i]);
  return r;
}

// A logit's place in the order of logits: larger logits have larger keys, a NaN the least.
__device__ __forceinline__ unsigned key_of(float l) {
  const unsigned u = __float_as_uint(l);
  if (l != l) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(unsigned key) {
  if (key == 0) return __uint_as_float(0x7fc00000u);
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// -0 and 0 are equal logits.
template <typename T>
__device__ __forceinline__ unsigned key_at(T l) { return key_of((float)l + 0.f); }

struct LogprobOut {
  const void* targets;
  float *logprob, *lse, *entropy, *top_logprobs;
  void* top_ids;
  int64_t vocab, stride;
  int top;
  bool wide;              // ids of 64 bits
};
__device__ __forceinline__ int64_t id_at(const void* ids, bool wide, int64_t row) {
  return wide ? static_cast<const int64_t*>(ids)[row] : static_cast<const int32_t*>(ids)[row];
}

// A row's results.
__device__ __forceinline__ void write_row(const LogprobOut& o, int64_t row, RowSums r, float target_logit, bool named) {
  const float log_s = logf(r.s);
  if (o.lse) o.lse[row] = r.top + log_s;
  if (o.entropy) o.entropy[row] = r.s == 0.f ? 0.f : log_s - r.t / r.s;
  if (o.logprob) o.logprob[row] = !named ? 0.f : (r.s == 0.f ? -INFINITY : (target_logit - r.top) - log_s);
}
__device__ __forceinline__ void write_top(const LogprobOut& o, int64_t row, int place, RowSums r, float logit, unsigned id) {
  o.top_logprobs[row * o.top + place] = r.s == 0.f ? -INFINITY : (logit - r.top) - logf(r.s);
  if (o.wide) static_cast<int64_t*>(o.top_ids)[row * o.top + place] = id;
  else static_cast<int32_t*>(o.top_ids)[row * o.top + place] = (int32_t)id;
}
template <typename T>
__device__ __forceinline__ float target_of(const LogprobOut& o, const T* logits, int64_t row, bool* named) {
  *named = false;
  if (!o.logprob) return 0.f;
  const int64_t id = id_at(o.targets, o.wide, row);
  *named = id >= 0 && id < o.vocab;
  return *named ? (float)logits[row * o.stride + id] : 0.f;
}

// ---- forward without the most probable tokens ----------------------------------------------------------------
// A workgroup streams a part of a row once, with the running largest logit and sums of its lanes; parts of a row that has several go to sums.
// 1000 x 131072 bf16: 48 us, 5.5 TB/s: the rate of a large copy.
// LANES: of a row, all of the workgroup's or a wave's.
template <typename T, int N, bool ENTROPY, bool PARTS, int LANES>
__global__ __launch_bounds__(256) void logprob_stream_kernel(LogprobOut o, const T* __restrict__ logits, int64_t rows, int64_t part, int parts,
                                                             RowSums* __restrict__ sums) {
  constexpr int K = 4;       // requests under way
  static_assert(LANES == 256 || (LANES == kWave && !PARTS), "a wave has a whole row");
  __shared__ RowSums red[4];
  const int64_t row = LANES == 256 ? blockIdx.x : (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int own = threadIdx.x % LANES;
  if (row >= rows) return;
  const int64_t from = blockIdx.y * part, to = min(from + part, o.vocab);
  const T* l = logits + row * o.stride;
  RowSums r = no_sums();
  for (int64_t at = from + own * N; at < to; at += LANES * N * K) {
    F32<N> v[K];
    float top = r.top;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t place = at + k * LANES * N, left = to - place;
      if (left >= N) {
        v[k] = widen<T, N>(load<N>(l + place));
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[k][i] = i < left ? (float)l[place + i] : -INFINITY;
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) top = fmaxf(top, top_of<N>(v[k]));
    if (top > r.top) raise(r, top);
#pragma unroll
    for (int k = 0; k < K; ++k) add_pack<N, ENTROPY>(r, v[k]);
  }
  r = group_sums<LANES>(r, red);
  if (own != 0) return;
  if (PARTS) {
    sums[row * parts + blockIdx.y] = r;
  } else {
    bool named;
    const float t = target_of<T>(o, logits, row, &named);
    write_row(o, row, r, t, named);
  }
}

// ---- forward with them ------------------------------------------------------------------------------------------
// A workgroup (a wave, for short rows) holds a part of a row in registers.  The part's tokens lie with 64 groups of lanes; the `top` groups with the largest maxima have a
// least maximum, below which none of the `top` most probable tokens can be.  What is not below it, few in general, is listed in LDS
// and ordered by counting.  Where it is more than the list holds (rows masked but for a few tokens, rows of few values), list_again finds a key with
// fewer above it.  A row is read once: 5 of 700 x 32768 fp32 in 19.8 us, 4.6 TB/s, and 4.0 for the join; 20 of 16 x 131072 bf16 in 8.0 and 4.3, most
// of it from one wait to the next.
constexpr int kTopGroups = 64;
// Tokens that a workgroup's list holds: a wave's is short, for as many workgroups as a CU takes.
__host__ __device__ constexpr int top_list(int threads) { return threads == kWave ? 512 : 1024; }

// A token in the order of the most probable ones: its logit's key, then its id, the lowest first.  0: no token.
typedef unsigned long long Token;
__device__ __forceinline__ Token token_of(float l, unsigned id) { return (Token)key_at(l) << 32 | ~id; }
__device__ __forceinline__ float logit_of(Token t) { return logit_of((unsigned)(t >> 32)); }
__device__ __forceinline__ unsigned id_of(Token t) { return ~(unsigned)t; }

__device__ __forceinline__ float wave_top(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  v = fmaxf(v, dpp<0x140>(v));
  return fmaxf(fmaxf(lane(v, 0), lane(v, 16)), fmaxf(lane(v, 32), lane(v, 48)));
}

// Tokens in front of one of a list's, which is filled up with "no token" to whole eights.
__device__ __forceinline__ int place_in(const Token* list, int count, Token token) {
  int place = 0;
  for (int j = 0; j < count; j += 8) {
    Token o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = list[j + k];
#pragma unroll
    for (int k = 0; k < 8; ++k) place += o[k] > token;
  }
  return place;
}

// Lists what can be among the `wanted` most probable of a part's tokens, read again: all above a key, fewer than the list holds, and of the tokens of this
// key the first ones.  The key is `least`, that of a logit that so many tokens reach, or, where too many lie above it, is halved up to from there; where so
// many do not (the rest are no numbers) it is zero.  Returns their number; `counts` holds a number a wave.
// 20 of 128 x 131072 bf16, masked but for 50: 46 us (a row as the model leaves it 19), 1024 x 50257 fp32 112 (47); 259 and 801 with one token after the
// other sought among all.
template <typename T, int N, int THREADS>
__device__ __forceinline__ int list_again(const T* l, int size, unsigned from, int wanted, unsigned least, Token* list, unsigned* counts,
                                          unsigned* listed) {
  constexpr int waves = THREADS / kWave, turn = THREADS * N, kTopList = top_list(THREADS);
  const int lane_of = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto pack_at = [&](int at) {
    const int left = size - at;
    Pack<T, N> v;
    if (left >= N) return load<N>(l + at);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < left ? l[at + i] : (T)0.f;
    return v;
  };
  // tokens above the key << 16 | tokens of the key
  auto count = [&](unsigned key) {
    unsigned n = 0;
#pragma unroll 1
    for (int at = threadIdx.x * N; at < size; at += turn) {
      const Pack<T, N> v = pack_at(at);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned own = key_at(v[i]);
        if (at + i < size) n += own > key ? 0x10000u : own == key;
      }
    }
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) n += __shfl_xor(n, m);
    __syncthreads();
    if (lane_of == 0) counts[wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll 1
    for (int w = 0; w < waves; ++w) n += counts[w];
    return n;
  };
  unsigned key = least, most = 0xffffffffu, n = count(key);
  if ((int)(n >> 16) + (int)(n & 0xffffu) < wanted) {
    key = 0;
    n = count(key);
  }
  while (n >> 16 > kTopList) {               // ends with key == most at the latest, which fewer than `wanted` are above
    const unsigned half = key + (most - key) / 2 + 1, m = count(half);
    if ((int)(m >> 16) + (int)(m & 0xffffu) >= wanted) {
      key = half;
      n = m;
    } else {
      most = half - 1;
    }
  }
  const int above = (int)(n >> 16), need = max(wanted - above, 0);
  for (int i = threadIdx.x; i < kTopList; i += THREADS) list[i] = 0;
  if (threadIdx.x == 0) *listed = 0;
  __syncthreads();
#pragma unroll 1
  for (int at = threadIdx.x * N; at < size; at += turn) {
    const Pack<T, N> v = pack_at(at);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at + i < size && key_at(v[i]) > key) list[atomicAdd(listed, 1u)] = token_of((float)v[i], from + at + i);
  }
  int taken = 0;
#pragma unroll 1
  for (int start = 0; start < size && taken < need; start += turn) {       // the same for all threads
    const int at = start + threadIdx.x * N;
    Pack<T, N> v{};
    if (at < size) v = pack_at(at);
    int own = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) own += at + i < size && key_at(v[i]) == key;
    int up_to = own;
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) {
      const int other = __shfl_up(up_to, m);
      if (lane_of >= m) up_to += other;
    }
    __syncthreads();
    if (lane_of == 63) counts[wave] = up_to;
    __syncthreads();
    int place = taken + up_to - own;
#pragma unroll 1
    for (int w = 0; w < waves; ++w) {
      if (w < wave) place += (int)counts[w];
      taken += (int)counts[w];
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at + i < size && key_at(v[i]) == key) {
        if (place < need) list[above + place] = token_of((float)v[i], from + at + i);
        ++place;
      }
  }
  __syncthreads();
  return above + min(taken, need);
}

template <typename T, int N, int K, int THREADS, bool PARTS>
__global__ __launch_bounds__(THREADS) void logprob_top_kernel(LogprobOut o, const T* __restrict__ logits, int64_t part, int parts,
                                                              RowSums* __restrict__ sums, Token* __restrict__ best) {
  constexpr int waves = THREADS / kWave, each = THREADS / kTopGroups;       // lanes of a group
  constexpr int kTopList = top_list(THREADS);
  static_assert(each == 1 || each == 4 || each == 16, "groups are lanes, whole rows or quarters of rows of 16 lanes");
  __shared__ float group_top[kTopGroups], sum[waves], weighted[waves], least_of;
  __shared__ unsigned listed;
  __shared__ alignas(16) Token list[kTopList];
  __shared__ unsigned counts[waves];
  const int64_t row = blockIdx.x;
  const int64_t from = blockIdx.y * part;
  const int size = (int)min(part, o.vocab - from);
  const T* const l = logits + row * o.stride + from;
  Pack<T, N> v[K];
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int place = ((int)threadIdx.x + k * THREADS) * N, left = size - place;
    if (left >= N) {
      v[k] = load<N>(l + place);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[k][i] = i < left ? l[place + i] : (T)-INFINITY;
    }
  }
  // (requested with the logits, used at the end)
  bool named = false;
  const float target = PARTS ? 0.f : target_of<T>(o, logits, row, &named);
  if (threadIdx.x == 0) listed = 0;
#pragma unroll
  for (int i = 0; i < kTopList; i += THREADS) list[i + threadIdx.x] = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) top = fmaxf(top, top_of<N>(widen<T, N>(v[k])));
  if (each >= 4) {
    top = fmaxf(top, dpp<0xB1>(top));
    top = fmaxf(top, dpp<0x4E>(top));
  }
  if (each == 16) {
    top = fmaxf(top, dpp<0x141>(top));
    top = fmaxf(top, dpp<0x140>(top));
  }
  if (threadIdx.x % each == 0) group_top[threadIdx.x / each] = top;
  __syncthreads();
  const float own = group_top[threadIdx.x & 63];
  RowSums r = no_sums();
  r.top = fmaxf(kLowest, wave_top(own));
  if (threadIdx.x < kWave) {
    // the least of the maxima that have fewer than `top` larger ones
    int larger = 0;
#pragma unroll 16
    for (int i = 0; i < kTopGroups; ++i) larger += lane(own, i) > own;
    const float least = -wave_top(larger < o.top ? -own : -INFINITY);
    if (threadIdx.x == 0) least_of = least;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) add_pack<N, true>(r, widen<T, N>(v[k]));
  r.s = wave_sum(r.s);
  r.t = wave_sum(r.t);
  if ((threadIdx.x & 63) == 0) {
    sum[threadIdx.x >> 6] = r.s;
    weighted[threadIdx.x >> 6] = r.t;
  }
  __syncthreads();
  r.s = r.t = 0.f;
#pragma unroll
  for (int w = 0; w < waves; ++w) {
    r.s += sum[w];
    r.t += weighted[w];
  }
  const float least = least_of;
  // (what is not a number is below no maximum)
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const F32<N> wide = widen<T, N>(v[k]);
    if (top_of<N>(wide) < least) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int place = ((int)threadIdx.x + k * THREADS) * N + i;
      if (!(wide[i] < least) && place < size) {
        const unsigned at = atomicAdd(&listed, 1u);
        if (at < kTopList) list[at] = token_of(wide[i], (unsigned)(from + place));
      }
    }
  }
  __syncthreads();
  const int wanted = min(o.top, size);     // tokens this part can give
  int count = (int)listed;
  if (count > kTopList) {                  // (of all threads, and once more after the list is cleared)
    __syncthreads();
    count = list_again<T, N, THREADS>(l, size, (unsigned)from, wanted, key_of(least), list, counts, &listed);
  }
  auto put = [&](int place, Token token) {
    if (PARTS) best[(row * parts + blockIdx.y) * o.top + place] = token;
    else write_top(o, row, place, r, logit_of(token), id_of(token));
  };
  for (int i = threadIdx.x; i < count; i += THREADS) {
    const Token token = list[i];
    const int place = place_in(list, count, token);
    if (place < wanted) put(place, token);
  }
  if (PARTS)
    for (int place = wanted + threadIdx.x; place < o.top; place += THREADS) put(place, 0);
  if (threadIdx.x != 0) return;
  if (PARTS) sums[row * parts + blockIdx.y] = r;
  else write_row(o, row, r, target, named);
}

// Joins a row's parts: their sums in order, and the most probable of their most probable tokens, by counting.
constexpr int kJoinThreads = 512;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void logprob_join_kernel(LogprobOut o, const T* __restrict__ logits, int parts,
                                                                    const RowSums* __restrict__ sums, const Token* __restrict__ best) {
  extern __shared__ Token tokens[];
  const int64_t row = blockIdx.x;
  bool named;
  const float target = target_of<T>(o, logits, row, &named);
  const int count = parts * o.top;
  for (int i = threadIdx.x; i < (count + 7) / 8 * 8; i += kJoinThreads) tokens[i] = i < count ? best[row * count + i] : 0;
  // (every thread for itself: the parts' sums come through scalar loads)
  RowSums r = no_sums();
  const RowSums* const of = sums + row * parts;
  for (int i = 0; i < parts; ++i) r.top = fmaxf(r.top, of[i].top);
  for (int i = 0; i < parts; ++i) {
    RowSums q = of[i];
    raise(q, r.top);
    r.s += q.s;
    r.t += q.t;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kJoinThreads) {
    const Token token = tokens[i];
    if (token == 0) continue;
    const int place = place_in(tokens, count, token);
    if (place < o.top) write_top(o, row, place, r, logit_of(token), id_of(token));
  }
  if (threadIdx.x == 0) write_row(o, row, r, target, named);
}

// ---- backward ---------------------------------------------------------------------------------------------
// One pass: p comes from lse.  16 bytes a lane and 4 requests under way reach the rate of a large copy: 16384 x 65536 bf16, 4.3 GB read and written, in
// 823 us, 5.2 TB/s.  grad may be logits: a lane writes what it has read.
template <typename T, int N, bool ENTROPY, int LANES>
__global__ __launch_bounds__(256) void logprob_backward_kernel(const T* logits, const void* __restrict__ targets, bool wide,
                                                               const float* __restrict__ lse_in, const float* __restrict__ dlogprob,
                                                               const float* __restrict__ entropy_in, const float* __restrict__ dentropy,
                                                               T* grad, int64_t rows, int64_t vocab, int64_t stride, int64_t grad_stride, int64_t part) {
  constexpr int K = 4;
  const int64_t row = LANES == 256 ? blockIdx.x : (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= rows) return;
  const int64_t from = blockIdx.y * part, to = min(from + part, vocab);
  int64_t id = -1;
  if (dlogprob) id = id_at(targets, wide, row);
  const bool named = id >= 0 && id < vocab;
  const float lse = lse_in[row], g = named ? dlogprob[row] : 0.f;
  const float entropy = ENTROPY ? entropy_in[row] : 0.f, ge = ENTROPY ? dentropy[row] : 0.f;
  const T* l = logits + row * stride;
  T* out = grad + row * grad_stride;
  const bool nothing = (!ENTROPY && !named) || lse == -INFINITY;
  for (int64_t at = from + threadIdx.x % LANES * N; at < to; at += LANES * N * K) {
    F32<N> v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t place = at + k * LANES * N;
      v[k] = F32<N>{};
      if (!nothing) v[k] = widen<T, N>(load_some<N>(l + place, to - place));
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t place = at + k * LANES * N;
      if (place >= to) break;
      F32<N> r = {};
      if (!nothing) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float lp = v[k][i] - lse;
          bool far;
          float p = exp_neg(-lp, &far);
          p = far ? p * 0x1p-32f : p;
          r[i] = -g * p;
          if (ENTROPY) r[i] -= ge * p * (fmaxf(lp, kFar) + entropy);
          if (place + i == id) r[i] += g;
        }
      }
      store_some<T, N>(out + place, r, to - place);
    }
  }
}

}  // namespace accop
