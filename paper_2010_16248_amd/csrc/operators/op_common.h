// Shared device-side helpers of the language-model operators (gfx950, wave64).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace accop {

constexpr int kWave = 64;

typedef __bf16 bf16;

// N consecutive elements that start anywhere (this part's wide global accesses need no alignment beyond the
// element's), and the same in fp32.
template <typename T, int N>
using Pack = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));
template <int N>
using F32 = float __attribute__((ext_vector_type(N)));

template <typename T, int N>
__device__ __forceinline__ F32<N> widen(const Pack<T, N>& v) {
  return __builtin_convertvector(v, F32<N>);
}

template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load(const T* p) {
  return *reinterpret_cast<const Pack<T, N>*>(p);
}
// Streaming ("non-temporal") access: for data that no later kernel of the step finds in a cache anyway.
template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load_stream(const T* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const Pack<T, N>*>(p));
}
// The first n of N elements (n <= 0: none); the others are zero and are not read.
template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load_some(const T* p, int64_t n) {
  if (n >= N) return load<N>(p);
  Pack<T, N> v;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < n ? p[i] : (T)0.0f;
  return v;
}

// fp32 values, rounded to T (to nearest even) and stored.
template <typename T, int N>
__device__ __forceinline__ void store(T* p, const F32<N>& v) {
  *reinterpret_cast<Pack<T, N>*>(p) = __builtin_convertvector(v, Pack<T, N>);
}
template <typename T, int N>
__device__ __forceinline__ void store_stream(T* p, const F32<N>& v) {
  __builtin_nontemporal_store(__builtin_convertvector(v, Pack<T, N>), reinterpret_cast<Pack<T, N>*>(p));
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, const F32<N>& v, int64_t n) {
  if (n >= N) {
    store<T, N>(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < n) p[i] = (T)v[i];
}

template <typename T, int N>
__device__ __forceinline__ void store_some_stream(T* p, const F32<N>& v, int64_t n) {
  if (n >= N) store_stream<T, N>(p, v);
  else store_some<T, N>(p, v, n);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane(float v, int l) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l));
}
// Sum over each row of 16 lanes, the same value in all of them.
__device__ __forceinline__ float row16_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  return v;
}
// Sum over the 64 lanes, the same value in every lane (lane exchanges inside rows of 16, then the four rows).
// All lanes must be active.
__device__ __forceinline__ float wave_sum(float v) {
  v = row16_sum(v);
  return (lane(v, 0) + lane(v, 16)) + (lane(v, 32) + lane(v, 48));
}

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

// The same for products with f, as SiLU and its derivative take them: half as many instructions.  Below f = -88.5 both are zero (a is below
// 2^-127 there); their NaN is left to f.
__device__ __forceinline__ Gates sigmoid(float f) {
  const float x = __builtin_amdgcn_fmed3f(f, -88.5f, 100.f);
  const float t = -1.44269502f * x;
  const float d = fmaf(t, -0.693147182f, -x);
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e, d, e);
  const float a = f < -88.5f ? 0.f : __builtin_amdgcn_rcpf(1.f + e);
  return {a, e * a};
}

__device__ __forceinline__ int64_t steps_of(const int32_t* lengths, int64_t batch, int64_t steps) {
  if (!lengths) return steps;
  const int64_t n = lengths[batch];
  return n < 0 ? 0 : (n < steps ? n : steps);
}

}  // namespace accop
