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

}  // namespace accop
