// One AdamW step over many tensors, moments in 32 or 8 bits.
#pragma once
#include "op_common.h"

namespace accop {

constexpr int kAdamBlock = 256;       // elements that share a scale: four per lane of a wave
// Elements per workgroup: a block per wave.  us at 1024, 2048, 4096, 8192: 51 M parameters 32 bits 270, 276, 280, 283; 8 bits 146, 160, 164, 167;
// VGG-19 shapes 8 bits 70, 74, 80, 88.
constexpr int kAdamTile = 1024;
constexpr int kAdamTensors = 64;      // tensors per launch (their table travels with the launch: 3.5 KiB)

struct AdamTensor {
  void* weights;
  const void* grads;
  void* copies;
  int64_t state;                      // first element in the moments
  int64_t n;
  uint32_t tile;                      // first tile in this launch
  float keep;                         // 1 - lr weight_decay
};

struct AdamArgs {
  AdamTensor t[kAdamTensors];
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  const float* grad_scale;
  float beta1, c1, beta2, c2, rate, up, eps;
  int count;
  uint32_t turn;                      // of the thresholds: step times the golden ratio
  bool dither_m, dither_v;
};

// Codes to nearest follow an average only while a step moves it by about half of what lies between two codes (3 to 6 %), or while the
// block's largest moves about by as much: sqrt(v) of random gradients, a tenth of what they were from step 2000 on, is held 1.03
// times too large after 5000 more steps at beta2 = 0.95, but 10 times at 0.98 and 7 times at 0.999, for good; m of gradients of
// 1 and a tenth of noise that fall to a tenth is held 1.01 times too large at beta1 = 0.9, 3.5 times at 0.95 and 9 times at 0.99.
// Above these betas a code is therefore rounded up where the part cut off reaches a threshold that goes through (0, 1) evenly over the
// steps, by the golden ratio (and over the elements, by other irrational numbers): on average nothing is lost (0.98 to 1.01 times in all of
// these cases), with less noise than random thresholds make, and the same bits for the same step.
constexpr double kNearestBeta1 = 0.9, kNearestBeta2 = 0.95;
// 2^32 times (sqrt(5) - 1) / 2 and the fractions of sqrt(2) and sqrt(3)
constexpr uint32_t kTurn = 0x9E3779B9u, kPhaseM = 0x6A09E667u, kPhaseV = 0xBB67AE85u;

constexpr float kTop = 448.0f;                 // largest e4m3 value
constexpr float kLeast = 0.001953125f;         // smallest positive e4m3 value, 2^-9
constexpr float kTiny = 7.8886090522101181e-31f;   // 2^-100

typedef float f4 __attribute__((ext_vector_type(4)));

// Four e4m3 codes as floats, and four floats as codes (to nearest even; conversions of this part).
__device__ __forceinline__ f4 decode4(uint32_t c) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ uint32_t encode4(const f4& v) {
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], c, true);
}

// Largest magnitude of a wave's 256 values as bits: the order of the bits is that of the magnitudes, with
// infinity and then NaN above all others, so that neither gets lost.
__device__ __forceinline__ uint32_t wave_top(const f4& v) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#define ACCOP_STEP(ctrl) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, ctrl, 0xf, 0xf, false))
  ACCOP_STEP(0xB1);
  ACCOP_STEP(0x4E);
  ACCOP_STEP(0x141);
  ACCOP_STEP(0x140);
#undef ACCOP_STEP
  const uint32_t a = __builtin_amdgcn_readlane((int)top, 0), b = __builtin_amdgcn_readlane((int)top, 16);
  const uint32_t c = __builtin_amdgcn_readlane((int)top, 32), d = __builtin_amdgcn_readlane((int)top, 48);
  return max(max(a, b), max(c, d));
}

// y cut to a code's value, or the next one where y's part beyond it and u in [0, 1) make up a spacing; NaN stays.
__device__ __forceinline__ float dithered(float y, float u) {
  const float a = fabsf(y);
  // of codes at a: 2^-9 up to 2^-6, else an eighth of a's power of two
  const uint32_t spacing = max(__float_as_uint(a) & 0x7f800000u, 0x3c800000u) - (3u << 23);
  const float r = floorf(a * __uint_as_float(0x7f000000u - spacing) + u) * __uint_as_float(spacing);
  return copysignf(r > kTop ? kTop : r, y);
}

// A block of 256 values (four per lane) as codes and a scale; dither: with the thresholds of phase + i step_phase for value i.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode_block(const f4& x, float* scale, bool dither, uint32_t phase, uint32_t step_phase) {
  const float top = __uint_as_float(wave_top(x));
  const bool held = !(top < kTiny);            // infinity, NaN: held, with an up of zero or NaN that makes the whole block NaN
  const float up = held ? kTop / top : 0.f;
  f4 y = x * up;
  if (dither)
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = dithered(y[i], (float)((phase + i * step_phase) >> 12) * 0x1p-20f);
  if (ROOT)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (up > 0.f && x[i] > 0.f && y[i] < kLeast) y[i] = kLeast;
  if ((threadIdx.x & 63) == 0) *scale = held ? top * (1.0f / kTop) : 0.f;
  return encode4(y);
}

// One pass over weights, gradients and moments, bound by memory: 51 M parameters 32 bits 264 us (5.4 TB/s), 8 bits with bf16 gradients and
// copy 141 (5.8), 11 M in 62 tensors 8 bits 34 (5.3); weights and gradients in bf16 32 bits 201 (5.6), 8 bits 103 (5.0).  Thresholds for codes of
// sqrt(v) 143 -> 146, of both 150 (fp32 gradients).  A wave holds a block of 256 elements, four per lane, so that the largest value of
// an 8-bit block is a reduction inside the wave; the root and the quotient are rounded correctly, which the memory hides.
// DITHER: some codes are dithered (a.dither_m, a.dither_v).
template <typename W, typename G, bool BITS8, bool DITHER>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamArgs a) {
  // the tensor of this tile
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].tile <= blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const int64_t n = a.t[lo].n;
  const int64_t tile0 = (int64_t)(blockIdx.x - a.t[lo].tile) * kAdamTile;
  W* const weights = static_cast<W*>(a.t[lo].weights);
  const G* const grads = static_cast<const G*>(a.t[lo].grads);
  bf16* const copies = static_cast<bf16*>(a.t[lo].copies);
  const int64_t state = a.t[lo].state;
  const float keep = a.t[lo].keep;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int r = 0; r < kAdamTile / (4 * kAdamBlock); ++r) {
    const int64_t block = tile0 + (r * 4 + wave) * kAdamBlock;   // first element of the wave's block
    if (block >= n) return;
    const int64_t i = block + 4 * l, left = n - i;
    f4 g = widen<G, 4>(load_some<4>(grads + i, left));
    f4 w = widen<W, 4>(load_some<4>(weights + i, left));
    f4 m, v, root;
    if (BITS8) {
      const int64_t b = (state + block) / kAdamBlock;
      m = decode4(static_cast<const uint32_t*>(a.m)[(state + i) / 4]) * a.m_scale[b];
      const f4 s = decode4(static_cast<const uint32_t*>(a.v)[(state + i) / 4]) * a.v_scale[b];
      v = s * s;
    } else {
      m = widen<float, 4>(load_some<4>(static_cast<const float*>(a.m) + state + i, left));
      v = widen<float, 4>(load_some<4>(static_cast<const float*>(a.v) + state + i, left));
    }
    if (a.grad_scale) g *= gs;
    m = a.beta1 * m + a.c1 * g;
    v = a.beta2 * v + (a.c2 * g) * g;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      root[k] = sqrtf(v[k]);
      w[k] = w[k] * keep - (a.rate * m[k]) / (root[k] * a.up + a.eps);
    }
    if (left > 0) {
      store_some_stream<W, 4>(weights + i, w, left);
      if (copies) store_some_stream<bf16, 4>(copies + i, w, left);
    }
    if (BITS8) {
      // codes beyond the tensor's end are zeros of zeros: the block's storage is whole
      const int64_t b = (state + block) / kAdamBlock;
      const uint32_t e = (uint32_t)(state + i);
      static_cast<uint32_t*>(a.m)[(state + i) / 4] =
          encode_block<false>(m, a.m_scale + b, DITHER && a.dither_m, e * kPhaseM + a.turn, kPhaseM);
      static_cast<uint32_t*>(a.v)[(state + i) / 4] =
          encode_block<true>(root, a.v_scale + b, DITHER && a.dither_v, e * kPhaseV + a.turn, kPhaseV);
    } else if (left > 0) {
      store_some_stream<float, 4>(static_cast<float*>(a.m) + state + i, m, left);
      store_some_stream<float, 4>(static_cast<float*>(a.v) + state + i, v, left);
    }
  }
}

}  // namespace accop
