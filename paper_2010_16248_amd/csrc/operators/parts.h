// Sums of parts that workgroups have left: rows of channels, added over the parts in their order.
#pragma once
#include "op_common.h"

namespace accop {

// Where the sums of the parts' rows go: rows [0, columns) are the columns of a channels x columns matrix, the two rows behind them vectors.
struct PartsTo {
  float* matrix;
  int columns;
  float* first;
  float* second;
};

// A workgroup takes 64 channels of one row, each of its 16 waves a run of consecutive parts.  2048 parts x 5 rows of 4096 channels: 6 us.
constexpr int kPartsThreads = 1024, kPartsAhead = 16;   // parts under way
__device__ __forceinline__ void parts_join(const float* parts, int64_t count, int rows, int64_t channels, const PartsTo& to, int accumulate,
                                           unsigned block, int row, float* fold) {
  constexpr int waves = kPartsThreads / kWave;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t c = (int64_t)block * kWave + l;
  float* at = row < to.columns ? to.matrix + c * to.columns + row : (row == to.columns ? to.first : to.second);
  if (row >= to.columns) {
    if (!at) return;
    at += c;
  }
  const int64_t share = (count + waves - 1) / waves, lo = w * share, hi = min(count, lo + share);
  float s = 0.f;
  if (c < channels)
    for (int64_t i = lo; i < hi; i += kPartsAhead) {
      float v[kPartsAhead];
#pragma unroll
      for (int k = 0; k < kPartsAhead; ++k) v[k] = i + k < hi ? parts[((i + k) * rows + row) * channels + c] : 0.f;
#pragma unroll
      for (int k = 0; k < kPartsAhead; ++k) s += v[k];
    }
  fold[w * kWave + l] = s;
  __syncthreads();
  if (w == 0 && c < channels) {
    s = 0.f;
    for (int i = 0; i < waves; ++i) s += fold[i * kWave + l];
    *at = accumulate ? *at + s : s;
  }
}

static __global__ __launch_bounds__(kPartsThreads) void parts_join_kernel(const float* __restrict__ parts, int64_t count, int rows,
                                                                          int64_t channels, PartsTo to, int accumulate) {
  __shared__ float fold[kPartsThreads];
  parts_join(parts, count, rows, channels, to, accumulate, blockIdx.x, (int)blockIdx.y, fold);
}

}  // namespace accop
