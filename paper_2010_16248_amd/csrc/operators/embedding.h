// Embedding lookup with scaling, and the table's gradient by sorted tokens.
#pragma once
#include "op_common.h"

namespace accop {

// ---- forward: out[t, :] = scale * table[id_t, :] ------------------------------------------------------
// A copy of rows, bound by memory (up to a few thousand rows: by the launch, 3 us).  A group of 2^lanes_log2 lanes takes a row,
// kLookupLoads requests per lane under way; grid.y splits rows of more columns.  The output is streamed, the rows are not: frequent
// tokens find theirs in a cache.  131072 tokens of 2048 bf16 146 us (4.4 TB/s of output and distinct rows; one request per lane and
// plain stores 211, four requests 147), 40000 of 672 fp32 24 (48).
constexpr int kLookupLoads = 2;

template <typename I, typename T, typename O, int N>
__global__ __launch_bounds__(256) void embedding_lookup_kernel(const I* __restrict__ ids, const T* __restrict__ table,
                                                               O* __restrict__ out, int64_t tokens, int64_t vocab,
                                                               int64_t dim, int64_t table_stride, int64_t out_stride,
                                                               float scale, int lanes_log2) {
  const int lanes = 1 << lanes_log2;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> lanes_log2;
  if (t >= tokens) return;
  const int64_t id = (int64_t)ids[t];
  const bool known = id >= 0 && id < vocab;
  const T* row = table + (known ? id : 0) * table_stride;
  O* to = out + t * out_stride;
  const int64_t c0 = (int64_t)blockIdx.y * kLookupLoads * lanes * N + (int64_t)(threadIdx.x & (lanes - 1)) * N;
  const int64_t pitch = (int64_t)lanes * N;
  Pack<T, N> v[kLookupLoads];
#pragma unroll
  for (int i = 0; i < kLookupLoads; ++i) v[i] = load_some<N>(row + c0 + i * pitch, known ? dim - (c0 + i * pitch) : 0);
#pragma unroll
  for (int i = 0; i < kLookupLoads; ++i) {
    const int64_t left = dim - (c0 + i * pitch);
    if (left > 0) store_some_stream<O, N>(to + c0 + i * pitch, widen<T, N>(v[i]) * scale, left);
  }
}

// ---- backward: order the tokens by id, ties by position ------------------------------------------------
// key = id, or vocab for an id outside the table (sorts behind all others and is left out).
template <typename I>
__device__ __forceinline__ uint32_t key_of_id(I id, uint32_t vocab) {
  const int64_t v = (int64_t)id;
  return v >= 0 && v < (int64_t)vocab ? (uint32_t)v : vocab;
}

// The zeros of the rows that no token asks for.  The launches that order the tokens wait for latencies and leave the
// memory idle, so each of them also clears a share of the last rows, whatever they will hold (Clear); the rest is cleared in
// the launch that sums, which knows the rows without tokens.
constexpr int kClearAhead = 4;
struct Clear {
  float* table;
  int64_t first, rows, dim, stride;   // rows [first, first + rows)
};

// Zeros over [p, p + n): thread `me` of `all`, whole 128-byte lines by neighbouring threads (a line written in two pieces costs
// the memory twice: rows of 1001 elements, 200 MB: 51 -> 43 us).
__device__ __forceinline__ void clear_span(float* p, int64_t n, int64_t me, int64_t all) {
  const F32<4> zero = {0.f, 0.f, 0.f, 0.f};
  const int64_t head = min(n, (int64_t)((128 - (reinterpret_cast<uintptr_t>(p) & 127)) & 127) / 4);
  if (me < head) p[me] = 0.f;
  p += head;
  n -= head;
  for (int64_t i = me * 4; i < n; i += all * 4 * kClearAhead) {
#pragma unroll
    for (int k = 0; k < kClearAhead; ++k)
      if (i + k * all * 4 < n) store_some_stream<float, 4>(p + i + k * all * 4, zero, n - (i + k * all * 4));
  }
}

__device__ __forceinline__ void clear_rows(const Clear& s, int64_t block, int64_t blocks) {
  float* table = s.table + s.first * s.stride;
  if (s.stride == s.dim) {
    // pieces of kClearAhead requests per thread, in order
    const int64_t piece = (int64_t)blockDim.x * 4 * kClearAhead, n = s.rows * s.dim;
    const int64_t head = min(n, (int64_t)((128 - (reinterpret_cast<uintptr_t>(table) & 127)) & 127) / 4);
    if (block == 0 && (int64_t)threadIdx.x < head) table[threadIdx.x] = 0.f;
    for (int64_t at = head + block * piece; at < n; at += blocks * piece)
      clear_span(table + at, min(piece, n - at), threadIdx.x, blockDim.x);
  } else {
    for (int64_t r = block; r < s.rows; r += blocks) clear_span(table + r * s.stride, s.dim, threadIdx.x, blockDim.x);
  }
}

// A wave clears those of kGapRows rows from `row` on whose bits are set.
constexpr int kGapRows = 4;
__device__ __forceinline__ void clear_gap_rows(const Clear& s, int64_t row, uint64_t gaps) {
  const int l = threadIdx.x & 63;
  if (gaps == (1ull << kGapRows) - 1 && s.stride == s.dim) {     // one piece
    clear_span(s.table + row * s.stride, kGapRows * s.dim, l, kWave);
    return;
  }
  while (gaps) {
    clear_span(s.table + (row + __builtin_ctzll(gaps)) * s.stride, s.dim, l, kWave);
    gaps &= gaps - 1;
  }
}

// A wave clears those of kGapRows rows from `row` on (below `rows`) that no token asks for.
__device__ __forceinline__ void clear_gaps(const Clear& s, int64_t row, int64_t rows, const uint32_t* __restrict__ skey, int64_t n) {
  const int l = threadIdx.x & 63;
  // lane l < kGapRows looks for its row in the order: the first place whose key is not below it
  const uint32_t mine = (uint32_t)min(row + (l & (kGapRows - 1)), rows - 1);
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (skey[mid] < mine) lo = mid + 1; else hi = mid;
  }
  const bool empty = l < kGapRows && row + l < rows && (lo == n || skey[lo] != mine);
  uint64_t gaps = __ballot(empty);
  clear_gap_rows(s, row, gaps);
}

template <int N>
__device__ __forceinline__ void to_row(float* to, const F32<N>& sum, const F32<N>& old, float scale, bool accumulate, int64_t left) {
  F32<N> v = sum * scale;
  if (accumulate) v = old + v;
  store_some<float, N>(to, v, left);
}

// A handful of tokens: one launch, nothing is ordered.  The wave of the first token of an id (and 64 N columns) finds the
// others by comparing all ids, 64 at a time, and adds their rows; other waves clear the rows of which no id is found.
// us per call at 32768 x 672 fp32, in one launch and in the three of the other way: 20 tokens 16.1 and 19.2, 512 tokens 17.6 and 22.3, added to
// what is there 7.8 and 15.2; 700 tokens 18.6 and 22.5.  500 tokens of two ids, which two waves add: 21.9 and 13.7, 1000 of them 43 and 18,
// hence the limit (kFewTokens).  Sixteen rows under way: 512 tokens 19.1.
constexpr int kFewAhead = 8;
template <typename I, typename T, int N, bool ACCUMULATE, bool EVEN>
__global__ __launch_bounds__(256) void embedding_few_kernel(const I* __restrict__ ids, int n, int64_t vocab, const T* __restrict__ grad,
                                                            int64_t grad_stride, float* __restrict__ table, int64_t table_stride,
                                                            int64_t dim, uint32_t across, uint32_t units, float scale, uint32_t gap_units) {
  const int l = threadIdx.x & 63;
  const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= units) {
    if (ACCUMULATE || unit - units >= gap_units) return;
    for (int64_t row = (int64_t)(unit - units) * kGapRows; row < vocab; row += (int64_t)gap_units * kGapRows) {
      uint32_t found = 0;
      for (int j = l; j < n; j += kWave) {
        const int64_t at = (int64_t)ids[j] - row;
        if (at >= 0 && at < kGapRows) found |= 1u << at;
      }
      uint32_t gaps = 0;
#pragma unroll
      for (int r = 0; r < kGapRows; ++r) gaps |= (row + r < vocab && __ballot(found >> r & 1) == 0) ? 1u << r : 0u;
      clear_gap_rows(Clear{table, 0, vocab, dim, table_stride}, row, gaps);
    }
    return;
  }
  const int i = (int)(unit / across);
  const int64_t id = (int64_t)ids[i];
  if (id < 0 || id >= vocab) return;
  for (int j = l; j - l < i; j += kWave)
    if (__ballot(j < i && (int64_t)ids[j] == id) != 0) return;
  const int64_t c = ((int64_t)(unit % across) * kWave + l) * N, left = EVEN ? min(dim - c, (int64_t)N) : dim - c;
  const bool mine = left > 0;
  const T* from = grad + (EVEN && !mine ? 0 : c);
  F32<N> acc = {};
  for (int j0 = i; j0 < n; j0 += kWave) {
    uint64_t same = __ballot(j0 + l < n && (int64_t)ids[min(j0 + l, n - 1)] == id);
    while (same) {
      // up to kFewAhead rows under way; behind the last one it is requested again
      const int here = min(kFewAhead, (int)__popcll(same));
      Pack<T, N> v[kFewAhead];
      int at = 0;
#pragma unroll
      for (int k = 0; k < kFewAhead; ++k) {
        if (same) {
          at = __builtin_ctzll(same);
          same &= same - 1;
        }
        const T* p = from + (int64_t)(j0 + at) * grad_stride;
        v[k] = EVEN ? load<N>(p) : load_some<N>(p, left);
      }
#pragma unroll
      for (int k = 0; k < kFewAhead; ++k)
        if (k < here) acc += widen<T, N>(v[k]);
    }
  }
  if (!mine) return;
  float* to = table + id * table_stride + c;
  F32<N> old = {};
  if (ACCUMULATE) old = widen<float, N>(EVEN ? load<N>(to) : load_some<N>(to, left));
  to_row<N>(to, acc, old, scale, ACCUMULATE, EVEN ? N : left);
}

// Few tokens: a token's place is the number of tokens that come before it, counted against all others.  A workgroup
// holds all keys in LDS and places 64 tokens (one per lane); its waves share the tokens to compare with, four per
// read: two operations per pair of tokens.  (672 columns, us per call, counted and sorted: 8192 tokens 33.0 and 34.2, 10000 37.4 and 36.4,
// 14000 46 and 40.)
constexpr int kRankThreads = 1024, kRankAhead = 4;   // ids under way per thread
template <typename I>
__global__ __launch_bounds__(kRankThreads) void embedding_rank_kernel(const I* __restrict__ ids, int n, uint32_t vocab,
                                                                     uint32_t* __restrict__ skey, uint32_t* __restrict__ spos,
                                                                     int rank_blocks, Clear clear) {
  if ((int)blockIdx.x >= rank_blocks) {
    clear_rows(clear, (int64_t)blockIdx.x - rank_blocks, (int64_t)gridDim.x - rank_blocks);
    return;
  }
  extern __shared__ uint32_t keys[];     // n, filled up to whole groups of four with keys above all others
  __shared__ uint32_t part[kRankThreads];
  constexpr int waves = kRankThreads / kWave;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (n + 3) >> 2;
  for (int j0 = threadIdx.x; j0 < 4 * groups; j0 += kRankAhead * kRankThreads) {
    I v[kRankAhead];
#pragma unroll
    for (int k = 0; k < kRankAhead; ++k) v[k] = ids[min(j0 + k * kRankThreads, n - 1)];
#pragma unroll
    for (int k = 0; k < kRankAhead; ++k) {
      const int j = j0 + k * kRankThreads;
      if (j < 4 * groups) keys[j] = j < n ? key_of_id(v[k], vocab) : 0xffffffffu;
    }
  }
  __syncthreads();
  const int first = blockIdx.x * kWave, i = first + l;
  const uint32_t mine = keys[min(i, n - 1)];
  const uint4* quads = reinterpret_cast<const uint4*>(keys);
  const int share = (groups + waves - 1) / waves, lo = min(w * share, groups), hi = min(lo + share, groups);
  // in front of the workgroup's own tokens an equal key counts, behind them it does not (16 groups are the workgroup's own)
  const int own = first >> 2;
  uint32_t before = 0;
#pragma unroll 4
  for (int j = lo; j < min(hi, own); ++j) {
    const uint4 k = quads[j];
    before += (uint32_t)(k.x <= mine) + (uint32_t)(k.y <= mine) + (uint32_t)(k.z <= mine) + (uint32_t)(k.w <= mine);
  }
  for (int j = max(lo, own); j < min(hi, own + kWave / 4); ++j)
    for (int q = 0; q < 4; ++q) {
      const uint32_t k = keys[4 * j + q];
      before += k < mine || (k == mine && 4 * j + q < i);
    }
#pragma unroll 4
  for (int j = max(lo, own + kWave / 4); j < hi; ++j) {
    const uint4 k = quads[j];
    before += (uint32_t)(k.x < mine) + (uint32_t)(k.y < mine) + (uint32_t)(k.z < mine) + (uint32_t)(k.w < mine);
  }
  part[threadIdx.x] = before;
  __syncthreads();
  if (w == 0 && i < n) {
    uint32_t place = 0;
    for (int k = 0; k < waves; ++k) place += part[k * kWave + l];
    skey[place] = mine;
    spos[place] = (uint32_t)i;
  }
}

// Many tokens: stable counting passes over digits of up to 10 key bits, lowest first.  A workgroup takes a tile of
// consecutive tokens, 1024 (kSortItems per thread) at a time.  (us per call with 1, 2, 4, 8 items: 20000 tokens of 672 columns 49, 51, 58, 72; 40000
// 73, 75, 78, 94; 131072 of 2048 254, 250, 255, 270.)
constexpr int kSortThreads = 1024, kSortItems = 1, kSortStep = kSortThreads * kSortItems, kSortTiles = 128;
constexpr int kSortDigitBits = 10, kSortDigits = 1 << kSortDigitBits;

// Where a pass finds its keys: in the ids (first pass: the position is the place) or in the last pass's order.
template <typename I, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const I* ids, const uint32_t* key, int64_t i, uint32_t vocab) {
  if (FIRST) return key_of_id(ids[i], vocab);
  return key[i];
}

template <typename I, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(const I* __restrict__ ids, const uint32_t* __restrict__ key,
                                                                      int64_t n, uint32_t vocab, int64_t tile, int shift, int digits,
                                                                      uint32_t* __restrict__ counts, int tiles, Clear clear) {
  if ((int)blockIdx.x >= tiles) {
    clear_rows(clear, (int64_t)blockIdx.x - tiles, (int64_t)gridDim.x - tiles);
    return;
  }
  __shared__ uint32_t count[kSortDigits];
  for (int d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * tile, hi = min(n, lo + tile);
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads)
    atomicAdd(&count[(sort_key<I, FIRST>(ids, key, i, vocab) >> shift) & (digits - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) counts[(int64_t)blockIdx.x * digits + d] = count[d];
}

constexpr int kCountAhead = 32;   // tiles' counts under way

template <typename I, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void embedding_place_kernel(const I* __restrict__ ids, const uint32_t* __restrict__ key,
                                                                      const uint32_t* __restrict__ pos, int64_t n, uint32_t vocab,
                                                                      int64_t tile, int shift, int digit_bits,
                                                                      const uint32_t* __restrict__ counts, int tiles,
                                                                      uint32_t* __restrict__ key_out, uint32_t* __restrict__ pos_out,
                                                                      Clear clear) {
  if ((int)blockIdx.x >= tiles) {
    clear_rows(clear, (int64_t)blockIdx.x - tiles, (int64_t)gridDim.x - tiles);
    return;
  }
  constexpr int waves = kSortThreads / kWave;
  __shared__ uint32_t base[kSortDigits];               // where the tile's next token of a digit goes
  __shared__ __align__(16) uint16_t seen[waves][kSortDigits];   // tokens of a digit in a wave, then in the waves before it
  __shared__ uint32_t sums[waves];
  const int digits = 1 << digit_bits;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, d = threadIdx.x;
  // all tiles' tokens of smaller digits, and of this digit those of the tiles in front (kSortDigits == kSortThreads)
  uint32_t all = 0, front = 0;
  if (d < digits)
    for (int t0 = 0; t0 < tiles; t0 += kCountAhead) {
      uint32_t c[kCountAhead];
#pragma unroll
      for (int k = 0; k < kCountAhead; ++k) c[k] = t0 + k < tiles ? counts[(int64_t)(t0 + k) * digits + d] : 0u;
#pragma unroll
      for (int k = 0; k < kCountAhead; ++k) {
        if (t0 + k < (int)blockIdx.x) front += c[k];
        all += c[k];
      }
    }
  uint32_t incl = all;
  for (int s = 1; s < kWave; s <<= 1) {
    const uint32_t o = __shfl_up(incl, s, kWave);
    if (l >= s) incl += o;
  }
  if (l == 63) sums[w] = incl;
  __syncthreads();
  uint32_t smaller = incl - all;
  for (int k = 0; k < w; ++k) smaller += sums[k];
  base[d] = smaller + front;
  const int64_t lo = blockIdx.x * tile, hi = min(n, lo + tile);
  for (int64_t step = lo; step < hi; step += kSortStep) {
    for (int k = threadIdx.x; k < waves * kSortDigits / 8; k += kSortThreads) reinterpret_cast<uint4*>(seen)[k] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    uint32_t k[kSortItems], p[kSortItems], rank[kSortItems];
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
      const int64_t i = step + w * (kWave * kSortItems) + r * kWave + l;
      k[r] = p[r] = 0;
      if (i < hi) {
        k[r] = sort_key<I, FIRST>(ids, key, i, vocab);
        p[r] = FIRST ? (uint32_t)i : pos[i];
      }
    }
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
      const int64_t i = step + w * (kWave * kSortItems) + r * kWave + l;
      const bool in = i < hi;
      const uint32_t dig = (k[r] >> shift) & (digits - 1);
      uint64_t same = __ballot(in);
      for (int b = 0; b < digit_bits; ++b) {
        const uint64_t ones = __ballot((dig >> b) & 1);
        same &= (dig >> b) & 1 ? ones : ~ones;
      }
      const uint32_t below = __popcll(same & ((1ull << l) - 1));
      const uint32_t had = in ? seen[w][dig] : 0;
      rank[r] = had + below;
      // the wave's lanes read and write its counts in turn
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (in && below == 0) seen[w][dig] = (uint16_t)(had + __popcll(same));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // tokens of a digit: waves in front of each wave; the tile's base moves on once all have read it
    uint32_t run = 0;
    if (d < digits)
      for (int k2 = 0; k2 < waves; ++k2) {
        const uint32_t c = seen[k2][d];
        seen[k2][d] = (uint16_t)run;
        run += c;
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
      const int64_t i = step + w * (kWave * kSortItems) + r * kWave + l;
      if (i < hi) {
        const uint32_t dig = (k[r] >> shift) & (digits - 1);
        const uint32_t to = base[dig] + seen[w][dig] + rank[r];
        key_out[to] = k[r];
        pos_out[to] = p[r];
      }
    }
    __syncthreads();
    if (d < digits) base[d] += run;
    __syncthreads();
  }
}

// ---- backward: sums over runs of equal ids ---------------------------------------------------------------
// A wave takes a chunk of consecutive places of the order and 64 N columns.  A run of equal ids inside the chunk is
// summed and written to its row; of a run that crosses the chunk's ends the part inside is left in the workspace:
// parts[2 c] for a run that began in an earlier chunk, parts[2 c + 1] for one that begins here and goes on.
// Bound by memory: 131072 tokens of 2048 bf16 added to 65537 rows 196 us (4.9 TB/s); by latency: 2800 of 672 fp32 12 us beside clearing 48 MB.
constexpr int kSumAhead = 8;     // rows under way
constexpr int kJoinRows = 16;    // parts under way

// EVEN: N divides the columns.  STREAM: gradients and rows go past the caches (131072 tokens x 2048 bf16 into 65537 rows: 271 ->
// 247 us, added to what is there 276 -> 253; 2800 tokens x 672 fp32: 25.7 -> 26.5).
template <typename T, int N, bool ACCUMULATE, bool EVEN, bool STREAM>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const uint32_t* __restrict__ skey, const uint32_t* __restrict__ spos,
                                                            int64_t n, int chunk, uint32_t vocab, const T* __restrict__ grad,
                                                            int64_t grad_stride, float* __restrict__ table, int64_t table_stride,
                                                            int64_t dim, uint32_t across, uint32_t units, float scale,
                                                            float* __restrict__ parts, int64_t gap_rows, uint32_t gap_units) {
  // neighbouring waves take neighbouring columns of one chunk; those beyond the chunks' clear rows [0, gap_rows)
  const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= units) {
    if (unit - units < gap_units)
      for (int64_t row = (int64_t)(unit - units) * kGapRows; row < gap_rows; row += (int64_t)gap_units * kGapRows)
        clear_gaps(Clear{table, 0, gap_rows, dim, table_stride}, row, gap_rows, skey, n);
    return;
  }
  const int64_t b = unit / across, lo = b * chunk, hi = min(n, lo + chunk);
  const int64_t c = ((int64_t)(unit % across) * kWave + (threadIdx.x & 63)) * N, left = EVEN ? min(dim - c, (int64_t)N) : dim - c;
  if (lo >= n) return;
  const bool mine = left > 0;          // every lane stays: each holds a place of the order for all of them
  const int count = (int)(hi - lo), l = threadIdx.x & 63;
  bool opened = lo == 0 || skey[lo - 1] != skey[lo];   // the run began in this chunk
  F32<N> acc = {};
  for (int part = 0; part < count; part += kWave - 1) {
    // lane l holds place part + l; 63 places at a time, so that the key behind each is there too
    const int64_t i = lo + part + l;
    const uint32_t keys = i < n ? skey[i] : 0xffffffffu, places = i < n ? spos[i] : 0u;
    const int here = min(kWave - 1, count - part);
    for (int j0 = 0; j0 < here; j0 += kSumAhead) {
      Pack<T, N> v[kSumAhead];
#pragma unroll
      for (int j = 0; j < kSumAhead; ++j) {
        // places behind the last one load it again, lanes without columns the first ones: no branch between the requests
        const int at = min(j0 + j, here - 1);
        const T* from = grad + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)places, at) * grad_stride + (EVEN && !mine ? 0 : c);
        v[j] = STREAM ? load_stream<N>(from) : EVEN ? load<N>(from) : load_some<N>(from, left);
      }
#pragma unroll
      for (int j = 0; j < kSumAhead; ++j) {
        const int at = j0 + j;
        if (at >= here) break;
        const uint32_t key = (uint32_t)__builtin_amdgcn_readlane((int)keys, at), next = (uint32_t)__builtin_amdgcn_readlane((int)keys, at + 1);
        if (key >= vocab) break;                         // nothing but ids outside the table from here on
        acc += widen<T, N>(v[j]);
        if (next != key) {                               // the run ends here
          if (mine) {
            if (opened) {
              float* to = table + (int64_t)key * table_stride + c;
              F32<N> old = {};
              if (ACCUMULATE) old = widen<float, N>(EVEN ? load<N>(to) : load_some<N>(to, left));
              if (STREAM) store_stream<float, N>(to, ACCUMULATE ? old + acc * scale : acc * scale);
              else to_row<N>(to, acc, old, scale, ACCUMULATE, EVEN ? N : left);
            } else {
              store_some<float, N>(parts + 2 * b * dim + c, acc, EVEN ? N : left);
            }
          }
          opened = true;
          acc = F32<N>{};
        } else if (part + at == count - 1) {             // ... or in a later chunk
          if (mine) store_some<float, N>(parts + (2 * b + (opened ? 1 : 0)) * dim + c, acc, EVEN ? N : left);
        }
      }
    }
  }
}

// The runs that cross chunks: the workgroup of the chunk where one begins adds its parts in order, its first wave those of
// short runs, all its waves a share each of long ones (a frequent token has thousands of rows).  131072 tokens 27 us, 2800 4.4.
constexpr int kJoinWaves = 4;
template <int N>
__global__ __launch_bounds__(kWave* kJoinWaves) void embedding_join_kernel(const uint32_t* __restrict__ skey, int64_t n, int chunk,
                                                                          int64_t chunks, uint32_t vocab,
                                                                          const float* __restrict__ parts, float* __restrict__ table,
                                                                          int64_t table_stride, int64_t dim, float scale, int accumulate) {
  const int64_t b = blockIdx.x, lo = b * chunk, hi = lo + chunk;
  if (hi >= n) return;
  const uint32_t row = skey[hi];
  if (row >= vocab || skey[hi - 1] != row || (lo > 0 && skey[lo] == row && skey[lo - 1] == row)) return;
  // the chunks that begin with the run's id
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t end = b + 1;
  for (;;) {
    const int64_t k = end + l;
    const uint64_t others = __ballot(k >= chunks || skey[min(k, chunks - 1) * chunk] != row);
    end += others ? __builtin_ctzll(others) : kWave;
    if (others) break;
  }
  const int64_t count = end - b - 1;
  const bool shared = count > kJoinRows;               // the same for the whole workgroup
  if (!shared && w > 0) return;
  const int64_t share = shared ? (count + kJoinWaves - 1) / kJoinWaves : count;
  const int64_t from = min(b + 1 + w * share, end), to_part = min(from + share, end);
  const int64_t c = ((int64_t)blockIdx.y * kWave + l) * N, left = dim - c;
  float* to = table + (int64_t)row * table_stride + c;
  F32<N> old = {}, acc = {};
  if (w == 0) {
    acc = widen<float, N>(load_some<N>(parts + (2 * b + 1) * dim + c, left));
    if (accumulate) old = widen<float, N>(load_some<N>(to, left));
  }
  for (int64_t k = from; k < to_part; k += kJoinRows) {
    Pack<float, N> v[kJoinRows];
#pragma unroll
    for (int j = 0; j < kJoinRows; ++j) v[j] = load_some<N>(parts + 2 * min(k + j, to_part - 1) * dim + c, left);
#pragma unroll
    for (int j = 0; j < kJoinRows; ++j)
      if (k + j < to_part) acc += widen<float, N>(v[j]);
  }
  if (shared) {
    __shared__ F32<N> of[kJoinWaves][kWave];
    of[w][l] = acc;
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int k = 1; k < kJoinWaves; ++k) acc += of[k][l];
  }
  if (left > 0) to_row<N>(to, acc, old, scale, accumulate != 0, left);
}

}  // namespace accop
