// Host side of the language-model operators declared in include/accordion.h: argument checks, workspace layout,
// choice of kernels and the launches.
#include "../../../include/accordion.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <memory>
#include <new>
#include <tuple>

#include "op_common.h"
#include "adamw.h"
#include "embedding.h"
#include "layernorm.h"
#include "recurrence.h"

using namespace accop;

namespace {

thread_local char g_error[256] = "no error";

int32_t fail(int32_t code, const char* msg) {
  std::snprintf(g_error, sizeof g_error, "%s", msg);
  return code;
}

#define REQUIRE(cond, msg) \
  do {                     \
    if (!(cond)) return fail(ACC_EINVAL, msg); \
  } while (0)

constexpr int kComputeUnits = 256;
constexpr int64_t kMaxStride = int64_t(1) << 40;
// A launch has fewer than 2^32 work items per axis: rows beyond this many go into further launches.
constexpr int64_t kRowsPerLaunch = int64_t(1) << 21;

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round256(int64_t bytes) { return up(bytes, 256) * 256; }
inline int type_bytes(int32_t t) { return t == ACC_BF16 ? 2 : 4; }
inline bool is_type(int32_t t) { return t == ACC_FLOAT || t == ACC_BF16; }
inline bool off_type(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes != 0; }

// A buffer's first byte and the bytes it spans; where its rows lie apart, the bytes of a row and a distance of which all
// distances between rows are multiples (0: none); where rows lie in blocks, the bytes of a block and the distance between blocks (0: none).
struct Span {
  const char* p;
  int64_t bytes, row = 0, every = 0, block = 0, far = 0;
};
inline Span rows_span(const void* p, int64_t rows, int64_t dim, int64_t stride, int elem) {
  return {static_cast<const char*>(p), p && rows > 0 ? ((rows - 1) * stride + dim) * elem : 0, dim * elem, rows > 1 ? stride * elem : 0};
}
// Whether pieces of a bytes from one place on and of b bytes from `to_b` behind it, both repeated every so many bytes, are apart.
inline bool pieces_apart(int64_t to_b, int64_t a, int64_t b, int64_t every) {
  const int64_t at = (to_b % every + every) % every;
  return at >= a && at <= every - b;
}
inline bool overlap(const Span& a, const Span& b) {
  if (!(a.bytes > 0 && b.bytes > 0 && a.p < b.p + b.bytes && b.p < a.p + a.bytes)) return false;
  if (a.every > 0 && a.every == b.every && pieces_apart(b.p - a.p, a.row, b.row, a.every)) return false;   // columns of one larger buffer
  return !(a.far > 0 && a.far == b.far && pieces_apart(b.p - a.p, a.block, b.block, a.far));               // steps of one
}
// Whether one of the first `written` buffers shares memory with any other.
bool any_overlap(const Span* s, int written, int all) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < all; ++j)
      if (overlap(s[i], s[j])) return true;
  return false;
}

int32_t check_workspace(const void* ws, size_t have, int64_t need) {
  if (need == 0) return ACC_OK;
  REQUIRE(ws, "workspace_dev is NULL");
  REQUIRE(reinterpret_cast<uintptr_t>(ws) % 256 == 0, "workspace_dev is not 256-byte aligned");
  if (have < (size_t)need) return fail(ACC_ENOSPACE, "workspace too small");
  return ACC_OK;
}

// A call's launches, in order: after one that fails nothing more is enqueued, and what other calls of this thread left behind as
// HIP's last error plays no role.
struct Queue {
  hipStream_t stream;
  hipError_t status = hipSuccess;
  explicit Queue(void* s) : stream(static_cast<hipStream_t>(s)) {}
};

template <typename... P, typename... A>
void enqueue(Queue& q, void (*kernel)(P...), dim3 grid, dim3 block, unsigned lds, const A&... args) {
  static_assert(sizeof...(P) == sizeof...(A), "a kernel's arguments");
  if (q.status != hipSuccess) return;
  std::tuple<P...> held{static_cast<P>(args)...};
  std::apply(
      [&](P&... each) {
        void* at[] = {static_cast<void*>(&each)...};
        q.status = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, lds, q.stream);
      },
      held);
}

int32_t launched(const Queue& q) {
  if (q.status == hipSuccess) return ACC_OK;
  (void)hipGetLastError();                 // it is reported here
  std::snprintf(g_error, sizeof g_error, "kernel launch failed: %s", hipGetErrorString(q.status));
  return ACC_EHIP;
}

#define LAUNCH(kernel, grid, block, queue, ...) enqueue(queue, kernel, grid, block, 0, __VA_ARGS__)

// ---- embedding --------------------------------------------------------------------------------------

constexpr int64_t kFewTokens = 512;     // up to here nothing is ordered (embedding_few_kernel)
constexpr int64_t kRankTokens = 8192;   // up to here the order is counted, from here on it is sorted by digits

int32_t check_embedding(const acc_embedding* e) {
  REQUIRE(e, "config is NULL");
  REQUIRE(e->vocab >= 1 && e->vocab <= (int64_t(1) << 31) - 2, "vocab out of range");
  REQUIRE(e->dim >= 1 && e->dim <= (int64_t(1) << 23), "dim out of range");
  REQUIRE(e->tokens >= 0 && e->tokens <= (int64_t(1) << 28), "tokens out of range");
  REQUIRE(e->index_bits == 32 || e->index_bits == 64, "index_bits must be 32 or 64");
  REQUIRE(is_type(e->table_type) && is_type(e->out_type), "unknown type");
  REQUIRE(e->accumulate == 0 || e->accumulate == 1, "accumulate must be 0 or 1");
  REQUIRE(std::isfinite(e->scale), "scale must be finite");
  REQUIRE(e->vocab == 1 || (e->table_stride >= e->dim && e->table_stride <= kMaxStride), "table_stride out of range");
  REQUIRE(e->tokens <= 1 || (e->out_stride >= e->dim && e->out_stride <= kMaxStride), "out_stride out of range");
  return ACC_OK;
}

// Waves that sum: fewer than a launch has (see kRowsPerLaunch).
constexpr int64_t kMostUnits = int64_t(1) << 25;

struct EmbeddingPlan {
  bool few, rank;
  int passes = 0, digit_bits = 0, tiles = 0, chunk = 0;
  int64_t tile = 0, chunks = 0;
  int64_t key[2], pos[2], counts, parts, bytes;   // offsets in the workspace
};

EmbeddingPlan plan_embedding(const acc_embedding& e) {
  EmbeddingPlan p{};
  const int64_t n = e.tokens;
  p.few = n <= kFewTokens;
  if (p.few) {
    p.chunks = n;                      // a token takes the place of a chunk
    return p;
  }
  p.rank = n <= kRankTokens;
  if (!p.rank) {
    int bits = 1;
    while ((e.vocab >> bits) != 0) ++bits;            // keys go up to vocab
    p.passes = (int)up(bits, kSortDigitBits);
    p.digit_bits = (int)up(bits, p.passes);
    p.tile = up(up(n, kSortTiles), kSortStep) * kSortStep;
    p.tiles = (int)up(n, p.tile);
  }
  // A wave goes through a chunk's tokens one after the other, and a few through the parts of a run, of which there may be one per
  // chunk: chunks of about sqrt(n) / 12 to sqrt(n) / 6, twice that where waves abound or runs are long (us at the shorter and the longer:
  // 86738 tokens of 62 columns 59 and 77, 20000 of 672 45 and 46, 131072 of 2048 264 and 249, 128345 of 348 in 425 rows 79 and 68; added to 65537 rows
  // in fp32, 131072 tokens of 672 columns 135 and 136, 1024 174 and 175, 1280 210 and 198, 1536 245 and 229, 2048 320 and 297).
  const int64_t scale = up(e.dim, kWave * 4) >= 8 || n > 32 * e.vocab ? 64 : 128;
  p.chunk = 8;
  while (p.chunk < 128 && scale * p.chunk * p.chunk < n) p.chunk *= 2;
  p.chunks = up(n, p.chunk);
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t o = at; at += round256(bytes); return o; };
  p.key[0] = take(4 * n);
  p.pos[0] = take(4 * n);
  p.key[1] = p.rank ? 0 : take(4 * n);
  p.pos[1] = p.rank ? 0 : take(4 * n);
  p.counts = p.rank ? 0 : take(4 * (int64_t)p.tiles << p.digit_bits);
  p.parts = take(8 * p.chunks * e.dim);
  p.bytes = at;
  return p;
}

// Lanes of a row with two requests each from here on, with one below.  us, one and two: 672 columns fp32 1024 tokens 3.0 and 3.2, 4096 4.4
// and 3.9, 65536 40 and 37; bf16 2048 3.3 and 3.3, 4096 3.9 and 3.7, 65536 25 and 20; rows of whole waves' requests the same either way.
constexpr int64_t kLookupMany = 4096;

template <typename I, typename T, typename O>
void lookup(const acc_embedding& e, const void* ids, const void* table, void* out, Queue& queue) {
  constexpr int N = sizeof(T) == 2 ? 8 : 4;
  int lanes_log2 = 3;
  // many tokens: lanes with all their requests under way; few: lanes for all columns
  const int each = e.tokens >= kLookupMany ? kLookupLoads : 1;
  while (lanes_log2 < 8 && ((int64_t)(N * each) << lanes_log2) < e.dim) ++lanes_log2;
  const int64_t across = up(e.dim, (int64_t)kLookupLoads * N << lanes_log2);
  for (int64_t t = 0; t < e.tokens; t += kRowsPerLaunch) {
    const int64_t n = std::min(kRowsPerLaunch, e.tokens - t);
    LAUNCH((embedding_lookup_kernel<I, T, O, N>), dim3((unsigned)up(n << lanes_log2, 256), (unsigned)across), dim3(256), queue,
           static_cast<const I*>(ids) + t, static_cast<const T*>(table), static_cast<O*>(out) + t * e.out_stride, n, e.vocab, e.dim,
           e.table_stride, e.out_stride, e.scale, lanes_log2);
  }
}

template <typename I, typename T>
void lookup_to(const acc_embedding& e, const void* ids, const void* table, void* out, Queue& queue) {
  e.out_type == ACC_BF16 ? lookup<I, T, bf16>(e, ids, table, out, queue) : lookup<I, T, float>(e, ids, table, out, queue);
}

constexpr int64_t kSumStream = 128 << 20;   // bytes of gradients that are streamed from here on (they fit no cache)
// Rows cleared beside the ordering of the tokens: what the memory takes while a launch of it lasts.
constexpr int64_t kClearRank = 40 << 20, kClearCount = 16 << 20, kClearPlace = 48 << 20;   // bytes

template <typename T>
void sum_runs(const acc_embedding& e, const EmbeddingPlan& p, const uint32_t* key, const uint32_t* pos, const void* grad,
              float* table, int64_t stride, float* parts, int64_t gap_rows, Queue& queue) {
  constexpr int N = 4;
  const int64_t across = up(e.dim, kWave * N), units = p.chunks * across;
  const int64_t gap_units = std::min<int64_t>(up(gap_rows, kGapRows), int64_t(1) << 20);
  const dim3 grid((unsigned)up(units + gap_units, 4));
  const bool stream_rows = e.tokens * e.dim * (int64_t)sizeof(T) > kSumStream;
#define SUM(ACCUMULATE, EVEN, STREAM)                                                                                              \
  LAUNCH((embedding_sum_kernel<T, N, ACCUMULATE, EVEN, STREAM>), grid, dim3(256), queue, key, pos, e.tokens, p.chunk,             \
         (uint32_t)e.vocab, static_cast<const T*>(grad), e.out_stride, table, stride, e.dim, (uint32_t)across, (uint32_t)units,    \
         e.scale, parts, gap_rows, (uint32_t)gap_units)
  if (e.dim % N != 0) {
    if (e.accumulate) SUM(true, false, false);
    else SUM(false, false, false);
  } else if (stream_rows) {
    if (e.accumulate) SUM(true, true, true);
    else SUM(false, true, true);
  } else {
    if (e.accumulate) SUM(true, true, false);
    else SUM(false, true, false);
  }
#undef SUM
}

template <typename I, typename T>
void sum_few(const acc_embedding& e, const I* ids, const void* grad, float* table, int64_t stride, Queue& queue) {
  constexpr int N = 4;
  const int64_t across = up(e.dim, kWave * N), units = e.tokens * across;
  const int64_t gap_units = e.accumulate ? 0 : std::min<int64_t>(up(e.vocab, kGapRows), int64_t(1) << 20);
  if (units + gap_units == 0) return;
#define FEW(ACCUMULATE, EVEN)                                                                                                     \
  LAUNCH((embedding_few_kernel<I, T, N, ACCUMULATE, EVEN>), dim3((unsigned)up(units + gap_units, 4)), dim3(256), queue, ids,     \
         (int)e.tokens, e.vocab, static_cast<const T*>(grad), e.out_stride, table, stride, e.dim, (uint32_t)across,               \
         (uint32_t)units, e.scale, (uint32_t)gap_units)
  if (e.dim % N == 0) {
    if (e.accumulate) FEW(true, true);
    else FEW(false, true);
  } else {
    if (e.accumulate) FEW(true, false);
    else FEW(false, false);
  }
#undef FEW
}

template <typename I>
void embedding_gradient(const acc_embedding& e, const EmbeddingPlan& p, const I* ids, const void* grad, float* table, char* ws,
                        Queue& queue) {
  uint32_t* key[2] = {reinterpret_cast<uint32_t*>(ws + p.key[0]), reinterpret_cast<uint32_t*>(ws + p.key[1])};
  uint32_t* pos[2] = {reinterpret_cast<uint32_t*>(ws + p.pos[0]), reinterpret_cast<uint32_t*>(ws + p.pos[1])};
  uint32_t* counts = reinterpret_cast<uint32_t*>(ws + p.counts);
  float* parts = reinterpret_cast<float*>(ws + p.parts);
  const uint32_t vocab = (uint32_t)e.vocab;
  const int64_t stride = e.vocab == 1 ? e.dim : e.table_stride;
  if (p.few) {
    if (e.out_type == ACC_BF16) sum_few<I, bf16>(e, ids, grad, table, stride, queue);
    else sum_few<I, float>(e, ids, grad, table, stride, queue);
    return;
  }
  // rows [0, dirty) are still to be cleared; share() takes the last ones of them off, as many as `bytes` hold
  int64_t dirty = e.accumulate ? 0 : e.vocab;
  auto share = [&](int64_t bytes) {
    const int64_t rows = std::min(dirty, std::max<int64_t>(1, bytes / (4 * e.dim)));
    dirty -= rows;
    return Clear{table, dirty, rows, e.dim, stride};
  };
  auto blocks = [&](const Clear& c) { return std::min<int64_t>(up(c.rows * c.dim, 4 * kClearAhead * 1024), 8 * kComputeUnits); };
  int at = 0;
  if (p.rank) {
    const int rank_blocks = (int)up(e.tokens, kWave);
    const Clear clear = share(kClearRank);
    if (rank_blocks + blocks(clear) > 0)
      enqueue(queue, embedding_rank_kernel<I>, dim3((unsigned)(rank_blocks + blocks(clear))), dim3(kRankThreads),
              (unsigned)round256(4 * e.tokens), ids, (int)e.tokens, vocab, key[0], pos[0], rank_blocks, clear);
  } else {
    for (int pass = 0; pass < p.passes; ++pass) {
      const int shift = pass * p.digit_bits, digits = 1 << p.digit_bits, to = pass & 1;
      const Clear c = share(kClearCount), d = share(kClearPlace);
      const dim3 count_grid((unsigned)(p.tiles + blocks(c))), place_grid((unsigned)(p.tiles + blocks(d)));
      if (pass == 0) {
        LAUNCH((embedding_count_kernel<I, true>), count_grid, dim3(kSortThreads), queue, ids, nullptr, e.tokens, vocab, p.tile, shift,
               digits, counts, p.tiles, c);
        LAUNCH((embedding_place_kernel<I, true>), place_grid, dim3(kSortThreads), queue, ids, nullptr, nullptr, e.tokens, vocab, p.tile,
               shift, p.digit_bits, counts, p.tiles, key[to], pos[to], d);
      } else {
        LAUNCH((embedding_count_kernel<I, false>), count_grid, dim3(kSortThreads), queue, ids, key[at], e.tokens, vocab, p.tile, shift,
               digits, counts, p.tiles, c);
        LAUNCH((embedding_place_kernel<I, false>), place_grid, dim3(kSortThreads), queue, ids, key[at], pos[at], e.tokens, vocab, p.tile,
               shift, p.digit_bits, counts, p.tiles, key[to], pos[to], d);
      }
      at = to;
    }
  }
  if (e.out_type == ACC_BF16) sum_runs<bf16>(e, p, key[at], pos[at], grad, table, stride, parts, dirty, queue);
  else sum_runs<float>(e, p, key[at], pos[at], grad, table, stride, parts, dirty, queue);
  LAUNCH((embedding_join_kernel<4>), dim3((unsigned)p.chunks, (unsigned)up(e.dim, kWave * 4)), dim3(kWave * kJoinWaves), queue, key[at], e.tokens,
         p.chunk, p.chunks, vocab, parts, table, stride, e.dim, e.scale, e.accumulate);
}

// ---- layer norm -------------------------------------------------------------------------------------

int32_t check_layernorm(const acc_layernorm* c, bool backward) {
  REQUIRE(c, "config is NULL");
  REQUIRE(c->rows >= 0 && c->rows < (int64_t(1) << 31), "rows out of range");
  REQUIRE(c->dim >= 1 && c->dim <= (int64_t(1) << 24), "dim out of range");
  REQUIRE(is_type(c->type), "unknown type");
  REQUIRE(std::isfinite(c->eps) && c->eps >= 0.f, "eps must be finite and not negative");
  REQUIRE(c->accumulate == 0 || c->accumulate == 1, "accumulate must be 0 or 1");
  if (c->rows > 1) {
    REQUIRE(c->x_stride >= c->dim && c->x_stride <= kMaxStride, "x_stride out of range");
    REQUIRE(c->y_stride >= c->dim && c->y_stride <= kMaxStride, "y_stride out of range");
    if (backward) REQUIRE(c->grad_x_stride >= c->dim && c->grad_x_stride <= kMaxStride, "grad_x_stride out of range");
  }
  return ACC_OK;
}

template <typename T>
void norm_forward(const acc_layernorm& c, const T* x, const float* w, const float* b, T* y, float* mean, float* rstd, int64_t rows,
                  Queue& queue) {
  constexpr int N = sizeof(T) == 2 ? 8 : 4;
  const int64_t packs = up(c.dim, N);
#define FORWARD(THREADS, K, BLOCK)                                                                                                \
  LAUNCH((layernorm_forward_kernel<T, N, THREADS, K, BLOCK>), dim3((unsigned)up(rows, BLOCK / THREADS)), dim3(BLOCK), queue, x, w, \
         b, y, mean, rstd, rows, (int)c.dim, c.x_stride, c.y_stride, c.eps)
  if (packs <= 16) FORWARD(16, 1, 256);
  else if (packs <= 32) FORWARD(16, 2, 256);
  else if (packs <= 64) FORWARD(64, 1, 256);
  else if (packs <= 128) FORWARD(64, 2, 256);
  else if (packs <= 256) FORWARD(64, 4, 256);
  else if (packs <= 512) FORWARD(256, 2, 256);
  else if (packs <= 1024) FORWARD(256, 4, 256);
  else if (packs <= 2048) FORWARD(256, 8, 256);
  else if (packs <= 4096) FORWARD(1024, 4, 1024);
  else
    LAUNCH((layernorm_forward_long_kernel<T, N>), dim3((unsigned)rows), dim3(256), queue, x, w, b, y, mean, rstd, (int)c.dim,
           c.x_stride, c.y_stride, c.eps);
#undef FORWARD
}

template <typename T>
void norm_forward_rows(const acc_layernorm& c, const void* x, const float* w, const float* b, void* y, float* mean, float* rstd,
                       Queue& queue) {
  for (int64_t r = 0; r < c.rows; r += kRowsPerLaunch)
    norm_forward<T>(c, static_cast<const T*>(x) + r * c.x_stride, w, b, static_cast<T*>(y) + r * c.y_stride, mean ? mean + r : nullptr,
                    rstd ? rstd + r : nullptr, std::min(kRowsPerLaunch, c.rows - r), queue);
}

// Parts that the backward pass leaves (two rows of dim each): enough workgroups to fill the chip, no more than rows.  Two per
// compute unit where a wave has a row, one where a workgroup has (4096 x 8192 bf16 with two: 58 us, with one 52; 5003 x 1001 fp32
// 18.4 and 18.7).
int64_t norm_parts(const acc_layernorm& c) {
  const int64_t packs = up(c.dim, c.type == ACC_BF16 ? 8 : 4);
  const int64_t at_once = packs <= 32 ? 16 : packs <= 256 ? 4 : 1;      // rows a workgroup has under way
  const int64_t most = (packs <= 256 ? 2 : 1) * kComputeUnits;
  // no more than keep the longest wave as short as it is
  const int64_t turns = std::max<int64_t>(1, up(c.rows, most * at_once));
  return std::max<int64_t>(1, up(c.rows, turns * at_once));
}

template <typename T>
void norm_backward(const acc_layernorm& c, const void* dy, const void* x, const float* w, const float* mean, const float* rstd,
                   void* dx, float* dw, float* db, float* parts, Queue& queue) {
  constexpr int N = sizeof(T) == 2 ? 8 : 4;
  const int64_t packs = up(c.dim, N);
  const unsigned count = (unsigned)norm_parts(c);
#define BACKWARD(THREADS, K, BLOCK)                                                                                               \
  LAUNCH((layernorm_backward_kernel<T, N, THREADS, K, BLOCK>), dim3(count), dim3(BLOCK), queue, static_cast<const T*>(dy),      \
         static_cast<const T*>(x), w, mean, rstd, static_cast<T*>(dx), c.rows, (int)c.dim, c.y_stride, c.x_stride,               \
         c.grad_x_stride, parts)
  if (packs <= 16) BACKWARD(16, 1, 256);
  else if (packs <= 32) BACKWARD(16, 2, 256);
  else if (packs <= 64) BACKWARD(64, 1, 256);
  else if (packs <= 128) BACKWARD(64, 2, 256);
  else if (packs <= 256) BACKWARD(64, 4, 256);
  else if (packs <= 512) BACKWARD(256, 2, 256);
  else if (packs <= 1024) BACKWARD(512, 2, 512);
  else if (packs <= 2048) BACKWARD(1024, 2, 1024);
  else if (N == 4 && packs <= 4096) BACKWARD(1024, N == 4 ? 4 : 2, 1024);
  else {
    for (int64_t r = 0; r < c.rows; r += kRowsPerLaunch)
      LAUNCH((layernorm_backward_long_kernel<T, N>), dim3((unsigned)std::min(kRowsPerLaunch, c.rows - r)), dim3(256), queue,
             static_cast<const T*>(dy) + r * c.y_stride, static_cast<const T*>(x) + r * c.x_stride, w, mean + r, rstd + r,
             static_cast<T*>(dx) + r * c.grad_x_stride, (int)c.dim, c.y_stride, c.x_stride, c.grad_x_stride);
    LAUNCH((layernorm_columns_kernel<T, N>), dim3(count, (unsigned)up(c.dim, 256 * N)), dim3(256), queue, static_cast<const T*>(dy),
           static_cast<const T*>(x), mean, rstd, c.rows, (int)c.dim, c.y_stride, c.x_stride, parts);
  }
#undef BACKWARD
  LAUNCH(layernorm_join_kernel, dim3((unsigned)up(c.dim, kWave), 2), dim3(1024), queue, parts, (int)count, (int)c.dim, dw, db,
         c.accumulate);
}

// ---- recurrence -------------------------------------------------------------------------------------

// Whether rows of `channels` elements at [batch, step] are apart, as they have to be where they are written.
bool rows_apart(const acc_recurrence& c, int64_t batch, int64_t step) {
  if (c.steps <= 1 && c.batch <= 1) return true;
  if (c.steps <= 1) return batch >= c.channels;
  if (c.batch <= 1) return step >= c.channels;
  if (step <= batch) return step >= c.channels && batch >= step * (c.steps - 1) + c.channels;
  return batch >= c.channels && step >= batch * (c.batch - 1) + c.channels;
}

bool strides_fit(const acc_recurrence& c, int64_t batch, int64_t step) {
  const int64_t most = int64_t(1) << 40;
  return (c.batch <= 1 || (batch >= 0 && batch <= most)) &&
         (c.steps <= 1 || (step >= 0 && step <= most && step * (double)c.steps < 1e18));
}

Span steps_span(const void* p, const acc_recurrence& c, int64_t batch, int64_t step) {
  if (!p || c.batch == 0 || c.steps == 0) return {static_cast<const char*>(p), 0};
  if (c.batch == 1) batch = 0;
  if (c.steps == 1) step = 0;
  const bool two = batch > 0 && step > 0;
  const int64_t near = two ? std::min(batch, step) : std::max(batch, step), far = std::max(batch, step);
  const int64_t block = ((near == step ? c.steps : c.batch) - 1) * near + c.channels;
  const int e = type_bytes(c.type);
  return {static_cast<const char*>(p), ((c.batch - 1) * batch + (c.steps - 1) * step + c.channels) * e, c.channels * e,
          near > 0 && far % near == 0 ? near * e : 0, block * e, two ? far * e : 0};
}

int32_t check_recurrence(const acc_recurrence* c, bool backward) {
  REQUIRE(c, "config is NULL");
  REQUIRE(c->batch >= 0 && c->batch <= 65535, "batch out of range");
  REQUIRE(c->steps >= 0 && c->steps < (int64_t(1) << 31), "steps out of range");
  REQUIRE(c->channels >= 1 && c->channels <= (int64_t(1) << 24), "channels out of range");
  REQUIRE(is_type(c->type), "unknown type");
  REQUIRE(strides_fit(*c, c->gate_batch, c->gate_step) && strides_fit(*c, c->input_batch, c->input_step) &&
              strides_fit(*c, c->out_batch, c->out_step),
          "stride out of range");
  if (!backward) {
    REQUIRE(rows_apart(*c, c->out_batch, c->out_step), "rows of out overlap");
    return ACC_OK;
  }
  REQUIRE(strides_fit(*c, c->grad_gate_batch, c->grad_gate_step) && strides_fit(*c, c->grad_input_batch, c->grad_input_step) &&
              strides_fit(*c, c->grad_out_batch, c->grad_out_step),
          "stride out of range");
  REQUIRE(rows_apart(*c, c->grad_gate_batch, c->grad_gate_step) && rows_apart(*c, c->grad_input_batch, c->grad_input_step),
          "rows of grad_gate or grad_input overlap");
  return ACC_OK;
}

// Whether rows start on whole pieces of memory.
bool whole_rows(const void* p, int64_t step_bytes) { return reinterpret_cast<uintptr_t>(p) % 64 == 0 && step_bytes % 64 == 0; }

RecurrenceShape shape_of(const acc_recurrence& c) {
  return {c.steps, c.channels, c.gate_batch, c.gate_step, c.input_batch, c.input_step, c.out_batch, c.out_step,
          c.grad_gate_batch, c.grad_gate_step, c.grad_input_batch, c.grad_input_step, c.grad_out_batch, c.grad_out_step};
}

// Up to kWalkSteps steps a lane walks them.  More: chunks, whose number of waves follows the steps.  us of the walk and of chunks, forward
// and backward: fp32 20 x 672 2 steps 3.3 and 4.7, 3.5 and 6.5; 16 steps 6.3 and 3.9, 6.6 and 8.1; 24 steps 8.0 and 4.8, 8.8 and 8.2;
// 512 x 1024 8 steps 10 and 18, 18 and 30; 16 steps 18 and 19, 34 and 40; 24 steps 25 and 27, 58 and 55; bf16 16 steps 13 and 17, 20 and 28,
// 32 steps 23 and 23, 39 and 38; 64 x 672 bf16 16 steps 7.0 and 5.1, 9.9 and 7.8.
constexpr int64_t kWalkSteps = 16;
constexpr int64_t kMostChunks = int64_t(1) << 22;   // work items per launch: see kRowsPerLaunch

struct RecurrencePlan {
  bool walk;
  int lane = 1;                            // channels per lane
  int wave_steps = 0, waves = 0, chunks = 0, groups = 0;
  int64_t channel_blocks = 0, chains = 0;
  int64_t slots = 0, group_slots = 0;      // chunks' and groups' words of a kind
  int64_t words = 0, bytes = 0;            // workspace: the counter, then the words
};

RecurrencePlan plan_recurrence(const acc_recurrence& c, bool backward) {
  RecurrencePlan p;
  p.lane = c.type == ACC_BF16 && c.channels > 1 ? 2 : 1;
  p.walk = c.steps <= kWalkSteps;
  if (p.walk) return p;
  p.wave_steps = backward && p.lane == 2 ? 8 : 16;
  p.waves = (int)std::min<int64_t>(kChunkWaves, up(c.steps, p.wave_steps));
  p.chunks = (int)up(c.steps, p.waves * p.wave_steps);
  p.channel_blocks = up(c.channels, kWave * p.lane);
  p.chains = p.channel_blocks * c.batch;
  if (p.chunks > 1) {
    p.groups = (int)up(p.chunks, kChunkGroup);
    p.slots = p.chains * p.chunks * kWave * p.lane;
    p.group_slots = p.groups > 1 ? p.chains * p.groups * kWave * p.lane : 0;
    p.words = 2 * p.slots + 3 * p.group_slots;
    p.bytes = 256 + round256(8 * p.words);
  }
  return p;
}

ChunkSlots chunk_slots(const RecurrencePlan& p, void* workspace, Queue& queue) {
  uint32_t* counter = static_cast<uint32_t*>(workspace);
  unsigned long long* words = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + 256);
  unsigned long long* const groups = words + 2 * p.slots;
  const ChunkSlots s = {words, words + p.slots, groups, groups + p.group_slots, groups + 2 * p.group_slots, counter, p.chains,
                        p.channel_blocks, p.chunks, p.groups};
  if (p.chunks > 1) LAUNCH(recurrence_clear_kernel, dim3((unsigned)up(p.words, 256)), dim3(256), queue, words, p.words, counter);
  return s;
}

template <typename T, int N, int S, bool ODD, bool STREAM>
void run_forward(const acc_recurrence& c, const RecurrencePlan& p, const void* gate, const void* input, const float* h0,
                 const int32_t* lengths, void* out, float* h_last, void* ws, Queue& queue) {
  if (p.walk) {
    LAUNCH((recurrence_forward_walk_kernel<T, N>), dim3((unsigned)up(c.channels, 256 * N), (unsigned)c.batch), dim3(256), queue,
           shape_of(c), static_cast<const T*>(gate), static_cast<const T*>(input), h0, lengths, static_cast<T*>(out), h_last);
    return;
  }
  const ChunkSlots slots = chunk_slots(p, ws, queue);
  LAUNCH((recurrence_forward_chunk_kernel<T, N, S, ODD, STREAM>), dim3((unsigned)(p.chains * p.chunks)), dim3(kWave * p.waves), queue, shape_of(c),
         slots, static_cast<const T*>(gate), static_cast<const T*>(input), h0, lengths, static_cast<T*>(out), h_last);
}

template <typename T, int N, int S, bool ODD, bool STREAM>
void run_backward(const acc_recurrence& c, const RecurrencePlan& p, const void* gate, const void* input, const void* out,
                  const float* h0, const int32_t* lengths, const void* dout, const float* dlast, void* dgate, void* dinput, float* dh0,
                  void* ws, Queue& queue) {
  if (p.walk) {
    LAUNCH((recurrence_backward_walk_kernel<T, N>), dim3((unsigned)up(c.channels, 256 * N), (unsigned)c.batch), dim3(256), queue,
           shape_of(c), static_cast<const T*>(gate), static_cast<const T*>(input), static_cast<const T*>(out), h0, lengths,
           static_cast<const T*>(dout), dlast, static_cast<T*>(dgate), static_cast<T*>(dinput), dh0);
    return;
  }
  const ChunkSlots slots = chunk_slots(p, ws, queue);
  LAUNCH((recurrence_backward_chunk_kernel<T, N, S, ODD, STREAM>), dim3((unsigned)(p.chains * p.chunks)), dim3(kWave * p.waves), queue, shape_of(c),
         slots, static_cast<const T*>(gate), static_cast<const T*>(input), static_cast<const T*>(out), h0, lengths,
         static_cast<const T*>(dout), dlast, static_cast<T*>(dgate), static_cast<T*>(dinput), dh0);
}

// ---- AdamW ------------------------------------------------------------------------------------------

int32_t check_adamw(const acc_adamw* c) {
  REQUIRE(c, "config is NULL");
  REQUIRE(c->n_tensors >= 0 && c->n_tensors <= (1 << 20), "n_tensors out of range");
  REQUIRE(c->n_tensors == 0 || c->sizes_host, "sizes_host is NULL");
  REQUIRE(is_type(c->weight_type) && is_type(c->grad_type), "unknown type");
  REQUIRE(c->state_bits == 8 || c->state_bits == 32, "state_bits must be 8 or 32");
  for (int32_t i = 0; i < c->n_tensors; ++i)
    REQUIRE(c->sizes_host[i] >= 0 && c->sizes_host[i] <= (int64_t(1) << 36), "tensor size out of range");
  return ACC_OK;
}

// Whether a tensor's weights or copy share memory with any tensor's weights, copy or gradients; -1: no host memory to find out.
// Layers of flat buffers, in order, are seen to be apart in one look at each; other tensors are sorted by their place.
int tensors_overlap(const acc_adamw& c, void* const* weights, const void* const* grads, void* const* copies) {
  struct Piece {
    uintptr_t from, to;
    bool written;
  };
  const int64_t bytes[3] = {type_bytes(c.weight_type), 2, type_bytes(c.grad_type)};
  auto piece = [&](int kind, int32_t i) -> Piece {
    const void* p = kind == 0 ? weights[i] : kind == 1 ? (copies ? copies[i] : nullptr) : grads[i];
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    return {from, p ? from + (uintptr_t)(c.sizes_host[i] * bytes[kind]) : from, kind < 2};
  };
  Piece all[3];
  bool in_order = true;
  for (int kind = 0; kind < 3; ++kind) {
    all[kind] = {~(uintptr_t)0, 0, kind < 2};
    for (int32_t i = 0; i < c.n_tensors; ++i) {
      const Piece p = piece(kind, i);
      if (p.from == p.to) continue;
      in_order = in_order && (kind == 2 || p.from >= all[kind].to);
      all[kind].from = std::min(all[kind].from, p.from);
      all[kind].to = std::max(all[kind].to, p.to);
    }
  }
  auto apart = [](const Piece& a, const Piece& b) { return a.to <= b.from || b.to <= a.from; };
  if (in_order && apart(all[0], all[1]) && apart(all[0], all[2]) && apart(all[1], all[2])) return 0;
  std::unique_ptr<Piece[]> pieces(new (std::nothrow) Piece[3 * (size_t)c.n_tensors]);
  if (!pieces) return -1;
  Piece* end = pieces.get();
  for (int kind = 0; kind < 3; ++kind)
    for (int32_t i = 0; i < c.n_tensors; ++i) {
      const Piece p = piece(kind, i);
      if (p.from != p.to) *end++ = p;
    }
  std::sort(pieces.get(), end, [](const Piece& a, const Piece& b) { return a.from < b.from; });
  uintptr_t written = 0, any = 0;           // how far the pieces so far reach
  for (const Piece* p = pieces.get(); p != end; ++p) {
    if (p->from < (p->written ? any : written)) return 1;
    any = std::max(any, p->to);
    if (p->written) written = std::max(written, p->to);
  }
  return 0;
}

// Elements per launch at most (see kRowsPerLaunch); larger tensors go in pieces.
constexpr int64_t kAdamPiece = int64_t(1) << 33;

int64_t state_elements(const acc_adamw& c, int64_t n) { return c.state_bits == 8 ? up(n, kAdamBlock) * kAdamBlock : n; }

template <typename W, typename G>
void adamw(const AdamArgs& a, int bits, unsigned tiles, Queue& queue) {
  if (bits == 32) LAUNCH((adamw_kernel<W, G, false, false>), dim3(tiles), dim3(256), queue, a);
  else if (a.dither_m || a.dither_v) LAUNCH((adamw_kernel<W, G, true, true>), dim3(tiles), dim3(256), queue, a);
  else LAUNCH((adamw_kernel<W, G, true, false>), dim3(tiles), dim3(256), queue, a);
}

}  // namespace

extern "C" {

const char* accordion_operator_error(void) { return g_error; }

int32_t accordion_embedding_forward(const acc_embedding* e, const void* ids_dev, const void* table_dev, void* out_dev,
                                    void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_embedding(e)) return rc;
  if (e->tokens == 0) return ACC_OK;
  REQUIRE(ids_dev && table_dev && out_dev, "a pointer is NULL");
  REQUIRE(!off_type(ids_dev, e->index_bits / 8) && !off_type(table_dev, type_bytes(e->table_type)) &&
              !off_type(out_dev, type_bytes(e->out_type)),
          "a pointer is not aligned to its element type");
  const Span s[3] = {rows_span(out_dev, e->tokens, e->dim, e->out_stride, type_bytes(e->out_type)),
                     rows_span(table_dev, e->vocab, e->dim, e->table_stride, type_bytes(e->table_type)),
                     {static_cast<const char*>(ids_dev), e->tokens * (e->index_bits / 8)}};
  REQUIRE(!any_overlap(s, 1, 3), "out_dev overlaps another buffer");
  if (e->index_bits == 32)
    e->table_type == ACC_BF16 ? lookup_to<int32_t, bf16>(*e, ids_dev, table_dev, out_dev, queue)
                              : lookup_to<int32_t, float>(*e, ids_dev, table_dev, out_dev, queue);
  else
    e->table_type == ACC_BF16 ? lookup_to<int64_t, bf16>(*e, ids_dev, table_dev, out_dev, queue)
                              : lookup_to<int64_t, float>(*e, ids_dev, table_dev, out_dev, queue);
  return launched(queue);
}

int32_t accordion_embedding_workspace_bytes(const acc_embedding* e, size_t* out_bytes) {
  REQUIRE(out_bytes, "out_bytes is NULL");
  if (const int32_t rc = check_embedding(e)) return rc;
  const EmbeddingPlan p = plan_embedding(*e);
  REQUIRE(p.chunks * up(e->dim, kWave * 4) <= kMostUnits, "tokens x dim out of range");
  *out_bytes = (size_t)p.bytes;
  return ACC_OK;
}

int32_t accordion_embedding_backward(const acc_embedding* e, const void* ids_dev, const void* grad_out_dev, float* grad_table_dev,
                                     void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_embedding(e)) return rc;
  REQUIRE(grad_table_dev, "grad_table_dev is NULL");
  REQUIRE(!off_type(grad_table_dev, 4), "a pointer is not aligned to its element type");
  if (e->tokens > 0) {
    REQUIRE(ids_dev && grad_out_dev, "a pointer is NULL");
    REQUIRE(!off_type(ids_dev, e->index_bits / 8) && !off_type(grad_out_dev, type_bytes(e->out_type)),
            "a pointer is not aligned to its element type");
  }
  const EmbeddingPlan p = plan_embedding(*e);
  REQUIRE(p.chunks * up(e->dim, kWave * 4) <= kMostUnits, "tokens x dim out of range");
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const Span s[4] = {rows_span(grad_table_dev, e->vocab, e->dim, e->table_stride, 4),
                     {static_cast<const char*>(workspace_dev), p.bytes},
                     rows_span(grad_out_dev, e->tokens, e->dim, e->out_stride, type_bytes(e->out_type)),
                     {static_cast<const char*>(ids_dev), e->tokens * (e->index_bits / 8)}};
  REQUIRE(!any_overlap(s, 2, 4), "grad_table_dev or workspace_dev overlaps another buffer");
  if (e->index_bits == 32)
    embedding_gradient(*e, p, static_cast<const int32_t*>(ids_dev), grad_out_dev, grad_table_dev, static_cast<char*>(workspace_dev),
                       queue);
  else
    embedding_gradient(*e, p, static_cast<const int64_t*>(ids_dev), grad_out_dev, grad_table_dev, static_cast<char*>(workspace_dev),
                       queue);
  return launched(queue);
}

int32_t accordion_layernorm_forward(const acc_layernorm* c, const void* x_dev, const float* weight_dev, const float* bias_dev,
                                    void* y_dev, float* mean_dev, float* rstd_dev, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_layernorm(c, false)) return rc;
  REQUIRE((mean_dev == nullptr) == (rstd_dev == nullptr), "mean_dev and rstd_dev go together");
  if (c->rows == 0) return ACC_OK;
  REQUIRE(x_dev && weight_dev && y_dev, "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(x_dev, e) && !off_type(y_dev, e) && !off_type(weight_dev, 4) && !off_type(bias_dev, 4) &&
              !off_type(mean_dev, 4) && !off_type(rstd_dev, 4),
          "a pointer is not aligned to its element type");
  const Span s[6] = {rows_span(y_dev, c->rows, c->dim, c->y_stride, e), rows_span(mean_dev, c->rows, 1, 1, 4),
                     rows_span(rstd_dev, c->rows, 1, 1, 4), rows_span(x_dev, c->rows, c->dim, c->x_stride, e),
                     rows_span(weight_dev, 1, c->dim, 0, 4), rows_span(bias_dev, 1, c->dim, 0, 4)};
  REQUIRE(!any_overlap(s, 3, 6), "a buffer that is written overlaps another one");
  if (c->type == ACC_BF16) norm_forward_rows<bf16>(*c, x_dev, weight_dev, bias_dev, y_dev, mean_dev, rstd_dev, queue);
  else norm_forward_rows<float>(*c, x_dev, weight_dev, bias_dev, y_dev, mean_dev, rstd_dev, queue);
  return launched(queue);
}

int32_t accordion_layernorm_workspace_bytes(const acc_layernorm* c, size_t* out_bytes) {
  REQUIRE(out_bytes, "out_bytes is NULL");
  if (const int32_t rc = check_layernorm(c, false)) return rc;
  *out_bytes = (size_t)round256(8 * norm_parts(*c) * c->dim);
  return ACC_OK;
}

int32_t accordion_layernorm_backward(const acc_layernorm* c, const void* grad_y_dev, const void* x_dev, const float* weight_dev,
                                     const float* mean_dev, const float* rstd_dev, void* grad_x_dev, float* grad_weight_dev,
                                     float* grad_bias_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_layernorm(c, true)) return rc;
  REQUIRE(weight_dev && grad_weight_dev, "a pointer is NULL");
  REQUIRE(c->rows == 0 || (grad_y_dev && x_dev && mean_dev && rstd_dev && grad_x_dev), "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(grad_y_dev, e) && !off_type(x_dev, e) && !off_type(grad_x_dev, e) && !off_type(weight_dev, 4) &&
              !off_type(mean_dev, 4) && !off_type(rstd_dev, 4) && !off_type(grad_weight_dev, 4) && !off_type(grad_bias_dev, 4),
          "a pointer is not aligned to its element type");
  const int64_t need = round256(8 * norm_parts(*c) * c->dim);
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, need)) return rc;
  const Span s[9] = {rows_span(grad_x_dev, c->rows, c->dim, c->grad_x_stride, e), rows_span(grad_weight_dev, 1, c->dim, 0, 4),
                     rows_span(grad_bias_dev, 1, c->dim, 0, 4), {static_cast<const char*>(workspace_dev), need},
                     rows_span(grad_y_dev, c->rows, c->dim, c->y_stride, e), rows_span(x_dev, c->rows, c->dim, c->x_stride, e),
                     rows_span(weight_dev, 1, c->dim, 0, 4), rows_span(mean_dev, c->rows, 1, 1, 4), rows_span(rstd_dev, c->rows, 1, 1, 4)};
  REQUIRE(!any_overlap(s, 4, 9), "a buffer that is written overlaps another one");
  float* parts = static_cast<float*>(workspace_dev);
  if (c->type == ACC_BF16)
    norm_backward<bf16>(*c, grad_y_dev, x_dev, weight_dev, mean_dev, rstd_dev, grad_x_dev, grad_weight_dev, grad_bias_dev, parts,
                        queue);
  else
    norm_backward<float>(*c, grad_y_dev, x_dev, weight_dev, mean_dev, rstd_dev, grad_x_dev, grad_weight_dev, grad_bias_dev, parts,
                         queue);
  return launched(queue);
}

int32_t accordion_recurrence_workspace_bytes(const acc_recurrence* c, size_t* out_bytes) {
  REQUIRE(out_bytes, "out_bytes is NULL");
  if (const int32_t rc = check_recurrence(c, false)) return rc;
  const RecurrencePlan f = plan_recurrence(*c, false), b = plan_recurrence(*c, true);
  REQUIRE(std::max(f.chains * f.chunks, b.chains * b.chunks) <= kMostChunks, "too many steps");
  *out_bytes = (size_t)std::max(f.bytes, b.bytes);
  return ACC_OK;
}

int32_t accordion_recurrence_forward(const acc_recurrence* c, const void* gate_dev, const void* input_dev, const float* h0_dev,
                                     const int32_t* lengths_dev, void* out_dev, float* h_last_dev, void* workspace_dev,
                                     size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_recurrence(c, false)) return rc;
  if (c->batch == 0) return ACC_OK;
  REQUIRE(c->steps == 0 || (gate_dev && input_dev && out_dev), "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(gate_dev, e) && !off_type(input_dev, e) && !off_type(out_dev, e) && !off_type(h0_dev, 4) &&
              !off_type(lengths_dev, 4) && !off_type(h_last_dev, 4),
          "a pointer is not aligned to its element type");
  const RecurrencePlan p = plan_recurrence(*c, false);
  REQUIRE(p.chains * p.chunks <= kMostChunks, "too many steps");
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const Span s[7] = {{static_cast<const char*>(workspace_dev), p.bytes}, steps_span(out_dev, *c, c->out_batch, c->out_step), rows_span(h_last_dev, c->batch, c->channels, c->channels, 4),
                     steps_span(gate_dev, *c, c->gate_batch, c->gate_step), steps_span(input_dev, *c, c->input_batch, c->input_step),
                     {reinterpret_cast<const char*>(lengths_dev), lengths_dev ? 4 * c->batch : 0},
                     rows_span(h0_dev == h_last_dev ? nullptr : h0_dev, c->batch, c->channels, c->channels, 4)};
  REQUIRE(!any_overlap(s, 3, 7), "a buffer that is written overlaps another one");
  const bool whole = whole_rows(out_dev, c->out_step * e);
  const auto run = c->type == ACC_FLOAT ? (whole ? run_forward<float, 1, 16, false, true> : run_forward<float, 1, 16, false, false>)
                   : p.lane == 1      ? run_forward<bf16, 1, 16, false, false>
                   : c->channels % 2  ? run_forward<bf16, 2, 16, true, false>
                   : whole            ? run_forward<bf16, 2, 16, false, true>
                                      : run_forward<bf16, 2, 16, false, false>;
  run(*c, p, gate_dev, input_dev, h0_dev, lengths_dev, out_dev, h_last_dev, workspace_dev, queue);
  return launched(queue);
}

int32_t accordion_recurrence_backward(const acc_recurrence* c, const void* gate_dev, const void* input_dev, const void* out_dev,
                                      const float* h0_dev, const int32_t* lengths_dev, const void* grad_out_dev,
                                      const float* grad_last_dev, void* grad_gate_dev, void* grad_input_dev, float* grad_h0_dev,
                                      void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_recurrence(c, true)) return rc;
  if (c->batch == 0) return ACC_OK;
  REQUIRE(c->steps == 0 || (gate_dev && input_dev && out_dev && grad_out_dev && grad_gate_dev && grad_input_dev), "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(gate_dev, e) && !off_type(input_dev, e) && !off_type(out_dev, e) && !off_type(grad_out_dev, e) &&
              !off_type(grad_gate_dev, e) && !off_type(grad_input_dev, e) && !off_type(h0_dev, 4) && !off_type(lengths_dev, 4) &&
              !off_type(grad_last_dev, 4) && !off_type(grad_h0_dev, 4),
          "a pointer is not aligned to its element type");
  const RecurrencePlan p = plan_recurrence(*c, true);
  REQUIRE(p.chains * p.chunks <= kMostChunks, "too many steps");
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const Span s[11] = {{static_cast<const char*>(workspace_dev), p.bytes},
                      steps_span(grad_gate_dev, *c, c->grad_gate_batch, c->grad_gate_step),
                      steps_span(grad_input_dev, *c, c->grad_input_batch, c->grad_input_step),
                      rows_span(grad_h0_dev, c->batch, c->channels, c->channels, 4),
                      steps_span(gate_dev, *c, c->gate_batch, c->gate_step),
                      steps_span(input_dev, *c, c->input_batch, c->input_step),
                      steps_span(out_dev, *c, c->out_batch, c->out_step),
                      steps_span(grad_out_dev, *c, c->grad_out_batch, c->grad_out_step),
                      rows_span(h0_dev, c->batch, c->channels, c->channels, 4),
                      rows_span(grad_last_dev, c->batch, c->channels, c->channels, 4),
                      {reinterpret_cast<const char*>(lengths_dev), lengths_dev ? 4 * c->batch : 0}};
  REQUIRE(!any_overlap(s, 4, 11), "a buffer that is written overlaps another one");
  const bool whole = whole_rows(grad_gate_dev, c->grad_gate_step * e) && whole_rows(grad_input_dev, c->grad_input_step * e);
  const auto run = c->type == ACC_FLOAT ? (whole ? run_backward<float, 1, 16, false, true> : run_backward<float, 1, 16, false, false>)
                   : p.lane == 1      ? run_backward<bf16, 1, 16, false, false>
                   : c->channels % 2  ? run_backward<bf16, 2, 8, true, false>
                   : whole            ? run_backward<bf16, 2, 8, false, true>
                                      : run_backward<bf16, 2, 8, false, false>;
  run(*c, p, gate_dev, input_dev, out_dev, h0_dev, lengths_dev, grad_out_dev, grad_last_dev, grad_gate_dev, grad_input_dev,
                              grad_h0_dev, workspace_dev, queue);
  return launched(queue);
}

int32_t accordion_adamw_state_elements(const acc_adamw* c, int64_t* out_elements) {
  REQUIRE(out_elements, "out_elements is NULL");
  if (const int32_t rc = check_adamw(c)) return rc;
  int64_t n = 0;
  for (int32_t i = 0; i < c->n_tensors; ++i) n += state_elements(*c, c->sizes_host[i]);
  *out_elements = n;
  return ACC_OK;
}

int32_t accordion_adamw_step(const acc_adamw* c, void* const* weights_host_array, const void* const* grads_host_array,
                             void* const* copies_host_array, void* m_dev, void* v_dev, float* m_scale_dev, float* v_scale_dev,
                             const float* grad_scale_dev, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_adamw(c)) return rc;
  REQUIRE(std::isfinite(c->lr) && c->lr >= 0 && std::isfinite(c->eps) && c->eps >= 0, "lr and eps must be finite and not negative");
  REQUIRE(c->beta1 >= 0 && c->beta1 < 1 && c->beta2 >= 0 && c->beta2 < 1, "betas must lie in [0, 1)");
  REQUIRE(c->step >= 1, "step counts from 1");
  REQUIRE(c->dither == 0 || c->dither == 1, "dither must be 0 or 1");
  int64_t elements = 0;
  for (int32_t i = 0; i < c->n_tensors; ++i) {
    const float wd = c->weight_decay_host ? c->weight_decay_host[i] : 0.f;
    REQUIRE(std::isfinite(wd) && wd >= 0.f, "weight decay must be finite and not negative");
    elements += state_elements(*c, c->sizes_host[i]);
  }
  if (elements == 0) return ACC_OK;
  REQUIRE(weights_host_array && grads_host_array && m_dev && v_dev, "a pointer is NULL");
  const bool bits8 = c->state_bits == 8;
  if (bits8) {
    REQUIRE(m_scale_dev && v_scale_dev, "8-bit moments need m_scale_dev and v_scale_dev");
  } else {
    REQUIRE(!m_scale_dev && !v_scale_dev, "32-bit moments have no scales");
  }
  REQUIRE(!off_type(m_dev, 4) && !off_type(v_dev, 4) && !off_type(m_scale_dev, 4) && !off_type(v_scale_dev, 4) &&
              !off_type(grad_scale_dev, 4),
          "a pointer is not aligned to its element type");
  const int64_t state_bytes = elements * (bits8 ? 1 : 4), scale_bytes = bits8 ? elements / kAdamBlock * 4 : 0;
  const Span st[5] = {{static_cast<const char*>(m_dev), state_bytes},
                      {static_cast<const char*>(v_dev), state_bytes},
                      {reinterpret_cast<const char*>(m_scale_dev), scale_bytes},
                      {reinterpret_cast<const char*>(v_scale_dev), scale_bytes},
                      {reinterpret_cast<const char*>(grad_scale_dev), grad_scale_dev ? 4 : 0}};
  REQUIRE(!any_overlap(st, 4, 5), "moments and scales overlap");
  const int we = type_bytes(c->weight_type), ge = type_bytes(c->grad_type);
  for (int32_t i = 0; i < c->n_tensors; ++i) {
    const int64_t n = c->sizes_host[i];
    if (n == 0) continue;
    void* const copy = copies_host_array ? copies_host_array[i] : nullptr;
    REQUIRE(weights_host_array[i] && grads_host_array[i], "a tensor's pointer is NULL");
    REQUIRE(!off_type(weights_host_array[i], we) && !off_type(grads_host_array[i], ge) && !off_type(copy, 2),
            "a pointer is not aligned to its element type");
    const Span t[8] = {rows_span(weights_host_array[i], 1, n, 0, we), rows_span(copy, 1, n, 0, 2), rows_span(grads_host_array[i], 1, n, 0, ge),
                       st[0], st[1], st[2], st[3], st[4]};
    REQUIRE(!any_overlap(t, 2, 8), "a tensor's weights or copy overlap another of its buffers or the state");
    for (int k = 0; k < 4; ++k) REQUIRE(!overlap(st[k], t[2]), "a gradient overlaps the state");
  }
  if (const int shared = tensors_overlap(*c, weights_host_array, grads_host_array, copies_host_array)) {
    REQUIRE(shared < 0, "weights or copies of a tensor overlap buffers of another tensor");
    return fail(ACC_ENOSPACE, "no host memory for the check of the tensors");
  }
  AdamArgs a;
  a.m = m_dev;
  a.v = v_dev;
  a.m_scale = m_scale_dev;
  a.v_scale = v_scale_dev;
  a.grad_scale = grad_scale_dev;
  a.beta1 = (float)c->beta1;
  a.c1 = (float)(1.0 - c->beta1);
  a.beta2 = (float)c->beta2;
  a.c2 = (float)(1.0 - c->beta2);
  a.rate = (float)(c->lr / (1.0 - std::pow(c->beta1, (double)c->step)));
  a.up = (float)(1.0 / std::sqrt(1.0 - std::pow(c->beta2, (double)c->step)));
  a.eps = (float)c->eps;
  a.turn = (uint32_t)c->step * kTurn;
  a.dither_m = bits8 && (c->dither || c->beta1 > kNearestBeta1);
  a.dither_v = bits8 && (c->dither || c->beta2 > kNearestBeta2);
  int64_t at = 0;
  int64_t tiles = 0;
  a.count = 0;
  auto flush = [&]() {
    if (a.count == 0) return;
    const bool wb = c->weight_type == ACC_BF16, gb = c->grad_type == ACC_BF16;
    if (wb) gb ? adamw<bf16, bf16>(a, c->state_bits, (unsigned)tiles, queue) : adamw<bf16, float>(a, c->state_bits, (unsigned)tiles, queue);
    else gb ? adamw<float, bf16>(a, c->state_bits, (unsigned)tiles, queue) : adamw<float, float>(a, c->state_bits, (unsigned)tiles, queue);
    a.count = 0;
    tiles = 0;
  };
  for (int32_t i = 0; i < c->n_tensors; ++i) {
    void* const copy = copies_host_array ? copies_host_array[i] : nullptr;
    for (int64_t from = 0; from < c->sizes_host[i]; from += kAdamPiece) {
      const int64_t n = std::min(kAdamPiece, c->sizes_host[i] - from);
      if (a.count == kAdamTensors || tiles + up(n, kAdamTile) > kAdamPiece / kAdamTile) flush();
      AdamTensor& t = a.t[a.count++];
      t.weights = static_cast<char*>(weights_host_array[i]) + from * we;
      t.grads = static_cast<const char*>(grads_host_array[i]) + from * ge;
      t.copies = copy ? static_cast<char*>(copy) + from * 2 : nullptr;
      t.state = at + from;
      t.n = n;
      t.tile = (uint32_t)tiles;
      t.keep = (float)(1.0 - c->lr * (double)(c->weight_decay_host ? c->weight_decay_host[i] : 0.f));
      tiles += up(n, kAdamTile);
    }
    at += state_elements(*c, c->sizes_host[i]);
  }
  flush();
  return launched(queue);
}

}  // extern "C"
