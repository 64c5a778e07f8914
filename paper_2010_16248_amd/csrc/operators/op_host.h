// Host side that the language-model operators share: errors, checks of strides, overlaps and workspaces, launches.
#pragma once
#include "../../../include/accordion.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <tuple>

namespace accop {

// Records what accordion_operator_error() says to the calling thread, and returns the code.
int32_t fail(int32_t code, const char* msg);

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
inline bool any_overlap(const Span* s, int written, int all) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < all; ++j)
      if (overlap(s[i], s[j])) return true;
  return false;
}

inline int32_t check_workspace(const void* ws, size_t have, int64_t need) {
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

// ACC_OK, or the error of the first launch that failed.
int32_t launched(const Queue& q);

#define LAUNCH(kernel, grid, block, queue, ...) enqueue(queue, kernel, grid, block, 0, __VA_ARGS__)

// Rows of a batch x steps x channels tensor: C has batch, steps, channels and type.
struct Rows {
  int64_t batch, steps, channels;
  int32_t type;
};

// Whether rows of `channels` elements at [batch, step] are apart, as they have to be where they are written.
template <typename C>
bool rows_apart(const C& c, int64_t batch, int64_t step) {
  if (c.steps <= 1 && c.batch <= 1) return true;
  if (c.steps <= 1) return batch >= c.channels;
  if (c.batch <= 1) return step >= c.channels;
  if (step <= batch) return step >= c.channels && batch >= step * (c.steps - 1) + c.channels;
  return batch >= c.channels && step >= batch * (c.batch - 1) + c.channels;
}

template <typename C>
bool strides_fit(const C& c, int64_t batch, int64_t step) {
  const int64_t most = int64_t(1) << 40;
  return (c.batch <= 1 || (batch >= 0 && batch <= most)) &&
         (c.steps <= 1 || (step >= 0 && step <= most && step * (double)c.steps < 1e18));
}

template <typename C>
Span steps_span(const void* p, const C& c, int64_t batch, int64_t step) {
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

// Whether rows start on whole pieces of memory.
inline bool whole_rows(const void* p, int64_t step_bytes) { return reinterpret_cast<uintptr_t>(p) % 64 == 0 && step_bytes % 64 == 0; }

}  // namespace accop
