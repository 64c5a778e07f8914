// Host side of the tokens' log probabilities: argument checks, workspace layout, choice of kernels and the launches.
#include "op_common.h"
#include "op_host.h"
#include "logprob.h"

using namespace accop;

namespace {

int32_t check_logprob(const acc_logprob* c) {
  REQUIRE(c, "config is NULL");
  REQUIRE(c->rows >= 0 && c->rows <= (int64_t(1) << 28), "rows out of range");
  REQUIRE(c->vocab >= 1 && c->vocab <= (int64_t(1) << 22), "vocab out of range");
  REQUIRE(c->index_bits == 32 || c->index_bits == 64, "index_bits must be 32 or 64");
  REQUIRE(is_type(c->type), "unknown type");
  REQUIRE(c->top >= 0 && c->top <= ACC_LOGPROB_TOP && c->top <= c->vocab, "top out of range");
  REQUIRE(c->rows <= 1 || (c->logits_stride >= c->vocab && c->logits_stride <= kMaxStride), "logits_stride out of range");
  return ACC_OK;
}

// Rows that a wave takes in one turn of its requests: four of them are a workgroup's.  us of a workgroup and of a wave for a row, forward and gradient: bf16
// 1 x 1000 4.5, 3.8 and 4.3, 4.1; 700 x 2000 6.5, 4.8 and 4.8, 5.2; 3000 x 2000 13.4, 10.0 and 6.3, 8.7; 14379 x 2000 46, 31 and 19, 27; 14379 x 64 30, 14 and
// 15, 11; fp32 700 x 1000 5.5, 4.1 and 4.2, 4.3; 14379 x 1000 36, 22 and 14, 20; 100000 x 1000 229, 165 and 77, 147.
bool short_row(const acc_logprob& c) { return c.vocab <= kWave * 4 * (c.type == ACC_BF16 ? 8 : 4); }

struct LogprobPlan {
  int packs = 0, threads = 256;         // with the most probable tokens: packs of a lane
  bool rows_at_once = false;            // without them: a row is a wave's
  int64_t part = 0, parts = 1;
  int64_t sums = 0, best = 0, bytes = 0;
};

// Without the most probable tokens: parts of a row where there are fewer rows than kLogprobGroups, as many as give so many workgroups, of kStreamPart elements
// at least.  us with one part a row and with 256, 512, 1024, 2048 workgroups: 1 x 131072 fp32 20.4, 7.6, 7.6, 7.8, 7.6 (parts of 2048 elements 12.3);
// 64 x 131072 bf16 21.6, 10.5, 9.2, 10.0, 9.9; 300 x 50257 16.4, 16.3, 15.0, 15.0, 15.1; 700 x 32768 fp32 17.5, 17.5, 17.5, 21.2, 20.7; 1000 x 9000 bf16 8.5,
// 8.6, 8.6, 11.7, 11.6; 1000 x 131072 48, 48, 48, 50, 53.
constexpr int64_t kLogprobGroups = 512, kStreamPart = 8192;
// Gradient: parts of a row, as many as give so many workgroups.  us with one part a row and with 512, 1024, 2048, 4096 workgroups: 1 x 131072 fp32 42, 4.0 (all);
// 64 x 131072 bf16 37, 10.6, 10.0, 10.0, 9.9; 300 x 50257 25, 18.0, 16.4, 15.5, 15.5; 700 x 32768 fp32 31, 31, 31, 30, 29; 1000 x 131072 bf16 112, 112, 123, 110,
// 107; 1000 x 9000 11.8, 11.8, 10.5, 10.5, 10.5.
constexpr int64_t kGradientGroups = 2048;
// Parts of 32768 tokens where so many workgroups of 1024 lanes take all rows in two turns, of 8192 (as many as kTopMostSmall) where there are more.
// us of parts of 8192 and of 32768, 20 tokens wanted: 1 x 32768 fp32 10.3 and 7.7, 1 x 131072 15.2 and 10.8, 128 x 131072 bf16 22.6 and 17.9,
// 700 x 16384 fp32 18.8 and 20.1, 700 x 65536 41.9 and 50.0, 4096 x 16384 57 and 91, 4096 x 65536 225 and 258; 700 x 32768 bf16 23.6 and 21.1.
constexpr int64_t kTopGroupsAtOnce = 512, kTopMostSmall = 64, kSmallPart = 256 * 32;

// A wave for a row: of up to 512 tokens (an element a lane at a time, so that all 64 groups have some), of up to 2048 where there are many rows, or where packs
// of n would leave some of the `top` largest groups empty.  us of a workgroup of 256 lanes and of a wave: bf16 1 x 500, 20 wanted 13.7 and 6.2;
// 700 x 283, 16 13.3 and 6.1; 14379 x 283, 16 131 and 19.6; fp32 64 x 500, 20 5.3 and 5.7; 14379 x 283, 16 36 and 18.9; bf16 700 x 1024, 5 5.9 and 6.6; 700 x 2000,
// 20 6.4 and 9.0, 64 71 and 37; 2000 x 2048, 20 9.7 and 9.7; 4096 x 2048, 20 15.3 and 12.9; 14379 x 1000, 20 44 and 29; fp32 14379 x 2048, 20 44 and 34,
// 64 142 and 146.
constexpr int64_t kTopWaveAlways = 512, kTopWaveMost = 2048, kTopWaveRows = 2048;

LogprobPlan plan_logprob(const acc_logprob& c) {
  LogprobPlan p;
  const int64_t n = c.type == ACC_BF16 ? 8 : 4;
  if (c.top > 0) {
    // parts that 256 lanes hold, or 1024
    p.packs = (int)(c.vocab <= 256 * n ? 1 : (c.vocab <= 256 * 8 ? 8 : 32) / n);
    const bool wave = c.vocab <= kTopWaveAlways || (c.vocab <= kTopWaveMost && (c.rows >= kTopWaveRows || c.top * 4 * n > c.vocab));
    if (wave) {
      p.threads = kWave;
      p.part = c.vocab <= kTopWaveAlways ? kTopWaveAlways : kTopWaveMost;
      p.parts = 1;
      return p;
    }
    if (c.vocab > kSmallPart && (c.rows * up(c.vocab, 4 * kSmallPart) <= kTopGroupsAtOnce || c.vocab > kTopMostSmall * kSmallPart)) p.threads = 1024;
    p.part = p.threads * n * p.packs;
  } else {
    p.part = c.vocab;
    p.rows_at_once = short_row(c);
    if (c.rows < kLogprobGroups) p.part = std::max(kStreamPart, up(c.vocab, up(kLogprobGroups, std::max<int64_t>(1, c.rows))));
    p.part = up(p.part, 64) * 64;
  }
  p.parts = up(c.vocab, p.part);
  if (p.parts == 1) return p;
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t o = at; at += round256(bytes); return o; };
  p.sums = take(sizeof(RowSums) * c.rows * p.parts);
  p.best = take(8 * c.rows * p.parts * c.top);
  p.bytes = at;
  return p;
}

template <typename T, int N, int K, int THREADS>
void top_rows(const LogprobPlan& p, const LogprobOut& o, const T* logits, int64_t rows, RowSums* sums, Token* best, Queue& queue) {
  const dim3 grid((unsigned)rows, (unsigned)p.parts);
  if constexpr (THREADS * N * K >= kSmallPart) {         // (rows of several parts)
    if (p.parts > 1) {
      LAUNCH((logprob_top_kernel<T, N, K, THREADS, true>), grid, dim3(THREADS), queue, o, logits, p.part, (int)p.parts, sums, best);
      return;
    }
  }
  LAUNCH((logprob_top_kernel<T, N, K, THREADS, false>), grid, dim3(THREADS), queue, o, logits, p.part, 1, sums, best);
}

template <typename T>
void forward(const acc_logprob& c, const LogprobPlan& p, const LogprobOut& all, const T* logits, char* ws, Queue& queue) {
  constexpr int N = sizeof(T) == 2 ? 8 : 4;
  for (int64_t r = 0; r < c.rows; r += kRowsPerLaunch) {
    const int64_t rows = std::min(kRowsPerLaunch, c.rows - r);
    LogprobOut o = all;
    if (o.targets) o.targets = static_cast<const char*>(o.targets) + r * (c.index_bits / 8);
    if (o.logprob) o.logprob += r;
    if (o.lse) o.lse += r;
    if (o.entropy) o.entropy += r;
    if (o.top_logprobs) o.top_logprobs += r * c.top;
    if (o.top_ids) o.top_ids = static_cast<char*>(o.top_ids) + r * c.top * (c.index_bits / 8);
    RowSums* const sums = reinterpret_cast<RowSums*>(ws + p.sums) + (p.parts > 1 ? r * p.parts : 0);
    Token* const best = reinterpret_cast<Token*>(ws + p.best) + (p.parts > 1 ? r * p.parts * c.top : 0);
    const T* const from = logits + r * c.logits_stride;
    if (c.top > 0) {
      if (p.threads == kWave && p.part == kTopWaveAlways) top_rows<T, 1, kTopWaveAlways / kWave, kWave>(p, o, from, rows, sums, best, queue);
      else if (p.threads == kWave) top_rows<T, N, kTopWaveMost / kWave / N, kWave>(p, o, from, rows, sums, best, queue);
      else if (p.threads == 1024) top_rows<T, N, 32 / N, 1024>(p, o, from, rows, sums, best, queue);
      else if (p.packs == 1) top_rows<T, N, 1, 256>(p, o, from, rows, sums, best, queue);
      else if (p.packs == 8 / N) top_rows<T, N, 8 / N, 256>(p, o, from, rows, sums, best, queue);
      else top_rows<T, N, 32 / N, 256>(p, o, from, rows, sums, best, queue);
    } else {
      const auto kernel = o.entropy ? (p.parts > 1      ? logprob_stream_kernel<T, N, true, true, 256>
                                       : p.rows_at_once ? logprob_stream_kernel<T, N, true, false, kWave>
                                                        : logprob_stream_kernel<T, N, true, false, 256>)
                                    : (p.parts > 1      ? logprob_stream_kernel<T, N, false, true, 256>
                                       : p.rows_at_once ? logprob_stream_kernel<T, N, false, false, kWave>
                                                        : logprob_stream_kernel<T, N, false, false, 256>);
      LAUNCH(kernel, p.rows_at_once ? dim3((unsigned)up(rows, 4)) : dim3((unsigned)rows, (unsigned)p.parts), dim3(256), queue, o, from, rows, p.part, (int)p.parts, sums);
    }
    if (p.parts > 1)
      enqueue(queue, logprob_join_kernel<T>, dim3((unsigned)rows), dim3(kJoinThreads),
              (unsigned)(8 * up(p.parts * c.top, 8) * 8), o, from, (int)p.parts, sums, best);
  }
}

template <typename T>
void backward(const acc_logprob& c, const T* logits, const void* targets, const float* lse, const float* dlogprob, const float* entropy,
              const float* dentropy, T* grad, Queue& queue) {
  constexpr int N = sizeof(T) == 2 ? 8 : 4;
  constexpr int64_t turn = 256 * N * 4;
  int64_t part = up(c.vocab, turn) * turn;
  while (part > turn && c.rows * up(c.vocab, part) < kGradientGroups) part = up(part / 2, turn) * turn;
  for (int64_t r = 0; r < c.rows; r += kRowsPerLaunch) {
    const int64_t rows = std::min(kRowsPerLaunch, c.rows - r);
    const bool four = short_row(c);
    const dim3 grid((unsigned)(four ? up(rows, 4) : rows), (unsigned)up(c.vocab, part));
    const T* const from = logits + r * c.logits_stride;
    const void* const ids = dlogprob ? static_cast<const char*>(targets) + r * (c.index_bits / 8) : nullptr;
    T* const to = grad + r * c.grad_stride;
    const auto kernel = dentropy ? (four ? logprob_backward_kernel<T, N, true, kWave> : logprob_backward_kernel<T, N, true, 256>)
                                 : (four ? logprob_backward_kernel<T, N, false, kWave> : logprob_backward_kernel<T, N, false, 256>);
    LAUNCH(kernel, grid, dim3(256), queue, from, ids, c.index_bits == 64, lse + r, dlogprob ? dlogprob + r : nullptr, dentropy ? entropy + r : nullptr,
           dentropy ? dentropy + r : nullptr, to, rows, c.vocab, c.logits_stride, c.grad_stride, part);
  }
}

Span bytes_span(const void* p, int64_t bytes) { return {static_cast<const char*>(p), p ? bytes : 0}; }

}  // namespace

extern "C" {

int32_t accordion_logprob_workspace_bytes(const acc_logprob* c, size_t* out_bytes) {
  REQUIRE(out_bytes, "out_bytes is NULL");
  if (const int32_t rc = check_logprob(c)) return rc;
  *out_bytes = (size_t)plan_logprob(*c).bytes;
  return ACC_OK;
}

int32_t accordion_logprob_forward(const acc_logprob* c, const void* logits_dev, const void* targets_dev, float* logprob_dev,
                                  float* lse_dev, float* entropy_dev, float* top_logprobs_dev, void* top_ids_dev, void* workspace_dev,
                                  size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_logprob(c)) return rc;
  if (c->rows == 0) return ACC_OK;
  REQUIRE(logits_dev, "logits_dev is NULL");
  REQUIRE(!logprob_dev || targets_dev, "logprob_dev needs targets_dev");
  REQUIRE(c->top == 0 || (top_logprobs_dev && top_ids_dev), "top_logprobs_dev or top_ids_dev is NULL");
  const int e = type_bytes(c->type), i = c->index_bits / 8;
  REQUIRE(!off_type(logits_dev, e) && !off_type(targets_dev, i) && !off_type(logprob_dev, 4) && !off_type(lse_dev, 4) &&
              !off_type(entropy_dev, 4) && !off_type(top_logprobs_dev, 4) && !off_type(top_ids_dev, i),
          "a pointer is not aligned to its element type");
  const LogprobPlan p = plan_logprob(*c);
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const Span s[8] = {bytes_span(workspace_dev, p.bytes), bytes_span(logprob_dev, 4 * c->rows), bytes_span(lse_dev, 4 * c->rows),
                     bytes_span(entropy_dev, 4 * c->rows), bytes_span(top_logprobs_dev, 4 * c->rows * c->top),
                     bytes_span(top_ids_dev, i * c->rows * c->top), rows_span(logits_dev, c->rows, c->vocab, c->logits_stride, e),
                     bytes_span(targets_dev, i * c->rows)};
  REQUIRE(!any_overlap(s, 6, 8), "a buffer that is written overlaps another one");
  const LogprobOut o = {targets_dev, logprob_dev, lse_dev, entropy_dev, top_logprobs_dev, top_ids_dev, c->vocab, c->logits_stride, c->top, c->index_bits == 64};
  char* const ws = static_cast<char*>(workspace_dev);
  if (c->type == ACC_BF16) forward(*c, p, o, static_cast<const bf16*>(logits_dev), ws, queue);
  else forward(*c, p, o, static_cast<const float*>(logits_dev), ws, queue);
  return launched(queue);
}

int32_t accordion_logprob_backward(const acc_logprob* c, const void* logits_dev, const void* targets_dev, const float* lse_dev,
                                   const float* grad_logprob_dev, const float* entropy_dev, const float* grad_entropy_dev,
                                   void* grad_logits_dev, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_logprob(c)) return rc;
  REQUIRE(c->rows <= 1 || (c->grad_stride >= c->vocab && c->grad_stride <= kMaxStride), "grad_stride out of range");
  if (c->rows == 0) return ACC_OK;
  REQUIRE(logits_dev && lse_dev && grad_logits_dev, "a pointer is NULL");
  REQUIRE(!grad_logprob_dev || targets_dev, "grad_logprob_dev needs targets_dev");
  REQUIRE(!grad_entropy_dev || entropy_dev, "grad_entropy_dev needs entropy_dev");
  const int e = type_bytes(c->type), i = c->index_bits / 8;
  REQUIRE(!off_type(logits_dev, e) && !off_type(targets_dev, i) && !off_type(lse_dev, 4) && !off_type(grad_logprob_dev, 4) &&
              !off_type(entropy_dev, 4) && !off_type(grad_entropy_dev, 4) && !off_type(grad_logits_dev, e),
          "a pointer is not aligned to its element type");
  const bool in_place = grad_logits_dev == logits_dev && (c->rows <= 1 || c->grad_stride == c->logits_stride);
  const Span s[7] = {rows_span(grad_logits_dev, c->rows, c->vocab, c->grad_stride, e),
                     rows_span(in_place ? nullptr : logits_dev, c->rows, c->vocab, c->logits_stride, e),
                     bytes_span(targets_dev, i * c->rows),
                     bytes_span(lse_dev, 4 * c->rows),
                     bytes_span(grad_logprob_dev, 4 * c->rows),
                     bytes_span(entropy_dev, 4 * c->rows),
                     bytes_span(grad_entropy_dev, 4 * c->rows)};
  REQUIRE(!any_overlap(s, 1, 7), "grad_logits_dev overlaps another buffer");
  if (c->type == ACC_BF16)
    backward(*c, static_cast<const bf16*>(logits_dev), targets_dev, lse_dev, grad_logprob_dev, entropy_dev, grad_entropy_dev,
             static_cast<bf16*>(grad_logits_dev), queue);
  else
    backward(*c, static_cast<const float*>(logits_dev), targets_dev, lse_dev, grad_logprob_dev, entropy_dev, grad_entropy_dev,
             static_cast<float*>(grad_logits_dev), queue);
  return launched(queue);
}

}  // extern "C"
