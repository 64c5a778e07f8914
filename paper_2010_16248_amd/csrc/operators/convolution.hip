// Host side of the short causal convolution: argument checks, workspace layout, choice of kernels and the launches.
#include "op_common.h"
#include "op_host.h"
#include "convolution.h"
#include "parts.h"

using namespace accop;

namespace {

int32_t check_convolution(const acc_convolution* c, bool backward) {
  REQUIRE(c, "config is NULL");
  REQUIRE(c->batch >= 0 && c->batch <= 65535, "batch out of range");
  REQUIRE(c->steps >= 0 && c->steps < (int64_t(1) << 31), "steps out of range");
  REQUIRE(c->channels >= 1 && c->channels <= (int64_t(1) << 23), "channels out of range");
  REQUIRE(c->width >= 1 && c->width <= ACC_CONVOLUTION_WIDTH, "width out of range");
  REQUIRE(is_type(c->type), "unknown type");
  REQUIRE(c->silu == 0 || c->silu == 1, "silu must be 0 or 1");
  REQUIRE(c->accumulate == 0 || c->accumulate == 1, "accumulate must be 0 or 1");
  REQUIRE(strides_fit(*c, c->x_batch, c->x_step) && strides_fit(*c, c->out_batch, c->out_step), "stride out of range");
  if (!backward) {
    REQUIRE(rows_apart(*c, c->out_batch, c->out_step), "rows of out overlap");
    return ACC_OK;
  }
  REQUIRE(strides_fit(*c, c->grad_x_batch, c->grad_x_step), "stride out of range");
  REQUIRE(rows_apart(*c, c->grad_x_batch, c->grad_x_step), "rows of grad_x overlap");
  return ACC_OK;
}

struct ConvolutionPlan {
  int lanes_log2 = 2;
  int64_t run = 0, runs = 0, across = 0, blocks = 0;   // blocks of 256 lanes
  int64_t bytes = 0;                                   // workspace of the backward pass
};

// Runs as long as leave the chip this many waves, from 8 to 128 steps.  us with runs of 8, 16, 32, 64, 128, 256 steps, width 4 with SiLU:
// bf16 8 x 4096 x 4096 forward 147, 133, 121, 124, 106, 139, backward 376, 281, 238, 221, 179, 179; fp32 forward 251, 237, 223, 215, 210, 219,
// backward 451, 393, 375, 334, 334, 342; bf16 1 x 2048 x 1536 forward 7.8, 10.3, 15.6, 26, 47, 89, backward 17, 17, 22, 32, 54, 97; width 3
// fp32 7 x 1999 x 1001 forward 23, 24, 24, 29, 50, 94, backward 51, 47, 46, 61, 101, 187.
constexpr int64_t kConvolutionWaves = 2048;

ConvolutionPlan plan_convolution(const acc_convolution& c, bool backward) {
  ConvolutionPlan p;
  const int pack = backward || c.type == ACC_FLOAT ? 4 : 8;
  while (p.lanes_log2 < 6 && ((int64_t)pack << p.lanes_log2) < c.channels) ++p.lanes_log2;
  p.across = up(c.channels, (int64_t)pack << p.lanes_log2);
  p.run = 128;
  const int64_t per_wave = kWave >> p.lanes_log2;
  while (p.run > 8 && c.batch * up(c.steps, p.run) * p.across / per_wave < kConvolutionWaves) p.run /= 2;
  while (c.batch * up(c.steps, p.run) > (int64_t(1) << 25)) p.run *= 2;     // lanes of a launch: see kRowsPerLaunch
  p.runs = std::max<int64_t>(1, up(c.steps, p.run));
  p.blocks = up((c.batch * p.runs) << p.lanes_log2, 256);
  p.bytes = round256(4 * p.blocks * (c.width + 1) * c.channels);
  return p;
}

// in_place: a state is replaced, which packs that share channels would read and write.
ConvolutionShape shape_of(const acc_convolution& c, const ConvolutionPlan& p, int pack, bool in_place) {
  return {c.batch, c.steps, c.channels, c.x_batch, c.x_step, c.out_batch, c.out_step, c.grad_x_batch, c.grad_x_step, p.run, p.runs, p.lanes_log2,
          c.channels >= pack && !in_place};
}

// Whether a wave has one run and every pack of N channels is or can be made whole.
template <int N>
bool full(const acc_convolution& c, const ConvolutionPlan& p, bool in_place) { return p.lanes_log2 == 6 && (c.channels % N == 0 || !in_place); }

template <typename F>
void with_width(int width, F&& run) {
  switch (width) {
    case 1: return run(std::integral_constant<int, 1>());
    case 2: return run(std::integral_constant<int, 2>());
    case 3: return run(std::integral_constant<int, 3>());
    case 4: return run(std::integral_constant<int, 4>());
    case 5: return run(std::integral_constant<int, 5>());
    case 6: return run(std::integral_constant<int, 6>());
    case 7: return run(std::integral_constant<int, 7>());
    default: return run(std::integral_constant<int, 8>());
  }
}

template <typename T, int N>
void forward(const acc_convolution& c, const ConvolutionPlan& p, const void* x, const float* weight, const float* bias, const float* state,
             const int32_t* lengths, void* out, float* last, Queue& queue) {
  with_width(c.width, [&](auto width) {
    constexpr int W = decltype(width)::value;
    const dim3 grid((unsigned)p.blocks, (unsigned)p.across);
    const bool in_place = state && state == last;
    const auto kernel = full<N>(c, p, in_place) ? convolution_forward_kernel<T, N, W, true> : convolution_forward_kernel<T, N, W, false>;
    LAUNCH(kernel, grid, dim3(256), queue, shape_of(c, p, N, in_place), static_cast<const T*>(x), weight, bias, state, lengths, static_cast<T*>(out), last,
           c.silu);
  });
}

template <typename T, int N>
void backward(const acc_convolution& c, const ConvolutionPlan& p, const void* x, const float* weight, const float* bias,
              const float* state, const int32_t* lengths, const void* dout, const float* dlast, void* dx, float* dstate, float* parts,
              Queue& queue) {
  with_width(c.width, [&](auto width) {
    constexpr int W = decltype(width)::value;
    const dim3 grid((unsigned)p.blocks, (unsigned)p.across);
    const auto kernel = full<N>(c, p, false) ? convolution_backward_kernel<T, N, W, true> : convolution_backward_kernel<T, N, W, false>;
    LAUNCH(kernel, grid, dim3(256), queue, shape_of(c, p, N, false), static_cast<const T*>(x), weight, bias, state, lengths,
           static_cast<const T*>(dout), dlast, static_cast<T*>(dx), dstate, parts, c.silu);
  });
}

Span floats(const void* p, int64_t n) { return {static_cast<const char*>(p), p ? 4 * n : 0}; }

}  // namespace

extern "C" {

int32_t accordion_convolution_forward(const acc_convolution* c, const void* x_dev, const float* weight_dev, const float* bias_dev,
                                      const float* state_dev, const int32_t* lengths_dev, void* out_dev, float* last_dev,
                                      void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_convolution(c, false)) return rc;
  if (c->batch == 0) return ACC_OK;
  REQUIRE(weight_dev && (c->steps == 0 || (x_dev && out_dev)), "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(x_dev, e) && !off_type(out_dev, e) && !off_type(weight_dev, 4) && !off_type(bias_dev, 4) && !off_type(state_dev, 4) &&
              !off_type(lengths_dev, 4) && !off_type(last_dev, 4),
          "a pointer is not aligned to its element type");
  const int64_t ends = c->batch * (c->width - 1) * c->channels;
  const Span s[7] = {steps_span(out_dev, *c, c->out_batch, c->out_step), floats(last_dev, ends), steps_span(x_dev, *c, c->x_batch, c->x_step),
                     floats(weight_dev, c->channels * c->width), floats(bias_dev, c->channels),
                     floats(state_dev == last_dev ? nullptr : state_dev, ends), floats(lengths_dev, c->batch)};
  REQUIRE(!any_overlap(s, 2, 7), "a buffer that is written overlaps another one");
  const ConvolutionPlan p = plan_convolution(*c, false);
  if (c->type == ACC_BF16) forward<bf16, 8>(*c, p, x_dev, weight_dev, bias_dev, state_dev, lengths_dev, out_dev, last_dev, queue);
  else forward<float, 4>(*c, p, x_dev, weight_dev, bias_dev, state_dev, lengths_dev, out_dev, last_dev, queue);
  return launched(queue);
}

int32_t accordion_convolution_workspace_bytes(const acc_convolution* c, size_t* out_bytes) {
  REQUIRE(out_bytes, "out_bytes is NULL");
  if (const int32_t rc = check_convolution(c, true)) return rc;       // (grad_out is only read: its rows may share memory)
  *out_bytes = (size_t)plan_convolution(*c, true).bytes;
  return ACC_OK;
}

int32_t accordion_convolution_backward(const acc_convolution* c, const void* x_dev, const float* weight_dev, const float* bias_dev,
                                       const float* state_dev, const int32_t* lengths_dev, const void* grad_out_dev,
                                       const float* grad_last_dev, void* grad_x_dev, float* grad_weight_dev, float* grad_bias_dev,
                                       float* grad_state_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_convolution(c, true)) return rc;
  const bool any = c->batch > 0 && c->steps > 0;
  REQUIRE(weight_dev && grad_weight_dev && (!any || (x_dev && grad_out_dev && grad_x_dev)), "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(x_dev, e) && !off_type(grad_out_dev, e) && !off_type(grad_x_dev, e) && !off_type(weight_dev, 4) &&
              !off_type(bias_dev, 4) && !off_type(state_dev, 4) && !off_type(lengths_dev, 4) && !off_type(grad_last_dev, 4) &&
              !off_type(grad_weight_dev, 4) && !off_type(grad_bias_dev, 4) && !off_type(grad_state_dev, 4),
          "a pointer is not aligned to its element type");
  const ConvolutionPlan p = plan_convolution(*c, true);
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const int64_t ends = c->batch * (c->width - 1) * c->channels;
  const Span s[12] = {{static_cast<const char*>(workspace_dev), p.bytes},
                      steps_span(grad_x_dev, *c, c->grad_x_batch, c->grad_x_step),
                      floats(grad_weight_dev, c->channels * c->width),
                      floats(grad_bias_dev, c->channels),
                      floats(grad_state_dev, ends),
                      steps_span(x_dev, *c, c->x_batch, c->x_step),
                      steps_span(grad_out_dev, *c, c->out_batch, c->out_step),
                      floats(weight_dev, c->channels * c->width),
                      floats(bias_dev, c->channels),
                      floats(state_dev, ends),
                      floats(grad_last_dev, ends),
                      floats(lengths_dev, c->batch)};
  REQUIRE(!any_overlap(s, 5, 12), "a buffer that is written overlaps another one");
  float* parts = static_cast<float*>(workspace_dev);
  if (p.blocks > 0) {
    if (c->type == ACC_BF16)
      backward<bf16, 4>(*c, p, x_dev, weight_dev, bias_dev, state_dev, lengths_dev, grad_out_dev, grad_last_dev, grad_x_dev,
                        grad_state_dev, parts, queue);
    else
      backward<float, 4>(*c, p, x_dev, weight_dev, bias_dev, state_dev, lengths_dev, grad_out_dev, grad_last_dev, grad_x_dev,
                         grad_state_dev, parts, queue);
  }
  LAUNCH(parts_join_kernel, dim3((unsigned)up(c->channels, kWave), (unsigned)(c->width + 1)), dim3(kPartsThreads), queue, parts, p.blocks,
         c->width + 1, c->channels, PartsTo{grad_weight_dev, c->width, grad_bias_dev, nullptr}, c->accumulate);
  return launched(queue);
}

}  // extern "C"
