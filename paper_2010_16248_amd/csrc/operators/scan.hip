// Host side of the selective state space scan: argument checks, workspace layout, choice of kernels and the launches.
#include "op_common.h"
#include "op_host.h"
#include "scan.h"

using namespace accop;

namespace {

constexpr int64_t kMostBackwardSteps = int64_t(1) << 21;   // chunks of a launch: below 2^16

Rows shared_rows(const acc_scan& c) { return {c.batch, c.steps, (int64_t)c.groups * c.states, c.type}; }

int32_t check_scan(const acc_scan* c, bool backward) {
  REQUIRE(c, "config is NULL");
  REQUIRE(c->batch >= 0 && c->batch <= 65535, "batch out of range");
  REQUIRE(c->steps >= 0 && c->steps < (int64_t(1) << 31), "steps out of range");
  REQUIRE(c->channels >= 1 && c->channels <= (int64_t(1) << 20), "channels out of range");
  REQUIRE(c->states >= 1 && c->states <= ACC_SCAN_STATES, "states out of range");
  REQUIRE(c->groups >= 1 && c->channels % c->groups == 0, "channels must be a multiple of groups");
  REQUIRE(is_type(c->type), "unknown type");
  REQUIRE(c->softplus == 0 || c->softplus == 1, "softplus must be 0 or 1");
  REQUIRE(c->accumulate == 0 || c->accumulate == 1, "accumulate must be 0 or 1");
  const Rows shared = shared_rows(*c);
  REQUIRE(strides_fit(*c, c->x_batch, c->x_step) && strides_fit(*c, c->delta_batch, c->delta_step) &&
              strides_fit(shared, c->b_batch, c->b_step) && strides_fit(shared, c->c_batch, c->c_step) &&
              strides_fit(*c, c->gate_batch, c->gate_step) && strides_fit(*c, c->out_batch, c->out_step),
          "stride out of range");
  if (!backward) return ACC_OK;
  REQUIRE(c->steps <= kMostBackwardSteps, "steps out of range");
  REQUIRE(strides_fit(*c, c->grad_x_batch, c->grad_x_step) && strides_fit(*c, c->grad_delta_batch, c->grad_delta_step) &&
              strides_fit(shared, c->grad_b_batch, c->grad_b_step) && strides_fit(shared, c->grad_c_batch, c->grad_c_step) &&
              strides_fit(*c, c->grad_gate_batch, c->grad_gate_step),
          "stride out of range");
  return ACC_OK;
}

// Up to here lanes share a channel and walk the steps: one launch, but every step waits for its own loads.  us of it and of the chunks' kernels at
// 1, 8, 12, 16, 20, 24, 32 steps: bf16 64 x 1344 channels x 16 states 5.1, 11.9, 15.9, 19.5, 24.2, 28.6, 37.5 and 17.1, 17.3, 19.0, 19.2, 21.9, 22.3, 25.9;
// 8 x 2048 x 16 3.6, 6.3, 8.0, 9.8, 11.4, 13.1, 16.7 and 8.0, 8.2, 9.4, 9.5, 10.7, 10.9, 12.1; fp32 64 x 4096 x 16 41.0 and 40.5 (16), 49.2 and 43.8 (20);
// 16 x 1024 x 64 15.6 and 17.6 (16), 21.2 and 19.7 (24); 16 x 1024 x 4 9.0 and 10.9 (16), 12.2 and 13.1 (24).
constexpr int64_t kScanWalkSteps = 16;
// Chunks of the forward pass cost every step a second time (scan_ends_kernel) and two more launches, for waves.  None up to 64 steps, and from kScanLone
// waves on without them; otherwise as long as leave kScanWaves, from 32 to 128 steps.  us without chunks and with chunks of 32, 64, 128, 256 steps,
// bf16, 16 states: 1 x 128 x 1536 (96 waves without chunks) 26, 19, 26; 8 x 128 x 768 (384) 26, 24, 27; 8 x 256 x 768 (384) 45, 30, 34, 42;
// 1 x 512 x 1536 (96) 84, 24, 27, 41, 71; 1 x 4096 x 1536 624, 77, 70, 69, 94; 20 x 512 x 1024 (1280) 105, 101, 93, 92, 109; 64 x 512 x 512 (2048) 109,
// 148, 134, 130, 130; 64 x 512 x 1024 (4096) 169, 277, 248, 232, 219; 8 x 4096 x 2048 (1024) 618, 547, 480, 464, 459; 4 states 64 x 512 x 1024 (1024) 151,
// 148, 141, 140, 166; 32 states 4 x 1024 x 1536 (768) 179, 116, 104, 99, 129; 64 states 2 x 2048 x 768 (192) 517, 115, 105, 122, 129.
// With lengths, from kScanRagged steps on, up to twice as many waves: without chunks the longest sequence's are the last ones.  32 x 4096 x 1024 (2048) without
// chunks 691 and with chunks of 128 548, and of one length 804 and 892; fp32 29 x 4370 x 1159 (2204) 899 and 690, 1085 and 1187; 64 x 2048 x 1024 (4096) 563
// and 562, 631 and 891; 64 x 512 x 512 (2048) 102 and 118.
constexpr int64_t kScanRagged = 2048;
// (256 steps are no slower where they too leave kScanWaves waves: 8 x 4096 x 2048 459 us for 464.  The rule stops at 128.)
constexpr int64_t kScanFew = 64, kScanLone = 2048, kScanWaves = 4096, kScanShortest = 32, kScanLongest = 128;
// Chunks of the backward pass: as long as leave this many workgroups and waves, from 16 to 256 steps.  us with chunks of 16, 32, 64, 128, 256 steps, bf16:
// 16 states (4 waves) 1 x 512 x 1536 (24 workgroups per chunk) 41, 44, 49, 79, 139; 2 x 2048 x 768 (24) 102, 87, 84, 106, 143; 4 x 1024 x 1536 (96) 166,
// 148, 138, 138, 189; 64 x 128 x 512 (512) 117, 107, 107, 105; 8 x 4096 x 2048 (256) 1730, 1359, 1195, 1155, 1132; 4 states (1 wave) 64 x 512 x 1024 (1024)
// 411, 354, 330, 331, 349; 64 states (8 waves) 2 x 2048 x 768 (24) 347, 274, 251, 299, 300.  Longer ones were not measured.  Next to the border of
// kBackwardWaves neither side is the better one throughout: 4 states 47 x 1024 x 1024 in chunks of 256 (3008 waves) 514 and of 128 466, 188 x 200 x 1024
// (3008) 401 and 462; 8 states (2 waves) 25 x 1024 x 960 (3000) 410 and 338.
constexpr int64_t kBackwardGroups = 768, kBackwardWaves = 3000, kBackwardShortest = 16, kBackwardLongest = 256;

struct ScanPlan {
  bool walk = false, large = false;
  int padded = 16, split = 1;               // states, filled up; waves of a workgroup
  int64_t group = 0, blocks = 0;            // channels of a group, blocks of 64 of them
  int64_t chunk = 0, chunks = 1, rows = 0;  // steps of a chunk, chunks, rows of a sequence's b and c
  int64_t packed = 0, ends = 0, starts = 0, sums = 0, marks = 0, parts = 0, shared_parts = 0, bytes = 0;   // offsets in the workspace
};

// ragged: there are lengths.
ScanPlan plan_scan(const acc_scan& c, bool backward, bool ragged) {
  ScanPlan p;
  p.walk = !backward && c.steps <= kScanWalkSteps;
  if (p.walk || c.batch == 0) return p;
  p.padded = c.states <= 4 ? 4 : c.states <= 8 ? 8 : c.states <= 16 ? 16 : c.states <= 32 ? 32 : 64;
  p.split = std::min(8, p.padded / 4);
  p.group = c.channels / c.groups;
  p.blocks = up(p.group, kWave);
  // A launch has fewer than 2^32 work items per axis: the last one of the backward pass has these and up to 2^30 more.
  p.large = (double)c.batch * c.groups * up(c.steps, kScanAhead) * kScanAhead * 2 * p.padded >= 3e9;
  if (p.large) return p;
  const int64_t groups = c.batch * c.groups * p.blocks;              // workgroups of one chunk
  if (backward) {
    p.chunk = kBackwardLongest;
    while (p.chunk > kBackwardShortest &&
           groups * up(c.steps, p.chunk) < std::max(kBackwardGroups, up(kBackwardWaves, p.split)))
      p.chunk /= 2;
  } else {
    p.chunk = std::max<int64_t>(1, c.steps);
    if (c.steps > kScanFew && groups * p.split < (ragged && c.steps >= kScanRagged ? 2 : 1) * kScanLone) {
      p.chunk = kScanLongest;
      while (p.chunk > kScanShortest && groups * p.split * up(c.steps, p.chunk) < kScanWaves) p.chunk /= 2;
    }
    while (up(c.steps, p.chunk) > 65535) p.chunk *= 2;
  }
  p.chunk = up(p.chunk, kScanAhead) * kScanAhead;
  p.chunks = std::max<int64_t>(1, up(c.steps, p.chunk));
  int64_t at = 0;
  auto take = [&](int64_t floats) { const int64_t o = at; at += round256(4 * floats); return o; };
  p.rows = up(c.steps, kScanAhead) * kScanAhead;
  const int64_t slots = p.chunks > 1 || (backward && c.steps > kScanAhead) ? c.batch * p.chunks * c.channels : 0;
  // (rows are requested ahead: up to a turn beyond the last)
  p.packed = take((c.batch * c.groups * p.rows + kScanAhead) * 2 * p.padded);
  p.ends = take(slots * p.padded);
  p.sums = take(slots);
  if (backward) {
    p.starts = take(slots * p.padded);
    p.marks = take(c.steps > kScanAhead ? c.batch * (p.rows / kScanAhead) * (p.padded + 1) * c.channels : 0);
    p.parts = take(c.batch * p.chunks * (c.states + 2) * c.channels);
    p.shared_parts = take(c.batch * c.groups * p.blocks * p.rows * 2 * p.padded);
  }
  p.bytes = at;
  return p;
}

ScanShape shape_of(const acc_scan& c, const ScanPlan& p) {
  return {c.steps, c.channels, c.x_batch, c.x_step, c.delta_batch, c.delta_step, c.gate_batch, c.gate_step, c.out_batch, c.out_step,
          c.grad_x_batch, c.grad_x_step, c.grad_delta_batch, c.grad_delta_step, c.grad_gate_batch, c.grad_gate_step,
          p.chunk, p.rows, (int)p.chunks, c.states, p.padded, c.groups, (int)(c.channels / c.groups), (int)p.blocks, c.softplus};
}

struct ScanIn {
  const void *x, *delta;
  const float* a;
  const void *b, *c;
  const float* d;
  const void* gate;
  const float *delta_bias, *h0;
  const int32_t* lengths;
};

template <typename T>
const T* as(const void* p) { return static_cast<const T*>(p); }

template <typename T>
void pack(const acc_scan& c, const ScanPlan& p, const ScanIn& in, float* to, Queue& queue) {
  const int64_t all = c.batch * c.groups * p.rows;
  if (all == 0) return;
  int fours_log2 = 1;
  while (4 << fours_log2 < 2 * p.padded) ++fours_log2;
  LAUNCH(scan_pack_kernel<T>, dim3((unsigned)up(all << fours_log2, 256)), dim3(256), queue, as<T>(in.b), as<T>(in.c), c.b_batch, c.b_step,
         c.c_batch, c.c_step, (unsigned)all, c.steps, (unsigned)p.rows, (unsigned)c.groups, c.states, p.padded, fours_log2, in.lengths, to);
}

template <typename T, int L>
void walk(const acc_scan& c, const ScanPlan& p, const ScanIn& in, void* out, float* h_last, Queue& queue) {
  LAUNCH((scan_walk_kernel<T, L>), dim3((unsigned)up(c.channels * L, 256), (unsigned)c.batch), dim3(256), queue, shape_of(c, p), as<T>(in.x),
         as<T>(in.delta), in.a, as<T>(in.b), as<T>(in.c), c.b_batch, c.b_step, c.c_batch, c.c_step, in.d, as<T>(in.gate), in.delta_bias,
         in.lengths, in.h0, static_cast<T*>(out), h_last);
}

dim3 carry_grid(const acc_scan& c, const ScanPlan& p, bool backward) {
  return dim3((unsigned)up(c.channels, kWave), (unsigned)(p.padded * (backward ? 2 : 1)), (unsigned)c.batch);
}
constexpr int64_t kCarryFill = 4096;        // waves that fill the chip
// More waves than one for a state's chunks where the states alone do not fill the chip.
dim3 carry_threads(const acc_scan& c, const ScanPlan& p) {
  const int64_t lone = c.batch * up(c.channels, kWave) * p.padded;
  return dim3((unsigned)(kWave * std::max<int64_t>(1, std::min({(int64_t)kCarryWaves, up(kCarryFill, lone), up(p.chunks, kCarryAhead)}))));
}

template <typename T, int NP, int WAVES>
void forward_ends(const acc_scan& c, const ScanPlan& p, const ScanIn& in, char* ws, Queue& queue) {
  auto at = [&](int64_t offset) { return reinterpret_cast<float*>(ws + offset); };
  LAUNCH((scan_ends_kernel<T, NP, WAVES, false>), dim3((unsigned)(c.groups * p.blocks), (unsigned)(p.chunks - 1), (unsigned)c.batch),
         dim3(kWave * WAVES), queue, shape_of(c, p), as<T>(in.x), as<T>(in.delta), in.a, at(p.packed), nullptr, in.delta_bias, in.lengths,
         nullptr, at(p.ends), nullptr, at(p.sums), nullptr);
}

template <typename T, int NP, int WAVES>
auto forward_kernel(const acc_scan& c, const ScanPlan& p) {
  return c.states == p.padded ? scan_forward_kernel<T, NP, WAVES, true> : scan_forward_kernel<T, NP, WAVES, false>;
}

template <typename T>
void forward(const acc_scan& c, const ScanPlan& p, const ScanIn& in, void* out, float* h_last, char* ws, Queue& queue) {
  if (p.walk) {
    if (c.states <= 4) walk<T, 1>(c, p, in, out, h_last, queue);
    else if (c.states <= 8) walk<T, 2>(c, p, in, out, h_last, queue);
    else if (c.states <= 16) walk<T, 4>(c, p, in, out, h_last, queue);
    else if (c.states <= 32) walk<T, 8>(c, p, in, out, h_last, queue);
    else walk<T, 16>(c, p, in, out, h_last, queue);
    return;
  }
  auto at = [&](int64_t offset) { return reinterpret_cast<float*>(ws + offset); };
  pack<T>(c, p, in, at(p.packed), queue);
  if (p.chunks > 1) {
    if (p.padded == 4) forward_ends<T, 4, 1>(c, p, in, ws, queue);
    else if (p.padded == 8) forward_ends<T, 4, 2>(c, p, in, ws, queue);
    else if (p.padded == 16) forward_ends<T, 4, 4>(c, p, in, ws, queue);
    else if (p.padded == 32) forward_ends<T, 4, 8>(c, p, in, ws, queue);
    else forward_ends<T, 8, 8>(c, p, in, ws, queue);
    LAUNCH(scan_carry_kernel<false>, carry_grid(c, p, false), carry_threads(c, p), queue, shape_of(c, p), in.a, in.h0, nullptr, at(p.ends),
           nullptr, at(p.sums));
  }
  const auto kernel = p.padded == 4    ? forward_kernel<T, 4, 1>(c, p)
                      : p.padded == 8  ? forward_kernel<T, 4, 2>(c, p)
                      : p.padded == 16 ? forward_kernel<T, 4, 4>(c, p)
                      : p.padded == 32 ? forward_kernel<T, 4, 8>(c, p)
                                       : forward_kernel<T, 8, 8>(c, p);
  LAUNCH(kernel, dim3((unsigned)(c.groups * p.blocks), (unsigned)p.chunks, (unsigned)c.batch), dim3((unsigned)(kWave * p.split)), queue,
         shape_of(c, p), as<T>(in.x), as<T>(in.delta), in.a, at(p.packed), in.d, as<T>(in.gate), in.delta_bias, in.lengths, in.h0, at(p.ends),
         static_cast<T*>(out), h_last);
}

struct ScanGradients {
  const void* out;
  const float* last;
  void *x, *delta;
  float* a;
  void *b, *c;
  float* d;
  void* gate;
  float *delta_bias, *h0;
};

template <typename T, int NP, int WAVES>
void backward_ends(const acc_scan& c, const ScanPlan& p, const ScanIn& in, const ScanGradients& g, char* ws, Queue& queue) {
  auto at = [&](int64_t offset) { return reinterpret_cast<float*>(ws + offset); };
  LAUNCH((scan_ends_kernel<T, NP, WAVES, true>), dim3((unsigned)(c.groups * p.blocks), (unsigned)p.chunks, (unsigned)c.batch),
         dim3(kWave * WAVES), queue, shape_of(c, p), as<T>(in.x), as<T>(in.delta), in.a, at(p.packed), as<T>(in.gate),
         in.delta_bias, in.lengths, as<T>(g.out), at(p.ends), at(p.starts), at(p.sums), at(p.marks));
}

template <typename T, int NP, int WAVES>
void backward_chunks(const acc_scan& c, const ScanPlan& p, const ScanIn& in, const ScanGradients& g, char* ws, Queue& queue) {
  auto at = [&](int64_t offset) { return reinterpret_cast<float*>(ws + offset); };
  const auto kernel = c.states == p.padded ? scan_backward_kernel<T, NP, WAVES, true> : scan_backward_kernel<T, NP, WAVES, false>;
  LAUNCH(kernel, dim3((unsigned)(c.groups * p.blocks), (unsigned)p.chunks, (unsigned)c.batch), dim3(kWave * WAVES),
         queue, shape_of(c, p), as<T>(in.x), as<T>(in.delta), in.a, at(p.packed), in.d, as<T>(in.gate), in.delta_bias, in.lengths, as<T>(g.out),
         in.h0, g.last, at(p.ends), at(p.starts), at(p.marks), static_cast<T*>(g.x), static_cast<T*>(g.delta), static_cast<T*>(g.gate), g.h0,
         at(p.parts), at(p.shared_parts));
}

template <typename T>
void backward(const acc_scan& c, const ScanPlan& p, const ScanIn& in, const ScanGradients& g, char* ws, Queue& queue) {
  auto at = [&](int64_t offset) { return reinterpret_cast<float*>(ws + offset); };
  if (c.batch > 0) {
    pack<T>(c, p, in, at(p.packed), queue);
    if (c.steps > kScanAhead) {
      if (p.padded == 4) backward_ends<T, 4, 1>(c, p, in, g, ws, queue);
      else if (p.padded == 8) backward_ends<T, 4, 2>(c, p, in, g, ws, queue);
      else if (p.padded == 16) backward_ends<T, 4, 4>(c, p, in, g, ws, queue);
      else if (p.padded == 32) backward_ends<T, 4, 8>(c, p, in, g, ws, queue);
      else backward_ends<T, 8, 8>(c, p, in, g, ws, queue);
    }
    if (p.chunks > 1)
      LAUNCH(scan_carry_kernel<true>, carry_grid(c, p, true), carry_threads(c, p), queue, shape_of(c, p), in.a, in.h0, g.last, at(p.ends),
             at(p.starts), at(p.sums));
    if (p.padded == 4) backward_chunks<T, 4, 1>(c, p, in, g, ws, queue);
    else if (p.padded == 8) backward_chunks<T, 4, 2>(c, p, in, g, ws, queue);
    else if (p.padded == 16) backward_chunks<T, 4, 4>(c, p, in, g, ws, queue);
    else if (p.padded == 32) backward_chunks<T, 4, 8>(c, p, in, g, ws, queue);
    else backward_chunks<T, 8, 8>(c, p, in, g, ws, queue);
  }
  const int64_t rows = c.batch * c.groups * c.steps, shared_blocks = up(rows * 2 * p.padded, kPartsThreads);
  LAUNCH(scan_join_kernel<T>, dim3((unsigned)(shared_blocks + up(c.channels, kWave) * (c.states + 2))), dim3(kPartsThreads), queue,
         at(p.shared_parts), rows, c.steps, p.rows, c.groups, (int)p.blocks, c.states, p.padded, in.lengths, static_cast<T*>(g.b),
         static_cast<T*>(g.c), c.grad_b_batch, c.grad_b_step, c.grad_c_batch, c.grad_c_step, (unsigned)shared_blocks, at(p.parts),
         c.batch * p.chunks, c.channels, PartsTo{g.a, c.states, g.d, g.delta_bias}, c.accumulate);
}

Span floats(const void* p, int64_t n) { return {static_cast<const char*>(p), p ? 4 * n : 0}; }

}  // namespace

extern "C" {

int32_t accordion_scan_workspace_bytes(const acc_scan* c, int32_t backward_pass, size_t* out_bytes) {
  REQUIRE(out_bytes, "out_bytes is NULL");
  REQUIRE(backward_pass == 0 || backward_pass == 1, "backward must be 0 or 1");
  if (const int32_t rc = check_scan(c, backward_pass)) return rc;
  const ScanPlan p = plan_scan(*c, backward_pass, true);      // (of one length it takes no more)
  REQUIRE(!p.large, "batch x steps x groups out of range");
  *out_bytes = (size_t)p.bytes;
  return ACC_OK;
}

int32_t accordion_scan_forward(const acc_scan* c, const void* x_dev, const void* delta_dev, const float* a_dev, const void* b_dev,
                               const void* c_dev, const float* d_dev, const void* gate_dev, const float* delta_bias_dev,
                               const float* h0_dev, const int32_t* lengths_dev, void* out_dev, float* h_last_dev, void* workspace_dev,
                               size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_scan(c, false)) return rc;
  REQUIRE(rows_apart(*c, c->out_batch, c->out_step), "rows of out overlap");
  if (c->batch == 0) return ACC_OK;
  REQUIRE(a_dev && (c->steps == 0 || (x_dev && delta_dev && b_dev && c_dev && out_dev)), "a pointer is NULL");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(x_dev, e) && !off_type(delta_dev, e) && !off_type(b_dev, e) && !off_type(c_dev, e) && !off_type(gate_dev, e) &&
              !off_type(out_dev, e) && !off_type(a_dev, 4) && !off_type(d_dev, 4) && !off_type(delta_bias_dev, 4) && !off_type(h0_dev, 4) &&
              !off_type(lengths_dev, 4) && !off_type(h_last_dev, 4),
          "a pointer is not aligned to its element type");
  const ScanPlan p = plan_scan(*c, false, lengths_dev != nullptr);
  REQUIRE(!p.large, "batch x steps x groups out of range");
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const Rows shared = shared_rows(*c);
  const int64_t ends = c->batch * c->channels * c->states;
  const Span s[13] = {{static_cast<const char*>(workspace_dev), p.bytes},
                      steps_span(out_dev, *c, c->out_batch, c->out_step),
                      floats(h_last_dev, ends),
                      steps_span(x_dev, *c, c->x_batch, c->x_step),
                      steps_span(delta_dev, *c, c->delta_batch, c->delta_step),
                      steps_span(b_dev, shared, c->b_batch, c->b_step),
                      steps_span(c_dev, shared, c->c_batch, c->c_step),
                      steps_span(gate_dev, *c, c->gate_batch, c->gate_step),
                      floats(a_dev, c->channels * c->states),
                      floats(d_dev, c->channels),
                      floats(delta_bias_dev, c->channels),
                      floats(h0_dev == h_last_dev ? nullptr : h0_dev, ends),
                      floats(lengths_dev, c->batch)};
  REQUIRE(!any_overlap(s, 3, 13), "a buffer that is written overlaps another one");
  const ScanIn in = {x_dev, delta_dev, a_dev, b_dev, c_dev, d_dev, gate_dev, delta_bias_dev, h0_dev, lengths_dev};
  char* const ws = static_cast<char*>(workspace_dev);
  if (c->type == ACC_BF16) forward<bf16>(*c, p, in, out_dev, h_last_dev, ws, queue);
  else forward<float>(*c, p, in, out_dev, h_last_dev, ws, queue);
  return launched(queue);
}

int32_t accordion_scan_backward(const acc_scan* c, const void* x_dev, const void* delta_dev, const float* a_dev, const void* b_dev,
                                const void* c_dev, const float* d_dev, const void* gate_dev, const float* delta_bias_dev,
                                const float* h0_dev, const int32_t* lengths_dev, const void* grad_out_dev, const float* grad_last_dev,
                                void* grad_x_dev, void* grad_delta_dev, float* grad_a_dev, void* grad_b_dev, void* grad_c_dev,
                                float* grad_d_dev, void* grad_gate_dev, float* grad_delta_bias_dev, float* grad_h0_dev,
                                void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  Queue queue(hip_stream);
  if (const int32_t rc = check_scan(c, true)) return rc;
  const Rows shared = shared_rows(*c);
  REQUIRE(rows_apart(*c, c->grad_x_batch, c->grad_x_step) && rows_apart(*c, c->grad_delta_batch, c->grad_delta_step) &&
              rows_apart(shared, c->grad_b_batch, c->grad_b_step) && rows_apart(shared, c->grad_c_batch, c->grad_c_step) &&
              (!gate_dev || rows_apart(*c, c->grad_gate_batch, c->grad_gate_step)),
          "rows of a gradient overlap");
  const bool any = c->batch > 0 && c->steps > 0;
  REQUIRE(a_dev && grad_a_dev, "a pointer is NULL");
  REQUIRE(!any || (x_dev && delta_dev && b_dev && c_dev && grad_out_dev && grad_x_dev && grad_delta_dev && grad_b_dev && grad_c_dev),
          "a pointer is NULL");
  REQUIRE(!any || (gate_dev == nullptr) == (grad_gate_dev == nullptr), "gate_dev and grad_gate_dev go together");
  REQUIRE(d_dev || !grad_d_dev, "grad_d_dev needs d_dev");
  REQUIRE(delta_bias_dev || !grad_delta_bias_dev, "grad_delta_bias_dev needs delta_bias_dev");
  const int e = type_bytes(c->type);
  REQUIRE(!off_type(x_dev, e) && !off_type(delta_dev, e) && !off_type(b_dev, e) && !off_type(c_dev, e) && !off_type(gate_dev, e) &&
              !off_type(grad_out_dev, e) && !off_type(grad_x_dev, e) && !off_type(grad_delta_dev, e) && !off_type(grad_b_dev, e) &&
              !off_type(grad_c_dev, e) && !off_type(grad_gate_dev, e) && !off_type(a_dev, 4) && !off_type(d_dev, 4) &&
              !off_type(delta_bias_dev, 4) && !off_type(h0_dev, 4) && !off_type(lengths_dev, 4) && !off_type(grad_last_dev, 4) &&
              !off_type(grad_a_dev, 4) && !off_type(grad_d_dev, 4) && !off_type(grad_delta_bias_dev, 4) && !off_type(grad_h0_dev, 4),
          "a pointer is not aligned to its element type");
  const ScanPlan p = plan_scan(*c, true, lengths_dev != nullptr);
  REQUIRE(!p.large, "batch x steps x groups out of range");
  if (const int32_t rc = check_workspace(workspace_dev, workspace_bytes, p.bytes)) return rc;
  const int64_t ends = c->batch * c->channels * c->states;
  const Span s[22] = {{static_cast<const char*>(workspace_dev), p.bytes},
                      steps_span(grad_x_dev, *c, c->grad_x_batch, c->grad_x_step),
                      steps_span(grad_delta_dev, *c, c->grad_delta_batch, c->grad_delta_step),
                      steps_span(grad_b_dev, shared, c->grad_b_batch, c->grad_b_step),
                      steps_span(grad_c_dev, shared, c->grad_c_batch, c->grad_c_step),
                      steps_span(grad_gate_dev, *c, c->grad_gate_batch, c->grad_gate_step),
                      floats(grad_a_dev, c->channels * c->states),
                      floats(grad_d_dev, c->channels),
                      floats(grad_delta_bias_dev, c->channels),
                      floats(grad_h0_dev, ends),
                      steps_span(x_dev, *c, c->x_batch, c->x_step),
                      steps_span(delta_dev, *c, c->delta_batch, c->delta_step),
                      steps_span(b_dev, shared, c->b_batch, c->b_step),
                      steps_span(c_dev, shared, c->c_batch, c->c_step),
                      steps_span(gate_dev, *c, c->gate_batch, c->gate_step),
                      steps_span(grad_out_dev, *c, c->out_batch, c->out_step),
                      floats(a_dev, c->channels * c->states),
                      floats(d_dev, c->channels),
                      floats(delta_bias_dev, c->channels),
                      floats(h0_dev, ends),
                      floats(grad_last_dev, ends),
                      floats(lengths_dev, c->batch)};
  REQUIRE(!any_overlap(s, 10, 22), "a buffer that is written overlaps another one");
  const ScanIn in = {x_dev, delta_dev, a_dev, b_dev, c_dev, d_dev, gate_dev, delta_bias_dev, h0_dev, lengths_dev};
  const ScanGradients g = {grad_out_dev, grad_last_dev, grad_x_dev, grad_delta_dev, grad_a_dev, grad_b_dev, grad_c_dev,
                           grad_d_dev, grad_gate_dev, grad_delta_bias_dev, grad_h0_dev};
  char* const ws = static_cast<char*>(workspace_dev);
  if (c->type == ACC_BF16) backward<bf16>(*c, p, in, g, ws, queue);
  else backward<float>(*c, p, in, g, ws, queue);
  return launched(queue);
}

}  // extern "C"
