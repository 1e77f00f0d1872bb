// Launchers of the language-model operators of include/pgc_ops.h.  Arguments have been
// checked by the C entry points; launchers only choose a kernel and enqueue it.
#pragma once
#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "pgc_ops.h"

namespace pgc {

struct DropoutArgs {
  const void* x;
  const void* residual;    // or null
  void* out;
  const int64_t* row_ids;  // or null: first_row + i
  int64_t rows, cols, x_stride, residual_stride, out_stride, first_row;
  uint64_t seed;
  uint32_t threshold;      // a field below it drops its value; up to 65536
  float factor;            // 65536 / (65536 - threshold), 0 at 65536
};
hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t stream);

// One row of logits per unit of work.  What becomes of its log-probability is the mode's.
enum class RowMode {
  kForward,    // logprobs and, if asked for, stats; with zero_grad also a 0 per row
  kBackward,   // gradient from stats and grad
  kPolicy,     // loss and gradient
};

struct LogitsArgs {
  const void* logits;
  const int32_t* targets;
  int64_t rows, cols, stride, out_stride;
  void* dlogits;           // kBackward, kPolicy (there null: no gradient)
  float* logprobs;         // kForward, kPolicy
  float* stats;            // kForward: written unless null; kBackward: read
  const float* grad;       // kBackward
  float* zero_grad;        // kForward: written as 0, unless null
  // kPolicy
  const float* old_logprobs;
  const float* advantages;
  const float* ref_logprobs;
  const float* weights;
  float* loss;
  float clip_low, clip_high, kl, scale;
};
hipError_t launch_logits(const LogitsArgs& a, RowMode mode, int dtype, hipStream_t stream);

struct PairArgs {
  const int32_t* targets;
  const int32_t* offsets;
  const float* logprobs;
  const float* ref_logprobs;   // or null
  const float* weights;        // or null
  float* loss;
  float* margins;
  float* grad;                 // the rows' gradients, written for the rows of pairs; or null
  double* chunk_sums;          // pair_chunk_places(rows, pairs) of them, as scratch memory
  int64_t rows, pairs, cols;
  double beta, smoothing, scale;
};
int64_t pair_chunk_places(int64_t rows, int64_t pairs);
hipError_t launch_pairs(const PairArgs& a, hipStream_t stream);

// The same and the gradient in one launch, for few rows (a.stats as RowMode::kForward wrote them; a.grad and
// p.grad are not used).
bool preference_sums_in_gradient(int64_t rows, int64_t cols, int64_t pairs, int dtype);
hipError_t launch_pair_gradient(const LogitsArgs& a, const PairArgs& p, int dtype, hipStream_t stream);

// Forward, pairs and backward of few logits in one launch, without a workspace (a.dlogits null: no
// gradient; p.logprobs and p.grad are not used).
bool preference_is_small(int64_t rows, int64_t cols, int64_t pairs, int dtype);
hipError_t launch_small_preference(const LogitsArgs& a, const PairArgs& p, int dtype, hipStream_t stream);

}  // namespace pgc
