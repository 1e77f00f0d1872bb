/*
 * pgc_ops.h -- C ABI of the operators that turn a language model's outputs into a
 * partition's loss and gradient, for coded gradient descent (pgc.h) on gfx950:
 * dropout, token log-probabilities, the preference loss of pairs of sequences and
 * the clipped policy loss, each forward and backward.
 *
 * Gradient coding combines copies of a partition's gradient that different workers
 * compute, so a partition's gradient must not depend on who computes it, nor with
 * which other rows: every result here is a function of a row's own data alone, is
 * summed in a fixed order without atomics, and dropout draws its mask from a seed
 * and the row's number in the data set.
 *
 * Conventions, as in pgc.h, and:
 *   - Calls are independent of any context.  They return a pgc_status; on failure
 *     pgc_ops_last_error() gives the reason.  Every argument that the host can see
 *     is checked before any work is enqueued.
 *   - All pointers are device pointers unless stated; `hip_stream` is a hipStream_t
 *     (NULL = the null stream) of the current device.  Work is enqueued and not
 *     synchronised.  Nothing is allocated; the calls can be captured into a graph.
 *   - Matrices are row-major; a stride is the number of values between the starts of
 *     two rows, at least the number of columns.  Data is aligned to its own type;
 *     nothing else is asked of addresses, strides and sizes.
 *   - Rows and columns number at most 2^31 - 1; a matrix may exceed 2^32 values.
 *   - An output may be the input of the same shape itself (same address and stride);
 *     apart from that an output must not overlap an input.  Matrices of one stride
 *     whose columns lie beside each other do not overlap.
 *   - Values are read as they are, computed with and summed in 32 bits (sequence
 *     sums in 64) and rounded once to the output's type, to nearest even.
 */
#ifndef PGC_OPS_H
#define PGC_OPS_H

#include "pgc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of a matrix's values. */
enum pgc_dtype {
  PGC_F32 = 0,
  PGC_BF16 = 1,
  PGC_F16 = 2
};

/* The reason for the calling thread's last failed call of this header (never NULL). */
const char* pgc_ops_last_error(void);

/* ---- Dropout ----------------------------------------------------------------------
 *
 * out[i][j] = residual[i][j] + (keep(r_i, j) ? x[i][j] * s : 0)
 *
 * r_i = row_ids ? row_ids[i] : first_row + i is the row's number in the data set.
 * keep(r, j) holds when the 16-bit field number j % 4 (lowest first) of
 * splitmix64(splitmix64(seed, r), j / 4) is at least T = floor(65536 p + 1/2), with
 * splitmix64(seed, index) the generator of pgc_splitmix64 (indices taken modulo
 * 2^64).  A value is kept with probability 1 - T / 65536 exactly and scaled by its
 * inverse s = 65536 / (65536 - T), so p is rounded to a multiple of 2^-16.  p = 1
 * keeps nothing.  A dropped value is not multiplied: NaN and infinities in dropped
 * places leave no trace.  The mask is never stored: the backward pass draws it again.
 * Use another seed for each step and layer, e.g. pgc_splitmix64(seed, t).
 */
typedef struct pgc_dropout_args {
  const void* x;           /* rows x cols (backward: the gradient of out) */
  const void* residual;    /* rows x cols, or NULL; same type */
  void* out;               /* rows x cols, same type (backward: the gradient of x) */
  const int64_t* row_ids;  /* rows numbers, or NULL */
  int64_t rows, cols;
  int64_t x_stride, residual_stride, out_stride;
  int64_t first_row;
  uint64_t seed;
  double p;                /* 0 <= p <= 1 */
  int32_t dtype;           /* enum pgc_dtype */
} pgc_dropout_args;

int pgc_dropout(const pgc_dropout_args* args, void* hip_stream);

/* dx[i][j] = keep(r_i, j) ? dout[i][j] * s : 0.  `residual` must be NULL (its gradient is dout). */
int pgc_dropout_backward(const pgc_dropout_args* args, void* hip_stream);

/* ---- Token log-probabilities ------------------------------------------------------
 *
 * For every row t of logits z and its target y_t:
 *   M_t = max_j z[t][j],  S_t = sum_j exp(z[t][j] - M_t)
 *   logprobs[t] = (z[t][y_t] - M_t) - ln S_t
 *   stats[t] = (M_t, ln S_t)          (the log of the whole sum is M_t + ln S_t)
 *
 * A target outside of [0, cols) stands for no token: logprobs and stats are 0, the
 * gradient's row is 0, and the row is not read.  -inf marks a token that cannot
 * occur.  A row of nothing but -inf has logprobs -inf, stats (-inf, 0) and gradient 0.
 * NaN or +inf in a row that is read makes that row's results NaN, and no other's.
 */
typedef struct pgc_logits {
  const void* data;
  int64_t rows, cols, stride;
  int32_t dtype;           /* enum pgc_dtype */
} pgc_logits;

/* logprobs: rows floats; stats: rows pairs of floats, 8-byte aligned, or NULL. */
int pgc_token_logprobs(const pgc_logits* logits, const int32_t* targets, float* logprobs,
                       float* stats, void* hip_stream);

/* dlogits[t][j] = grad[t] ([j = y_t] - exp(z[t][j] - M_t - ln S_t)), in the type of the
 * logits.  stats: as pgc_token_logprobs wrote them.  A row whose grad is 0 gets zeros
 * and is not read, whatever its logits hold. */
int pgc_token_logprobs_backward(const pgc_logits* logits, const int32_t* targets,
                                const float* stats, const float* grad, void* dlogits,
                                int64_t dlogits_stride, void* hip_stream);

/* ---- Preference loss of pairs of sequences ----------------------------------------
 *
 * Rows are the tokens of 2 * pairs sequences one after the other: sequence q holds the
 * rows [offsets[q], offsets[q + 1]); pair i prefers sequence 2 i to sequence 2 i + 1.
 * With l_t the log-probability of row t's target (above) and w_i the pair's weight:
 *   h_i = beta (sum over sequence 2 i of (l_t - ref_t) - sum over sequence 2 i + 1)
 *   loss[i] = -(1 - label_smoothing) ln sigma(h_i) - label_smoothing ln sigma(-h_i)
 *   dlogits = scale * d(sum_i w_i loss[i]) / dz
 * Rows without a token count in no sum.  A sequence may be empty (its sum is 0).  Rows
 * of no pair, and of pairs whose gradient is 0 (w_i = 0), get gradient 0.
 * offsets must not decrease; values outside of [0, rows] are taken as the nearest bound.
 * h[i] is written to margins, l_t to logprobs.  A token that cannot occur makes its
 * pair's margin infinite: the loss is then the limit, with a term of weight 0 left out
 * (0 for h = inf without smoothing).  Infinite sums on both sides make the pair NaN.
 */
typedef struct pgc_preference_args {
  const int32_t* targets;       /* rows */
  const int32_t* offsets;       /* 2 * pairs + 1 */
  const float* ref_logprobs;    /* rows: l_t under the reference model, or NULL for 0 */
  const float* pair_weights;    /* pairs, or NULL for 1 */
  int64_t pairs;
  double beta;                  /* finite */
  double label_smoothing;       /* in [0, 1] */
  double scale;                 /* finite; e.g. 1 / pairs for the partition's mean */
  float* loss;                  /* pairs (not weighted) */
  float* margins;               /* pairs */
  float* logprobs;              /* rows */
  void* dlogits;                /* rows x cols in the logits' type, or NULL: the loss alone */
  int64_t dlogits_stride;
} pgc_preference_args;

/* Bytes of device workspace that the call on such logits (their data is not looked at)
 * and so many pairs needs: a multiple of 256, 0 for small ones.  Host only. */
int pgc_preference_workspace_bytes(const pgc_logits* logits, int64_t pairs, size_t* bytes);

/* workspace: at least that many bytes, 256-byte aligned, used until the stream has
 * passed the call; may be NULL where none are needed. */
int pgc_preference_loss(const pgc_logits* logits, const pgc_preference_args* args,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Clipped policy loss with a KL term -------------------------------------------
 *
 * For every row t with target y_t (an action), l_t its log-probability, advantage a_t:
 *   r = exp(l_t - old_t),  b = min(max(r, 1 - clip_low), 1 + clip_high)
 *   loss[t] = -min(r a_t, b a_t) + kl (exp(ref_t - l_t) - (ref_t - l_t) - 1)
 *   dlogits = scale * d(sum_t w_t loss[t]) / dz
 * The gradient of the first term is -r a_t where r a_t <= b a_t and 0 where the bound
 * holds; a_t = 0 contributes 0 whatever r is.  A row without a token or with w_t = 0 has
 * loss, logprobs and gradient 0 and is not read.  A target that cannot occur (l_t = -inf)
 * has r = 0, and with kl > 0 and a finite ref_t the loss +inf, the limit; the gradient's
 * factor is then -inf, so that no value of that row's gradient is finite (all are 0 where
 * the whole row is -inf).
 */
typedef struct pgc_policy_args {
  const int32_t* targets;       /* rows */
  const float* old_logprobs;    /* rows: l_t under the policy that sampled */
  const float* advantages;      /* rows */
  const float* ref_logprobs;    /* rows; may be NULL when kl = 0 */
  const float* token_weights;   /* rows, or NULL for 1 */
  double clip_low;              /* in [0, 1] */
  double clip_high;             /* >= 0, finite */
  double kl;                    /* finite */
  double scale;                 /* finite; e.g. 1 / rows for the mean */
  float* loss;                  /* rows (not weighted) */
  float* logprobs;              /* rows */
  void* dlogits;                /* rows x cols in the logits' type, or NULL: the loss alone */
  int64_t dlogits_stride;
} pgc_policy_args;

int pgc_policy_loss(const pgc_logits* logits, const pgc_policy_args* args, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* PGC_OPS_H */
