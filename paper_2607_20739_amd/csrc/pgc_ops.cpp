// C entry points of the language-model operators (include/pgc_ops.h): argument checks
// and launches.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "pgc_ops.h"
#include "pgc_ops_kernels.h"

namespace {

constexpr int64_t kMaxExtent = 2147483647;
constexpr size_t kAlign = 256;

thread_local char g_error[256] = "";

__attribute__((format(printf, 2, 3))) int fail(int status, const char* format, ...) {
  va_list list;
  va_start(list, format);
  std::vsnprintf(g_error, sizeof(g_error), format, list);
  va_end(list);
  return status;
}

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? PGC_OK : fail(PGC_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

int value_bytes(int dtype) { return dtype == PGC_F32 ? 4 : 2; }

// Finite also in the 32 bits that the kernels compute with.
bool finite32(double v) { return std::isfinite(static_cast<float>(v)); }

bool known(int dtype) { return dtype == PGC_F32 || dtype == PGC_BF16 || dtype == PGC_F16; }

struct Span {
  const char* name;
  uintptr_t at = 0;
  size_t bytes = 0;
  int64_t stride = 0, row = 0;   // of a matrix: bytes from row to row and of a row; 0: an array
};

// A matrix's or an array's bytes, from its first value to its last.
Span matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t stride, int value) {
  const size_t last = rows > 0 ? static_cast<size_t>(rows - 1) * stride + cols : 0;
  return {name, reinterpret_cast<uintptr_t>(p), last * value, stride * value, cols * value};
}
Span array(const char* name, const void* p, int64_t count, int value) {
  return {name, reinterpret_cast<uintptr_t>(p), static_cast<size_t>(count) * value};
}

int check_pointer(const Span& s, int align, bool required) {
  if (s.at == 0) return required && s.bytes > 0 ? fail(PGC_EINVAL, "%s is NULL", s.name) : PGC_OK;
  if (s.at % align != 0) return fail(PGC_EINVAL, "%s must be %d-byte aligned", s.name, align);
  return PGC_OK;
}

// Whether two matrices are columns of one wider matrix that lie beside each other.
bool side_by_side(const Span& a, const Span& b) {
  if (a.stride == 0 || a.stride != b.stride) return false;
  const uintptr_t stride = static_cast<uintptr_t>(a.stride);
  const uintptr_t from_b = a.at >= b.at ? (a.at - b.at) % stride : (stride - (b.at - a.at) % stride) % stride;
  return from_b >= static_cast<uintptr_t>(b.row) && from_b + a.row <= stride;
}

// An output may be an input itself where both are matrices of the same shape, else they
// must lie apart.
int check_apart(const Span& out, const Span& in, bool may_be_same) {
  if (out.at == 0 || in.at == 0 || out.bytes == 0 || in.bytes == 0) return PGC_OK;
  if (may_be_same && out.at == in.at && out.stride == in.stride) return PGC_OK;
  if (out.at < in.at + in.bytes && in.at < out.at + out.bytes && !side_by_side(out, in))
    return fail(PGC_EINVAL, "%s overlaps %s", out.name, in.name);
  return PGC_OK;
}

int check_extents(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > kMaxExtent || cols < 0 || cols > kMaxExtent)
    return fail(PGC_EINVAL, "rows and columns must lie in [0, 2^31 - 1]");
  return PGC_OK;
}

int check_pairs(int64_t pairs) {
  return pairs < 0 || pairs > kMaxExtent / 2 ? fail(PGC_EINVAL, "pairs must lie in [0, 2^30 - 1]") : PGC_OK;
}

int check_stride(const char* name, int64_t stride, int64_t cols) {
  if (stride < cols || stride > (int64_t{1} << 40))
    return fail(PGC_EINVAL, "%s stride must lie in [columns, 2^40]", name);
  return PGC_OK;
}

#define CHECK(expr)                       \
  do {                                    \
    const int status_ = (expr);           \
    if (status_ != PGC_OK) return status_; \
  } while (0)

int dropout(const pgc_dropout_args* a, void* stream) {
  if (!known(a->dtype)) return fail(PGC_EINVAL, "unknown dtype %d", a->dtype);
  CHECK(check_extents(a->rows, a->cols));
  if (!(a->p >= 0.0 && a->p <= 1.0)) return fail(PGC_EINVAL, "p must lie in [0, 1]");
  const int b = value_bytes(a->dtype);
  CHECK(check_stride("x", a->x_stride, a->cols));
  CHECK(check_stride("out", a->out_stride, a->cols));
  if (a->residual) CHECK(check_stride("residual", a->residual_stride, a->cols));
  if (a->rows == 0 || a->cols == 0) return PGC_OK;
  const Span x = matrix("x", a->x, a->rows, a->cols, a->x_stride, b);
  const Span out = matrix("out", a->out, a->rows, a->cols, a->out_stride, b);
  const Span residual = matrix("residual", a->residual, a->rows, a->cols, a->residual_stride, b);
  const Span ids = array("row_ids", a->row_ids, a->rows, 8);
  CHECK(check_pointer(x, b, true));
  CHECK(check_pointer(out, b, true));
  CHECK(check_pointer(residual, b, false));
  CHECK(check_pointer(ids, 8, false));
  CHECK(check_apart(out, x, true));
  CHECK(check_apart(out, residual, true));
  CHECK(check_apart(out, ids, false));
  pgc::DropoutArgs k{};
  k.x = a->x;
  k.residual = a->residual;
  k.out = a->out;
  k.row_ids = a->row_ids;
  k.rows = a->rows;
  k.cols = a->cols;
  k.x_stride = a->x_stride;
  k.residual_stride = a->residual_stride;
  k.out_stride = a->out_stride;
  k.first_row = a->first_row;
  k.seed = a->seed;
  k.threshold = static_cast<uint32_t>(std::floor(a->p * 65536.0 + 0.5));
  k.factor = k.threshold == 65536 ? 0.f : static_cast<float>(65536.0 / (65536.0 - k.threshold));
  return launched(pgc::launch_dropout(k, a->dtype, static_cast<hipStream_t>(stream)), "dropout kernel");
}

// The logits and their targets, with the columns' lower bound.
int check_logits(const pgc_logits* z, const int32_t* targets) {
  if (!known(z->dtype)) return fail(PGC_EINVAL, "unknown dtype %d", z->dtype);
  CHECK(check_extents(z->rows, z->cols));
  if (z->cols < 1) return fail(PGC_EINVAL, "logits need at least one column");
  CHECK(check_stride("logits", z->stride, z->cols));
  const int b = value_bytes(z->dtype);
  CHECK(check_pointer(matrix("logits", z->data, z->rows, z->cols, z->stride, b), b, true));
  return check_pointer(array("targets", targets, z->rows, 4), 4, true);
}

// An array of `count` floats that is read or written.
int check_floats(const char* name, const float* p, int64_t count, bool required) {
  return check_pointer(array(name, p, count, 4), 4, required);
}

// A gradient matrix beside the logits (which it may replace).
int check_dlogits(const pgc_logits* z, const void* dlogits, int64_t stride) {
  CHECK(check_stride("dlogits", stride, z->cols));
  const int b = value_bytes(z->dtype);
  const Span out = matrix("dlogits", dlogits, z->rows, z->cols, stride, b);
  CHECK(check_pointer(out, b, true));
  return check_apart(out, matrix("logits", z->data, z->rows, z->cols, z->stride, b), true);
}

// Outputs against inputs and against each other (outs[0 .. n_outs) first).
int check_all_apart(const Span* outs, int n_outs, const Span* ins, int n_ins) {
  for (int i = 0; i < n_outs; ++i) {
    for (int j = 0; j < n_ins; ++j) CHECK(check_apart(outs[i], ins[j], false));
    for (int j = 0; j < i; ++j) CHECK(check_apart(outs[i], outs[j], false));
  }
  return PGC_OK;
}

pgc::LogitsArgs logits_args(const pgc_logits* z, const int32_t* targets) {
  pgc::LogitsArgs k{};
  k.logits = z->data;
  k.targets = targets;
  k.rows = z->rows;
  k.cols = z->cols;
  k.stride = z->stride;
  return k;
}

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

}  // namespace

extern "C" {

const char* pgc_ops_last_error(void) { return g_error; }

int pgc_dropout(const pgc_dropout_args* args, void* hip_stream) {
  if (args == nullptr) return fail(PGC_EINVAL, "null arguments");
  return dropout(args, hip_stream);
}

int pgc_dropout_backward(const pgc_dropout_args* args, void* hip_stream) {
  if (args == nullptr) return fail(PGC_EINVAL, "null arguments");
  if (args->residual != nullptr) return fail(PGC_EINVAL, "the backward pass takes no residual");
  return dropout(args, hip_stream);
}

int pgc_token_logprobs(const pgc_logits* logits, const int32_t* targets, float* logprobs,
                       float* stats, void* hip_stream) {
  if (logits == nullptr) return fail(PGC_EINVAL, "null arguments");
  CHECK(check_logits(logits, targets));
  const int64_t rows = logits->rows;
  CHECK(check_floats("logprobs", logprobs, rows, true));
  CHECK(check_pointer(array("stats", stats, rows, 8), 8, false));
  const Span outs[] = {array("logprobs", logprobs, rows, 4), array("stats", stats, rows, 8)};
  const Span ins[] = {matrix("logits", logits->data, rows, logits->cols, logits->stride, value_bytes(logits->dtype)),
                      array("targets", targets, rows, 4)};
  CHECK(check_all_apart(outs, 2, ins, 2));
  if (rows == 0) return PGC_OK;
  pgc::LogitsArgs k = logits_args(logits, targets);
  k.logprobs = logprobs;
  k.stats = stats;
  return launched(pgc::launch_logits(k, pgc::RowMode::kForward, logits->dtype, static_cast<hipStream_t>(hip_stream)),
                  "log-probability kernel");
}

int pgc_token_logprobs_backward(const pgc_logits* logits, const int32_t* targets, const float* stats,
                                const float* grad, void* dlogits, int64_t dlogits_stride, void* hip_stream) {
  if (logits == nullptr) return fail(PGC_EINVAL, "null arguments");
  CHECK(check_logits(logits, targets));
  const int64_t rows = logits->rows;
  CHECK(check_pointer(array("stats", stats, rows, 8), 8, true));
  CHECK(check_floats("grad", grad, rows, true));
  CHECK(check_dlogits(logits, dlogits, dlogits_stride));
  const Span outs[] = {matrix("dlogits", dlogits, rows, logits->cols, dlogits_stride, value_bytes(logits->dtype))};
  const Span ins[] = {array("targets", targets, rows, 4), array("stats", stats, rows, 8), array("grad", grad, rows, 4)};
  CHECK(check_all_apart(outs, 1, ins, 3));
  if (rows == 0) return PGC_OK;
  pgc::LogitsArgs k = logits_args(logits, targets);
  k.stats = const_cast<float*>(stats);
  k.grad = grad;
  k.dlogits = dlogits;
  k.out_stride = dlogits_stride;
  return launched(pgc::launch_logits(k, pgc::RowMode::kBackward, logits->dtype, static_cast<hipStream_t>(hip_stream)),
                  "log-probability gradient kernel");
}

// The rows' (M, ln S) pairs, their gradients, then the sums of long pairs' chunks; nothing where one launch
// does it all.
int pgc_preference_workspace_bytes(const pgc_logits* logits, int64_t pairs, size_t* bytes) {
  if (logits == nullptr || bytes == nullptr) return fail(PGC_EINVAL, "null arguments");
  if (!known(logits->dtype)) return fail(PGC_EINVAL, "unknown dtype %d", logits->dtype);
  CHECK(check_extents(logits->rows, logits->cols));
  CHECK(check_pairs(pairs));
  const size_t rows = static_cast<size_t>(logits->rows);
  const bool none = pgc::preference_is_small(logits->rows, logits->cols, pairs, logits->dtype);
  const size_t sums = 8 * static_cast<size_t>(pgc::pair_chunk_places(logits->rows, pairs));
  *bytes = none ? 0 : align_up(8 * rows) + align_up(4 * rows) + align_up(sums);
  return PGC_OK;
}

int pgc_preference_loss(const pgc_logits* logits, const pgc_preference_args* a, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
  if (logits == nullptr || a == nullptr) return fail(PGC_EINVAL, "null arguments");
  CHECK(check_logits(logits, a->targets));
  const int64_t rows = logits->rows, pairs = a->pairs;
  CHECK(check_pairs(pairs));
  if (!finite32(a->beta) || !finite32(a->scale)) return fail(PGC_EINVAL, "beta and scale must be finite");
  if (!(a->label_smoothing >= 0.0 && a->label_smoothing <= 1.0))
    return fail(PGC_EINVAL, "label_smoothing must lie in [0, 1]");
  CHECK(check_pointer(array("offsets", a->offsets, 2 * pairs + 1, 4), 4, true));
  CHECK(check_floats("ref_logprobs", a->ref_logprobs, rows, false));
  CHECK(check_floats("pair_weights", a->pair_weights, pairs, false));
  CHECK(check_floats("loss", a->loss, pairs, true));
  CHECK(check_floats("margins", a->margins, pairs, true));
  CHECK(check_floats("logprobs", a->logprobs, rows, true));
  if (a->dlogits) CHECK(check_dlogits(logits, a->dlogits, a->dlogits_stride));
  size_t need = 0;
  CHECK(pgc_preference_workspace_bytes(logits, pairs, &need));
  const Span ws = {"workspace", reinterpret_cast<uintptr_t>(workspace), need};
  CHECK(check_pointer(ws, kAlign, true));
  if (workspace_bytes < need)
    return fail(PGC_EINVAL, "workspace too small: need %zu bytes", need);
  const int b = value_bytes(logits->dtype);
  const Span outs[] = {array("loss", a->loss, pairs, 4), array("margins", a->margins, pairs, 4),
                       array("logprobs", a->logprobs, rows, 4), ws,
                       matrix("dlogits", a->dlogits, rows, logits->cols, a->dlogits_stride, b)};
  const Span ins[] = {array("targets", a->targets, rows, 4), array("offsets", a->offsets, 2 * pairs + 1, 4),
                      array("ref_logprobs", a->ref_logprobs, rows, 4),
                      array("pair_weights", a->pair_weights, pairs, 4)};
  CHECK(check_all_apart(outs, 5, ins, 4));
  const Span z = matrix("logits", logits->data, rows, logits->cols, logits->stride, b);
  CHECK(check_all_apart(outs, 4, &z, 1));
  if (rows == 0 && pairs == 0) return PGC_OK;

  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  float* stats = static_cast<float*>(workspace);
  float* grad = reinterpret_cast<float*>(static_cast<char*>(workspace) + align_up(8 * static_cast<size_t>(rows)));
  pgc::LogitsArgs k = logits_args(logits, a->targets);
  k.logprobs = a->logprobs;
  pgc::PairArgs p{};
  p.targets = a->targets;
  p.offsets = a->offsets;
  p.logprobs = a->logprobs;
  p.ref_logprobs = a->ref_logprobs;
  p.weights = a->pair_weights;
  p.loss = a->loss;
  p.margins = a->margins;
  p.grad = a->dlogits ? grad : nullptr;
  p.chunk_sums = reinterpret_cast<double*>(reinterpret_cast<char*>(grad) + align_up(4 * static_cast<size_t>(rows)));
  p.rows = rows;
  p.cols = logits->cols;
  p.pairs = pairs;
  p.beta = a->beta;
  p.smoothing = a->label_smoothing;
  p.scale = a->scale;
  if (need == 0 && rows > 0) {
    k.dlogits = a->dlogits;
    k.out_stride = a->dlogits_stride;
    return launched(pgc::launch_small_preference(k, p, logits->dtype, stream), "preference loss kernel");
  }
  const bool sums_in_gradient = rows > 0 && a->dlogits && pgc::preference_sums_in_gradient(rows, logits->cols, pairs, logits->dtype);
  if (rows > 0) {
    k.stats = stats;
    k.zero_grad = sums_in_gradient ? nullptr : grad;
    CHECK(launched(pgc::launch_logits(k, pgc::RowMode::kForward, logits->dtype, stream), "log-probability kernel"));
  }
  if (sums_in_gradient) {
    k.dlogits = a->dlogits;
    k.out_stride = a->dlogits_stride;
    return launched(pgc::launch_pair_gradient(k, p, logits->dtype, stream), "pair gradient kernel");
  }
  if (pairs > 0) CHECK(launched(pgc::launch_pairs(p, stream), "pair kernel"));
  if (rows > 0 && a->dlogits) {
    k.grad = grad;
    k.dlogits = a->dlogits;
    k.out_stride = a->dlogits_stride;
    CHECK(launched(pgc::launch_logits(k, pgc::RowMode::kBackward, logits->dtype, stream),
                   "log-probability gradient kernel"));
  }
  return PGC_OK;
}

int pgc_policy_loss(const pgc_logits* logits, const pgc_policy_args* a, void* hip_stream) {
  if (logits == nullptr || a == nullptr) return fail(PGC_EINVAL, "null arguments");
  CHECK(check_logits(logits, a->targets));
  const int64_t rows = logits->rows;
  if (!(a->clip_low >= 0.0 && a->clip_low <= 1.0)) return fail(PGC_EINVAL, "clip_low must lie in [0, 1]");
  if (!(a->clip_high >= 0.0) || !finite32(a->clip_high))
    return fail(PGC_EINVAL, "clip_high must be finite and not negative");
  if (!finite32(a->kl) || !finite32(a->scale)) return fail(PGC_EINVAL, "kl and scale must be finite");
  CHECK(check_floats("old_logprobs", a->old_logprobs, rows, true));
  CHECK(check_floats("advantages", a->advantages, rows, true));
  CHECK(check_floats("ref_logprobs", a->ref_logprobs, rows, a->kl != 0.0));
  CHECK(check_floats("token_weights", a->token_weights, rows, false));
  CHECK(check_floats("loss", a->loss, rows, true));
  CHECK(check_floats("logprobs", a->logprobs, rows, true));
  if (a->dlogits) CHECK(check_dlogits(logits, a->dlogits, a->dlogits_stride));
  const int b = value_bytes(logits->dtype);
  const Span outs[] = {array("loss", a->loss, rows, 4), array("logprobs", a->logprobs, rows, 4),
                       matrix("dlogits", a->dlogits, rows, logits->cols, a->dlogits_stride, b)};
  const Span ins[] = {array("targets", a->targets, rows, 4), array("old_logprobs", a->old_logprobs, rows, 4),
                      array("advantages", a->advantages, rows, 4), array("ref_logprobs", a->ref_logprobs, rows, 4),
                      array("token_weights", a->token_weights, rows, 4)};
  CHECK(check_all_apart(outs, 3, ins, 5));
  const Span z = matrix("logits", logits->data, rows, logits->cols, logits->stride, b);
  CHECK(check_all_apart(outs, 2, &z, 1));
  if (rows == 0) return PGC_OK;
  pgc::LogitsArgs k = logits_args(logits, a->targets);
  k.old_logprobs = a->old_logprobs;
  k.advantages = a->advantages;
  k.kl = static_cast<float>(a->kl);
  k.ref_logprobs = k.kl != 0.f ? a->ref_logprobs : nullptr;   // of a factor that 32 bits round to 0, 0 * inf would stay
  k.weights = a->token_weights;
  k.loss = a->loss;
  k.logprobs = a->logprobs;
  k.dlogits = a->dlogits;
  k.out_stride = a->dlogits_stride;
  k.clip_low = static_cast<float>(1.0 - a->clip_low);
  k.clip_high = static_cast<float>(1.0 + a->clip_high);
  k.scale = static_cast<float>(a->scale);
  return launched(pgc::launch_logits(k, pgc::RowMode::kPolicy, logits->dtype, static_cast<hipStream_t>(hip_stream)),
                  "policy loss kernel");
}

}  // extern "C"
