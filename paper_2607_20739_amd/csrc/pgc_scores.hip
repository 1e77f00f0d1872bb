// Scores of tokens under rows of logits and their gradient (include/pgc_ops.h), for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_ops_kernels.h"

#pragma clang fp contract(off)

namespace pgc {
namespace {

constexpr int kThreads = 256;

// A logit and its column: the larger comes first, of equal ones the lower column.
struct Entry {
  float value;
  uint32_t column;
  __device__ __forceinline__ bool before(const Entry& o) const { return value > o.value || (value == o.value && column < o.column); }
};
constexpr uint32_t kNoColumn = 0xFFFFFFFFu;

// Over the block's threads, in all of them.
template <class V, class Join>
__device__ __forceinline__ V block_join(V v, Join join) {
  __shared__ V all[kThreads];
  __syncthreads();
  all[threadIdx.x] = v;
  for (int d = kThreads / 2; d > 0; d /= 2) {
    __syncthreads();
    if (threadIdx.x < static_cast<uint32_t>(d)) all[threadIdx.x] = join(all[threadIdx.x], all[threadIdx.x + d]);
  }
  __syncthreads();
  return all[0];
}

// A block per row: the maximum, the sums, then the top tokens one by one.
template <class T>
__global__ __launch_bounds__(kThreads)
void scores_kernel(ScoresArgs a) {
  const int64_t row = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const int64_t y = a.targets ? a.targets[row] : 0;
  const bool first = threadIdx.x == 0;
  auto write = [&](float lp, float entropy, float top, float log_sum) {
    if (!first) return;
    if (a.targets) a.logprobs[row] = lp;
    if (a.entropy) a.entropy[row] = entropy;
    if (a.stats) {
      a.stats[2 * row] = top;
      a.stats[2 * row + 1] = log_sum;
    }
  };
  auto write_top = [&](int i, float lp, int32_t token) {
    a.top_logprobs[row * a.top + i] = lp;
    a.top_tokens[row * a.top + i] = token;
  };
  if (a.targets && (y < 0 || y >= a.cols)) {
    write(0.f, 0.f, 0.f, 0.f);
    for (int i = threadIdx.x; i < a.top; i += kThreads) write_top(i, 0.f, -1);
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  float top = -INFINITY, bad = 0.f;
  for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
    const float v = static_cast<float>(z[j]);
    top = fmaxf(top, v);
    if (!(v < INFINITY)) bad = 1.f;
  }
  top = block_join(top, [](float x, float y) { return fmaxf(x, y); });
  bad = block_join(bad, [](float x, float y) { return fmaxf(x, y); });
  if (bad != 0.f || top == -INFINITY) {
    if (bad != 0.f) write(NAN, NAN, NAN, NAN);
    else write(-INFINITY, 0.f, -INFINITY, 0.f);
    for (int i = threadIdx.x; i < a.top; i += kThreads) write_top(i, bad != 0.f ? NAN : -INFINITY, -1);
    return;
  }
  float sum = 0.f, weighted = 0.f;
  for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
    const float d = static_cast<float>(z[j]) - top, e = expf(d);
    sum += e;
    if (e > 0.f) weighted += e * d;
  }
  sum = block_join(sum, [](float x, float y) { return x + y; });
  weighted = block_join(weighted, [](float x, float y) { return x + y; });
  const float log_sum = logf(sum);
  write(a.targets ? (static_cast<float>(z[y]) - top) - log_sum : 0.f, log_sum - weighted / sum, top, log_sum);
  Entry last{INFINITY, 0};
  for (int i = 0; i < a.top; ++i) {
    Entry best{-INFINITY, kNoColumn};
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
      const Entry e{static_cast<float>(z[j]), static_cast<uint32_t>(j)};
      if (last.before(e) && e.before(best) && e.value > -INFINITY) best = e;
    }
    last = best = block_join(best, [](const Entry& x, const Entry& y) { return x.before(y) ? x : y; });
    if (first) write_top(i, (best.value - top) - log_sum, best.column == kNoColumn ? -1 : static_cast<int32_t>(best.column));
  }
}

template <class T>
__global__ __launch_bounds__(kThreads)
void scores_gradient_kernel(ScoresArgs a) {
  const int64_t row = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const int64_t y = a.targets ? a.targets[row] : -1;
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
  const bool counts = a.targets == nullptr || (y >= 0 && y < a.cols);
  const float g = a.grad_logprobs && counts ? a.grad_logprobs[row] : 0.f, e = a.grad_entropy && counts ? a.grad_entropy[row] : 0.f;
  const float top = a.stats[2 * row], log_sum = a.stats[2 * row + 1];
  const bool none = (g == 0.f && e == 0.f) || (top == -INFINITY && log_sum == 0.f);
  const float rest = e == 0.f ? 0.f : a.entropy[row] - log_sum;
  for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
    float v = 0.f;
    if (!none) {
      const float d = static_cast<float>(z[j]) - top, p = expf(d - log_sum);
      v = p * (-g - e * (fmaxf(d, -1e4f) + rest));
      if (j == y) v += g;
    }
    dz[j] = static_cast<T>(v);
  }
}

dim3 grid_of(int64_t rows) {
  const int64_t x = std::min<int64_t>(rows, 1 << 20);
  return dim3(static_cast<uint32_t>(x), static_cast<uint32_t>((rows + x - 1) / x));
}

}  // namespace

size_t scores_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_scores(const ScoresArgs& a, int dtype, void*, hipStream_t stream) {
  const dim3 grid = grid_of(a.rows);
  if (dtype == PGC_F32) scores_kernel<float><<<grid, kThreads, 0, stream>>>(a);
  else if (dtype == PGC_BF16) scores_kernel<__bf16><<<grid, kThreads, 0, stream>>>(a);
  else scores_kernel<_Float16><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_scores_gradient(const ScoresArgs& a, int dtype, hipStream_t stream) {
  const dim3 grid = grid_of(a.rows);
  if (dtype == PGC_F32) scores_gradient_kernel<float><<<grid, kThreads, 0, stream>>>(a);
  else if (dtype == PGC_BF16) scores_gradient_kernel<__bf16><<<grid, kThreads, 0, stream>>>(a);
  else scores_gradient_kernel<_Float16><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pgc
