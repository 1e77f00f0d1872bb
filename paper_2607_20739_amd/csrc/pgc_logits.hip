// Token log-probabilities, their gradient, the policy loss and the preference loss's pair
// sums (include/pgc_ops.h), for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_ops_kernels.h"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWave = 64;
constexpr int64_t kMaxBlocks = 1 << 20;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// A row's maximum and the sum of exp(z - maximum).  A maximum of -inf (nothing seen yet,
// or nothing but -inf) counts as 0 in differences, which keeps -inf - -inf out of them.
struct Stat {
  float top, sum;
};

__device__ __forceinline__ float finite_top(float top) { return top == -INFINITY ? 0.f : top; }

__device__ __forceinline__ Stat join(Stat a, Stat b) {
  const float top = fmaxf(a.top, b.top), base = finite_top(top);
  return {top, a.sum * exp2f((a.top - base) * kLog2E) + b.sum * exp2f((b.top - base) * kLog2E)};
}

// What a row's gradient is made of: g (onehot - exp(z - top - log_sum)).
struct RowGrad {
  float g, top, log_sum;
};

// The row's loss and the factor of its gradient, from its log-probability.
__device__ __forceinline__ float policy_row(const LogitsArgs& a, int64_t row, float lp, float* loss) {
  const float adv = a.advantages[row], weight = a.weights ? a.weights[row] : 1.f;
  const float ratio = expf(lp - a.old_logprobs[row]);
  const float bounded = ratio < a.clip_low ? a.clip_low : ratio > a.clip_high ? a.clip_high : ratio;
  const float free = ratio * adv, bound = bounded * adv;
  float l = 0.f, slope = 0.f;
  if (adv != 0.f) {
    l = free > bound ? -bound : -free;
    slope = free > bound ? 0.f : -free;
  } else if (lp != lp) {
    l = slope = lp;
  }
  if (a.ref_logprobs) {
    const float d = a.ref_logprobs[row] - lp, e = expm1f(d);
    l += a.kl * (e - d);
    slope -= a.kl * e;
  }
  *loss = l;
  return slope * a.scale * weight;
}

template <class T, RowMode kMode>
__global__ __launch_bounds__(kThreads)
void logits_kernel(LogitsArgs a) {
  const int lane = threadIdx.x % kWave;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave; row < a.rows;
       row += static_cast<int64_t>(gridDim.x) * (kThreads / kWave)) {
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const int32_t y = a.targets[row];
    bool counts = y >= 0 && y < a.cols;
    RowGrad r{0.f, 0.f, 0.f};
    if constexpr (kMode == RowMode::kBackward) {
      r = {counts ? a.grad[row] : 0.f, a.stats[2 * row], a.stats[2 * row + 1]};
    } else {
      if (kMode == RowMode::kPolicy && a.weights && a.weights[row] == 0.f) counts = false;
      float lp = 0.f, loss = 0.f;
      if (counts) {
        Stat s{-INFINITY, 0.f};
        for (int64_t j = lane; j < a.cols; j += kWave) {
          const float v = static_cast<float>(z[j]), top = fmaxf(s.top, v), base = finite_top(top);
          s = {top, s.sum * exp2f((s.top - base) * kLog2E) + exp2f((v - base) * kLog2E)};
        }
        for (int d = 1; d < kWave; d *= 2) s = join(s, {__shfl_xor(s.top, d, kWave), __shfl_xor(s.sum, d, kWave)});
        r.top = s.top;
        if (s.top == -INFINITY && s.sum == 0.f) {
          lp = -INFINITY;
        } else {
          r.log_sum = kLn2 * log2f(s.sum);
          lp = (static_cast<float>(z[y]) - s.top) - r.log_sum;
        }
        if (kMode == RowMode::kPolicy) r.g = policy_row(a, row, lp, &loss);
      }
      if (lane == 0) {
        a.logprobs[row] = lp;
        if (kMode == RowMode::kPolicy) a.loss[row] = loss;
        if (kMode == RowMode::kForward && a.stats) {
          a.stats[2 * row] = r.top;
          a.stats[2 * row + 1] = r.log_sum;
        }
        if (kMode == RowMode::kForward && a.zero_grad) a.zero_grad[row] = 0.f;
      }
    }
    if (kMode == RowMode::kForward || a.dlogits == nullptr) continue;
    T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
    const bool none = r.g == 0.f || (r.top == -INFINITY && r.log_sum == 0.f);
    for (int64_t j = lane; j < a.cols; j += kWave) {
      float v = 0.f;
      if (!none) {
        const float p = exp2f(((static_cast<float>(z[j]) - r.top) - r.log_sum) * kLog2E);
        v = j == y ? r.g - r.g * p : -r.g * p;
      }
      dz[j] = static_cast<T>(v);
    }
  }
}

template <class T>
hipError_t launch_typed(const LogitsArgs& a, RowMode mode, hipStream_t stream) {
  const int64_t rows_per_block = kThreads / kWave;
  const int blocks = static_cast<int>(std::min((a.rows + rows_per_block - 1) / rows_per_block, kMaxBlocks));
  switch (mode) {
    case RowMode::kForward: logits_kernel<T, RowMode::kForward><<<blocks, kThreads, 0, stream>>>(a); break;
    case RowMode::kBackward: logits_kernel<T, RowMode::kBackward><<<blocks, kThreads, 0, stream>>>(a); break;
    case RowMode::kPolicy: logits_kernel<T, RowMode::kPolicy><<<blocks, kThreads, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

// One block per pair: the two sequences' sums of l - ref in 64 bits, in a fixed order,
// then the loss and the gradient of every row.
__global__ __launch_bounds__(kThreads)
void pair_kernel(PairArgs a) {
  __shared__ double sums[kThreads / kWave];
  for (int64_t pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    int64_t at[3];
    for (int k = 0; k < 3; ++k)
      at[k] = std::min<int64_t>(std::max<int64_t>(a.offsets[2 * pair + k], 0), a.rows);
    double sum = 0.0;
    for (int64_t t = at[0] + threadIdx.x; t < at[2]; t += kThreads) {
      const int32_t y = a.targets[t];
      if (y < 0 || y >= a.cols) continue;
      const double v = static_cast<double>(a.logprobs[t]) - (a.ref_logprobs ? a.ref_logprobs[t] : 0.f);
      sum += t < at[1] ? v : -v;
    }
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d, kWave);
    __syncthreads();
    if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = sum;
    __syncthreads();
    double h = 0.0;
    for (int w = 0; w < kThreads / kWave; ++w) h += sums[w];
    h *= a.beta;
    const double rest = log1p(exp(-fabs(h)));
    const double minus = rest + fmax(-h, 0.0), plus = rest + fmax(h, 0.0);   // -ln sigma(h), -ln sigma(-h)
    if (threadIdx.x == 0) {
      a.margins[pair] = static_cast<float>(h);
      a.loss[pair] = static_cast<float>(h != h ? h : (1.0 - a.smoothing) * minus + a.smoothing * plus);
    }
    if (a.grad == nullptr) continue;
    const double weight = a.weights ? a.weights[pair] : 1.f;
    const double slope = a.smoothing * (1.0 / (1.0 + exp(-h))) - (1.0 - a.smoothing) * (1.0 / (1.0 + exp(h)));
    const float g = weight == 0.0 ? 0.f : static_cast<float>(slope * a.beta * a.scale * weight);
    for (int64_t t = at[0] + threadIdx.x; t < at[2]; t += kThreads) a.grad[t] = t < at[1] ? g : -g;
  }
}

}  // namespace

hipError_t launch_logits(const LogitsArgs& a, RowMode mode, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PGC_F32: return launch_typed<float>(a, mode, stream);
    case PGC_BF16: return launch_typed<__bf16>(a, mode, stream);
    default: return launch_typed<_Float16>(a, mode, stream);
  }
}

hipError_t launch_pairs(const PairArgs& a, hipStream_t stream) {
  pair_kernel<<<static_cast<int>(std::min(a.pairs, kMaxBlocks)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pgc
