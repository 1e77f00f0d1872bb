// Token log-probabilities, their gradient, the policy loss and the preference loss's pair
// sums (include/pgc_ops.h), for gfx950.
//
// A row of logits belongs to a group of LANES lanes (4 to 1,024): lane i takes the 16-byte
// vectors i, i + LANES, ... counted from the row's first value, wherever that lies in memory
// (loads and stores work at any alignment), and the last values that fill no vector go to one
// lane each.  Which lane sums what, and hence every bit of the result, depends on the number of
// columns alone.  Each lane keeps a running maximum and sum; lanes and waves join theirs once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_lanes.h"
#include "pgc_ops_kernels.h"

namespace pgc {
namespace {

constexpr int kWave = 64, kBlock = 256;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef u4v u4v_unaligned __attribute__((aligned(2)));

// 16 bytes of a row and the values in them.
template <class T>
struct Vec {
  static constexpr int kN = 16 / sizeof(T);
  typedef T Packed __attribute__((ext_vector_type(kN)));
  typedef float Floats __attribute__((ext_vector_type(kN)));

  // Vector `first + lane` of a row; `first` is the same for all lanes, so the address is a
  // scalar and a lane's 32-bit offset.
  static __device__ __forceinline__ u4v load(const T* row, uint32_t first, uint32_t lane) {
    const char* p = reinterpret_cast<const char*>(row) + static_cast<uint64_t>(first) * 16 + lane * 16;
    return __builtin_nontemporal_load(reinterpret_cast<const u4v_unaligned*>(p));
  }
  static __device__ __forceinline__ void store(T* row, uint32_t first, uint32_t lane, u4v v) {
    char* p = reinterpret_cast<char*>(row) + static_cast<uint64_t>(first) * 16 + lane * 16;
    __builtin_nontemporal_store(v, reinterpret_cast<u4v_unaligned*>(p));
  }
  static __device__ __forceinline__ Floats floats(u4v v) {
    return __builtin_convertvector(__builtin_bit_cast(Packed, v), Floats);
  }
  static __device__ __forceinline__ u4v packed(Floats f) {
    return __builtin_bit_cast(u4v, __builtin_convertvector(f, Packed));
  }
  // A vector of -inf: counts for nothing in a maximum or a sum.
  static __device__ __forceinline__ u4v none() {
    const uint32_t bits = sizeof(T) == 4 ? 0xFF800000u : std::is_same_v<T, __bf16> ? 0xFF80FF80u : 0xFC00FC00u;
    return u4v{bits, bits, bits, bits};
  }
};

// 2^x by the hardware's instruction; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A maximum and the sum of exp(z - maximum) of some of a row's values.  A maximum of -inf
// (nothing seen yet, or nothing but -inf) counts as 0 in differences, which keeps -inf - -inf
// out of them.  NaN never becomes the maximum, but the sum.
struct Stat {
  float top, sum;
};

__device__ __forceinline__ float finite_top(float top) { return top == -INFINITY ? 0.f : top; }

template <class T, int U>
__device__ __forceinline__ void add_few(Stat& s, const u4v* h) {
  constexpr int kN = Vec<T>::kN;
  float top = s.top;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const auto f = Vec<T>::floats(h[i]);
#pragma unroll
    for (int k = 0; k < kN; ++k) top = fmaxf(top, f[k]);
  }
  const float base = finite_top(top);
  float sum = s.sum * exp2_fast((s.top - base) * kLog2E);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    auto f = Vec<T>::floats(h[i]);
#pragma unroll
    for (int k = 0; k < kN; ++k) f[k] = exp2_fast((f[k] - base) * kLog2E);
#pragma unroll
    for (int w = kN / 2; w >= 1; w /= 2)
#pragma unroll
      for (int k = 0; k < w; ++k) f[k] += f[k + w];
    sum += f[0];
  }
  s = {top, sum};
}

// U vectors, four at a time: their 32 values are all that is unpacked at once.
template <class T, int U>
__device__ __forceinline__ void add_vectors(Stat& s, const u4v (&h)[U]) {
  constexpr int kFew = U < 4 ? U : 4;
  static_assert(U % kFew == 0, "whole groups");
#pragma unroll
  for (int i = 0; i < U; i += kFew) add_few<T, kFew>(s, h + i);
}

__device__ __forceinline__ void add_value(Stat& s, float v) {
  const float top = fmaxf(s.top, v), base = finite_top(top);
  s = {top, s.sum * exp2_fast((s.top - base) * kLog2E) + exp2_fast((v - base) * kLog2E)};
}

template <int LANES>
__device__ __forceinline__ float lane_group_max(float v) {
  if constexpr (LANES >= 2) v = fmaxf(v, dpp_move<kDppSwap1>(v));
  if constexpr (LANES >= 4) v = fmaxf(v, dpp_move<kDppSwap2>(v));
  if constexpr (LANES >= 8) v = fmaxf(v, dpp_move<kDppHalfMirror>(v));
  if constexpr (LANES >= 16) v = fmaxf(v, dpp_move<kDppMirror>(v));
  if constexpr (LANES >= 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
  if constexpr (LANES >= 64) v = fmaxf(v, __shfl_xor(v, 32, 64));
  return v;
}

// Joined over LANES lanes of a wave; every lane ends with the result.
template <int LANES>
__device__ __forceinline__ Stat join_lanes(Stat s) {
  const float top = lane_group_max<LANES>(s.top);
  return {top, lane_group_sum<LANES>(s.sum * exp2_fast((s.top - finite_top(top)) * kLog2E))};
}

// A group of LANES lanes and its row: block `group` of the launch holds kRows of them.
template <int LANES>
struct Place {
  static constexpr int kThreads = LANES < kBlock ? kBlock : LANES;
  static constexpr int kRows = kThreads / LANES;
  __device__ static uint32_t lane() { return threadIdx.x % LANES; }
  __device__ static int64_t row(int64_t group) {
    if constexpr (LANES >= kThreads) return group;
    uint32_t r = threadIdx.x / LANES;
    if constexpr (LANES >= kWave) r = __builtin_amdgcn_readfirstlane(r);
    return group * kRows + r;
  }
  static int64_t groups(int64_t rows) { return (rows + kRows - 1) / kRows; }
};

// Grids of up to 2^31 groups (of one dimension, HIP takes fewer threads than that needs).
constexpr int64_t kGridX = 1 << 20, kGridYZ = 65535;

// What the policy loss reads of a row besides its logits.
struct PolicyRow {
  float advantage, old_logprob, ref_logprob, weight;
};

__device__ __forceinline__ PolicyRow policy_row(const LogitsArgs& a, int64_t row) {
  return {a.advantages[row], a.old_logprobs[row], a.ref_logprobs ? a.ref_logprobs[row] : 0.f,
          a.weights ? a.weights[row] : 1.f};
}

// The row's loss from its log-probability, and the factor of its gradient.
__device__ __forceinline__ float policy_slope(const LogitsArgs& a, const PolicyRow& r, float lp, float* loss) {
  const float ratio = expf(lp - r.old_logprob);
  const float bounded = ratio < a.clip_low ? a.clip_low : ratio > a.clip_high ? a.clip_high : ratio;
  const float free = ratio * r.advantage, bound = bounded * r.advantage;
  float l = 0.f, slope = 0.f;
  if (r.advantage != 0.f) {
    l = free > bound ? -bound : -free;
    slope = free > bound ? 0.f : -free;
  } else if (lp != lp) {
    l = slope = lp;
  }
  if (a.ref_logprobs) {
    const float d = r.ref_logprob - lp, e = expm1f(d);
    l += a.kl * (e - d);
    slope -= a.kl * e;
  }
  *loss = l;
  return slope * a.scale * r.weight;
}

// A row's gradient g (onehot(y) - exp(z - top - log_sum)), value by value.  The exponential is
// taken 2^24 times larger and g as much smaller, so that what lies below 2^-126 is not lost
// before the product.
template <class T>
struct RowGradient {
  float g, scaled, top, shift;
  bool none;

  __device__ RowGradient(float g_, float top_, float log_sum)
      : g(g_), scaled(-g_ * 0x1p-24f), top(top_), shift(24.f - log_sum * kLog2E),
        none(g_ == 0.f || (top_ == -INFINITY && log_sum == 0.f)) {}

  __device__ __forceinline__ float of(float z) const {
    return scaled * exp2_fast(__builtin_fmaf(z - top, kLog2E, shift));
  }
  // Gradient of the vector that starts at column `first`.
  __device__ __forceinline__ u4v of_vector(u4v z, uint32_t y_in_vector) const {
    constexpr uint32_t kN = Vec<T>::kN;
    auto f = Vec<T>::floats(z);
#pragma unroll
    for (uint32_t k = 0; k < kN; ++k) f[k] = of(f[k]);
    if (y_in_vector < kN) {
#pragma unroll
      for (uint32_t k = 0; k < kN; ++k) f[k] += k == y_in_vector ? g : 0.f;
    }
    return Vec<T>::packed(f);
  }
};

// kForward and kPolicy.  The policy loss holds a lane's first HOLD vectors in registers from
// the sum to the gradient, so rows of up to LANES * HOLD vectors are read once; of longer ones
// the rest is read again.  Forward alone goes through the row HOLD vectors at a time.
template <class T, RowMode kMode, int LANES, int HOLD, bool kLonger>
__global__ __launch_bounds__(Place<LANES>::kThreads)
void row_kernel(LogitsArgs a) {
  constexpr int kN = Vec<T>::kN, kWaves = LANES / kWave, kMore = HOLD < 4 ? HOLD : 4;
  constexpr bool kPolicy = kMode == RowMode::kPolicy;
  __shared__ Stat parts[kWaves > 1 ? kWaves : 1];
  __shared__ float target_logit;
  const uint32_t lane = Place<LANES>::lane(), cols = static_cast<uint32_t>(a.cols);
  const uint32_t full = cols / kN, rem = cols % kN;
  const int64_t row = Place<LANES>::row(static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x);
  if (row < a.rows) {
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const int32_t y = a.targets[row];
    PolicyRow pr{};
    if constexpr (kPolicy) pr = policy_row(a, row);
    const bool counts = y >= 0 && y < a.cols && !(kPolicy && pr.weight == 0.f);
    u4v held[HOLD];
    float tail = -INFINITY, lp = 0.f, loss = 0.f, g = 0.f, log_sum = 0.f;
    Stat s{-INFINITY, 0.f};
    if (counts) {
#pragma unroll
      for (int i = 0; i < HOLD; ++i) {
        const uint32_t first = i * LANES;
        held[i] = first + lane < full ? Vec<T>::load(z, first, lane) : Vec<T>::none();
      }
      if (lane < rem) tail = static_cast<float>(z[full * kN + lane]);
      float zy = kWaves > 1 && threadIdx.x != 0 ? 0.f : static_cast<float>(z[y]);
      add_vectors<T>(s, held);
      if constexpr (kLonger) {
        for (uint32_t v0 = HOLD * LANES; v0 < full; v0 += kMore * LANES) {
          u4v more[kMore];
#pragma unroll
          for (int i = 0; i < kMore; ++i) {
            const uint32_t first = v0 + i * LANES;
            more[i] = first + lane < full ? Vec<T>::load(z, first, lane) : Vec<T>::none();
          }
          add_vectors<T>(s, more);
        }
      }
      if (lane < rem) add_value(s, tail);
      s = join_lanes<(LANES < kWave ? LANES : kWave)>(s);
      if constexpr (kWaves > 1) {
        // The target's logit is read by one wave, before the others can write over it.
        if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave] = s;
        if (threadIdx.x == 0) target_logit = zy;
        __syncthreads();
        s = join_lanes<(kWaves > 1 ? kWaves : 1)>(parts[threadIdx.x % kWaves]);
        zy = target_logit;
      }
      if (s.top == -INFINITY && s.sum == 0.f) {
        lp = -INFINITY;
      } else {
        log_sum = kLn2 * log2f(s.sum);
        lp = (zy - s.top) - log_sum;
      }
      if constexpr (kPolicy) g = policy_slope(a, pr, lp, &loss);
    }
    if (lane == 0) {
      a.logprobs[row] = lp;
      if constexpr (kPolicy) a.loss[row] = loss;
      if (kMode == RowMode::kForward && a.stats) {
        a.stats[2 * row] = counts ? s.top : 0.f;
        a.stats[2 * row + 1] = log_sum;
      }
      if (kMode == RowMode::kForward && a.zero_grad) a.zero_grad[row] = 0.f;
    }
    if constexpr (kPolicy) {
      if (a.dlogits == nullptr) return;
      T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
      const RowGradient<T> grad(g, s.top, log_sum);
      const uint32_t yv = static_cast<uint32_t>(y);
#pragma unroll
      for (int i = 0; i < HOLD; ++i) {
        const uint32_t first = i * LANES;
        asm("" : "+v"(held[i]));   // unpacked anew: twice the registers would go to its values
        if (first + lane < full)
          Vec<T>::store(dz, first, lane, grad.none ? u4v{0, 0, 0, 0} : grad.of_vector(held[i], yv - (first + lane) * kN));
      }
      if constexpr (kLonger)
        for (uint32_t first = HOLD * LANES; first < full; first += LANES)
          if (first + lane < full)
            Vec<T>::store(dz, first, lane, grad.none ? u4v{0, 0, 0, 0}
                                                     : grad.of_vector(Vec<T>::load(z, first, lane), yv - (first + lane) * kN));
      if (lane < rem) {
        const uint32_t j = full * kN + lane;
        dz[j] = static_cast<T>(grad.none ? 0.f : grad.of(tail) + (j == yv ? g : 0.f));
      }
    }
  }
}

// kBackward: every value by itself.  A group of LANES lanes takes LANES * U vectors of a row;
// the runs of a longer row go to different blocks.
template <class T, int LANES, int U>
__global__ __launch_bounds__(Place<LANES>::kThreads)
void gradient_kernel(LogitsArgs a) {
  constexpr int kN = Vec<T>::kN;
  const uint32_t lane = Place<LANES>::lane(), cols = static_cast<uint32_t>(a.cols);
  const uint32_t full = cols / kN, rem = cols % kN;
  const int64_t row = Place<LANES>::row(static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y);
  if (row >= a.rows) return;
  const int32_t y = a.targets[row];
  const float g = a.grad[row], top = a.stats[2 * row], log_sum = a.stats[2 * row + 1];
  const RowGradient<T> grad(y >= 0 && y < a.cols ? g : 0.f, top, log_sum);
  const uint32_t yv = static_cast<uint32_t>(y);
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
  const uint32_t v0 = blockIdx.x * (LANES * U);
  if (grad.none) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (v0 + i * LANES + lane < full) Vec<T>::store(dz, v0 + i * LANES, lane, u4v{0, 0, 0, 0});
  } else {
    u4v h[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      h[i] = u4v{0, 0, 0, 0};
      if (v0 + i * LANES + lane < full) h[i] = Vec<T>::load(z, v0 + i * LANES, lane);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t first = v0 + i * LANES;
      if (first + lane < full) Vec<T>::store(dz, first, lane, grad.of_vector(h[i], yv - (first + lane) * kN));
    }
  }
  if (blockIdx.x == gridDim.x - 1 && lane < rem) {
    const uint32_t j = full * kN + lane;
    dz[j] = static_cast<T>(grad.none ? 0.f : grad.of(static_cast<float>(z[j])) + (j == yv ? grad.g : 0.f));
  }
}

template <class T, RowMode kMode, int LANES, int HOLD, bool kLonger = false>
hipError_t launch_rows(const LogitsArgs& a, hipStream_t stream) {
  const int64_t groups = Place<LANES>::groups(a.rows), x = std::min(groups, kGridX);
  const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>((groups + x - 1) / x));
  row_kernel<T, kMode, LANES, HOLD, kLonger><<<grid, Place<LANES>::kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <class T, int LANES, int U>
hipError_t launch_gradient(const LogitsArgs& a, hipStream_t stream) {
  constexpr int64_t kRun = int64_t{LANES} * U;
  const int64_t full = a.cols / Vec<T>::kN, groups = Place<LANES>::groups(a.rows), y = std::min(groups, kGridYZ);
  const dim3 grid(static_cast<uint32_t>(std::max<int64_t>(1, (full + kRun - 1) / kRun)), static_cast<uint32_t>(y),
                  static_cast<uint32_t>((groups + y - 1) / y));
  gradient_kernel<T, LANES, U><<<grid, Place<LANES>::kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

// Lanes and vectors per lane by the row's whole vectors.
template <class T, RowMode kMode>
hipError_t launch_by_row(const LogitsArgs& a, hipStream_t stream) {
  const int64_t full = a.cols / Vec<T>::kN;
  if constexpr (sizeof(T) == 4)
    if (full <= 4) return launch_rows<T, kMode, 4, 1>(a, stream);
  if (full <= 8) return launch_rows<T, kMode, 8, 1>(a, stream);
  if (full <= 16) return launch_rows<T, kMode, 16, 1>(a, stream);
  if (full <= 32) return launch_rows<T, kMode, 32, 1>(a, stream);
  if (full <= 64) return launch_rows<T, kMode, 64, 1>(a, stream);
  if (full <= 128) return launch_rows<T, kMode, 64, 2>(a, stream);
  if (full <= 256) return launch_rows<T, kMode, 64, 4>(a, stream);
  if (full <= 512) return launch_rows<T, kMode, 64, 8>(a, stream);
  if (full <= 1024) return launch_rows<T, kMode, 256, 4>(a, stream);
  if constexpr (kMode == RowMode::kForward) {
    return launch_rows<T, kMode, 1024, 4, true>(a, stream);
  } else {
    if (full <= 2048) return launch_rows<T, kMode, 256, 8>(a, stream);
    if (full <= 4096) return launch_rows<T, kMode, 512, 8>(a, stream);
    if (full <= 8192) return launch_rows<T, kMode, 1024, 8>(a, stream);
    if (full <= 16384) return launch_rows<T, kMode, 1024, 16>(a, stream);
    return launch_rows<T, kMode, 1024, 16, true>(a, stream);
  }
}

template <class T>
hipError_t launch_gradient_by_row(const LogitsArgs& a, hipStream_t stream) {
  const int64_t full = a.cols / Vec<T>::kN;
  if constexpr (sizeof(T) == 4)
    if (full <= 4) return launch_gradient<T, 4, 1>(a, stream);
  if (full <= 8) return launch_gradient<T, 8, 1>(a, stream);
  if (full <= 16) return launch_gradient<T, 16, 1>(a, stream);
  if (full <= 32) return launch_gradient<T, 32, 1>(a, stream);
  if (full <= 64) return launch_gradient<T, 64, 1>(a, stream);
  if (full <= 128) return launch_gradient<T, 64, 2>(a, stream);
  if (full <= 256) return launch_gradient<T, 64, 4>(a, stream);
  return launch_gradient<T, 256, 4>(a, stream);
}

template <class T>
hipError_t launch_typed(const LogitsArgs& a, RowMode mode, hipStream_t stream) {
  switch (mode) {
    case RowMode::kForward: return launch_by_row<T, RowMode::kForward>(a, stream);
    case RowMode::kPolicy: return launch_by_row<T, RowMode::kPolicy>(a, stream);
    default: return launch_gradient_by_row<T>(a, stream);
  }
}

// One block per pair: the two sequences' sums of l - ref in 64 bits, in a fixed order,
// then the loss and the gradient of every row.
__global__ __launch_bounds__(kBlock)
void pair_kernel(PairArgs a) {
  __shared__ double sums[kBlock / kWave];
  for (int64_t pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    int64_t at[3];
    for (int k = 0; k < 3; ++k)
      at[k] = std::min<int64_t>(std::max<int64_t>(a.offsets[2 * pair + k], 0), a.rows);
    double sum = 0.0;
    for (int64_t t = at[0] + threadIdx.x; t < at[2]; t += kBlock) {
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
    for (int w = 0; w < kBlock / kWave; ++w) h += sums[w];
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
    for (int64_t t = at[0] + threadIdx.x; t < at[2]; t += kBlock) a.grad[t] = t < at[1] ? g : -g;
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
  pair_kernel<<<static_cast<int>(std::min(a.pairs, kGridX)), kBlock, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pgc
