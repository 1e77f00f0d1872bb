// The norm of many gradients and the AdamW step over many tensors (include/pgc_ops.h), for gfx950.
//
// Memory bounds both: a value's arithmetic is some 20 to 60 instructions.  What many tensors ask for is
// few launches: up to 48 (64) of them go to one by value, in its arguments, so that nothing has to be
// copied to the device first, and a block finds its tensor among them by one comparison per lane.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_ops_kernels.h"

// A product and a sum are rounded apart, so that states have the same bits however the code is laid out.
#pragma clang fp contract(off)

namespace pgc {
namespace {

constexpr int kWave = 64, kThreads = 256, kEach = 4;      // values of a lane at a time: a wave's make a block of 8-bit states
constexpr int kStateBlock = kWave * kEach;

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4_at4 __attribute__((aligned(4), may_alias));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef u2 u2_at2 __attribute__((aligned(2), may_alias));
typedef uint32_t u1_at1 __attribute__((aligned(1), may_alias));
typedef uint16_t u16_raw __attribute__((may_alias));
typedef uint32_t u32_raw __attribute__((may_alias));
typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
typedef _Float16 hf4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// Which of up to 64 tensors block `block` belongs to: the last whose first block is no later.  (Tensors
// without values have no blocks: the next one has the same first.)
__device__ __forceinline__ int32_t tensor_of(const int32_t* first, int32_t tensors, int32_t block) {
  const int32_t lane = threadIdx.x % kWave;
  return uniform(__popcll(__ballot(lane < tensors && first[lane] <= block))) - 1;
}

// Four neighbouring values from number i on, `n` of which are there, as they lie in memory.
__device__ __forceinline__ u4 load4(const void* p, int64_t i, int n, int dtype) {
  u4 r{0, 0, 0, 0};
  if (dtype == PGC_F32) {
    const auto* q = static_cast<const float*>(p) + i;
    if (n == kEach) return *reinterpret_cast<const u4_at4*>(q);
    for (int k = 0; k < n; ++k) r[k] = reinterpret_cast<const u32_raw*>(q)[k];
  } else {
    const auto* q = static_cast<const uint16_t*>(p) + i;
    if (n == kEach) {
      const u2 v = *reinterpret_cast<const u2_at2*>(q);
      return u4{v[0], v[1], 0, 0};
    }
    for (int k = 0; k < n; ++k) r[k / 2] |= static_cast<uint32_t>(reinterpret_cast<const u16_raw*>(q)[k]) << 16 * (k % 2);
  }
  return r;
}

__device__ __forceinline__ f4 floats(u4 r, int dtype) {
  if (dtype == PGC_F32) return __builtin_bit_cast(f4, r);
  const u2 h{r[0], r[1]};
  if (dtype == PGC_BF16) return __builtin_convertvector(__builtin_bit_cast(bf4, h), f4);
  return __builtin_convertvector(__builtin_bit_cast(hf4, h), f4);
}

__device__ __forceinline__ void store4(void* p, int64_t i, int n, int dtype, f4 v) {
  if (dtype == PGC_F32) {
    auto* q = static_cast<float*>(p) + i;
    if (n == kEach) *reinterpret_cast<u4_at4*>(q) = __builtin_bit_cast(u4, v);
    else for (int k = 0; k < n; ++k) q[k] = v[k];
    return;
  }
  const u2 h = dtype == PGC_BF16 ? __builtin_bit_cast(u2, __builtin_convertvector(v, bf4)) : __builtin_bit_cast(u2, __builtin_convertvector(v, hf4));
  auto* q = static_cast<uint16_t*>(p) + i;
  if (n == kEach) *reinterpret_cast<u2_at2*>(q) = h;
  else for (int k = 0; k < n; ++k) reinterpret_cast<u16_raw*>(q)[k] = static_cast<uint16_t>(h[k / 2] >> 16 * (k % 2));
}

// ---- states in 8 bits -----------------------------------------------------------------------

__device__ __forceinline__ uint32_t load_codes(const void* p, int64_t i, int n) {
  const uint8_t* q = static_cast<const uint8_t*>(p) + i;
  if (n == kEach) return *reinterpret_cast<const u1_at1*>(q);
  uint32_t r = 0;
  for (int k = 0; k < n; ++k) r |= static_cast<uint32_t>(q[k]) << 8 * k;
  return r;
}
__device__ __forceinline__ void store_codes(void* p, int64_t i, int n, uint32_t codes) {
  uint8_t* q = static_cast<uint8_t*>(p) + i;
  if (n == kEach) *reinterpret_cast<u1_at1*>(q) = codes;
  else for (int k = 0; k < n; ++k) q[k] = static_cast<uint8_t>(codes >> 8 * k);
}

// Floats of 4 significant bits by their number: the float's bits shifted right.
constexpr int kShift = 20, kNoNumber = 0x7F8;   // from here on: infinities and NaN
constexpr int kSigned = 127, kUnsigned = 255;   // levels

// Number of the nearest one (ties to even) of |x|.
__device__ __forceinline__ int number_of(float x) {
  const uint32_t size = __float_as_uint(x) & 0x7FFFFFFFu;
  return static_cast<int>((size + 0x7FFFFu + (size >> kShift & 1)) >> kShift);
}

// Four values out of their codes and their block's scale.
template <int kLevels>
__device__ __forceinline__ f4 decode(uint32_t codes, float scale) {
  const int bits = __float_as_int(scale), base = (bits >> kShift) - kLevels;
  const bool finite = (bits & 0x7FFFFFFF) < (kNoNumber << kShift);
  f4 v;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint32_t code = codes >> 8 * k & 0xFF;
    const int c = code & kLevels, number = std::max(base + c, 0);
    uint32_t x = c == 0 ? 0 : static_cast<uint32_t>(number) << kShift;
    if (kLevels == kSigned) x |= (code & 0x80) << 24;
    v[k] = finite ? __uint_as_float(x) : NAN;
  }
  return v;
}

// Their codes, from their numbers and the block's largest.
template <int kLevels>
__device__ __forceinline__ uint32_t encode(f4 v, const int (&number)[kEach], int largest) {
  uint32_t codes = 0;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int c = number[k] - largest + kLevels;
    const uint32_t bits = __float_as_uint(v[k]);
    uint32_t code;
    if (kLevels == kSigned) code = c <= -8 || bits << 1 == 0 ? 0 : std::max(c, 1) | (bits >> 24 & 0x80);
    else code = v[k] == 0.f ? 0 : std::max(c, 1);
    codes |= (code & 0xFF) << 8 * k;
  }
  return codes;
}

__device__ __forceinline__ int wave_max(int v) {
  for (int d = 1; d < kWave; d *= 2) v = std::max(v, __shfl_xor(v, d, kWave));
  return uniform(v);
}

// The largest number of a block, at least `levels`.
template <int kLevels>
__device__ __forceinline__ int largest_of(const int (&number)[kEach]) {
  int most = kLevels;
#pragma unroll
  for (int k = 0; k < kEach; ++k) most = std::max(most, number[k]);
  return wave_max(most);
}
// The scale that stands for it.
__device__ __forceinline__ float scale_of(int largest) { return largest >= kNoNumber ? NAN : __int_as_float(largest << kShift); }

// ---- the step ---------------------------------------------------------------------------------

struct Rates {
  float rate, decay, spread;
};

template <bool k8>
__global__ __launch_bounds__(kThreads)
void adamw_kernel(AdamwArgs a) {
  const int32_t block = static_cast<int32_t>(blockIdx.x), at = tensor_of(a.first, a.tensors, block);
  const AdamwTensor& t = a.tensor[at];
  const int64_t from = static_cast<int64_t>(block - a.first[at]) * a.chunk, to = std::min<int64_t>(from + a.chunk, t.count);
  const float factor = a.factor ? *a.factor : 1.f;
  if (a.factor && !(fabsf(factor) < INFINITY)) return;
  Rates r{a.rate, t.decay, a.spread};
  if (a.lr_at || a.step_at) {
    const double lr = a.lr_at ? static_cast<double>(*a.lr_at) : a.lr, step = static_cast<double>(a.step_at ? *a.step_at : a.step);
    r.rate = static_cast<float>(lr / -expm1(step * a.log_beta1));
    r.spread = static_cast<float>(1.0 / sqrt(-expm1(step * a.log_beta2)));
    if (a.lr_at) r.decay = static_cast<float>(lr * t.decay);
  }
  void *param = t.param, *m_at = t.m, *v_at = t.v, *copy = t.copy;
  const void* grad = t.grad;
  float* scales = t.scales;
  const int64_t count = t.count;
  const int param_dtype = t.param_dtype, grad_dtype = t.grad_dtype, copy_dtype = t.copy_dtype;
  for (int64_t i = from + threadIdx.x * kEach; i - static_cast<int>(threadIdx.x) * kEach < to; i += kThreads * kEach) {
    const int n = static_cast<int>(std::min<int64_t>(std::max<int64_t>(count - i, 0), kEach));
    const u4 xr = load4(param, i, n, param_dtype), gr = load4(grad, i, n, grad_dtype);
    f4 m, v;
    const int64_t state_block = i / kStateBlock;
    if constexpr (k8) {
      const uint32_t mc = load_codes(m_at, i, n), vc = load_codes(v_at, i, n);
      float2 scale{0.f, 0.f};
      if (n > 0) scale = *reinterpret_cast<const float2*>(scales + 2 * state_block);
      m = decode<kSigned>(mc, scale.x);
      v = decode<kUnsigned>(vc, scale.y);
    } else {
      m = floats(load4(m_at, i, n, PGC_F32), PGC_F32);
      v = floats(load4(v_at, i, n, PGC_F32), PGC_F32);
    }
    f4 x = floats(xr, param_dtype), g = floats(gr, grad_dtype);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      g[k] = g[k] * factor;
      m[k] = m[k] * a.beta1 + g[k] * a.rest1;
      v[k] = v[k] * a.beta2 + g[k] * g[k] * a.rest2;
      x[k] = x[k] - (x[k] * r.decay + m[k] / (sqrtf(v[k]) * r.spread + a.eps) * r.rate);
    }
    store4(param, i, n, param_dtype, x);
    if (copy) store4(copy, i, n, copy_dtype, x);
    if constexpr (k8) {
      int mn[kEach], vn[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        mn[k] = k < n ? number_of(m[k]) : 0;
        vn[k] = k < n ? number_of(v[k]) : 0;
      }
      const int m_most = largest_of<kSigned>(mn), v_most = largest_of<kUnsigned>(vn);
      store_codes(m_at, i, n, encode<kSigned>(m, mn, m_most));
      store_codes(v_at, i, n, encode<kUnsigned>(v, vn, v_most));
      if (n > 0 && threadIdx.x % kWave == 0)
        *reinterpret_cast<float2*>(scales + 2 * state_block) = float2{scale_of(m_most), scale_of(v_most)};
    } else {
      store4(m_at, i, n, PGC_F32, m);
      store4(v_at, i, n, PGC_F32, v);
    }
  }
}

__global__ __launch_bounds__(kThreads)
void state_values_kernel(StateArgs a) {
  const int32_t block = static_cast<int32_t>(blockIdx.x), at = tensor_of(a.first, a.tensors, block);
  const int64_t count = a.count[at], from = static_cast<int64_t>(block - a.first[at]) * a.chunk, to = std::min<int64_t>(from + a.chunk, count);
  for (int64_t i = from + threadIdx.x * kEach; i < to; i += kThreads * kEach) {
    const int n = static_cast<int>(std::min<int64_t>(count - i, kEach));
    const float2 scale = *reinterpret_cast<const float2*>(a.scales[at] + 2 * (i / kStateBlock));
    store4(a.m_values[at], i, n, a.dtype[at], decode<kSigned>(load_codes(a.m[at], i, n), scale.x));
    store4(a.v_values[at], i, n, a.dtype[at], decode<kUnsigned>(load_codes(a.v[at], i, n), scale.y));
  }
}

// ---- the norm ---------------------------------------------------------------------------------

// The sum over a block's threads, in thread 0: lanes, then waves one after the other.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double sums[THREADS / kWave];
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d, kWave);
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = v;
  __syncthreads();
  double total = 0.0;
  for (int w = 0; w < THREADS / kWave; ++w) total += sums[w];
  return total;
}

// Squares in 64 bits, where none of 32 bits or fewer overflows or vanishes.
__global__ __launch_bounds__(kThreads)
void norm_sums_kernel(NormArgs a) {
  const int32_t block = static_cast<int32_t>(blockIdx.x), at = tensor_of(a.first, a.tensors, block);
  const int64_t count = a.count[at], from = static_cast<int64_t>(block - a.first[at]) * a.chunk, to = std::min<int64_t>(from + a.chunk, count);
  const void* data = a.data[at];
  const int dtype = a.dtype[at];
  double sum = 0.0;
  for (int64_t i = from + threadIdx.x * kEach; i < to; i += kThreads * kEach) {
    const int n = static_cast<int>(std::min<int64_t>(count - i, kEach));
    const f4 g = floats(load4(data, i, n, dtype), dtype);
#pragma unroll
    for (int k = 0; k < kEach; ++k) sum = __builtin_fma(static_cast<double>(g[k]), static_cast<double>(g[k]), sum);
  }
  sum = block_sum<kThreads>(sum);
  if (threadIdx.x == 0) a.sums[block] = sum;
}

constexpr int kEndThreads = 1024;
__global__ __launch_bounds__(kEndThreads)
void norm_end_kernel(NormEnd a) {
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < a.count; i += kEndThreads) sum += a.sums[i];
  sum = block_sum<kEndThreads>(sum);
  if (threadIdx.x != 0) return;
  const double norm = fabs(a.scale) * sqrt(sum);
  if (a.norm) *a.norm = static_cast<float>(norm);
  if (a.factor) {
    const double factor = norm > a.max_norm ? a.scale * (a.max_norm / norm) : a.scale;
    *a.factor = static_cast<float>(sum < INFINITY ? factor : NAN);
  }
}

}  // namespace

int32_t norm_chunk(int64_t values) { return values <= (int64_t{1} << 24) ? 4096 : 32768; }

hipError_t launch_norm_sums(const NormArgs& a, int64_t blocks, hipStream_t stream) {
  norm_sums_kernel<<<static_cast<uint32_t>(blocks), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_norm_end(const NormEnd& a, hipStream_t stream) {
  norm_end_kernel<<<1, kEndThreads, 0, stream>>>(a);
  return hipGetLastError();
}

int32_t adamw_chunk(int64_t values) { return values <= (int64_t{1} << 24) ? 4096 : 16384; }

hipError_t launch_adamw(const AdamwArgs& a, int64_t blocks, int state_bits, hipStream_t stream) {
  if (state_bits == 8) adamw_kernel<true><<<static_cast<uint32_t>(blocks), kThreads, 0, stream>>>(a);
  else adamw_kernel<false><<<static_cast<uint32_t>(blocks), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_state_values(const StateArgs& a, int64_t blocks, hipStream_t stream) {
  state_values_kernel<<<static_cast<uint32_t>(blocks), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace pgc
