// Dropout whose mask is a function of a seed, a row's number and a column
// (include/pgc_ops.h), for gfx950.
//
// One 64-bit output of the counter generator decides four neighbouring values, so a
// thread computes the two 64-bit products of SplitMix64's finaliser per four values and
// no mask is stored: the backward pass is the same kernel on the gradient.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_ops_kernels.h"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWave = 64;
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;
// Grids of up to 2^31 groups of rows.
constexpr int64_t kGridYZ = 65535;

typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef u4v u4v_unaligned __attribute__((aligned(2), may_alias));

__device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

__device__ __forceinline__ uint32_t field(uint64_t bits, int k) {
  return static_cast<uint32_t>(bits >> (16 * k)) & 0xFFFF;
}

// A group of LANES lanes takes LANES * U vectors of 16 bytes of a row, the runs of a longer row
// go to different blocks, and the values that fill no vector to one lane each.
template <class T, bool kResidual, int LANES, int U>
__global__ __launch_bounds__(kThreads)
void dropout_kernel(DropoutArgs a) {
  constexpr uint32_t kN = 16 / sizeof(T), kRows = kThreads / LANES;
  typedef T Packed __attribute__((ext_vector_type(kN)));
  typedef float Floats __attribute__((ext_vector_type(kN)));
  const uint32_t lane = threadIdx.x % LANES, cols = static_cast<uint32_t>(a.cols);
  const uint32_t full = cols / kN, rem = cols % kN, v0 = blockIdx.x * (LANES * U);
  int64_t row = static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y;
  if constexpr (kRows > 1) {
    uint32_t r = threadIdx.x / LANES;
    if constexpr (LANES >= kWave) r = __builtin_amdgcn_readfirstlane(r);
    row = row * kRows + r;
  }
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* res = kResidual ? static_cast<const T*>(a.residual) + row * a.residual_stride : nullptr;
  T* out = static_cast<T*>(a.out) + row * a.out_stride;

  u4v h[U] = {}, r[kResidual ? U : 1] = {};
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint64_t first = static_cast<uint64_t>(v0 + i * LANES) * 16;
    if (v0 + i * LANES + lane < full) {
      h[i] = __builtin_nontemporal_load(
          reinterpret_cast<const u4v_unaligned*>(reinterpret_cast<const char*>(x) + first + lane * 16));
      if (kResidual)
        r[i] = __builtin_nontemporal_load(
            reinterpret_cast<const u4v_unaligned*>(reinterpret_cast<const char*>(res) + first + lane * 16));
    }
  }
  const uint64_t id = a.row_ids ? static_cast<uint64_t>(a.row_ids[row])
                                : static_cast<uint64_t>(a.first_row) + static_cast<uint64_t>(row);
  const uint64_t key = mix64(a.seed + (id + 1) * kGamma);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t v = v0 + i * LANES + lane;
    if (v >= full) continue;
    auto f = __builtin_convertvector(__builtin_bit_cast(Packed, h[i]), Floats);
#pragma unroll
    for (uint32_t w = 0; w < kN / 4; ++w) {
      const uint64_t bits = mix64(key + (static_cast<uint64_t>(v) * (kN / 4) + w + 1) * kGamma);
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k)
        f[4 * w + k] = field(bits, k) >= a.threshold ? f[4 * w + k] * a.factor : 0.f;
    }
    if constexpr (kResidual) f += __builtin_convertvector(__builtin_bit_cast(Packed, r[i]), Floats);
    const u4v o = __builtin_bit_cast(u4v, __builtin_convertvector(f, Packed));
    __builtin_nontemporal_store(o, reinterpret_cast<u4v_unaligned*>(reinterpret_cast<char*>(out) +
                                       static_cast<uint64_t>(v0 + i * LANES) * 16 + lane * 16));
  }
  if (blockIdx.x == gridDim.x - 1 && lane < rem) {
    const uint32_t j = full * kN + lane;
    const uint64_t bits = mix64(key + (static_cast<uint64_t>(j / 4) + 1) * kGamma);
    float f = field(bits, j % 4) >= a.threshold ? static_cast<float>(x[j]) * a.factor : 0.f;
    if constexpr (kResidual) f += static_cast<float>(res[j]);
    out[j] = static_cast<T>(f);
  }
}

template <class T, bool kResidual, int LANES, int U>
hipError_t launch(const DropoutArgs& a, hipStream_t stream) {
  constexpr int64_t kRows = kThreads / LANES, kRun = int64_t{LANES} * U;
  const int64_t full = a.cols / (16 / static_cast<int64_t>(sizeof(T)));
  const int64_t groups = (a.rows + kRows - 1) / kRows, y = std::min(groups, kGridYZ);
  const dim3 grid(static_cast<uint32_t>(std::max<int64_t>(1, (full + kRun - 1) / kRun)), static_cast<uint32_t>(y),
                  static_cast<uint32_t>((groups + y - 1) / y));
  dropout_kernel<T, kResidual, LANES, U><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

// Lanes and vectors per lane by the row's whole vectors.
template <class T, bool kResidual>
hipError_t launch_by_row(const DropoutArgs& a, hipStream_t stream) {
  const int64_t full = a.cols / (16 / static_cast<int64_t>(sizeof(T)));
  if (full <= 8) return launch<T, kResidual, 8, 1>(a, stream);
  if (full <= 16) return launch<T, kResidual, 16, 1>(a, stream);
  if (full <= 32) return launch<T, kResidual, 32, 1>(a, stream);
  if (full <= 64) return launch<T, kResidual, 64, 1>(a, stream);
  if (full <= 128) return launch<T, kResidual, 64, 2>(a, stream);
  if (full <= 256) return launch<T, kResidual, 64, 4>(a, stream);
  return launch<T, kResidual, 256, 4>(a, stream);
}

template <class T>
hipError_t launch_typed(const DropoutArgs& a, hipStream_t stream) {
  return a.residual ? launch_by_row<T, true>(a, stream) : launch_by_row<T, false>(a, stream);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PGC_F32: return launch_typed<float>(a, stream);
    case PGC_BF16: return launch_typed<__bf16>(a, stream);
    default: return launch_typed<_Float16>(a, stream);
  }
}

}  // namespace pgc
