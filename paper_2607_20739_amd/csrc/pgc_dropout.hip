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

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 20;
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

__device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

template <class T>
__global__ __launch_bounds__(kThreads)
void dropout_kernel(DropoutArgs a) {
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const uint64_t id = a.row_ids ? static_cast<uint64_t>(a.row_ids[i])
                                  : static_cast<uint64_t>(a.first_row) + static_cast<uint64_t>(i);
    const uint64_t key = mix64(a.seed + (id + 1) * kGamma);
    const T* x = static_cast<const T*>(a.x) + i * a.x_stride;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + i * a.residual_stride : nullptr;
    T* out = static_cast<T*>(a.out) + i * a.out_stride;
    for (int64_t word = threadIdx.x; 4 * word < a.cols; word += kThreads) {
      const uint64_t bits = mix64(key + (static_cast<uint64_t>(word) + 1) * kGamma);
      for (int k = 0; k < 4 && 4 * word + k < a.cols; ++k) {
        const uint32_t field = static_cast<uint32_t>(bits >> (16 * k)) & 0xFFFF;
        float v = field >= a.threshold ? static_cast<float>(x[4 * word + k]) * a.factor : 0.f;
        if (res) v += static_cast<float>(res[4 * word + k]);
        out[4 * word + k] = static_cast<T>(v);
      }
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t stream) {
  const int blocks = static_cast<int>(std::min(a.rows, kMaxBlocks));
  switch (dtype) {
    case PGC_F32: dropout_kernel<float><<<blocks, kThreads, 0, stream>>>(a); break;
    case PGC_BF16: dropout_kernel<__bf16><<<blocks, kThreads, 0, stream>>>(a); break;
    default: dropout_kernel<_Float16><<<blocks, kThreads, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace pgc
