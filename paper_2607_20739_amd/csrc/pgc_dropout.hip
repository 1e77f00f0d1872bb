// Dropout whose mask is a function of a seed, a row's number and a column
// (include/pgc_ops.h), for gfx950.
//
// One 64-bit output of the counter generator decides four neighbouring values: two 64-bit
// products, about 40 instruction slots, 10 per value, against some 30 that the memory's rate leaves.
// So no mask is stored, and the backward pass is the same kernel on the gradient.  Memory bounds
// it, given several 16-byte loads in flight per lane.
//
// Measured (MI355X): 65,536 x 8,192 bf16 364 us, 5.9 TB/s; 32,768 x 8,192 fp32 337 us, 6.4 TB/s;
// 1,048,576 x 200 bf16 142 us, 5.9 TB/s, of 100 columns 91 us, 4.6 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_ops_kernels.h"

// A product and a sum are rounded apart wherever in a row a value lies.
#pragma clang fp contract(off)

namespace pgc {
namespace {

constexpr int kThreads = 256;
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;
// Grids of up to 2^31 blocks (of one dimension, HIP takes fewer threads than that needs).
constexpr int64_t kGridX = 1 << 20, kGridYZ = 65535;

typedef uint32_t u4v __attribute__((ext_vector_type(4)));
// As they lie in memory: beside single values there, at any alignment.
typedef u4v u4v_unaligned __attribute__((aligned(2), may_alias));
typedef uint32_t u2v_unaligned __attribute__((ext_vector_type(2), aligned(2), may_alias));
typedef uint32_t u1v_unaligned __attribute__((aligned(2), may_alias));
typedef uint16_t u16_raw __attribute__((may_alias));

__device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

__device__ __forceinline__ uint32_t field(uint64_t bits, int k) {
  return static_cast<uint32_t>(bits >> (16 * k)) & 0xFFFF;
}

__device__ __forceinline__ uint64_t row_key(const DropoutArgs& a, int64_t row) {
  const uint64_t id = a.row_ids ? static_cast<uint64_t>(a.row_ids[row])
                                : static_cast<uint64_t>(a.first_row) + static_cast<uint64_t>(row);
  return mix64(a.seed + (id + 1) * kGamma);
}

__device__ __forceinline__ uint64_t draw(uint64_t key, uint32_t word) {
  return mix64(key + (static_cast<uint64_t>(word) + 1) * kGamma);
}

// 16 bytes of a row.
template <class T>
struct Vec {
  static constexpr uint32_t kN = 16 / sizeof(T);
  typedef T Packed __attribute__((ext_vector_type(kN)));
  typedef float Floats __attribute__((ext_vector_type(kN)));

  // Value `column` of a row, plus 16 bytes for each further lane: a scalar address and a lane's offset.
  static __device__ __forceinline__ const char* at(const T* row, uint32_t column, uint32_t lane) {
    return reinterpret_cast<const char*>(row + column) + lane * 16;
  }
  static __device__ __forceinline__ u4v load(const T* row, uint32_t column, uint32_t lane) {
    return __builtin_nontemporal_load(reinterpret_cast<const u4v_unaligned*>(at(row, column, lane)));
  }
  static __device__ __forceinline__ void store(T* row, uint32_t column, uint32_t lane, u4v v) {
    __builtin_nontemporal_store(v, reinterpret_cast<u4v_unaligned*>(const_cast<char*>(at(row, column, lane))));
  }
  // The vector whose first value is column `word` * 4 + `shift` of the row with this key.
  template <bool kResidual>
  static __device__ __forceinline__ u4v dropped(const DropoutArgs& a, uint64_t key, uint32_t word, uint32_t shift, u4v x, u4v residual) {
    auto f = __builtin_convertvector(__builtin_bit_cast(Packed, x), Floats);
    uint64_t bits[kN / 4];
#pragma unroll
    for (uint32_t w = 0; w < kN / 4; ++w) bits[w] = draw(key, word + w);
    if (shift > 0) {   // the fields that many further on
      const uint64_t next = draw(key, word + kN / 4);
      if (kN == 8) bits[0] = bits[0] >> 16 * shift | bits[kN / 4 - 1] << (64 - 16 * shift);
      bits[kN / 4 - 1] = bits[kN / 4 - 1] >> 16 * shift | next << (64 - 16 * shift);
    }
#pragma unroll
    for (uint32_t k = 0; k < kN; ++k) f[k] = field(bits[k / 4], k % 4) >= a.threshold ? f[k] * a.factor : 0.f;
    if constexpr (kResidual) f += __builtin_convertvector(__builtin_bit_cast(Packed, residual), Floats);
    return __builtin_bit_cast(u4v, __builtin_convertvector(f, Packed));
  }
};

// The 16 bytes moved down by `bytes` (the same in all lanes, below 16).
__device__ __forceinline__ u4v moved_down(u4v v, uint32_t bytes) {
  uint64_t lo = static_cast<uint64_t>(v[1]) << 32 | v[0], hi = static_cast<uint64_t>(v[3]) << 32 | v[2];
  if (bytes >= 8) {
    lo = hi;
    hi = 0;
  }
  const uint32_t shift = bytes % 8 * 8;
  if (shift > 0) {
    lo = lo >> shift | hi << (64 - shift);
    hi >>= shift;
  }
  return u4v{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
}

// The first `bytes` (the same in all lanes, below 16) to `p`.
__device__ __forceinline__ void store_first(char* p, u4v v, uint32_t bytes) {
  if (bytes & 8) {
    *reinterpret_cast<u2v_unaligned*>(p) = u2v_unaligned{v[0], v[1]};
    p += 8;
    v = moved_down(v, 8);
  }
  if (bytes & 4) {
    *reinterpret_cast<u1v_unaligned*>(p) = v[0];
    p += 4;
    v = moved_down(v, 4);
  }
  if (bytes & 2) *reinterpret_cast<u16_raw*>(p) = static_cast<uint16_t>(v[0]);
}

// One value by itself.
template <class T, bool kResidual>
__device__ __forceinline__ void drop_value(const DropoutArgs& a, uint64_t key, const T* x, const T* res, T* out, uint32_t column) {
  float f = field(draw(key, column / 4), column % 4) >= a.threshold ? static_cast<float>(x[column]) * a.factor : 0.f;
  asm("" : "+v"(f));   // rounded to 32 bits first, as in a vector: fp16's product and conversion would be fused
  if constexpr (kResidual) f += static_cast<float>(res[column]);
  out[column] = static_cast<T>(f);
}

// Rows of at most kShortVectors vectors: a block takes the vectors of several rows one after the
// other, so that no lane is without one and neighbouring lanes have neighbouring memory.  The rows'
// keys are drawn once, into LDS.  A row's last vector, where it is not whole, is loaded from the row's
// last 16 bytes, moved into place, and stored in up to three pieces.
constexpr uint32_t kShortVectors = 512;
template <class T, bool kResidual, int U>
__global__ __launch_bounds__(kThreads)
void short_dropout_kernel(DropoutArgs a, uint32_t rows_per_block) {
  constexpr uint32_t kN = Vec<T>::kN;
  __shared__ uint64_t keys[kThreads];
  const uint32_t cols = static_cast<uint32_t>(a.cols), vectors = (cols + kN - 1) / kN, rem = cols % kN;
  const int64_t first = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * rows_per_block;
  if (first >= a.rows) return;
  const uint32_t rows = a.rows - first < rows_per_block ? static_cast<uint32_t>(a.rows - first) : rows_per_block;
  const T* x = static_cast<const T*>(a.x) + first * a.x_stride;
  const T* res = kResidual ? static_cast<const T*>(a.residual) + first * a.residual_stride : nullptr;
  T* out = static_cast<T*>(a.out) + first * a.out_stride;
  if (cols < kN) {   // no vectors
    if (threadIdx.x < rows) keys[threadIdx.x] = row_key(a, first + threadIdx.x);
    __syncthreads();
    for (uint32_t n = threadIdx.x; n < rows * cols; n += kThreads) {
      const uint32_t t = n / cols;
      drop_value<T, kResidual>(a, keys[t], x + t * a.x_stride, res + t * a.residual_stride, out + t * a.out_stride, n - t * cols);
    }
    return;
  }
  const uint32_t inverse = (1u << 20) / vectors + 1;   // n / vectors = n * inverse >> 20 for n up to 1,024, vectors up to 513
  u4v h[U] = {}, r[kResidual ? U : 1] = {};
  uint32_t row[U], v[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t n = i * kThreads + threadIdx.x;
    row[i] = n * inverse >> 20;
    v[i] = n - row[i] * vectors;
    const uint32_t column = v[i] + 1 < vectors ? v[i] * kN : cols - kN;
    if (row[i] < rows) {
      h[i] = Vec<T>::load(x + row[i] * a.x_stride, column, 0);
      if (kResidual) r[i] = Vec<T>::load(res + row[i] * a.residual_stride, column, 0);
    }
  }
  if (threadIdx.x < rows) keys[threadIdx.x] = row_key(a, first + threadIdx.x);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (row[i] >= rows) continue;
    const bool part = rem > 0 && v[i] + 1 == vectors;
    if (part) {
      h[i] = moved_down(h[i], (kN - rem) * sizeof(T));
      if (kResidual) r[kResidual ? i : 0] = moved_down(r[kResidual ? i : 0], (kN - rem) * sizeof(T));
    }
    const u4v o = Vec<T>::template dropped<kResidual>(a, keys[row[i]], v[i] * (kN / 4), 0, h[i], r[kResidual ? i : 0]);
    T* to = out + row[i] * a.out_stride;
    if (part) store_first(reinterpret_cast<char*>(to + v[i] * kN), o, rem * sizeof(T));
    else Vec<T>::store(to, v[i] * kN, 0, o);
  }
}

// Longer rows: a block takes kThreads * U vectors of a row, which start at the row's first cache
// line, and the values that fill no vector, one per lane: the first block those before, the last one
// those after.  The fields of vectors that start at no multiple of 4 columns come from three draws,
// not two.  65,536 x 8,191 bf16 368 us, 390 with the vectors at the row's first multiple of 4 bytes
// (8,192 columns: 361); 32,768 x 16,385 346 and 375.
constexpr uint32_t kLine = 128;
template <class T, bool kResidual, int U>
__global__ __launch_bounds__(kThreads)
void dropout_kernel(DropoutArgs a) {
  constexpr uint32_t kN = Vec<T>::kN;
  const int64_t row = static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y;
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* res = kResidual ? static_cast<const T*>(a.residual) + row * a.residual_stride : nullptr;
  T* out = static_cast<T*>(a.out) + row * a.out_stride;
  const uint32_t head = static_cast<uint32_t>(-reinterpret_cast<uintptr_t>(x) % kLine / sizeof(T));
  const uint32_t lane = threadIdx.x, cols = static_cast<uint32_t>(a.cols);
  const uint32_t full = (cols - head) / kN, rem = cols - head - full * kN, v0 = blockIdx.x * (kThreads * U);
  u4v h[U] = {}, r[kResidual ? U : 1] = {};
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t column = (v0 + i * kThreads) * kN + head;
    if (v0 + i * kThreads + lane < full) {
      h[i] = Vec<T>::load(x, column, lane);
      if (kResidual) r[i] = Vec<T>::load(res, column, lane);
    }
  }
  const uint64_t key = row_key(a, row);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const uint32_t v = v0 + i * kThreads + lane;
    if (v < full)
      Vec<T>::store(out, (v0 + i * kThreads) * kN + head, lane,
                    Vec<T>::template dropped<kResidual>(a, key, v * (kN / 4) + head / 4, head % 4, h[i], r[kResidual ? i : 0]));
  }
  if (blockIdx.x == gridDim.x - 1 && lane < rem) drop_value<T, kResidual>(a, key, x, res, out, cols - rem + lane);
  if (blockIdx.x == 0 && lane < head) drop_value<T, kResidual>(a, key, x, res, out, lane);
}

template <class T, bool kResidual>
hipError_t launch_short(const DropoutArgs& a, hipStream_t stream) {
  constexpr int kU = 4;
  const int64_t vectors = (a.cols + Vec<T>::kN - 1) / Vec<T>::kN;
  const int64_t per = std::min<int64_t>(kThreads, kThreads * kU / vectors);
  const int64_t blocks = (a.rows + per - 1) / per, x = std::min(blocks, kGridX);
  const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>((blocks + x - 1) / x));
  short_dropout_kernel<T, kResidual, kU><<<grid, kThreads, 0, stream>>>(a, static_cast<uint32_t>(per));
  return hipGetLastError();
}

template <class T, bool kResidual, int U>
hipError_t launch_long(const DropoutArgs& a, hipStream_t stream) {
  constexpr int64_t kRun = int64_t{kThreads} * U;
  const int64_t full = a.cols / Vec<T>::kN;
  const int64_t y = std::min(a.rows, kGridYZ);
  const dim3 grid(static_cast<uint32_t>(std::max<int64_t>(1, (full + kRun - 1) / kRun)), static_cast<uint32_t>(y),
                  static_cast<uint32_t>((a.rows + y - 1) / y));
  dropout_kernel<T, kResidual, U><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

// Kernel by the row's whole vectors.  Packing pays up to 512 vectors (131,072 x 1,400 bf16 128 us, a wave
// per row 167; 65,536 x 4,000 177 and 204).  Longer fp32 rows do best with one
// load in flight per lane (32,768 x 4,400: 182 us, four 258), 16-bit ones with four (65,536 x
// 8,192: 364 us, one 459).
template <class T, bool kResidual>
hipError_t launch_by_row(const DropoutArgs& a, hipStream_t stream) {
  const int64_t full = a.cols / Vec<T>::kN;
  if (full <= kShortVectors) return launch_short<T, kResidual>(a, stream);
  if constexpr (sizeof(T) == 4) return launch_long<T, kResidual, 1>(a, stream);
  else return launch_long<T, kResidual, 4>(a, stream);
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
