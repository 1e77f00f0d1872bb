// Rows of logits as waves read them: vectors of 16 bytes at any alignment, lanes and waves to a row, and the
// reductions over them.  Shared by the kernels of token log-probabilities and losses and of scores.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "pgc_lanes.h"

// A product and a sum are rounded apart unless a fused operation is written: otherwise the compiler
// fuses them in some copies of the same code and not in others, and bits would depend on where a
// row lies.
#pragma clang fp contract(off)

namespace pgc {
namespace {

constexpr int kWave = 64, kBlock = 256;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef uint32_t u4v __attribute__((ext_vector_type(4)));
// As they lie in memory: beside single values there, at any alignment.
typedef u4v u4v_unaligned __attribute__((aligned(2), may_alias));
typedef uint16_t u16_raw __attribute__((may_alias));
typedef uint32_t u32_raw __attribute__((may_alias));

// 16 bytes of a row and the values in them.
template <class T>
struct Vec {
  static constexpr int kN = 16 / sizeof(T);
  typedef T Packed __attribute__((ext_vector_type(kN)));
  typedef float Floats __attribute__((ext_vector_type(kN)));

  // Vector `first + lane` of a row; `first` is the same for all lanes, so the address is a
  // scalar and a lane's 32-bit offset.
  template <bool kAgain = false>   // whether its line is read again soon
  static __device__ __forceinline__ u4v load(const T* row, uint32_t first, uint32_t lane) {
    const auto* p = reinterpret_cast<const u4v_unaligned*>(at(row, first, lane));
    if constexpr (kAgain) return *p;
    return __builtin_nontemporal_load(p);
  }
  template <bool kCached = false>
  static __device__ __forceinline__ void store(T* row, uint32_t first, uint32_t lane, u4v v) {
    auto* p = reinterpret_cast<u4v_unaligned*>(const_cast<char*>(at(row, first, lane)));
    if constexpr (kCached) *p = v;
    else __builtin_nontemporal_store(v, p);
  }
  static __device__ __forceinline__ const char* at(const T* row, uint32_t first, uint32_t lane) {
    return reinterpret_cast<const char*>(row) + static_cast<uint64_t>(first) * 16 + lane * 16;
  }
  static __device__ __forceinline__ Floats floats(u4v v) {
    return __builtin_convertvector(__builtin_bit_cast(Packed, v), Floats);
  }
  static __device__ __forceinline__ u4v packed(Floats f) {
    return __builtin_bit_cast(u4v, __builtin_convertvector(f, Packed));
  }
  // One value as it lies in memory, and as a number: apart, so that nothing waits for the load.
  static __device__ __forceinline__ uint32_t raw(const T* p) {
    if constexpr (sizeof(T) == 4) return *reinterpret_cast<const u32_raw*>(p);
    else return *reinterpret_cast<const u16_raw*>(p);
  }
  static __device__ __forceinline__ float value(uint32_t raw) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw);
    else return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(raw)));
  }
  static constexpr uint32_t kRawNone = sizeof(T) == 4 ? 0xFF800000u : std::is_same_v<T, __bf16> ? 0xFF80u : 0xFC00u;
  // A vector of -inf: counts for nothing in a maximum or a sum.
  static __device__ __forceinline__ u4v none() {
    constexpr uint32_t bits = sizeof(T) == 4 ? kRawNone : kRawNone * 0x10001u;
    return u4v{bits, bits, bits, bits};
  }
};

// 2^x by the hardware's instruction; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A maximum of -inf (nothing seen yet, or nothing but -inf) counts as 0 in differences, which keeps -inf - -inf
// out of them.
__device__ __forceinline__ float finite_top(float top) { return top == -INFINITY ? 0.f : top; }

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

// Groups of LANES lanes, kRows of them to a block, and their rows.
template <int LANES>
struct Place {
  static constexpr int kThreads = LANES <= kWave ? kBlock : LANES;   // rows that share a block share no barrier
  static constexpr int kRows = kThreads / LANES;
  __device__ static uint32_t lane() { return threadIdx.x % LANES; }
  __device__ static int64_t row(int64_t block) {
    if constexpr (LANES >= kThreads) return block;
    uint32_t r = threadIdx.x / LANES;
    if constexpr (LANES >= kWave) r = __builtin_amdgcn_readfirstlane(r);
    return block * kRows + r;
  }
  static int64_t blocks(int64_t rows) { return (rows + kRows - 1) / kRows; }
};

// Grids of up to 2^31 blocks (of one dimension, HIP takes fewer threads than that needs).
constexpr int64_t kGridX = 1 << 20, kGridYZ = 65535;

// A short row as one of LANES lanes sees it: its vectors are lane, lane + LANES, ..., HOLD of them.
// The row's last vector ends with the row and may overlap the one before it (both have the same
// gradient; in the sums only one counts the values that both hold).
template <class T, int LANES, int HOLD>
struct ShortVectors {
  static constexpr uint32_t kN = Vec<T>::kN;
  uint32_t lane, cols, vectors, overlap;

  __device__ __forceinline__ explicit ShortVectors(uint32_t cols_)
      : lane(Place<LANES>::lane()), cols(cols_), vectors((cols_ + kN - 1) / kN), overlap(vectors * kN - cols_) {}
  __device__ __forceinline__ uint32_t number(int i) const { return i * LANES + lane; }
  // First column of vector v, and how many of its values others have.
  __device__ __forceinline__ uint32_t start(uint32_t v) const { return v + 1 < vectors ? v * kN : cols - kN; }
  __device__ __forceinline__ uint32_t skipped(uint32_t v) const { return v + 1 < vectors ? 0 : v < vectors ? overlap : kN; }

  __device__ __forceinline__ void load(const T* z, u4v (&h)[HOLD]) const {
    if (cols >= kN) {
#pragma unroll
      for (int i = 0; i < HOLD; ++i) h[i] = Vec<T>::template load<true>(z + start(number(i)), 0, 0);
    } else {                // fewer values than a vector: at its end
      T v[kN];
      for (uint32_t k = 0; k < kN; ++k) v[k] = z[k < overlap ? 0 : k - overlap];
      __builtin_memcpy(&h[0], v, sizeof(v));
    }
  }
};

// The whole vectors of a long row.  The values left over, 1 to kN of them, go to a lane each, so that
// the vectors of a shifted row, too, end within it.
template <class T>
__device__ __forceinline__ uint32_t long_row_vectors(uint32_t cols) { return (cols - 1) / Vec<T>::kN; }

// A long row as a wave sees it: a run of neighbouring vectors, `whole` times 64 and `part` more.
//
// Loads are issued by all lanes at all times (past the run's end the last vector stands in), so
// that the number in flight is known where one is waited for, and the sum starts when the first
// vectors have come.
//
// Values of 16 bits may start at an address that is no multiple of 4, where a load of 16 bytes
// takes longer (rows of 131,071 bf16 logits: 412 us where aligned ones take 320).  The run is then
// loaded from the second value on, and `values` puts the vectors together that the row has when
// counted from its first value, from two lanes' loads each.
template <class T>
struct VectorRun {
  static constexpr uint32_t kN = Vec<T>::kN;
  uint32_t lane, begin, whole, part;
  uint32_t last;                // the last vector, counted from the one that z points to
  uint32_t odd;                 // 1 where shifted
  const T* z;                   // the run's first vector as it is loaded; of an empty run the row's last

  // Up to `most` vectors from number `first` on of the row's `full` ones (at least one).
  __device__ __forceinline__ VectorRun(const T* row, uint32_t full, uint32_t first, uint32_t most) {
    lane = threadIdx.x % kWave;
    begin = first < full ? first : full - 1;
    const uint32_t count = first < full ? (full - begin < most ? full - begin : most) : 0;
    whole = count / kWave;
    part = count % kWave;
    last = count > 0 ? count - 1 : 0;
    odd = sizeof(T) == 2 ? static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row) >> 1) & 1 : 0;
    z = row + odd + static_cast<uint64_t>(begin) * kN;
  }
  __device__ __forceinline__ bool any(uint32_t i) const { return i < whole || (i == whole && part > 0); }
  __device__ __forceinline__ uint32_t vector(uint32_t i) const {
    const uint32_t v = i * kWave + lane;
    return v < last ? v : last;
  }
  template <bool kAgain = false>
  __device__ __forceinline__ u4v load(uint32_t i) const { return Vec<T>::template load<kAgain>(z, 0, vector(i)); }
  // From memory to LDS without a wait, lane by lane.
  __device__ __forceinline__ void load_to_lds(uint32_t i, u4v* to) const {
    const char* from = Vec<T>::at(z, 0, vector(i));
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)from,
                                     (__attribute__((address_space(3))) uint32_t*)to, 16, 0, 0);
  }
  // The value before the run's first loaded one, raw, in lane 0 of a shifted row; 16 bits higher it
  // is the carry that `values` starts from.
  __device__ __forceinline__ uint32_t before() const { return sizeof(T) == 2 ? Vec<T>::raw(z - (lane == 0 ? odd : 0)) : 0; }

  // The row's vector, counted from its first value, out of what was loaded.
  __device__ __forceinline__ u4v values(u4v h, uint32_t& carry) const {
    if (sizeof(T) == 4 || !odd) return h;
    // Lane 0 takes `carry`, the others the lane below's last value (DPP wave shift by one).
    const uint32_t below = __builtin_amdgcn_update_dpp(static_cast<int>(carry), static_cast<int>(h[3]), 0x138, 0xF, 0xF, false);
    carry = __builtin_amdgcn_readlane(static_cast<int>(h[3]), kWave - 1);
    return u4v{__builtin_amdgcn_alignbit(h[0], below, 16), __builtin_amdgcn_alignbit(h[1], h[0], 16),
               __builtin_amdgcn_alignbit(h[2], h[1], 16), __builtin_amdgcn_alignbit(h[3], h[2], 16)};
  }
};

}  // namespace
}  // namespace pgc
