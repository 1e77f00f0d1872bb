// Token log-probabilities, their gradient and that of the scores, the policy loss and the preference
// loss (include/pgc_ops.h), for gfx950.
//
// All of it is one exponential and a handful of additions per logit, so memory bounds it: a row
// should come in once and its gradient leave once, with enough loads in flight throughout.  Sums of
// exponentials run beside the maximum (a running pair per lane, joined over lanes and waves
// once), so one pass suffices for the log-probability; the policy loss keeps the row on the chip
// from there to the gradient.  The preference loss needs whole sequences before its first
// gradient, so its rows are read twice.
//
// Rows of up to 128 vectors of 16 bytes belong to 1 to 32 lanes of a wave, longer ones to 1 to 16
// waves.  Which lane sums what, and hence every bit of the result, depends on the number of
// columns alone, not on where the row lies nor on the rows beside it.
//
// Measured (MI355X; GB of logits read and gradients written per second): forward of 16,384 rows of
// 131,072 bf16 602 us, 7.1 TB/s; policy loss of 4,096 rows of 65,536 fp16 176 us, 5.8 TB/s; of 8,192
// rows of 131,071 bf16 810 us, 5.3; gradient of 8,192 rows of 131,072 bf16 704 us, 6.1.  A copy of a
// gigabyte by the runtime moves 5.0, a read alone 7.2.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pgc_ops_kernels.h"
#include "pgc_rows.h"

// A product and a sum are rounded apart unless a fused operation is written: otherwise the compiler
// fuses them in some copies of the same code and not in others, and bits would depend on where a
// row lies.
#pragma clang fp contract(off)

namespace pgc {
namespace {

// A maximum and the sum of exp(z - maximum) of some of a row's values.  A maximum of -inf
// (nothing seen yet, or nothing but -inf) counts as 0 in differences, which keeps -inf - -inf
// out of them.  NaN never becomes the maximum, but the sum.
struct Stat {
  float top, sum;
};

// U vectors at once: one rescaling of the sum so far, and the lanes' additions in a tree.
template <class T, int U>
__device__ __forceinline__ void add_vectors(Stat& s, const u4v (&h)[U]) {
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

// The same of one vector that is unpacked already.
template <uint32_t N, class Floats>
__device__ __forceinline__ void add_floats(Stat& s, Floats f) {
  float top = s.top;
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) top = fmaxf(top, f[k]);
  const float base = finite_top(top);
  float sum = s.sum * exp2_fast((s.top - base) * kLog2E);
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) f[k] = exp2_fast((f[k] - base) * kLog2E);
#pragma unroll
  for (uint32_t w = N / 2; w >= 1; w /= 2)
#pragma unroll
    for (uint32_t k = 0; k < w; ++k) f[k] += f[k + w];
  s = {top, sum + f[0]};
}

__device__ __forceinline__ void add_value(Stat& s, float v) {
  const float top = fmaxf(s.top, v), base = finite_top(top);
  s = {top, s.sum * exp2_fast((s.top - base) * kLog2E) + exp2_fast((v - base) * kLog2E)};
}

// Joined over LANES lanes of a wave; every lane ends with the result.
template <int LANES>
__device__ __forceinline__ Stat join_lanes(Stat s) {
  const float top = lane_group_max<LANES>(s.top);
  return {top, lane_group_sum<LANES>(s.sum * exp2_fast((s.top - finite_top(top)) * kLog2E))};
}

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
    l += a.kl * (d == INFINITY ? d : e - d);   // a token that cannot occur: the limit, not inf - inf
    slope -= a.kl * e;
  }
  *loss = l;
  return slope * a.scale * r.weight;
}

// A row's gradient g (onehot(y) - exp(z - top) / sum), value by value.  The exponential is taken 8
// times larger, which costs near the maximum no more than its own rounding, so that for |g| up
// to 8 nothing is lost that 32 bits hold.
template <class T>
struct RowGradient {
  float g, scaled, top;
  bool none;   // zeros: no gradient comes in, or nothing can occur

  __device__ __forceinline__ RowGradient(float g_, float top_, float inverse_sum, bool empty)
      : g(g_), scaled(-g_ * inverse_sum * 0.125f), top(top_), none(g_ == 0.f || empty) {}
  // From the maximum and the log of the sum.
  static __device__ __forceinline__ RowGradient of_stats(float g, float top, float log_sum) {
    return RowGradient(g, top, expf(-log_sum), top == -INFINITY && log_sum == 0.f);
  }

  __device__ __forceinline__ float of(float z, bool target) const {
    const float v = scaled * exp2_fast(__builtin_fmaf(z - top, kLog2E, 3.f));
    return target ? v + g : v;
  }
  // Gradient of a vector, as if the target were in none.
  __device__ __forceinline__ u4v of_vector(u4v z) const {
    constexpr uint32_t kN = Vec<T>::kN;
    if (none) return u4v{0, 0, 0, 0};
    auto f = Vec<T>::floats(z);
#pragma unroll
    for (uint32_t k = 0; k < kN; ++k) f[k] = of(f[k], false);
    return Vec<T>::packed(f);
  }
};

// The gradient of the scores: g (onehot(y) - p) - e p (ln p + H), from the row's stats and entropy H.  With d = z - top the
// factor of p is a + b d, b = -e and a = -g - e (H - ln sum).
// p is taken 2^8 times larger and the factor as much smaller, so that factors of up to 2^8 lose nothing that 32 bits hold.
template <class T>
struct ScoresGradient {
  float g, a, b, top, log2_inverse;
  bool none;   // zeros, as above

  __device__ __forceinline__ ScoresGradient(float g_, float e, float top_, float log_sum, float entropy)
      : g(g_), a((e == 0.f ? -g_ : -g_ - e * (entropy - log_sum)) * 0x1p-8f), b(-e * 0x1p-8f), top(top_), log2_inverse(8.f - log_sum * kLog2E),
        none((g_ == 0.f && e == 0.f) || (top_ == -INFINITY && log_sum == 0.f)) {}

  __device__ __forceinline__ float of(float z, bool target) const {
    const float d = z - top, p = exp2_fast(__builtin_fmaf(d, kLog2E, log2_inverse));
    const float v = p * __builtin_fmaf(b, fmaxf(d, -200.f), a);   // at -inf, where p is 0, the factor has to be finite
    return target ? v + g : v;
  }
  __device__ __forceinline__ u4v of_vector(u4v z) const {
    constexpr uint32_t kN = Vec<T>::kN;
    if (none) return u4v{0, 0, 0, 0};
    auto f = Vec<T>::floats(z);
#pragma unroll
    for (uint32_t k = 0; k < kN; ++k) f[k] = of(f[k], false);
    return Vec<T>::packed(f);
  }
};

// The row's log-probability from its joined maximum and sum.
__device__ __forceinline__ float row_logprob(Stat s, float target_logit, float* log_sum) {
  if (s.top == -INFINITY && s.sum == 0.f) return -INFINITY;
  *log_sum = kLn2 * log2f(s.sum);
  return (target_logit - s.top) - *log_sum;
}

__device__ __forceinline__ void write_forward(const LogitsArgs& a, int64_t row, float lp, float top, float log_sum) {
  a.logprobs[row] = lp;
  if (a.stats) {
    a.stats[2 * row] = log_sum != log_sum ? log_sum : top;   // fmaxf leaves NaN out
    a.stats[2 * row + 1] = log_sum;
  }
  if (a.zero_grad) a.zero_grad[row] = 0.f;
}

// A pair's sum runs in a fixed order, whoever adds it up: by chunks of kChunk rows from the pair's first on.
// In a chunk kPairWaves waves' lanes take four neighbouring rows each, then the lanes of a wave are
// added up, then the waves one after the other.  Chunk c belongs to lane c % 64; each lane adds up its
// own, then the lanes.
constexpr int kPairThreads = 1024, kPairWaves = kPairThreads / kWave, kChunk = 4 * kPairThreads;

// A pair's rows: sequence 2 i is [at[0], at[1]), sequence 2 i + 1 [at[1], at[2]).
struct PairRows {
  int64_t at[3];

  __device__ __forceinline__ PairRows(const PairArgs& a, int64_t pair) {
    for (int k = 0; k < 3; ++k) at[k] = bounded(a, a.offsets[2 * pair + k]);
  }
  static __device__ __forceinline__ int64_t bounded(const PairArgs& a, int64_t offset) {
    return std::min<int64_t>(std::max<int64_t>(offset, 0), a.rows);
  }
  __device__ __forceinline__ int64_t chunks() const { return (at[2] - at[0] + kChunk - 1) / kChunk; }
};

// From the pair's sum of l - ref, preferred rows less the others, in 64 bits: the gradient of the
// preferred rows' log-probabilities (the others' is the negative), and the loss and the margin.
__device__ __forceinline__ float pair_slope(const PairArgs& a, int64_t pair, double sum) {
  const double h = sum * a.beta, e = exp(-fabs(h)), large = 1.0 / (1.0 + e), small = e / (1.0 + e);   // sigma(|h|), sigma(-|h|)
  const double weight = a.weights ? a.weights[pair] : 1.f;
  const double up = h >= 0 ? large : small, down = h >= 0 ? small : large;
  const double slope = h != h ? h : a.smoothing * up - (1.0 - a.smoothing) * down;
  return weight == 0.0 ? 0.f : static_cast<float>(slope * a.beta * a.scale * weight);
}
__device__ __forceinline__ void write_pair(const PairArgs& a, int64_t pair, double sum) {
  const double h = sum * a.beta, rest = log1p(exp(-fabs(h)));
  const double minus = rest + fmax(-h, 0.0), plus = rest + fmax(h, 0.0);   // -ln sigma(h), -ln sigma(-h)
  a.margins[pair] = static_cast<float>(h);
  // A term of weight 0 is left out: an infinite margin makes one of them infinite.
  const double loss = (a.smoothing == 1.0 ? 0.0 : (1.0 - a.smoothing) * minus) + (a.smoothing == 0.0 ? 0.0 : a.smoothing * plus);
  a.loss[pair] = static_cast<float>(h != h ? h : loss);
}

typedef float f4_unaligned __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i4_unaligned __attribute__((ext_vector_type(4), aligned(4)));

// Four rows' part of the sum, from row t of the pair's on.
struct FourRows {
  i4_unaligned y;
  f4_unaligned lp, ref;

  __device__ __forceinline__ void load(const PairArgs& a, const PairRows& rows, int64_t t) {
    y = i4_unaligned{-1, -1, -1, -1};
    lp = ref = f4_unaligned{0.f, 0.f, 0.f, 0.f};
    if (t + 4 <= rows.at[2]) {
      y = *reinterpret_cast<const i4_unaligned*>(a.targets + t);
      lp = *reinterpret_cast<const f4_unaligned*>(a.logprobs + t);
      if (a.ref_logprobs) ref = *reinterpret_cast<const f4_unaligned*>(a.ref_logprobs + t);
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (t + k >= rows.at[2]) break;
        y[k] = a.targets[t + k];
        lp[k] = a.logprobs[t + k];
        if (a.ref_logprobs) ref[k] = a.ref_logprobs[t + k];
      }
    }
  }
  __device__ __forceinline__ double sum(const PairArgs& a, const PairRows& rows, int64_t t) const {
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (y[k] < 0 || y[k] >= a.cols) continue;
      const double v = static_cast<double>(lp[k]) - ref[k];
      sum += t + k < rows.at[1] ? v : -v;
    }
    return sum;
  }
};

__device__ __forceinline__ double add_lanes(double sum) {
  for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d, kWave);
  return sum;
}

// By a block of kPairThreads, all of which get the slope.  One wave takes the 64-bit functions (all 16 take
// 1 us longer), and the last writes the loss and the margin while the others go on.  `part` gives a
// thread's part of a chunk, from the row that it is given on.
constexpr int kChunksAtOnce = 16;
struct PairSums {
  double sums[kChunksAtOnce][kPairWaves];
  float slope;
};
template <class Part>
__device__ __forceinline__ float block_pair_slope(const PairArgs& a, int64_t pair, const PairRows& rows, PairSums& shared, Part part) {
  const int64_t chunks = rows.chunks();
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const bool first = wave == 0, last = wave == kPairWaves - 1;
  double sum = 0.0;
  auto wave_sum = [&](int64_t c) { return add_lanes(part(rows.at[0] + c * kChunk + 4 * threadIdx.x)); };
  auto chunk_sum = [&](int c) {
    double total = 0.0;
    for (int w = 0; w < kPairWaves; ++w) total += shared.sums[c][w];
    return total;
  };
  if (chunks == 1) {   // the same without the lanes' last sum
    const double v = wave_sum(0);
    if (lane == 0) shared.sums[0][wave] = v;
    __syncthreads();
    if (first || last) sum = chunk_sum(0);
  } else {
    for (int64_t c0 = 0; c0 < chunks; c0 += kChunksAtOnce) {
      if (c0 > 0) __syncthreads();   // before the sums of the next chunks
      const int n = static_cast<int>(std::min<int64_t>(chunks - c0, kChunksAtOnce));
      for (int c = 0; c < n; ++c) {
        const double v = wave_sum(c0 + c);
        if (lane == 0) shared.sums[c][wave] = v;
      }
      __syncthreads();
      if ((first || last) && (c0 + lane % kChunksAtOnce) % kWave == lane && lane % kChunksAtOnce < n) sum += chunk_sum(lane % kChunksAtOnce);
    }
    if (first || last) sum = add_lanes(sum);
  }
  if (first) {
    const float slope = pair_slope(a, pair, sum);
    if (lane == 0) shared.slope = slope;
  }
  __syncthreads();
  if (last && lane == 0) write_pair(a, pair, sum);
  return shared.slope;
}

// By one wave, of one chunk; two waves' rows at a time are in flight.
__device__ __forceinline__ double wave_pair_sum(const PairArgs& a, const PairRows& rows) {
  const uint32_t lane = threadIdx.x % kWave;
  double h = 0.0;
  for (int w = 0; w < kPairWaves; w += 2) {
    const int64_t t0 = rows.at[0] + 4 * (w * kWave + lane), t1 = t0 + 4 * kWave;
    if (rows.at[0] + 4 * w * kWave >= rows.at[2]) break;   // the others' sums are 0
    FourRows r0, r1;
    r0.load(a, rows, t0);
    r1.load(a, rows, t1);
    h += add_lanes(r0.sum(a, rows, t0));
    h += add_lanes(r1.sum(a, rows, t1));
  }
  return h;
}

// How many of `count` keys, which do not decrease, are at most v, by a wave: each step looks at 64 of them.
template <class Key>
__device__ __forceinline__ int64_t keys_up_to(int64_t count, int64_t v, Key key) {
  const uint32_t lane = threadIdx.x % kWave;
  int64_t from = 0;
  while (true) {
    const int64_t step = (count + kWave - 1) / kWave, at = lane * step;
    const uint64_t below = __ballot(at < count && key(from + (at < count ? at : 0)) <= v);
    const int64_t n = __popcll(below);
    if (step == 1 || n == 0) return from + n;
    from += (n - 1) * step;
    count = std::min(count - (n - 1) * step, step);
  }
}
__device__ __forceinline__ int64_t offsets_up_to(const PairArgs& a, int64_t row) {
  return keys_up_to(2 * a.pairs + 1, row, [&](int64_t k) -> int64_t { return a.offsets[k]; });
}

// Where the gradient kernels take a row's factor from: memory, or the row's pair.  A wave calls with
// the rows [first, end) that its lanes have, and each lane's own.
struct GivenFactors {
  static constexpr bool kPairs = false, kScores = false;
};
// Of the scores: those of the log-probability and of the entropy, either of which may be missing.  Without targets
// every row counts.
struct ScoresFactors {
  static constexpr bool kPairs = false, kScores = true;
  const float* grad_logprobs;
  const float* grad_entropy;
  const float* entropy;

  template <class T>
  __device__ __forceinline__ ScoresGradient<T> gradient(const LogitsArgs& a, int64_t row, bool counts) const {
    const float g = counts && grad_logprobs ? grad_logprobs[row] : 0.f, e = counts && grad_entropy ? grad_entropy[row] : 0.f;
    return ScoresGradient<T>(g, e, a.stats[2 * row], a.stats[2 * row + 1], e == 0.f ? 0.f : entropy[row]);
  }
};
struct PairFactors {
  static constexpr bool kPairs = true, kScores = false;
  PairArgs p;

  __device__ __forceinline__ float operator()(int64_t first, int64_t end, int64_t row) const {
    float g = 0.f;
    for (int64_t r = first; r < end;) {
      const int64_t n = offsets_up_to(p, r);
      if (n > 2 * p.pairs) break;                              // past the last pair
      if (n == 0) {                                            // before the first
        r = std::max<int64_t>(r + 1, p.offsets[0]);
        continue;
      }
      const int64_t pair = (n - 1) / 2;
      const PairRows rows(p, pair);
      const float slope = pair_slope(p, pair, wave_pair_sum(p, rows));
      if (row >= r && row < rows.at[2]) g = row < rows.at[1] ? slope : -slope;
      r = std::max(r + 1, rows.at[2]);
    }
    return g;
  }
  // The pair's loss and margin.
  __device__ __forceinline__ void write(int64_t pair) const {
    const double sum = wave_pair_sum(p, PairRows(p, pair));
    if (threadIdx.x % kWave == 0) write_pair(p, pair, sum);
  }
};

int64_t pairs_of(const GivenFactors&) { return 0; }
int64_t pairs_of(const ScoresFactors&) { return 0; }
int64_t pairs_of(const PairFactors& f) { return f.p.pairs; }

// ... with what becomes of the vectors.
template <class T, int LANES, int HOLD>
struct ShortRow : ShortVectors<T, LANES, HOLD> {
  using ShortVectors<T, LANES, HOLD>::ShortVectors;
  using ShortVectors<T, LANES, HOLD>::kN;
  using ShortVectors<T, LANES, HOLD>::vectors;
  using ShortVectors<T, LANES, HOLD>::overlap;
  using ShortVectors<T, LANES, HOLD>::number;
  using ShortVectors<T, LANES, HOLD>::skipped;

  __device__ __forceinline__ Stat stat(const u4v (&h)[HOLD]) const {
    Stat s{-INFINITY, 0.f};
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      auto f = Vec<T>::floats(h[i]);
      if ((i + 1) * LANES >= vectors) {
        const uint32_t skip = skipped(number(i));
#pragma unroll
        for (uint32_t k = 0; k < kN; ++k) f[k] = k < skip ? -INFINITY : f[k];
      }
      add_floats<kN>(s, f);
    }
    return join_lanes<LANES>(s);
  }
  // The gradient of a row of fewer values than a vector.
  template <class Gradient>
  __device__ __forceinline__ void store_few(T* dz, const Gradient& grad, u4v z, uint32_t y, float target_logit) const {
    T v[kN];
    const u4v d = grad.of_vector(z);
    __builtin_memcpy(v, &d, sizeof(v));
    for (uint32_t k = overlap; k < kN; ++k) dz[k - overlap] = v[k];
    if (!grad.none) dz[y] = static_cast<T>(grad.of(target_logit, true));
  }
};

// How many waves have a row of `rows` short ones.
template <int LANES>
__host__ __device__ __forceinline__ int64_t short_row_waves(int64_t rows) { return (rows + kWave / LANES - 1) / (kWave / LANES); }

// A short row's gradient, from the registers to memory: through LDS, to as many lanes as the wave's rows have vectors.
template <class T, int LANES, int HOLD>
__device__ __forceinline__ void store_turned(const LogitsArgs& a, const ShortRow<T, LANES, HOLD>& at, const u4v* mine, int64_t first) {
  constexpr uint32_t kRows = kWave / LANES;
  const uint32_t vectors = at.vectors;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // lanes of one wave: LDS keeps their order
  __builtin_amdgcn_wave_barrier();
  const uint32_t inverse = 65536 / vectors + 1;   // n / vectors = n * inverse >> 16 for n up to 256, vectors up to 128
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    const uint32_t n = i * kWave + threadIdx.x % kWave, r = n * inverse >> 16, v = n - r * vectors;
    if (r < kRows && first + r < a.rows) Vec<T>::store(static_cast<T*>(a.dlogits) + (first + r) * a.out_stride + at.start(v), 0, 0, mine[n]);
  }
}

// The scores' gradient of a short row, by all lanes of a wave at once.
template <class T, int LANES, int HOLD>
__device__ __forceinline__ void store_short_scores(const LogitsArgs& a, const ScoresFactors& factors, const ShortRow<T, LANES, HOLD>& at,
                                                   u4v* turned, int64_t row, int64_t first, bool there, int32_t y) {
  constexpr uint32_t kN = Vec<T>::kN;
  const bool has_target = y >= 0 && y < a.cols;
  if (HOLD == 1 && !there) return;
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
  u4v h[HOLD] = {};
  float target_logit = 0.f;
  ScoresGradient<T> grad(0.f, 0.f, 0.f, 0.f, 0.f);
  if (there) grad = factors.gradient<T>(a, row, a.targets == nullptr || has_target);
  if (!grad.none) {
    at.load(z, h);
    if (has_target) target_logit = Vec<T>::value(Vec<T>::raw(z + y));
  }
  const uint32_t yv = static_cast<uint32_t>(y);
  const bool to_target = !grad.none && has_target;
  if (at.cols < kN) {
    if (!there) return;
    T v[kN];
    const u4v d = grad.of_vector(h[0]);
    __builtin_memcpy(v, &d, sizeof(v));
    for (uint32_t k = at.overlap; k < kN; ++k) dz[k - at.overlap] = v[k];
    if (to_target) dz[yv] = static_cast<T>(grad.of(target_logit, true));
    return;
  }
  if constexpr (HOLD == 1) {
    Vec<T>::store(dz, 0, 0, grad.of_vector(h[0]));
    if (to_target) dz[yv] = static_cast<T>(grad.of(target_logit, true));   // after its vector, by the same lane
  } else {
    u4v* mine = turned + threadIdx.x / kWave * (kWave * HOLD);          // the wave's rows, one after the other
    u4v* line = mine + threadIdx.x % kWave / LANES * at.vectors;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      const uint32_t v = at.number(i);
      if (v >= at.vectors) continue;
      line[v] = grad.of_vector(h[i]);
      if (to_target && yv - at.start(v) < kN) {
        const T d = static_cast<T>(grad.of(target_logit, true));
        __builtin_memcpy(reinterpret_cast<char*>(line + v) + (yv - at.start(v)) * sizeof(T), &d, sizeof(T));
      }
    }
    store_turned<T, LANES, HOLD>(a, at, mine, first);
  }
}

// All modes for short rows, 64 / LANES of them to a wave.  What bounds them is the number of
// instructions: few lanes per row, each with several vectors, spare the joins and the row's own
// arithmetic (1,048,576 rows of 100 bf16, 13 vectors, on 16 lanes: forward 79 us; on 4: 46).  Their
// stores would scatter (policy loss 120 us), so a row's gradient goes through LDS to as many
// lanes as it has vectors (84 us, 5.0 TB/s).
template <class T, RowMode kMode, int LANES, int HOLD, class Factors>
__global__ __launch_bounds__(kBlock)
void short_row_kernel(LogitsArgs a, Factors factors) {
  constexpr uint32_t kN = Vec<T>::kN, kRows = kWave / LANES;
  const ShortRow<T, LANES, HOLD> at(static_cast<uint32_t>(a.cols));
  constexpr bool kPolicy = kMode == RowMode::kPolicy, kForward = kMode == RowMode::kForward;
  constexpr bool kTurn = !kForward && HOLD > 1;
  __shared__ u4v turned[kTurn ? kBlock * HOLD : 1];
  const uint32_t vectors = at.vectors;
  const int64_t block = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x, row = Place<LANES>::row(block);
  const int64_t wave = block * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), first = wave * kRows;
  if constexpr (Factors::kPairs) {   // the waves after the last row's take a pair each
    const int64_t pair = wave - short_row_waves<LANES>(a.rows);
    if (pair >= 0) {
      if (pair < factors.p.pairs) factors.write(pair);
      return;
    }
  }
  const bool there = row < a.rows;
  if (!kTurn && !Factors::kPairs && !there) return;
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  const int32_t y = there && (!Factors::kScores || a.targets) ? a.targets[row] : -1;
  u4v h[HOLD];
  uint32_t target = 0;
  float lp = 0.f, loss = 0.f, g = 0.f, log_sum = 0.f;
  Stat s{-INFINITY, 0.f};
  bool counts = y >= 0 && y < a.cols;
  if constexpr (Factors::kScores) {
    store_short_scores<T, LANES, HOLD>(a, factors, at, turned, row, first, there, y);
    return;
  }
  PolicyRow pr{};
  if constexpr (kPolicy) {
    if (there) pr = policy_row(a, row);
    counts = counts && pr.weight != 0.f;
  }
  if constexpr (kMode == RowMode::kBackward) {
    if (counts) {
      if constexpr (!Factors::kPairs) g = a.grad[row];
      s.top = a.stats[2 * row];
      log_sum = a.stats[2 * row + 1];
    }
    counts = counts && (Factors::kPairs || g != 0.f);
  }
  if (counts) {
    target = Vec<T>::raw(z + y);
    at.load(z, h);
    if constexpr (kForward || kPolicy) {
      s = at.stat(h);
      lp = row_logprob(s, Vec<T>::value(target), &log_sum);
    }
    if constexpr (kPolicy) g = policy_slope(a, pr, lp, &loss);
  }
  if constexpr (Factors::kPairs) {
    const float factor = factors(first, std::min<int64_t>(first + kRows, a.rows), row);
    g = counts ? factor : 0.f;
    if (!kTurn && !there) return;
  }
  if constexpr (kForward) {
    if (at.lane == 0) write_forward(a, row, lp, counts ? s.top : 0.f, log_sum);
    return;
  }
  if constexpr (kPolicy) {
    if (at.lane == 0 && there) {
      a.logprobs[row] = lp;
      a.loss[row] = loss;
    }
    if (a.dlogits == nullptr) return;
  }
  T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
  const RowGradient<T> grad = kPolicy ? RowGradient<T>(g, s.top, 1.f / s.sum, s.top == -INFINITY && s.sum == 0.f)
                                      : RowGradient<T>::of_stats(g, s.top, log_sum);
  const uint32_t yv = static_cast<uint32_t>(y);
  if (at.cols < kN) {
    if (there) at.store_few(dz, grad, h[0], yv, Vec<T>::value(target));
    return;
  }
  if constexpr (!kTurn) {
    Vec<T>::store(dz, 0, 0, grad.of_vector(h[0]));
    if (!grad.none) dz[yv] = static_cast<T>(grad.of(Vec<T>::value(target), true));   // after its vector, by the same lane
  } else {
    u4v* mine = turned + threadIdx.x / kWave * (kWave * HOLD);          // the wave's rows, one after the other
    u4v* line = mine + threadIdx.x % kWave / LANES * vectors;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      const uint32_t v = at.number(i);
      if (v >= vectors) continue;
      line[v] = grad.of_vector(h[i]);
      if (!grad.none && yv - at.start(v) < kN) {
        const T d = static_cast<T>(grad.of(Vec<T>::value(target), true));
        __builtin_memcpy(reinterpret_cast<char*>(line + v) + (yv - at.start(v)) * sizeof(T), &d, sizeof(T));
      }
    }
    store_turned<T, LANES, HOLD>(a, at, mine, first);
  }
}

// ... with what becomes of the vectors.
template <class T>
struct WaveRun : VectorRun<T> {
  using VectorRun<T>::VectorRun;
  using VectorRun<T>::kN;
  using VectorRun<T>::lane;
  using VectorRun<T>::begin;
  using VectorRun<T>::whole;
  using VectorRun<T>::part;
  using VectorRun<T>::odd;
  using VectorRun<T>::any;
  using VectorRun<T>::values;

  // Maximum and sum of the vectors i0 .. i0 + N - 1, as loaded.
  template <int N>
  __device__ __forceinline__ void add(Stat& s, uint32_t i0, const u4v* loaded, uint32_t& carry) const {
    if (!any(i0)) return;
    u4v h[N];
#pragma unroll
    for (int k = 0; k < N; ++k) h[k] = values(loaded[k], carry);
    if (i0 + N > whole) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (!(i0 + k < whole || (i0 + k == whole && lane < part))) h[k] = Vec<T>::none();
    }
    add_vectors<T>(s, h);
  }
  // Gradient of vector i, as loaded, to the row at dz.
  __device__ __forceinline__ void store(T* dz, const RowGradient<T>& grad, uint32_t i, u4v v) const {
    if (!any(i)) return;
    T* out = dz + odd + static_cast<uint64_t>(begin) * kN;
    const u4v d = grad.of_vector(v);
    if (i < whole) Vec<T>::store(out, i * kWave, lane, d);
    else if (lane < part) Vec<T>::store(out, i * kWave, lane, d);
  }
  // Of a row whose vectors are shared out, those before `held` one by one and the others by `group`s: whose
  // has the target.
  __device__ __forceinline__ uint32_t stored_by(uint32_t y, uint32_t held, uint32_t group, uint32_t parts) const {
    const uint32_t i = ((y - odd) / kN - begin) / kWave;
    return (i < held ? i : (i - held) / group) % parts;
  }
  // The target's gradient, by the lane that stored its vector.
  __device__ __forceinline__ void store_target(T* dz, const RowGradient<T>& grad, uint32_t y, float target_logit) const {
    const uint32_t v = (y - odd) / kN - begin;    // of y = 0 in a shifted row: past any run
    if (!grad.none && v < whole * kWave + part && v % kWave == lane) dz[y] = static_cast<T>(grad.of(target_logit, true));
  }
};

// Waves' parts of a row.
template <int WAVES>
struct RowParts {
  Stat stat[WAVES];
  float target_logit;
};

// Maximum and sum of this wave's part of a long row, of which a block has WAVES: U vectors in flight
// per lane, the waves' runs side by side, so that the block reads neighbouring memory.
template <class T, int WAVES, int U>
__device__ __forceinline__ Stat long_row_part(const T* z, uint32_t cols, uint32_t tid) {
  constexpr uint32_t kN = Vec<T>::kN;
  const uint32_t full = long_row_vectors<T>(cols), rem = cols - full * kN;
  const uint32_t tail = Vec<T>::raw(z + full * kN + (tid < rem ? tid : rem - 1));
  Stat s{-INFINITY, 0.f};
  for (uint32_t first = __builtin_amdgcn_readfirstlane(tid / kWave) * (kWave * U); first < full; first += WAVES * kWave * U) {
    const WaveRun<T> run(z, full, first, kWave * U);
    const uint32_t before = run.before();
    u4v h[U];
#pragma unroll
    for (int i = 0; i < U; ++i) h[i] = run.load(i);
    uint32_t carry = before << 16;
    run.template add<U>(s, 0, h, carry);
  }
  if (tid < rem) add_value(s, Vec<T>::value(tail));
  return join_lanes<kWave>(s);
}

// kForward for long rows: a block (or, with WAVES = 1, a wave) per row, whose waves take U vectors per
// lane in turn.
template <class T, int WAVES, int U>
__global__ __launch_bounds__(Place<WAVES * kWave>::kThreads)
void long_forward_kernel(LogitsArgs a) {
  constexpr int LANES = WAVES * kWave;
  __shared__ RowParts<WAVES> parts;
  const int64_t row = Place<LANES>::row(static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x);
  if (row >= a.rows) return;
  const uint32_t tid = Place<LANES>::lane();
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  const int32_t y = __builtin_amdgcn_readfirstlane(a.targets[row]);
  const bool counts = y >= 0 && y < a.cols;
  float lp = 0.f, log_sum = 0.f;
  Stat s{-INFINITY, 0.f};
  if (counts) {
    const uint32_t target = Vec<T>::raw(z + y);
    s = long_row_part<T, WAVES, U>(z, static_cast<uint32_t>(a.cols), tid);
    if constexpr (WAVES > 1) {
      if (tid % kWave == 0) parts.stat[tid / kWave] = s;
      __syncthreads();
      s = join_lanes<WAVES>(parts.stat[tid % WAVES]);
    }
    lp = row_logprob(s, Vec<T>::value(target), &log_sum);
  }
  if (tid == 0) write_forward(a, row, lp, counts ? s.top : 0.f, log_sum);
}

// The same value in all lanes, to a scalar register.
__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// What a row's turn in the policy loss starts from, besides its vectors.
template <class T>
struct PolicyTurn {
  PolicyRow row;
  int32_t y;

  __device__ __forceinline__ void read(const LogitsArgs& a, int64_t r) {
    y = a.targets[r];
    row = policy_row(a, r);
  }
  __device__ __forceinline__ void make_uniform() {
    y = uniform(y);
    row = {uniform(row.advantage), uniform(row.old_logprob), uniform(row.ref_logprob), uniform(row.weight)};
  }
  __device__ __forceinline__ bool counts(const LogitsArgs& a) const {
    return uniform(static_cast<int32_t>(y >= 0 && y < a.cols && row.weight != 0.f)) != 0;
  }
};

// This lane's part of a row's values outside of its vectors, and their gradient.
template <class T>
struct RowEnds {
  uint32_t tail;   // value full * kN + tid, of the first rem lanes (the others: the row's last)
  uint32_t head;   // lane 0 of the first wave, shifted rows: the first value

  __device__ __forceinline__ void load(const WaveRun<T>& run, const T* z, uint32_t full, uint32_t tid, uint32_t rem) {
    tail = Vec<T>::raw(z + full * Vec<T>::kN + (tid < rem ? tid : rem - 1));
    head = run.before();
  }
  __device__ __forceinline__ void store(T* dz, const RowGradient<T>& grad, uint32_t full, uint32_t odd, uint32_t tid,
                                        uint32_t rem, uint32_t y) const {
    if (tid < rem && !(odd && tid == 0)) {   // a shifted row's vectors go one value further
      const uint32_t j = full * Vec<T>::kN + tid;
      dz[j] = static_cast<T>(grad.none ? 0.f : grad.of(Vec<T>::value(tail), j == y));
    }
    if (odd && tid == 0) dz[0] = static_cast<T>(grad.none ? 0.f : grad.of(Vec<T>::value(head), y == 0));
  }
};

// A row's loss and gradient factor from the lanes' maxima and sums; one lane writes the loss.
template <class T, int WAVES>
__device__ __forceinline__ RowGradient<T> finish_policy_row(const LogitsArgs& a, int64_t row, const PolicyTurn<T>& turn, bool counts,
                                                            Stat s, float target_logit, RowParts<WAVES>& parts, uint32_t tid, bool writes) {
  float lp = 0.f, loss = 0.f, g = 0.f, log_sum = 0.f;
  if (counts) {
    s = join_lanes<kWave>(s);
    if constexpr (WAVES > 1) {
      // One wave reads the target's logit, before the others can write over it in place.
      if (tid % kWave == 0) parts.stat[tid / kWave] = s;
      if (tid == 0) parts.target_logit = target_logit;
      __syncthreads();
      s = join_lanes<WAVES>(parts.stat[tid % WAVES]);
      target_logit = parts.target_logit;
    }
    lp = row_logprob(s, target_logit, &log_sum);
    g = policy_slope(a, turn.row, lp, &loss);
  }
  if (tid == 0 && writes) {
    a.logprobs[row] = lp;
    a.loss[row] = loss;
  }
  return RowGradient<T>(uniform(g), uniform(s.top), uniform(1.f / s.sum), uniform(s.top) == -INFINITY && uniform(s.sum) == 0.f);
}

// kPolicy for long rows: a block (or, with WAVES = 1, a wave) per row.  Two blocks or more share a
// CU, so that one's loads and stores go on while another computes (12,289 rows of 50,021 bf16: 454 us;
// one block of 16 waves per CU 580, the same with the next row's loads among the stores 566).
// From the sum to the gradient a lane keeps its first HOLD vectors in registers and the next STAGE
// in LDS, where they are loaded without passing through registers; the rest of a row that is
// longer still is read again.  8 waves of 16 + 9 vectors hold 102,400 16-bit values at two blocks
// to a CU: rows of 131,072 bf16 take 741 us so, 805 held whole by one block of 16 waves.
//
// kSplit, for few rows: as many blocks as blockIdx.z counts all take the row's sum, whose order stays the
// same, and each the gradient of every so-manieth vector.  Not in place: a block would change what
// another has yet to read.
template <class T, int WAVES, int HOLD, int STAGE, bool kSplit>
__global__ __launch_bounds__(Place<WAVES * kWave>::kThreads)
void long_policy_kernel(LogitsArgs a) {
  constexpr int kN = Vec<T>::kN, LANES = WAVES * kWave;
  // Vectors unpacked at once: with LDS in use as well, fewer, to stay within 128 registers.
  constexpr int kFew = STAGE > 0 ? 16 / kN : HOLD % 4 == 0 ? 4 : HOLD % 3 == 0 ? 3 : HOLD % 2 == 0 ? 2 : 1;
  __shared__ RowParts<WAVES> parts;
  __shared__ u4v stage[STAGE > 0 ? WAVES * STAGE * kWave : 1];
  const int64_t row = Place<LANES>::row(static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x);
  if (row >= a.rows) return;
  const uint32_t tid = Place<LANES>::lane(), cols = static_cast<uint32_t>(a.cols);
  const uint32_t full = long_row_vectors<T>(cols), rem = cols - full * kN, wave = uniform(static_cast<int32_t>(tid / kWave));
  const uint32_t per = (full + LANES - 1) / LANES * kWave;
  const uint32_t part = kSplit ? blockIdx.z : 0, parts_of_row = kSplit ? gridDim.z : 1;
  auto mine_to_store = [&](uint32_t i) { return !kSplit || i % parts_of_row == part; };
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  const WaveRun<T> run(z, full, wave * per, per);
  PolicyTurn<T> turn;
  turn.read(a, row);
  turn.make_uniform();
  const bool counts = turn.counts(a);
  u4v held[HOLD];
  u4v* mine = stage + wave * (STAGE * kWave);
  RowEnds<T> ends;
  uint32_t target = 0;
  Stat s{-INFINITY, 0.f};
  if (counts) {
    target = Vec<T>::raw(z + turn.y);
    ends.load(run, z, full, tid, rem);
#pragma unroll
    for (int i = 0; i < HOLD; ++i) held[i] = run.load(i);
    if constexpr (STAGE > 0) {
#pragma unroll
      for (int i = 0; i < STAGE; ++i) run.load_to_lds(HOLD + i, mine + i * kWave);
    }
    uint32_t carry = ends.head << 16;
#pragma unroll
    for (int i = 0; i < HOLD; i += kFew) run.template add<kFew>(s, i, held + i, carry);
    if constexpr (STAGE > 0) {
      constexpr int kThree = 3;
      static_assert(STAGE % kThree == 0, "whole groups");
      for (int i = 0; i < STAGE; i += kThree) {
        u4v h[kThree];
#pragma unroll
        for (int k = 0; k < kThree; ++k) h[k] = mine[(i + k) * kWave + run.lane];
        run.template add<kThree>(s, HOLD + i, h, carry);
      }
      for (uint32_t i = HOLD + STAGE; run.any(i); i += kFew) {
        u4v h[kFew];
#pragma unroll
        for (int k = 0; k < kFew; ++k) h[k] = run.template load<true>(i + k);
        run.template add<kFew>(s, i, h, carry);
      }
    }
    if (tid < rem) add_value(s, Vec<T>::value(ends.tail));
  }
  const RowGradient<T> grad = finish_policy_row<T, WAVES>(a, row, turn, counts, s, Vec<T>::value(target), parts, tid, part == 0);
  if (a.dlogits == nullptr) return;
  T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
  const uint32_t y = static_cast<uint32_t>(turn.y);
  constexpr int kMore = STAGE > 0 ? 4 : 1;
  u4v more[kMore];   // what is read again: on its way while the rest is stored
  auto load_more = [&](uint32_t i) {
    if (grad.none || !run.any(i)) return;
#pragma unroll
    for (int k = 0; k < kMore; ++k) more[k] = run.load(i + k);
  };
  const uint32_t first_more = HOLD + STAGE + part * kMore;
  if constexpr (STAGE > 0) load_more(first_more);
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    if (!mine_to_store(i)) continue;
    asm("" : "+v"(held[i]));   // unpacked anew: twice the registers would go to its values
    run.store(dz, grad, i, held[i]);
  }
  if constexpr (STAGE > 0) {
#pragma unroll 1
    for (int i = 0; i < STAGE; ++i)
      if (mine_to_store(HOLD + i)) run.store(dz, grad, HOLD + i, mine[i * kWave + run.lane]);
    for (uint32_t i = first_more; run.any(i); i += kMore * parts_of_row) {
#pragma unroll
      for (int k = 0; k < kMore; ++k) run.store(dz, grad, i + k, more[k]);
      load_more(i + kMore * parts_of_row);
    }
  }
  if (!kSplit || run.stored_by(y, HOLD + STAGE, kMore, parts_of_row) == part) run.store_target(dz, grad, y, Vec<T>::value(target));
  if (part == 0) ends.store(dz, grad, full, run.odd, tid, rem, y);
}

// kBackward of longer rows: every value by itself.  A group of LANES lanes takes LANES * U vectors of
// a row; the runs of a longer row go to different blocks.  Nothing is summed, so the vectors may start
// anywhere: they start at the row's first cache line, and each value before it goes to a lane of its
// own.  8,192 x 131,071 bf16 737 us against 774 with the vectors at the row's first multiple of 4
// bytes and 765 at that of 16; 131,072 x 2,001 187 against 213.
constexpr uint32_t kLine = 128;
template <class T, int LANES, int U, class Factors>
__global__ __launch_bounds__(Place<LANES>::kThreads)
void gradient_kernel(LogitsArgs a, Factors factors) {
  constexpr uint32_t kN = Vec<T>::kN;
  const int64_t row = Place<LANES>::row(static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y);
  if (row >= a.rows) {
    if constexpr (Factors::kPairs) {   // the groups after the last row's take a pair each
      const int64_t pair = row - a.rows;
      if (pair < factors.p.pairs && blockIdx.x == 0 && Place<LANES>::lane() < kWave) factors.write(pair);
    }
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.stride;
  T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
  const uint32_t head = static_cast<uint32_t>(-reinterpret_cast<uintptr_t>(z) % kLine / sizeof(T));
  const uint32_t lane = Place<LANES>::lane(), cols = static_cast<uint32_t>(a.cols);
  const uint32_t full = (cols - head) / kN, rem = cols - head - full * kN, v0 = blockIdx.x * (LANES * U);
  const int32_t y = !Factors::kScores || a.targets ? a.targets[row] : -1;
  const bool has_token = y >= 0 && y < a.cols;
  u4v h[U];
  auto load = [&] {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      h[i] = u4v{0, 0, 0, 0};
      if (v0 + i * LANES + lane < full) h[i] = Vec<T>::load(z + head, v0 + i * LANES, lane);
    }
  };
  float g = 0.f;
  if constexpr (Factors::kPairs) {
    if (has_token) {
      load();      // while the pair is summed
      if constexpr (Place<LANES>::kRows > 1) {
        g = factors(row, row + 1, row);
      } else {     // once per block: by each of 8 waves, 486 rows of 22,737 fp16 take 6 us longer
        __shared__ float factor;
        if (threadIdx.x < kWave) {
          g = factors(row, row + 1, row);
          if (threadIdx.x == 0) factor = g;
        }
        __syncthreads();
        g = factor;
      }
    }
  } else if constexpr (!Factors::kScores) {
    g = a.grad[row];
  }
  const auto grad = [&] {
    if constexpr (Factors::kScores) {
      return factors.template gradient<T>(a, row, a.targets == nullptr || has_token);
    } else {
      const float top = a.stats[2 * row], log_sum = a.stats[2 * row + 1];
      return RowGradient<T>::of_stats(has_token ? g : 0.f, top, log_sum);
    }
  }();
  // Columns outside of the vectors: up to kN - 1 at the end, less than a cache line at the start.
  const uint32_t yv = static_cast<uint32_t>(y), last = cols - rem + lane;
  const bool has_tail = blockIdx.x == gridDim.x - 1 && lane < rem, has_head = blockIdx.x == 0 && lane < head;
  if (grad.none) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (v0 + i * LANES + lane < full) Vec<T>::store(dz + head, v0 + i * LANES, lane, u4v{0, 0, 0, 0});
    if (has_tail) dz[last] = static_cast<T>(0.f);
    if (has_head) dz[lane] = static_cast<T>(0.f);
    return;
  }
  const uint32_t target = (yv - head) / kN - v0;   // the target's vector, and whether this lane has it (without a target, past the last)
  const bool has_target = target < LANES * U && target + v0 < full && target % LANES == lane;
  uint32_t z_target = 0, z_tail = 0, z_head = 0;
  if constexpr (!Factors::kPairs) load();
  if (has_target) z_target = Vec<T>::raw(z + yv);
  if (has_tail) z_tail = Vec<T>::raw(z + last);
  if (has_head) z_head = Vec<T>::raw(z + lane);
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (v0 + i * LANES + lane < full) Vec<T>::store(dz + head, v0 + i * LANES, lane, grad.of_vector(h[i]));
  if (has_target) dz[yv] = static_cast<T>(grad.of(Vec<T>::value(z_target), true));
  if (has_tail) dz[last] = static_cast<T>(grad.of(Vec<T>::value(z_tail), last == yv));
  if (has_head) dz[lane] = static_cast<T>(grad.of(Vec<T>::value(z_head), lane == yv));
}

// One block per kRows rows.
template <int LANES, class Kernel>
hipError_t launch_rows(Kernel kernel, const LogitsArgs& a, hipStream_t stream) {
  const int64_t blocks = Place<LANES>::blocks(a.rows), x = std::min(blocks, kGridX);
  const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>((blocks + x - 1) / x));
  kernel<<<grid, Place<LANES>::kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

// A short row's kernel; with pairs, a wave more for each.
template <class T, RowMode kMode, int LANES, int HOLD, class Factors>
hipError_t launch_short_rows(const LogitsArgs& a, const Factors& factors, hipStream_t stream) {
  constexpr int64_t kWaves = kBlock / kWave;
  const int64_t blocks = (short_row_waves<LANES>(a.rows) + pairs_of(factors) + kWaves - 1) / kWaves, x = std::min(blocks, kGridX);
  const dim3 grid(static_cast<uint32_t>(x), static_cast<uint32_t>((blocks + x - 1) / x));
  short_row_kernel<T, kMode, LANES, HOLD><<<grid, kBlock, 0, stream>>>(a, factors);
  return hipGetLastError();
}

template <class T, int LANES, int U, class Factors>
hipError_t launch_gradient(const LogitsArgs& a, const Factors& factors, hipStream_t stream) {
  constexpr int64_t kRun = int64_t{LANES} * U;
  const int64_t full = a.cols / Vec<T>::kN, blocks = Place<LANES>::blocks(a.rows + pairs_of(factors)), y = std::min(blocks, kGridYZ);
  const dim3 grid(static_cast<uint32_t>(std::max<int64_t>(1, (full + kRun - 1) / kRun)), static_cast<uint32_t>(y),
                  static_cast<uint32_t>((blocks + y - 1) / y));
  gradient_kernel<T, LANES, U><<<grid, Place<LANES>::kThreads, 0, stream>>>(a, factors);
  return hipGetLastError();
}

// Rows of up to 128 vectors: lanes by the number of vectors.
template <class T, RowMode kMode, class Factors = GivenFactors>
hipError_t launch_short(const LogitsArgs& a, hipStream_t stream, const Factors& factors = {}) {
  const int64_t vectors = (a.cols + Vec<T>::kN - 1) / Vec<T>::kN;
  if (vectors <= 1) return launch_short_rows<T, kMode, 1, 1>(a, factors, stream);
  if (vectors <= 2) return launch_short_rows<T, kMode, 1, 2>(a, factors, stream);
  if (vectors <= 4) return launch_short_rows<T, kMode, 1, 4>(a, factors, stream);
  if (vectors <= 8) return launch_short_rows<T, kMode, 2, 4>(a, factors, stream);
  if (vectors <= 16) return launch_short_rows<T, kMode, 4, 4>(a, factors, stream);
  if (vectors <= 32) return launch_short_rows<T, kMode, 8, 4>(a, factors, stream);
  if (vectors <= 64) return launch_short_rows<T, kMode, 16, 4>(a, factors, stream);
  return launch_short_rows<T, kMode, 32, 4>(a, factors, stream);
}
constexpr int64_t kShortVectors = 128;

// Whether a wave that has a row to itself takes three vectors per lane at a time, not four: where
// that leaves fewer empty ones in its one or two turns.
bool in_threes(int64_t full) { return full <= 192 || (full > 256 && full <= 384); }

template <class T>
hipError_t launch_forward(const LogitsArgs& a, hipStream_t stream) {
  const int64_t vectors = (a.cols + Vec<T>::kN - 1) / Vec<T>::kN, full = a.cols / Vec<T>::kN;
  if (vectors <= kShortVectors) return launch_short<T, RowMode::kForward>(a, stream);
  // Fewer waves leave fewer of them without a vector; more have more loads in flight for one row.
  // 9,000 bf16 columns (1,125 vectors): 82 us on 2 waves, 87 on 4, 106 on 8, 166 on 16; 131,073: 87,
  // 81, 80 and 79.
  if (in_threes(full)) return launch_rows<64>(long_forward_kernel<T, 1, 3>, a, stream);
  if (full <= 512) return launch_rows<64>(long_forward_kernel<T, 1, 4>, a, stream);
  if (full <= 1536) return launch_rows<128>(long_forward_kernel<T, 2, 4>, a, stream);
  if (full <= 2048) return launch_rows<256>(long_forward_kernel<T, 4, 4>, a, stream);
  if (full <= 12288) return launch_rows<512>(long_forward_kernel<T, 8, 4>, a, stream);
  return launch_rows<1024>(long_forward_kernel<T, 16, 4>, a, stream);
}

// Few long rows of a gradient that replaces no logits: four to eight blocks for each, up to one per CU.  16
// rows of 65,536 bf16 9.0 us, by a block each 11.6; 64 10.5 and 12.4; 64 of 32,768 fp32 8.2 and 8.8; one of
// 131,072 bf16 15.7 and 19.3.  Two blocks for each of 100 rows of 32,768 fp32 take 9.5, one 8.9; rows of up
// to 7,168 vectors gain nothing.
constexpr int64_t kCus = 256, kFewestParts = 4, kMostParts = 8;
template <class T, int WAVES, int HOLD, int STAGE>
hipError_t launch_long_policy(const LogitsArgs& a, hipStream_t stream) {
  constexpr int LANES = WAVES * kWave;
  if constexpr (HOLD == 16) {   // past 7,168 vectors
    const int64_t parts = std::min(kCus / a.rows, kMostParts);
    if (parts >= kFewestParts && a.dlogits && a.dlogits != a.logits) {
      const dim3 grid(static_cast<uint32_t>(a.rows), 1, static_cast<uint32_t>(parts));
      long_policy_kernel<T, WAVES, HOLD, STAGE, true><<<grid, LANES, 0, stream>>>(a);
      return hipGetLastError();
    }
  }
  return launch_rows<LANES>(long_policy_kernel<T, WAVES, HOLD, STAGE, false>, a, stream);
}

// Waves and vectors per lane by the row's vectors.
template <class T>
hipError_t launch_policy(const LogitsArgs& a, hipStream_t stream) {
  const int64_t vectors = (a.cols + Vec<T>::kN - 1) / Vec<T>::kN, full = a.cols / Vec<T>::kN;
  if (vectors <= kShortVectors) return launch_short<T, RowMode::kPolicy>(a, stream);
  if (full <= 192) return launch_long_policy<T, 1, 3, 0>(a, stream);
  if (full <= 256) return launch_long_policy<T, 1, 4, 0>(a, stream);
  if (full <= 384) return launch_long_policy<T, 1, 6, 0>(a, stream);
  if (full <= 512) return launch_long_policy<T, 1, 8, 0>(a, stream);
  if (full <= 768) return launch_long_policy<T, 4, 3, 0>(a, stream);
  if (full <= 1024) return launch_long_policy<T, 4, 4, 0>(a, stream);
  if (full <= 1536) return launch_long_policy<T, 4, 6, 0>(a, stream);
  if (full <= 2048) return launch_long_policy<T, 4, 8, 0>(a, stream);
  if (full <= 3072) return launch_long_policy<T, 8, 6, 0>(a, stream);
  if (full <= 4096) return launch_long_policy<T, 8, 8, 0>(a, stream);
  if (full <= 5120) return launch_long_policy<T, 8, 10, 0>(a, stream);
  if (full <= 6144) return launch_long_policy<T, 8, 12, 0>(a, stream);
  if (full <= 7168) return launch_long_policy<T, 8, 14, 0>(a, stream);
  if (full <= 8192) return launch_long_policy<T, 8, 16, 0>(a, stream);
  // Past 20,480 vectors what 16 waves of one block hold more outweighs the second block: 2,048 rows of
  // 131,072 fp32 391 us, 433 by 8 waves; of 80,000 232 and 234; of 65,600 195 and 180.
  if (full > 20480) return launch_long_policy<T, 16, 16, 9>(a, stream);
  return launch_long_policy<T, 8, 16, 9>(a, stream);
}

template <class T, class Factors = GivenFactors>
hipError_t launch_backward(const LogitsArgs& a, hipStream_t stream, const Factors& factors = {}) {
  const int64_t vectors = (a.cols + Vec<T>::kN - 1) / Vec<T>::kN;
  if (vectors <= kShortVectors) return launch_short<T, RowMode::kBackward>(a, stream, factors);
  // Runs that leave few lanes of a row's last one empty: 9,000 bf16 columns (1,125 vectors) 166 us in
  // runs of 512, 209 of 1,024; 20,000 (2,500) 169 and 163.  fp32 does best with a load per lane
  // (24,000 columns 163 us, with two 176).
  // 384 vectors and fewer: 2,501 bf16 columns 161 us in runs of 384, 168 in runs of 512; 3,501 (438) 270
  // and 215.
  if (vectors <= 256) return launch_gradient<T, 64, 4>(a, factors, stream);
  if (vectors <= 384) return launch_gradient<T, 128, 3>(a, factors, stream);
  if (vectors <= 512) return launch_gradient<T, 256, 2>(a, factors, stream);
  if constexpr (sizeof(T) == 4) {
    if (vectors > 768) return launch_gradient<T, 256, 1>(a, factors, stream);
  } else {
    if (vectors > 1024 && vectors <= 1536) return launch_gradient<T, 256, 2>(a, factors, stream);
  }
  return launch_gradient<T, 512, 2>(a, factors, stream);
}

template <class T>
hipError_t launch_typed(const LogitsArgs& a, RowMode mode, hipStream_t stream) {
  switch (mode) {
    case RowMode::kForward: return launch_forward<T>(a, stream);
    case RowMode::kPolicy: return launch_policy<T>(a, stream);
    default: return launch_backward<T>(a, stream);
  }
}

// The rows' part of the gradient of a pair, or of a chunk of it.
__device__ __forceinline__ void write_rows(const PairArgs& a, const PairRows& rows, int64_t from, int64_t to, float g) {
  for (int64_t t = from + 4 * threadIdx.x; t < to; t += kChunk) {
    f4_unaligned v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = t + k < rows.at[1] ? g : -g;
    if (t + 4 <= to) *reinterpret_cast<f4_unaligned*>(a.grad + t) = v;
    else
      for (int64_t u = t; u < to; ++u) a.grad[u] = v[u - t];
  }
}

__global__ __launch_bounds__(kPairThreads)
void pair_kernel(PairArgs a) {
  __shared__ PairSums shared;
  for (int64_t pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    const PairRows rows(a, pair);
    const float g = block_pair_slope(a, pair, rows, shared, [&](int64_t t) {
      FourRows r;
      r.load(a, rows, t);
      return r.sum(a, rows, t);
    });
    if (a.grad) write_rows(a, rows, rows.at[0], rows.at[2], g);
    __syncthreads();   // before the sums of the next pair
  }
}

// Long pairs, a block for each chunk: first the chunks' sums, then, in a second launch, each block adds up its
// pair's.  Chunk c of pair i has the place first row / kChunk + i + c, so that all chunks have places in
// [0, rows / kChunk + pairs), each its own.
struct ChunkPlace {
  int64_t pair, first;   // the pair's first place; pair -1: none (also where offsets decrease)

  __device__ __forceinline__ ChunkPlace(const PairArgs& a, int64_t place) {
    auto first_place = [&](int64_t i) { return PairRows::bounded(a, a.offsets[2 * i]) / kChunk + i; };
    pair = keys_up_to(a.pairs, place, first_place) - 1;
    first = pair < 0 ? 0 : first_place(pair);
    if (first > place) pair = -1;
  }
};

__global__ __launch_bounds__(kPairThreads)
void chunk_sum_kernel(PairArgs a) {
  __shared__ double sums[kPairWaves];
  const ChunkPlace at(a, blockIdx.x);
  if (at.pair < 0) return;
  const PairRows rows(a, at.pair);
  const int64_t t = rows.at[0] + (blockIdx.x - at.first) * kChunk + 4 * threadIdx.x;
  FourRows r;
  r.load(a, rows, t);
  double sum = add_lanes(r.sum(a, rows, t));
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int w = 0; w < kPairWaves; ++w) sum += sums[w];
    a.chunk_sums[blockIdx.x] = sum;
  }
}

__global__ __launch_bounds__(kPairThreads)
void chunk_gradient_kernel(PairArgs a) {
  __shared__ float slope;
  const ChunkPlace at(a, blockIdx.x);
  if (at.pair < 0) return;
  const PairRows rows(a, at.pair);
  const int64_t chunks = rows.chunks(), c = blockIdx.x - at.first;
  if (c > 0 && c >= chunks) return;   // a pair's first place also without rows
  double sum = 0.0;
  if (threadIdx.x < kWave) {
    for (int64_t k = threadIdx.x; k < chunks; k += kWave) sum += a.chunk_sums[at.first + k];
    sum = add_lanes(sum);
    const float g = pair_slope(a, at.pair, sum);
    if (threadIdx.x == 0) slope = g;
  }
  __syncthreads();
  const int64_t from = rows.at[0] + c * kChunk;
  if (a.grad) write_rows(a, rows, from, std::min(rows.at[2], from + kChunk), slope);
  if (c == 0 && threadIdx.x == 0) write_pair(a, at.pair, sum);
}

// The whole preference loss in one launch, for few logits: a block per pair takes its rows' sums,
// the pair's loss and, reading the rows again out of the caches, their gradients; what it needs of
// a row again stays in LDS.  Rows before
// the first pair and after the last go with those.  Every value is computed as by the kernels that
// take one step each, to the same bits.
constexpr int64_t kSmallRows = kChunk;
template <class T, int LANES, int HOLD, int U>   // as for short rows; U > 0: long rows, a wave for each
__global__ __launch_bounds__(kPairThreads)
void small_preference_kernel(LogitsArgs a, PairArgs p) {
  constexpr uint32_t kN = Vec<T>::kN;
  constexpr int kGroups = kPairThreads / LANES, kAhead = U > 0 ? U : HOLD;
  __shared__ PairSums shared;
  __shared__ double shares[kSmallRows];          // l - ref, of rows that count
  __shared__ float tops[kSmallRows], log_sums[kSmallRows], target_logits[kSmallRows];
  __shared__ int32_t targets[kSmallRows];        // -1: no token, or no row of the pair
  const int64_t pair = blockIdx.x;
  const PairRows rows(p, pair);
  const int64_t from = pair == 0 ? 0 : rows.at[0], to = pair == p.pairs - 1 ? a.rows : rows.at[2];
  const uint32_t cols = static_cast<uint32_t>(a.cols), lane = threadIdx.x % LANES;
  uint32_t group = threadIdx.x / LANES;
  if constexpr (LANES == kWave) group = __builtin_amdgcn_readfirstlane(group);
  const ShortRow<T, LANES, HOLD> at(cols);
  int32_t next_y = from + group < to ? a.targets[from + group] : -1;
  for (int64_t row = from + group; row < to; row += kGroups) {
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const int32_t y = next_y;
    if (row + kGroups < to) next_y = a.targets[row + kGroups];   // on its way with this row
    const float ref = p.ref_logprobs ? p.ref_logprobs[row] : 0.f;
    const bool counts = y >= 0 && y < a.cols;
    float lp = 0.f, log_sum = 0.f, target_logit = 0.f;
    Stat s{0.f, 0.f};
    if (counts) {
      const uint32_t target = Vec<T>::raw(z + y);
      if constexpr (U == 0) {
        u4v h[HOLD];
        at.load(z, h);
        s = at.stat(h);
      } else {
        s = long_row_part<T, 1, U>(z, cols, lane);
      }
      target_logit = Vec<T>::value(target);
      lp = row_logprob(s, target_logit, &log_sum);
    }
    if (lane == 0) {
      a.logprobs[row] = lp;
      shares[row] = counts ? static_cast<double>(lp) - ref : 0.0;
      tops[row] = s.top;
      log_sums[row] = log_sum;
      target_logits[row] = target_logit;
      targets[row] = counts && row >= rows.at[0] && row < rows.at[2] ? y : -1;
    }
  }
  __syncthreads();
  // A row's last vector, which overlaps the one before it, is loaded before either is stored, and the
  // first row's first vectors while the pair's loss is computed.
  const uint32_t last = at.vectors - 1;
  auto load = [&](int64_t row, u4v (&h)[kAhead], u4v& end) {
    if (cols < kN || row >= to || targets[row] < 0) return;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) h[i] = Vec<T>::template load<true>(z + at.start(std::min(i * LANES + lane, last)), 0, 0);
    if (lane == last % LANES) end = Vec<T>::template load<true>(z + at.start(last), 0, 0);
  };
  u4v h[kAhead] = {}, end{};
  if (a.dlogits) load(from + group, h, end);
  const float g = block_pair_slope(p, pair, rows, shared, [&](int64_t t) {
    double sum = 0.0;
    for (int64_t u = t; u < t + 4 && u < rows.at[2]; ++u) sum += u < rows.at[1] ? shares[u] : -shares[u];
    return sum;
  });
  if (a.dlogits == nullptr) return;
  for (int64_t row = from + group; row < to; row += kGroups) {
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    T* dz = static_cast<T*>(a.dlogits) + row * a.out_stride;
    const int32_t y = targets[row];
    const RowGradient<T> grad = RowGradient<T>::of_stats(y < 0 ? 0.f : row < rows.at[1] ? g : -g, tops[row], log_sums[row]);
    const uint32_t yv = static_cast<uint32_t>(y);
    const float target_logit = target_logits[row];
    if (cols < kN) {
      if constexpr (U == 0) {
        u4v few[HOLD] = {};
        if (!grad.none) at.load(z, few);
        at.store_few(dz, grad, few[0], yv, target_logit);
      }
      continue;
    }
    u4v next[kAhead] = {}, next_end{};
    load(row + kGroups, next, next_end);
    for (uint32_t v0 = 0; v0 < at.vectors; v0 += kAhead * LANES) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t v = v0 + i * LANES + lane;
        if (v >= at.vectors) continue;
        u4v x = h[i];
        if (v0 > 0 && !grad.none) x = Vec<T>::template load<true>(z + at.start(v), 0, 0);
        Vec<T>::template store<true>(dz + at.start(v), 0, 0, grad.of_vector(v == last ? end : x));
        if (!grad.none && yv - at.start(v) < kN) dz[yv] = static_cast<T>(grad.of(target_logit, true));
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) h[i] = next[i];
    end = next_end;
  }
}

// So many logits, and so many per pair, go through one launch, in which a pair has but one CU, whose exponentials
// bound it.  The longest pair decides, and the host knows the average.  As calls, in 1 to 16 pairs of rows of 57 to
// 2,000, two launches take 10 to 11 us, and one is faster up to 17,000 (short fp16 rows) to 48,000 (2,000 bf16) logits
// per pair of equal lengths, up to 12,000 to 32,000 where lengths go from 1 to 3; the limit is the middle of these.
// 4 pairs of 24 rows of 1,000 fp32 8.7 us and 10.9 in two (lengths from 1 to 3: 10.8 and 10.9), of 32 rows 10.8 and
// 10.7, of 48 13.7 and 10.8; but 3 of 88 rows of 269 fp16, which take one, 11.8 and 10.9 (from 1 to 3: 15.3 and 10.8).
// In a graph two win from 10,000 to 27,000 on (24 rows of 1,000 fp32 8.6 and 7.7).  More pairs than CUs take turns: 512
// of 8 rows of 128 fp16 11.7, 1,000 of 4 rows of 100 fp32 17.8 (two launches 10.2), of 4 rows of 20 18.1 (20.7).
// A pair that has all 524,288 logits takes 76 us (2,048 rows of 256 bf16) to 106 (4,096 of 128 fp32).
constexpr int64_t kSmallLogits = int64_t{1} << 19, kSmallPairLogits = 24576;
// Few rows (on average, of a pair) and bytes take two launches, the second of which sums the pairs again
// for every row, or part of one: 566 rows of 3,902 bf16 in 55 pairs 11.9 us a call, three launches 14.2 (in a graph
// 10.3 and 12.0); 1,000 in 10 pairs 12.6 and 14.7; 4,000 of 1,500 in 20 14.0 and 15.5; but 2,000 of 3,902 18.3 and
// 17.4, 486 of 22,737 fp16 in 43 23.7 and 21.4, 4,096 of 20,000 152 and 80.  A wave sums its rows' pairs in
// turn, but of rows past the limit above it has few: 4,000 of 256 bf16 in 1,000 pairs 10.7 and 17.9 (lengths from 1 to 3:
// 16.0 and 17.8), 4,000 of 200 in 4,000 23 and 45.  A single pair among thousands that has all the rows costs 16 loads in turn.
constexpr int64_t kLongPairRows = 20480;
constexpr int64_t kFewRows = kChunk, kFewPairRows = 512, kFewBytes = int64_t{1} << 23, kFewBytesOfWaves = int64_t{1} << 24;

template <class T>
hipError_t launch_small(const LogitsArgs& a, const PairArgs& p, hipStream_t stream) {
  const int64_t vectors = (a.cols + Vec<T>::kN - 1) / Vec<T>::kN;
  auto run = [&](auto kernel) {
    kernel<<<static_cast<uint32_t>(p.pairs), kPairThreads, 0, stream>>>(a, p);
    return hipGetLastError();
  };
  if (vectors <= 1) return run(small_preference_kernel<T, 1, 1, 0>);
  if (vectors <= 2) return run(small_preference_kernel<T, 1, 2, 0>);
  if (vectors <= 4) return run(small_preference_kernel<T, 1, 4, 0>);
  if (vectors <= 8) return run(small_preference_kernel<T, 2, 4, 0>);
  if (vectors <= 16) return run(small_preference_kernel<T, 4, 4, 0>);
  if (vectors <= 32) return run(small_preference_kernel<T, 8, 4, 0>);
  if (vectors <= 64) return run(small_preference_kernel<T, 16, 4, 0>);
  if (vectors <= kShortVectors) return run(small_preference_kernel<T, 32, 4, 0>);
  if (in_threes(a.cols / Vec<T>::kN)) return run(small_preference_kernel<T, 64, 1, 3>);
  return run(small_preference_kernel<T, 64, 1, 4>);
}

}  // namespace

hipError_t launch_logits(const LogitsArgs& a, RowMode mode, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PGC_F32: return launch_typed<float>(a, mode, stream);
    case PGC_BF16: return launch_typed<__bf16>(a, mode, stream);
    default: return launch_typed<_Float16>(a, mode, stream);
  }
}

// Few rows need no launch between their log-probabilities and their gradient.
bool preference_sums_in_gradient(int64_t rows, int64_t cols, int64_t pairs, int dtype) {
  const int64_t row_bytes = cols * (dtype == PGC_F32 ? 4 : 2);
  return pairs > 0 && pairs <= kFewRows && rows <= std::min(kFewRows, kFewPairRows * pairs) &&
         rows * row_bytes <= (row_bytes <= 4 * kWave * 16 ? kFewBytesOfWaves : kFewBytes);   // a wave or less to a row, or more
}

hipError_t launch_pair_gradient(const LogitsArgs& a, const PairArgs& p, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PGC_F32: return launch_backward<float>(a, stream, PairFactors{p});
    case PGC_BF16: return launch_backward<__bf16>(a, stream, PairFactors{p});
    default: return launch_backward<_Float16>(a, stream, PairFactors{p});
  }
}

hipError_t launch_scores_gradient(const ScoresArgs& s, int dtype, hipStream_t stream) {
  LogitsArgs a{};
  a.logits = s.logits;
  a.targets = s.targets;
  a.rows = s.rows;
  a.cols = s.cols;
  a.stride = s.stride;
  a.out_stride = s.out_stride;
  a.dlogits = s.dlogits;
  a.stats = s.stats;
  const ScoresFactors factors{s.grad_logprobs, s.grad_entropy, s.entropy};
  switch (dtype) {
    case PGC_F32: return launch_backward<float>(a, stream, factors);
    case PGC_BF16: return launch_backward<__bf16>(a, stream, factors);
    default: return launch_backward<_Float16>(a, stream, factors);
  }
}

int64_t pair_chunk_places(int64_t rows, int64_t pairs) { return rows / kChunk + pairs; }

hipError_t launch_pairs(const PairArgs& a, hipStream_t stream) {
  // Long pairs on average: 1,048,576 rows of 20 fp16 in one pair 36 us, by a block per pair 214; 170,950 of 58
  // bf16 in 4 21 and 28; 104,502 of 12 fp32 in 10 15.8 and 13.8.
  if (a.rows / kLongPairRows >= a.pairs) {
    const uint32_t places = static_cast<uint32_t>(pair_chunk_places(a.rows, a.pairs));
    chunk_sum_kernel<<<places, kPairThreads, 0, stream>>>(a);
    chunk_gradient_kernel<<<places, kPairThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  pair_kernel<<<static_cast<int>(std::min(a.pairs, kGridX)), kPairThreads, 0, stream>>>(a);
  return hipGetLastError();
}

bool preference_is_small(int64_t rows, int64_t cols, int64_t pairs, int dtype) {
  const int64_t row_bytes = cols * (dtype == PGC_F32 ? 4 : 2);
  return pairs > 0 && pairs <= kSmallRows && rows <= kSmallRows && row_bytes < 513 * 16 &&
         rows * cols <= std::min(kSmallLogits, kSmallPairLogits * pairs);
}

hipError_t launch_small_preference(const LogitsArgs& a, const PairArgs& p, int dtype, hipStream_t stream) {
  switch (dtype) {
    case PGC_F32: return launch_small<float>(a, p, stream);
    case PGC_BF16: return launch_small<__bf16>(a, p, stream);
    default: return launch_small<_Float16>(a, p, stream);
  }
}

}  // namespace pgc
