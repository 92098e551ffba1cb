// Drawing the next tokens: one token per row of logits, with temperature, top-k, top-p and min-p, from given random numbers.
//
// With x = logit / temperature, a token weighs w = exp(x - largest x). The kept tokens are a prefix of the row in the order (larger logit first, of
// equal ones the lower index): the shorter one of what top-k, top-p and min-p leave. The draw is the lowest index at which the sum of kept
// weights, taken in index order, passes u times their total. A token is a whole number that has one right value, so weights and sums are held in 64
// bits, and no sum's order depends on the order in which threads arrive: where those meet they add integers.
//
// What bounds it: the logits are read from memory once (and once more from the caches where a cut has to be found); a launch or a fp64 operation
// per token cost as much. So a row is never sorted. It is cut into slices, a workgroup each:
//   1 slices   the largest logit; a histogram of tokens and their weights over bins of a quarter octave (factor 2^(1/4)) of weight. Where there
//              is no filter the sum of weights alone.
//   2 decide   (filters only, a workgroup per row) adds up the row's histograms and sees in which bins the cuts lie.
//   3 collect  (filters only) every slice's workgroup makes a finer histogram of those bins, 256 parts, and a list of their tokens.
//   4 draw     a workgroup per row: finds the parts in which the cuts lie, compares the few tokens of such a part with each other, then finds
//              the slice with the drawn token from the slices' kept weights, and the token in it.
// A weight in a histogram is an integer in steps of 2^-35 of its bin's middle, in 64 bits beside the count; without filters it is
// rounded to 2^-34 of its octave's middle, at most 2^-34.5 of itself. A logit's place on the scale of bins is a product in twice 64 bits, so what all
// logits of a row have in common, a large number at a low temperature, costs a weight nothing. Equal logits have equal weights, and the sum
// of up to 2^17 tokens that all have the largest one is exact.
//
// us of the four kernels: 1 row of 32000 tokens, bf16, all filters 5, 4, 6, 21 (chains of latencies: the draw's are some 15 steps of 0.3 to 2); 128 rows of 131072,
// bf16 16, 6, 13, 28; 200 of 150001, f16, top-p 27, 7, 22, 24; 777 of 32768, fp32 26, 6, 23, 36; 64 of 131072, fp32, no filter 12 and 8. The first kernel without
// its histogram takes 10, 13 and 19 of the 16, 27 and 25: 18 operations and an atomic per token, and what a launch of so many loads takes to begin and end.
#include <float.h>
#include <math.h>

#include "paged_kv.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kBins = 256;                 // of weight; the last one has all that is lighter, whose weight does not count (2^-63 of the largest)
constexpr int kCountBits = 14;             // of a slice's bin: tokens below, weight in steps of kStep above
constexpr double kStep = 0x1p-35;
// A slice's histogram in LDS: neighbours add to different copies, and what is too light for the bins goes to places of its own per lane, or masked
// tokens would all wait for one (200 x 150001 tokens, 70 % of them masked: 86 us with 1 copy and 1 place, 38 with 4 copies and 1 place, 30 with both).
constexpr int kCopies = 4, kPlaces = kBins - 1 + 64;
// Tokens of a slice. (Half as many, twice as many slices: 1 row of 32000 tokens 33.6 us for 34.8, 1 of 262144 45 for 40.)
constexpr int kSlice = 8192, kSliceThreads = 256;
constexpr int kMostDraw = 1024, kHeld = 2048, kRanked = 256;   // tokens that are held in LDS, and that are compared with each other
constexpr int kParts = 256;                // of the cut bins
constexpr int kListed = 1024;              // tokens of a slice's cut bins that are listed; where it has more, they are looked for in the slice again
constexpr int kMostVocab = 1 << 20, kMostSlices = kMostVocab / kSlice + 1;

struct Slice {
  double top;       // middle of the bin, or octave (no filter), of the largest x
  double sum;       // weights relative to 2^top (no filter)
  float most;       // largest logit; -infinity: none
  int32_t first;    // its lowest index (greedy)
  int32_t nan, pad;
};
// What a row's filters come to, by bins.
struct Cut {
  int32_t from, upto;      // bins in which the last kept token may be; kBins: all are kept
  int32_t k_bin, k_left;   // bin in which top-k ends, tokens it keeps there; kBins: nowhere
  int32_t p_on, k_too;     // k_too: that bin, behind `upto`, matters for the weight that top-p takes a share of
  double all;              // weight of all tokens
  double least;            // least number that a logit may be for min-p
  double upto_weight[kBins];   // weight of bins 0 .. b, relative to the middle of bin 0
  int32_t upto_count[kBins];
};
struct Entry {
  uint32_t key, index;
};

struct Params {
  const char *logits;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t *top_k;
  int32_t *tokens;
  float *logprob;
  float all_temperature, all_top_p, all_min_p;
  int32_t all_top_k;
  int64_t row_stride;      // elements
  int32_t n_rows, vocab, n_slices, filters;
  Slice *slices;           // [row][slice]
  unsigned long long *bins;   // [row][slice][kBins]
  Cut *cuts;               // [row]
  unsigned long long *parts;   // [row][slice][2][kParts]: of bins from .. upto, as many of each; of the bin of top-k where k_too
  int32_t *listed;         // [row][slice]: tokens in them
  Entry *lists;            // [row][slice][kListed]
};

struct Row {
  double per_bin;          // bins per unit of logit; not 0
  float t, p, m;
  int k;
  bool greedy, filtered;
};
__device__ __forceinline__ Row row_of(const Params &p, int r) {
  Row w;
  const float t = p.temperature ? p.temperature[r] : p.all_temperature;
  w.t = t;
  w.p = p.top_p ? p.top_p[r] : p.all_top_p;
  w.m = p.min_p ? p.min_p[r] : p.all_min_p;
  w.k = p.top_k ? p.top_k[r] : p.all_top_k;
  if (!(w.p < 1.0f)) w.p = 1.0f;
  if (!(w.m > 0.0f)) w.m = 0.0f;
  if (w.m > 1.0f) w.m = 1.0f;
  if (w.k <= 0 || w.k >= p.vocab) w.k = 0;
  // An infinite temperature: logits that are numbers weigh the same, so all of them lie within 2^-60 of a bin, and min-p cuts nothing; +infinity is
  // far from them even then (number_of).
  const bool hot = t == INFINITY;
  if (hot) w.m = 0.0f;
  w.greedy = !(t > 0.0f);
  w.filtered = !w.greedy && (w.k > 0 || w.p < 1.0f || w.m > 0.0f);
  w.per_bin = hot ? 0x1p-190 : 4.0 * 1.4426950408889634 / static_cast<double>(t);
  return w;
}

// ---- logits
template <typename T>
__device__ __forceinline__ float as_float(T x);
template <>
__device__ __forceinline__ float as_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float as_float<__bf16>(__bf16 x) { return static_cast<float>(x); }
template <>
__device__ __forceinline__ float as_float<_Float16>(_Float16 x) { return static_cast<float>(x); }

// 16 bytes of logits from place `at` of the row's aligned grid, whose place `skew` is the row's first; places outside of the row are -infinity.
template <typename T, int N = 16 / sizeof(T)>
__device__ __forceinline__ void load16(const T *grid, int at, int skew, int vocab, float (&x)[N]) {
  if (at >= skew && at + N <= skew + vocab) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(grid + at);
    T v[N];
    __builtin_memcpy(v, &w, 16);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = as_float(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = at + i >= skew && at + i < skew + vocab ? as_float(grid[at + i]) : -INFINITY;
  }
}
template <typename T>
struct RowAt {
  const T *grid;   // 16-byte aligned
  int skew;
  __device__ __forceinline__ RowAt(const Params &p, int r) {
    const char *a = p.logits + r * p.row_stride * static_cast<int64_t>(sizeof(T));
    skew = static_cast<int>((reinterpret_cast<uintptr_t>(a) & 15) / sizeof(T));
    grid = reinterpret_cast<const T *>(a) - skew;
  }
};

// A slice's logits, kVectors x 16 bytes per thread, neighbours by neighbours. All are asked for before any is waited for, which takes a branch
// that is the same for all of them.
template <typename T, int kVectors, int N = 16 / sizeof(T)>
__device__ __forceinline__ void load_slice(const RowAt<T> &row, const Params &p, int s, float (&x)[kVectors][N]) {
  const int at = s * kSlice + static_cast<int>(threadIdx.x) * N;
  if (s * kSlice >= row.skew && (s + 1) * kSlice <= row.skew + p.vocab) {
    u32x4 w[kVectors];
#pragma unroll
    for (int v = 0; v < kVectors; ++v) w[v] = *reinterpret_cast<const u32x4 *>(row.grid + at + v * kSliceThreads * N);
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
      T t[N];
      __builtin_memcpy(t, &w[v], 16);
#pragma unroll
      for (int i = 0; i < N; ++i) x[v][i] = as_float(t[i]);
    }
  } else {
#pragma unroll
    for (int v = 0; v < kVectors; ++v) load16(row.grid, at + v * kSliceThreads * N, row.skew, p.vocab, x[v]);
  }
}

// Order-preserving key; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
// Larger logits first, of equal ones the lower index.
__device__ __forceinline__ unsigned long long rank_of(uint32_t key, uint32_t index) { return static_cast<unsigned long long>(~key) << 32 | index; }
// A logit's place on the scale of bins (or octaves): the nearest bin's middle by the rounded product, and how far from it the product itself is,
// -1/2 to 1/2 and what its rounding may add. From places of 2^36 on (kFar) that is taken as 0: neighbouring logits in 32 bits are 2^12 bins apart
// there, so what is not equal to the largest one weighs nothing beside it (596 bins are the lightest weight that min-p can keep, 1075 octaves the
// lightest number). Places never decrease with the logit, bin by bin and within a bin.
constexpr double kFar = 0x1p36;
struct Place {
  double bin, rest;
};
// Not of places beyond kFar, whose rest may be anything.
__device__ __forceinline__ Place near_place_of(double x, double per_bin) {
  Place a;
  a.bin = rint(x * per_bin);
  a.rest = fma(x, per_bin, -a.bin);
  return a;
}
__device__ __forceinline__ Place place_of(double x, double per_bin) {
  Place a = near_place_of(x, per_bin);
  if (!(fabs(a.bin) < kFar)) a.rest = 0.0;
  return a;
}
__device__ __forceinline__ double number_of(float x) { return x == INFINITY ? 0x1p300 : static_cast<double>(x); }
__device__ __forceinline__ int bin_of(double top, double bin) { return static_cast<int>(fmin(top - bin, kBins - 1.0)); }   // (a NaN's: the last one)

// 2^(z / 4) for |z| <= 1/2 in steps of kStep, with 1 added in the kCountBits bits below: a polynomial through the function's values at Chebyshev's
// points, 1.3e-13 off at most, times 2^49. The last addition leaves its whole part in the sum's mantissa.
__device__ __forceinline__ unsigned long long step_and_one(double z) {
  double s = 0x1p49 * 3.7615098597694156e-08;
  s = fma(s, z, 0x1p49 * 1.3025126327701222e-06);
  s = fma(s, z, 0x1p49 * 3.757081572373334e-05);
  s = fma(s, z, 0x1p49 * 0.0008672516469677146);
  s = fma(s, z, 0x1p49 * 0.01501415668497826);
  s = fma(s, z, 0x1p49 * 0.1732867951415776);
  s = fma(s, z, 0x1p52 + 0x1p49 + (1 << (kCountBits - 1)));
  const unsigned long long b = __double_as_longlong(s);
  return static_cast<unsigned long long>(static_cast<uint32_t>(b >> 32) & 0xfffff) << 32 | ((static_cast<uint32_t>(b) & (0u - (1u << kCountBits))) | 1u);
}
static_assert(kCountBits == 14, "2^49 of weight and the count's bits make steps of 2^-35");
__device__ __forceinline__ unsigned long long steps_of(double z) { return step_and_one(z) >> kCountBits; }
// 2^z for |z| <= 1/2, rounded to 2^-34: the same, 1.1e-12 off at most.
__device__ __forceinline__ double in_octave(double z) {
  double s = 1.3255224883636123e-06;
  s = fma(s, z, 1.531007940226575e-05);
  s = fma(s, z, 0.000154034558524266);
  s = fma(s, z, 0.001333345056800051);
  s = fma(s, z, 0.009618129159402605);
  s = fma(s, z, 0.05550410941205933);
  s = fma(s, z, 0.24022650695812986);
  s = fma(s, z, 0.6931471805459334);
  return fma(s, z, 1.0 + 0x1.8p18) - 0x1.8p18;
}
// 2^(-b / 4): the middle of bin b, relative to that of bin 0
__device__ __forceinline__ double middle_of(int b) {
  const double r = b & 2 ? 0.7071067811865476 : 1.0;
  return ldexp(b & 1 ? r * 0.8408964152537145 : r, -(b >> 2));
}

// Over the lanes of a wave: within rows of 16, then rows to the rows behind them.
template <int kControl, int kRowMask, typename V>
__device__ __forceinline__ V moved(V x, V none) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "");
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), kControl, kRowMask, 0xf, false));
  } else {
    const unsigned long long a = __builtin_bit_cast(unsigned long long, x), n = __builtin_bit_cast(unsigned long long, none);
    const uint32_t lo = __builtin_amdgcn_update_dpp(static_cast<int>(n), static_cast<int>(a), kControl, kRowMask, 0xf, false),
                   hi = __builtin_amdgcn_update_dpp(static_cast<int>(n >> 32), static_cast<int>(a >> 32), kControl, kRowMask, 0xf, false);
    return __builtin_bit_cast(V, static_cast<unsigned long long>(hi) << 32 | lo);
  }
}
template <typename V, typename F>
__device__ __forceinline__ V wave_scan(V x, V none, F &&join) {   // inclusive
  x = join(moved<0x111, 0xf>(x, none), x);
  x = join(moved<0x112, 0xf>(x, none), x);
  x = join(moved<0x114, 0xf>(x, none), x);
  x = join(moved<0x118, 0xf>(x, none), x);
  x = join(moved<0x142, 0xa>(x, none), x);
  return join(moved<0x143, 0xc>(x, none), x);
}
template <typename V>
__device__ __forceinline__ V of_lane(V x, int lane) {   // (the same lane for all)
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
  } else {
    const unsigned long long a = __builtin_bit_cast(unsigned long long, x);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(a), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(a >> 32), lane);
    return __builtin_bit_cast(V, static_cast<unsigned long long>(hi) << 32 | lo);
  }
}
template <typename V>
__device__ __forceinline__ V of_last_lane(V x) { return of_lane(x, 63); }
template <typename V>
__device__ __forceinline__ V wave_sums(V x) {
  return wave_scan(x, V(0), [](V a, V b) { return a + b; });
}
template <typename V>
__device__ __forceinline__ V wave_sum(V x) { return of_last_lane(wave_sums(x)); }
__device__ __forceinline__ float wave_max(float x) { return of_last_lane(wave_scan(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); })); }
template <typename V>
__device__ __forceinline__ V wave_min(V x, V most) {
  return of_last_lane(wave_scan(x, most, [](V a, V b) { return a < b ? a : b; }));
}
// Inclusive sums over a workgroup's threads; `waves` is LDS of a number per wave (16 at most).
template <int kThreads, typename V>
__device__ __forceinline__ V block_scan(V x, V *waves) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  x = wave_sums(x);
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  return x + wave_sum(lane < wave ? waves[lane & (kThreads / 64 - 1)] : V(0));
}

// The first, or last, thread of a workgroup for which `is`: one lane of a wave asks, for atomics of many lanes to one address go one by one.
__device__ __forceinline__ void first_thread(bool is, int *found) {
  const unsigned long long m = __ballot(is);
  if (m != 0 && (threadIdx.x & 63) == 0) atomicMin(found, static_cast<int>(threadIdx.x) + __ffsll(m) - 1);
}
__device__ __forceinline__ void last_thread(bool is, int *found) {
  const unsigned long long m = __ballot(is);
  if (m != 0 && (threadIdx.x & 63) == 0) atomicMax(found, static_cast<int>(threadIdx.x) + 63 - __clzll(m));
}

// ---- 1
template <typename T, int kVectors>   // 16-byte vectors per thread
__device__ __forceinline__ void one_slice(const Params &p, int r, int s) {
  constexpr int N = 16 / sizeof(T);
  __shared__ unsigned long long hist[kCopies][kPlaces];
  __shared__ double sums[kSliceThreads / 64];
  __shared__ float tops[kSliceThreads / 64];
  __shared__ int firsts[kSliceThreads / 64], nans[kSliceThreads / 64];
  const Row w = row_of(p, r);
  const RowAt<T> row(p, r);
  float x[kVectors][N];
  float most = -INFINITY;
  bool nan = false;
  load_slice(row, p, s, x);
  if (w.filtered)
#pragma unroll
    for (int i = 0; i < kCopies; ++i) hist[i][threadIdx.x] = 0;
#pragma unroll
  for (int v = 0; v < kVectors; ++v)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      most = fmaxf(most, x[v][i]);
      nan |= x[v][i] != x[v][i];
    }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  most = wave_max(most);
  const bool wave_nan = __any(nan);
  if (lane == 0) {
    tops[wave] = most;
    nans[wave] = wave_nan;
  }
  __syncthreads();
  bool any_nan = false;
  for (int i = 0; i < kSliceThreads / 64; ++i) {
    most = fmaxf(most, tops[i]);
    any_nan |= nans[i] != 0;
  }
  Slice out{};
  out.most = most;
  out.nan = any_nan;
  if (!any_nan && most > -INFINITY) {
    const auto each = [&](auto &&f) {
#pragma unroll
      for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int i = 0; i < N; ++i) f(x[v][i]);
    };
    const double unit = w.filtered ? w.per_bin : 0.25 * w.per_bin;
    out.top = place_of(number_of(most), unit).bin;
    const bool far = fabs(out.top) >= kFar;   // then what is not equal to the largest logit weighs nothing
    if (far && !w.greedy) each([&](float &y) { y = y == most ? 0.0f : -INFINITY; });
    const double top = far ? 0.0 : out.top;
    if (w.greedy) {
      int first = INT32_MAX;
#pragma unroll
      for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int i = N - 1; i >= 0; --i) {
          const int at = s * kSlice + (v * kSliceThreads + static_cast<int>(threadIdx.x)) * N + i - row.skew;
          if (x[v][i] == most && at < first) first = at;
        }
      first = wave_min(first, INT32_MAX);
      if (lane == 0) firsts[wave] = first;
      __syncthreads();
      for (int i = 0; i < kSliceThreads / 64; ++i) first = firsts[i] < first ? firsts[i] : first;
      out.first = first;
    } else if (!w.filtered) {
      double sum = 0.0;
      each([&](float y) {   // (far below the largest one, where `rest` is any number, or a NaN for -infinity, the weight is 0)
        const Place a = near_place_of(static_cast<double>(y), unit);
        sum += ldexp(in_octave(fmin(fmax(a.rest, -0.75), 0.75)), static_cast<int>(fmax(a.bin - top, -2000.0)));
      });
      sum = wave_sum(sum);
      if (lane == 0) sums[wave] = sum;
      __syncthreads();
      out.sum = 0.0;
      for (int i = 0; i < kSliceThreads / 64; ++i) out.sum += sums[i];
    } else {
      const double lightest = kBins - 1.0 + lane;
      unsigned long long *mine = hist[threadIdx.x % kCopies];
      each([&](float y) {
        const Place a = near_place_of(static_cast<double>(y), unit);
        const int b = static_cast<int>(fmin(top - a.bin, lightest));   // (of -infinity: the lane's own, whether the difference is infinite or a NaN)
        atomicAdd(&mine[b], step_and_one(a.rest));
      });
    }
  }
  if (w.filtered) {
    __syncthreads();
    unsigned long long sum = 0;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) sum += hist[i][threadIdx.x];
    p.bins[(static_cast<int64_t>(r) * p.n_slices + s) * kBins + threadIdx.x] = sum;
  }
  if (threadIdx.x == 0) p.slices[static_cast<int64_t>(r) * p.n_slices + s] = out;
}
template <typename T>
__global__ __launch_bounds__(kSliceThreads) void sample_slices_kernel(Params p) {
  const int r = blockIdx.x / p.n_slices, s = blockIdx.x - r * p.n_slices;
  one_slice<T, kSlice * static_cast<int>(sizeof(T)) / 16 / kSliceThreads>(p, r, s);
}

// ---- what both other kernels begin with: the row's largest logit and whether there is a draw
struct Whole {
  float most;
  bool nan;
  double top;
};
__device__ __forceinline__ Whole whole_of(const Params &p, int r) {   // by every wave for itself
  Whole a{-INFINITY, false, 0.0};
  const Slice *const s = p.slices + static_cast<int64_t>(r) * p.n_slices;
  for (int i = threadIdx.x & 63; i < p.n_slices; i += 64) {
    a.most = fmaxf(a.most, s[i].most);
    a.nan |= s[i].nan != 0;
  }
  a.most = wave_max(a.most);
  a.nan = __any(a.nan);
  return a;
}
// The least number that a logit may be to be kept by min-p: the sum of the largest one and b = t log(m), rounded up (its rounding error is what the
// three subtractions find). Rounding keeps the order of numbers, so a kept logit's place is not behind this one's, nor one that is not kept ahead.
__device__ __forceinline__ double least_of(float most, double b) {
#pragma clang fp contract(off)
  const double a = number_of(most), sum = a + b, of_b = sum - a;
  const double lost = (a - (sum - of_b)) + (b - of_b);
  if (!(lost > 0.0)) return sum;
  const long long bits = __double_as_longlong(sum);
  return __longlong_as_double(sum > 0.0 ? bits + 1 : bits - 1);   // (a sum of 0 is exact)
}
// Bins that a slice's are behind the row's.
__device__ __forceinline__ int behind(double top, double slice_top) { return static_cast<int>(fmin(top - slice_top, 1e6)); }

// ---- 2
__global__ __launch_bounds__(kBins) void sample_decide_kernel(Params p) {
  __shared__ double weight[kBins];
  __shared__ unsigned long long steps[kBins];
  __shared__ int count[kBins], off[kMostSlices], found[3];
  __shared__ double dwaves[kBins / 64];
  __shared__ int iwaves[kBins / 64];
  const int r = blockIdx.x, b = threadIdx.x;
  const Row w = row_of(p, r);
  if (!w.filtered) return;
  const Slice *const slices = p.slices + static_cast<int64_t>(r) * p.n_slices;
  const unsigned long long *const bins = p.bins + static_cast<int64_t>(r) * p.n_slices * kBins;
  steps[b] = 0;
  count[b] = 0;
  if (b < 3) found[b] = kBins;
  // the row's histogram, 16 slices at a time: their numbers are asked for before it is known how far they have to be moved
  constexpr int kAtOnce = 16;
  unsigned long long h[kAtOnce];
  const auto ask = [&](int base) {
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) h[j] = base + j < p.n_slices ? bins[(base + j) * kBins + b] : 0;
  };
  ask(0);
  const double t_log_m = w.m > 0.0f ? static_cast<double>(w.t) * log(static_cast<double>(w.m)) : 0.0;   // (while the numbers are on their way)
  Whole all = whole_of(p, r);
  if (all.nan || all.most == -INFINITY) return;
  all.top = place_of(number_of(all.most), w.per_bin).bin;
  for (int i = b; i < p.n_slices; i += kBins) off[i] = slices[i].most > -INFINITY ? behind(all.top, slices[i].top) : kBins;
  __syncthreads();
  for (int base = 0; base < p.n_slices; base += kAtOnce) {
    if (base > 0) ask(base);
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (base + j < p.n_slices && b < kBins - 1 && b + off[base + j] < kBins - 1 && h[j] != 0) {
        atomicAdd(&steps[b + off[base + j]], h[j] >> kCountBits);
        atomicAdd(&count[b + off[base + j]], static_cast<int>(h[j] & ((1u << kCountBits) - 1)));
      }
  }
  __syncthreads();
  weight[b] = block_scan<kBins>(static_cast<double>(steps[b]) * kStep * middle_of(b), dwaves);
  const int upto_here = block_scan<kBins>(count[b], iwaves);
  count[b] = upto_here;
  __syncthreads();
  const double total = weight[kBins - 1];
  // top-k ends in the first bin up to which there are k tokens
  first_thread(w.k > 0 && count[b] >= w.k, &found[0]);
  __syncthreads();
  const int k_bin = found[0], k_ahead = k_bin > 0 && k_bin < kBins ? count[k_bin - 1] : 0, k_left = k_bin < kBins ? w.k - k_ahead : 0;
  const bool k_inside = k_bin < kBins && count[k_bin] > w.k;
  const bool p_on = w.p < 1.0f;
  int from = kBins, upto = kBins;
  if (p_on) {
    // the weight that top-k leaves is known to within its last bin; the last token of top-p lies in one of these bins
    const double k_low = k_bin == kBins ? total : k_inside ? (k_bin > 0 ? weight[k_bin - 1] : 0.0) + k_left * middle_of(k_bin + 1) : weight[k_bin];
    const double k_high = k_bin == kBins ? total : weight[k_bin];
    const double low = w.p * k_low * (1.0 - 1e-9), high = w.p * k_high * (1.0 + 1e-9);
    first_thread(weight[b] >= low, &found[1]);
    first_thread(weight[b] >= high, &found[2]);
    __syncthreads();
    from = found[1];
    upto = found[2];
    if (upto > k_bin) upto = k_bin;
    if (from > upto) from = upto;
  } else if (k_bin < kBins) {
    from = upto = k_bin;
  }
  const double least = least_of(all.most, t_log_m);
  if (w.m > 0.0f) {
    const int m_bin = bin_of(all.top, place_of(least, w.per_bin).bin);
    if (m_bin < from) from = m_bin;
    if (m_bin < upto) upto = m_bin;
  }
  if (from > kBins - 2)
    from = upto = kBins;
  else if (upto > kBins - 2)
    upto = kBins - 2;
  Cut *const c = p.cuts + r;
  c->upto_weight[b] = weight[b];
  c->upto_count[b] = count[b];
  if (b == 0) {
    c->from = from;
    c->upto = upto;
    c->k_bin = k_bin;
    c->k_left = k_left;
    c->k_too = p_on && k_inside && k_bin > upto;
    c->p_on = p_on;
    c->all = total;
    c->least = least;
  }
}

// Logits among which are all of bins `first` .. `last`, few others, and never -infinity.
struct Interval {
  float low, high;
};
__device__ __forceinline__ Interval interval_of(double top, double first, double last, double per_bin) {
  if (!(per_bin > 0.0)) return Interval{-FLT_MAX, INFINITY};
  const double high = (top - first + 0.5) / per_bin, low = (top - last - 0.5) / per_bin;
  return Interval{fmaxf(static_cast<float>(low - fabs(low) * 1e-6 - 3e-45), -FLT_MAX), static_cast<float>(high + fabs(high) * 1e-6 + 3e-45)};
}
// A bin's part, of n: the lightest tokens are in the last one. (`rest` may be past 1/2 by 2^-18, which the conversion makes part 0 as well.)
__device__ __forceinline__ int part_of(double rest, int n) {
  const int i = static_cast<int>((0.5 - rest) * n);
  return i < n - 1 ? i : n - 1;
}

// ---- 3
template <typename T, int kVectors>
__device__ __forceinline__ void collect(const Params &p, int r, int s) {
  constexpr int N = 16 / sizeof(T);
  static_assert(kVectors * N <= 32, "a bit per logit");
  __shared__ unsigned long long parts[2][kParts];
  __shared__ int n;
  const RowAt<T> row(p, r);
  float x[kVectors][N];
  load_slice(row, p, s, x);
  const Row w = row_of(p, r);
  if (!w.filtered) return;
  const Whole all = whole_of(p, r);
  if (all.nan || all.most == -INFINITY) return;
  const Cut &c = p.cuts[r];
  const int from = c.from, upto = c.upto, k_bin = c.k_too ? c.k_bin : -1;
  if (from == kBins && k_bin < 0) return;
  const double top = place_of(number_of(all.most), w.per_bin).bin;
  parts[0][threadIdx.x] = 0;
  parts[1][threadIdx.x] = 0;
  if (threadIdx.x == 0) n = 0;
  __syncthreads();
  Interval a = {INFINITY, -INFINITY}, b = a;   // (none)
  if (from < kBins) a = interval_of(top, from, upto, w.per_bin);
  if (k_bin >= 0) b = interval_of(top, k_bin, k_bin, w.per_bin);
  uint32_t hits = 0;
#pragma unroll
  for (int v = 0; v < kVectors; ++v)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((x[v][i] >= a.low && x[v][i] <= a.high) || (x[v][i] >= b.low && x[v][i] <= b.high)) hits |= 1u << (v * N + i);
  const int per_bin = kParts / (upto - from + 1);
  Entry *const list = p.lists + (static_cast<int64_t>(r) * p.n_slices + s) * kListed;
  while (hits) {
    const int j = __ffs(hits) - 1;
    hits &= hits - 1;
    const int place = s * kSlice + (j / N * kSliceThreads + static_cast<int>(threadIdx.x)) * N + j % N;
    const float y = as_float(row.grid[place]);
    const Place q = place_of(number_of(y), w.per_bin);
    const int bin = bin_of(top, q.bin);
    if ((bin < from || bin > upto) && bin != k_bin) continue;
    if (bin == k_bin)
      atomicAdd(&parts[1][part_of(q.rest, kParts)], step_and_one(q.rest));
    else
      atomicAdd(&parts[0][(bin - from) * per_bin + part_of(q.rest, per_bin)], step_and_one(q.rest));
    const int at = atomicAdd(&n, 1);   // (their order does not matter)
    if (at < kListed) list[at] = Entry{key_of(y), static_cast<uint32_t>(place - row.skew)};
  }
  __syncthreads();
  const int64_t slot = static_cast<int64_t>(r) * p.n_slices + s;
  if (threadIdx.x == 0) p.listed[slot] = n;
  if (n > 0) {
    p.parts[slot * 2 * kParts + threadIdx.x] = parts[0][threadIdx.x];
    if (k_bin >= 0) p.parts[(slot * 2 + 1) * kParts + threadIdx.x] = parts[1][threadIdx.x];
  }
}
template <typename T>
__global__ __launch_bounds__(kSliceThreads) void sample_collect_kernel(Params p) {
  const int r = blockIdx.x / p.n_slices, s = blockIdx.x - r * p.n_slices;
  collect<T, kSlice * static_cast<int>(sizeof(T)) / 16 / kSliceThreads>(p, r, s);
}

// ---- 4
struct DrawLds {
  unsigned long long ranks[kHeld];
  unsigned long long near[kRanked], steps[kRanked];
  unsigned long long part[kMostDraw];
  int part_count[kMostDraw];
  double dwaves[kMostDraw / 64];
  unsigned long long low, high, rank;
  double of_slice[kMostSlices];
  double top_of_slice[kMostSlices];   // -infinity: it has no token
  double upto_weight[kBins];
  int upto_count[kBins];
  float tops[kMostDraw / 64];
  int flags[kMostDraw / 64];
  unsigned long long cut_steps[kMostSlices];
  int listed[kMostSlices];
  double d;
  int i[4];
};
// A row that is drawn from.
template <typename T, int kDrawThreads>
struct Drawn {
  const Params &p;
  DrawLds &l;
  const Row &w;
  int r;
  double top;
  int from, upto, k_bin;   // k_bin: -1 where it has no parts of its own
  bool unlisted;           // some slice's tokens are not listed
  int lanes;               // threads per slice that read its list
  Entry mine;              // first one that this thread reads
  __device__ __forceinline__ Place place(uint32_t key) const { return place_of(number_of(of_key(key)), w.per_bin); }
  __device__ __forceinline__ int parts_of(int bin) const { return bin == k_bin ? kParts : kParts / (upto - from + 1); }
  __device__ __forceinline__ int first_part(int bin) const { return bin == k_bin ? kParts : (bin - from) * parts_of(bin); }
  // Calls f(key, index) for the tokens in the cut bins, or for those of them that `in` has.
  template <typename F>
  __device__ __forceinline__ void each(int t, int r, Interval in, F &&f) const {
    const int s_mine = t / lanes, n = s_mine < p.n_slices && l.listed[s_mine] <= kListed ? l.listed[s_mine] : 0;
    const Entry *const list = p.lists + (static_cast<int64_t>(r) * p.n_slices + s_mine) * kListed;
    Entry e = mine;
#pragma unroll 1
    for (int i = t & (lanes - 1); i < n; i += lanes) {
      if (i >= lanes) e = list[i];
      f(e.key, e.index);
    }
    if (!unlisted) return;
    constexpr int N = 16 / sizeof(T), kUnits = 4;   // a slice is the work of 4 waves
    const RowAt<T> row(p, r);
#pragma unroll 1
    for (int u = t >> 6; u < p.n_slices * kUnits; u += kDrawThreads / 64) {
      const int s = u / kUnits;
      if (l.listed[s] <= kListed) continue;
      const int begin = s * kSlice + u % kUnits * (kSlice / kUnits), end = begin + kSlice / kUnits;
#pragma unroll 1
      for (int at = begin + (t & 63) * N; at < end; at += 64 * N) {
        float x[N];
        load16(row.grid, at, row.skew, p.vocab, x);
        uint32_t hits = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[i] >= in.low && x[i] <= in.high) hits |= 1u << i;
        while (hits) {
          const int i = __ffs(hits) - 1;
          hits &= hits - 1;
          f(key_of(as_float(row.grid[at + i])), static_cast<uint32_t>(at + i - row.skew));
        }
      }
    }
  }
};

struct Reached {
  unsigned long long rank;   // of the last token
  double weight;             // up to it
  int part;                  // of its bin
  int held;                  // tokens of this part, if l.ranks has them all; -1: it does not
};
// The last token of bin `bin` (with the weight `before` ahead of it) that is kept: the `left`th one, or (left == 0) the first one at which the weight
// reaches `goal`. It is in one part of the bin; where that has many tokens, they are cut into 256 by their ranks until few are left, and
// these are compared with each other.
template <typename T, int kDrawThreads>
__device__ __forceinline__ Reached resolve(const Drawn<T, kDrawThreads> &row, int bin, double before, int left, double goal) {
  const Params &p = row.p;
  DrawLds &l = row.l;
  int t = threadIdx.x, r = row.r;
  asm volatile("" : "+v"(t), "+s"(r));   // (or what depends on them alone would be held in registers across both calls)
  const int n_parts = row.parts_of(bin);
  const double unit = kStep * middle_of(bin);
  Reached out;
  // the part
  {
    const int j = t & (kParts - 1), set = t / kParts;
    unsigned long long steps = 0;
    int count = 0;
    if (j < n_parts) {
      const unsigned long long *const parts = p.parts + static_cast<int64_t>(r) * p.n_slices * 2 * kParts + row.first_part(bin) + j;
#pragma unroll 4
      for (int s = set; s < p.n_slices; s += kDrawThreads / kParts) {
        const unsigned long long h = l.listed[s] > 0 ? parts[s * 2 * kParts] : 0;
        steps += h >> kCountBits;
        count += static_cast<int>(h & ((1u << kCountBits) - 1));
      }
    }
    __syncthreads();
    l.part[t] = steps;
    l.part_count[t] = count;
    if (t == 0) {
      l.i[0] = l.i[1] = 0;
      l.rank = 0;
    }
    __syncthreads();
  }
  int n = 0;   // tokens that are left
  // the first of 256 numbers in l.part at which the goal is reached (the last one that has tokens, if rounding leaves none): every wave looks
  // for itself, 4 numbers per lane
  const auto choose = [&](int sets) {
    constexpr int kOwn = kParts / 64;
    const int lane = t & 63;
    int c[kOwn], c_upto[kOwn], c_sum = 0;
    double m[kOwn], m_upto[kOwn], m_sum = 0.0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      unsigned long long steps = 0;
      c[i] = 0;
      for (int set = 0; set < sets; ++set) {
        c[i] += l.part_count[set * kParts + kOwn * lane + i];
        steps += l.part[set * kParts + kOwn * lane + i];
      }
      m[i] = static_cast<double>(steps) * unit;
      c_upto[i] = c_sum += c[i];
      m_upto[i] = m_sum += m[i];
    }
    const int c_ahead = wave_sums(c_sum) - c_sum;
    const double m_ahead = before + (wave_sums(m_sum) - m_sum);
    int first = kOwn, last = -1;
#pragma unroll
    for (int i = kOwn - 1; i >= 0; --i)
      if (c[i] > 0) {
        if (left > 0 ? c_ahead + c_upto[i] >= left : m_ahead + m_upto[i] >= goal) first = i;
        if (last < 0) last = i;
      }
    const unsigned long long reached = __ballot(first < kOwn), any = __ballot(last >= 0);
    const int src = reached ? __ffsll(reached) - 1 : any ? 63 - __clzll(any) : 0, i_mine = reached ? first : last < 0 ? 0 : last;
    int c_mine = 0, c_before = 0;
    double m_before = 0.0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (i == i_mine) {
        c_mine = c[i];
        c_before = c_ahead + c_upto[i] - c[i];
        m_before = m_ahead + (m_upto[i] - m[i]);
      }
    n = of_lane(c_mine, src);
    if (left > 0) left -= of_lane(c_before, src);
    before = of_lane(m_before, src);
    return kOwn * src + of_lane(i_mine, src);
  };
  out.part = choose(kDrawThreads / kParts);
  out.held = -1;
  unsigned long long low = 0, high = ~0ull;
  const Interval in = interval_of(row.top, bin + (out.part - 0.01) / n_parts, bin - 1 + (out.part + 1.01) / n_parts, row.w.per_bin);
  int n_held = -1;   // tokens in l.ranks, if all that are left are there
  const auto each = [&](auto &&f) {
    if (n_held >= 0) {
      for (int i = t; i < n_held; i += kDrawThreads) {
        const unsigned long long rank = l.ranks[i];
        if (rank >= low && rank <= high) f(rank);
      }
    } else {
      row.each(t, r, in, [&](uint32_t key, uint32_t index) {
        const unsigned long long rank = rank_of(key, index);
        if (rank < low || rank > high) return;
        const Place a = row.place(key);
        if (bin_of(row.top, a.bin) == bin && part_of(a.rest, n_parts) == out.part) f(rank);
      });
    }
  };
  const auto hold = [&](unsigned long long rank, unsigned long long *ranks, int most, int *count) {
    const int at = atomicAdd(count, 1);
    if (at >= most) return;
    ranks[at] = rank;
    if (at < kRanked) l.steps[at] = steps_of(row.place(~static_cast<uint32_t>(rank >> 32)).rest);
  };
  bool whole = true;
  while (n_held < 0 || n > kRanked) {
    if (n_held < 0 && n <= kHeld) {
      each([&](unsigned long long rank) { hold(rank, l.ranks, kHeld, &l.i[0]); });
      __syncthreads();
      n_held = l.i[0] < kHeld ? l.i[0] : kHeld;
      if (whole) out.held = n_held;
      continue;
    }
    whole = false;
    __syncthreads();
    if (t == 0) {
      l.low = ~0ull;
      l.high = ~0ull;
    }
    if (t < kParts) {
      l.part[t] = 0;
      l.part_count[t] = 0;
    }
    __syncthreads();
    unsigned long long least = ~0ull, most = 0;
    each([&](unsigned long long rank) {
      least = rank < least ? rank : least;
      most = rank > most ? rank : most;
    });
    least = wave_min(least, ~0ull);
    most = wave_min(~most, ~0ull);   // (the complement of the largest)
    if ((t & 63) == 0) {
      atomicMin(&l.low, least);
      atomicMin(&l.high, most);
    }
    __syncthreads();
    low = l.low;
    high = ~l.high;
    int shift = 0;
    while (((high - low) >> shift) >= kParts) ++shift;
    each([&](unsigned long long rank) {
      const int part = static_cast<int>((rank - low) >> shift);
      atomicAdd(&l.part_count[part], 1);
      atomicAdd(&l.part[part], steps_of(row.place(~static_cast<uint32_t>(rank >> 32)).rest));
    });
    __syncthreads();
    low += static_cast<unsigned long long>(choose(1)) << shift;
    const unsigned long long rest = (1ull << shift) - 1;   // (low + rest may leave 64 bits, behind the lowest logits)
    if (high - low > rest) high = low + rest;
  }
  // the few that are left, and their weights
  const bool here = n_held <= kRanked;
  if (!here) {
    each([&](unsigned long long rank) { hold(rank, l.near, kRanked, &l.i[1]); });
    __syncthreads();
  }
  const unsigned long long *const near = here ? l.ranks : l.near;
  const int n_near = here ? n_held : l.i[1] < kRanked ? l.i[1] : kRanked;
  constexpr int kSets = kDrawThreads / kRanked;   // threads per token, each compares it with some of the others
  const int mine = t & (kRanked - 1), set = t / kRanked, each_set = (n_near + kSets - 1) / kSets;
  const unsigned long long rank = mine < n_near ? near[mine] : 0;
  int ahead = 0;
  unsigned long long steps = 0;
#pragma unroll 4
  for (int j = set * each_set; j < (set + 1) * each_set && j < n_near; ++j) {
    const bool before_it = near[j] < rank;
    ahead += before_it;
    steps += before_it ? l.steps[j] : 0;
  }
  l.part_count[t] = ahead;
  l.part[t] = steps;
  __syncthreads();
  if (t < n_near) {
    for (int i = 1; i < kSets; ++i) {
      ahead += l.part_count[i * kRanked + t];
      steps += l.part[i * kRanked + t];
    }
    const double upto = before + static_cast<double>(steps + l.steps[t]) * unit;
    // (the last of all, if rounding leaves none)
    const bool last = left > 0 ? ahead + 1 == (left < n_near ? left : n_near)
                               : (upto >= goal || ahead + 1 == n_near) && !(before + static_cast<double>(steps) * unit >= goal && ahead > 0);
    if (last) {
      l.rank = rank;
      l.d = upto;
    }
  }
  __syncthreads();
  out.rank = l.rank;
  out.weight = l.d;
  return out;
}

template <typename T, int kDrawThreads>
__global__ __launch_bounds__(kDrawThreads, 4) void sample_draw_kernel(Params p) {
  constexpr int N = 16 / sizeof(T);
  __shared__ DrawLds l;
  const int r = blockIdx.x, t = threadIdx.x;
  static_assert(kMostSlices <= kDrawThreads && kBins <= kDrawThreads, "one per thread");
  // all that the first kernels wrote is asked for at once (what they left out is not used)
  const Slice slice_t = t < p.n_slices ? p.slices[static_cast<int64_t>(r) * p.n_slices + t] : Slice{0.0, 0.0, -INFINITY, INT32_MAX, 0, 0};
  const Cut &c = p.cuts[r];
  double upto_weight = 0.0, weight_of_all = 0.0, least_there = 0.0;
  int upto_count = 0, listed = 0, from = 0, upto = 0, k_bin = 0, k_left = 0, p_on = 0, k_too = 0;
  if (p.filters) {
    from = c.from;
    upto = c.upto;
    k_bin = c.k_bin;
    k_left = c.k_left;
    p_on = c.p_on;
    k_too = c.k_too;
    weight_of_all = c.all;
    least_there = c.least;
    if (t < kBins) {
      upto_weight = c.upto_weight[t];
      upto_count = c.upto_count[t];
    }
    if (t < p.n_slices) listed = p.listed[static_cast<int64_t>(r) * p.n_slices + t];
  }
  float u = p.u[r];
  const Row w = row_of(p, r);
  // the lists: some threads per slice
  int lanes = kDrawThreads;
  while (lanes * p.n_slices > kDrawThreads) lanes >>= 1;
  static_assert(kDrawThreads <= kListed, "a thread's first entry lies in its slice's list");
  Entry mine_e{0, 0};
  if (p.filters && t / lanes < p.n_slices) mine_e = p.lists[(static_cast<int64_t>(r) * p.n_slices + t / lanes) * kListed + (t & (lanes - 1))];
  if (!w.filtered || (from == kBins && !k_too)) listed = 0;
  if (t < p.n_slices) {
    l.listed[t] = listed;
    l.cut_steps[t] = 0;
    l.top_of_slice[t] = slice_t.most > -INFINITY ? slice_t.top : -INFINITY;
  }
  if (t < kBins) {
    l.upto_weight[t] = upto_weight;
    l.upto_count[t] = upto_count;
  }
  Whole all{wave_max(slice_t.most), false, 0.0};
  const int flags = __any(slice_t.nan) | __any(listed > kListed) << 1;
  if ((t & 63) == 0) {
    l.tops[t >> 6] = all.most;
    l.flags[t >> 6] = flags;
  }
  if (t == 0) {
    l.i[2] = INT32_MAX;
    l.i[3] = -1;
  }
  __syncthreads();
  int all_flags = 0;
  for (int i = 0; i < kDrawThreads / 64; ++i) {
    all.most = fmaxf(all.most, l.tops[i]);
    all_flags |= l.flags[i];
  }
  all.nan = all_flags & 1;
  if (all.nan || all.most == -INFINITY) {
    if (t == 0) {
      p.tokens[r] = -1;
      if (p.logprob) p.logprob[r] = NAN;
    }
    return;
  }
  if (w.greedy) {
    const int first = wave_min(slice_t.most == all.most ? slice_t.first : INT32_MAX, INT32_MAX);
    if ((t & 63) == 0) atomicMin(&l.i[2], first);
    __syncthreads();
    if (t == 0) {
      p.tokens[r] = l.i[2];
      if (p.logprob) p.logprob[r] = 0.0f;
    }
    return;
  }
  const double unit = w.filtered ? w.per_bin : 0.25 * w.per_bin;   // what the slices' tops are in
  all.top = place_of(number_of(all.most), unit).bin;
  // ---- the kept tokens: rank <= last, logit >= least
  unsigned long long last = ~0ull;
  double least = -INFINITY;
  if (!w.filtered) {
    // (a slice in which every token's weight is rounded to 0 has none, whatever their sum is)
    if (t < p.n_slices) l.of_slice[t] = slice_t.most > -INFINITY && slice_t.top - all.top > -1075.0 ? ldexp(slice_t.sum, static_cast<int>(slice_t.top - all.top)) : 0.0;
  } else {
    const Drawn<T, kDrawThreads> row{p, l, w, r, all.top, from, upto, k_too ? k_bin : -1, (all_flags & 2) != 0, lanes, mine_e};
    if (w.m > 0.0f) least = least_there;
    int end = kBins, end_part = 0, held = -1;   // bin and part that have the last kept token
    double goal = 0.0;
    const auto weight_ahead = [&](int b) { return b > 0 ? l.upto_weight[b - 1] : 0.0; };
    const auto tokens_in = [&](int b) { return l.upto_count[b] - (b > 0 ? l.upto_count[b - 1] : 0); };
    // first top-k's last token, where it can be the last one and where top-p takes a share of the weight up to it; then top-p's
    double kept = k_bin < kBins ? l.upto_weight[k_bin] : weight_of_all;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
      int bin = k_bin, left = k_left;
      if (turn == 0) {
        if (bin == kBins || (bin > row.upto && row.k_bin < 0)) continue;
      } else {
        if (!p_on || row.from == kBins) break;
        goal = static_cast<double>(w.p) * kept;
        left = 0;
        bin = row.from;
        while (bin < row.upto && l.upto_weight[bin] < goal) ++bin;
        // (where min-p ends ahead of it, the bin has no token that counts)
        if (tokens_in(bin) == 0 || l.upto_weight[bin] < goal * (1.0 - 1e-9)) break;
      }
      const Reached at = resolve(row, bin, weight_ahead(bin), left, goal);
      if (turn == 0) kept = at.weight;
      if (at.rank < last) {
        last = at.rank;
        end = bin;
        end_part = at.part;
        held = at.held;
      } else {
        held = -1;
      }
    }
    if (w.m > 0.0f) {
      const Place at = place_of(least, w.per_bin);
      const int m_bin = bin_of(all.top, at.bin), m_part = m_bin <= row.upto && row.upto < kBins ? part_of(at.rest, row.parts_of(m_bin)) : 0;
      if (m_bin < end || (m_bin == end && m_part < end_part)) {
        end = m_bin;
        end_part = m_part;
        held = -1;
      }
    }
    // ---- the slices' kept weights: all bins ahead of `end`, of that the parts ahead of `end_part`, and what is kept in it
    const bool inside = end < kBins - 1;
    if (inside) {
      __syncthreads();
      const int skew = RowAt<T>(p, r).skew, n_parts = row.parts_of(end);
      const auto keep = [&](unsigned long long rank) {
        const float x = of_key(~static_cast<uint32_t>(rank >> 32));
        if (rank <= last && number_of(x) >= least)
          atomicAdd(&l.cut_steps[(static_cast<uint32_t>(rank) + skew) / kSlice], steps_of(place_of(number_of(x), w.per_bin).rest));
      };
      if (held >= 0)
        for (int i = threadIdx.x; i < held; i += kDrawThreads) keep(l.ranks[i]);
      else
        row.each(t, r, interval_of(all.top, end + (end_part - 0.01) / n_parts, end - 1 + (end_part + 1.01) / n_parts, w.per_bin), [&](uint32_t key, uint32_t index) {
          const Place a = row.place(key);
          if (bin_of(all.top, a.bin) == end && part_of(a.rest, n_parts) == end_part) keep(rank_of(key, index));
        });
    }
    __syncthreads();
    const unsigned long long *const bins = p.bins + static_cast<int64_t>(r) * p.n_slices * kBins;
    const unsigned long long *const parts = p.parts + static_cast<int64_t>(r) * p.n_slices * 2 * kParts + (inside ? row.first_part(end) : 0);
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int i = threadIdx.x >> 6; i < p.n_slices; i += kDrawThreads / 64) {
      double sum = 0.0;
      unsigned long long steps = 0;
      const int off = behind(all.top, l.top_of_slice[i]);
      if (off < kBins) {
#pragma unroll
        for (int j = 0; j < kBins / 64; ++j) {
          const int b = 64 * j + lane;
          if (b < kBins - 1 && b + off < end && b + off < kBins - 1) sum += static_cast<double>(bins[i * kBins + b] >> kCountBits) * kStep * middle_of(b + off);
        }
        if (inside && l.listed[i] > 0)
#pragma unroll
          for (int j = 0; j < kParts / 64; ++j)
            if (64 * j + lane < end_part) steps += parts[i * 2 * kParts + 64 * j + lane] >> kCountBits;
      }
      sum = wave_sum(sum);
      steps = wave_sum(steps);
      if (lane == 0) l.of_slice[i] = sum + (inside ? static_cast<double>(steps + l.cut_steps[i]) * kStep * middle_of(end) : 0.0);
    }
  }
  __syncthreads();
  // ---- the slice: the first one up to which the weight passes the goal (the last one that has any, if rounding leaves none)
  u = u > 0.0f ? (u < 1.0f ? u : 0x1.fffffep-1f) : 0.0f;
  int slice = 0;
  double total = 0.0, before = 0.0;
  // every wave for itself, 64 slices at a time
  for (int b = 0; b < p.n_slices; b += 64) {
    const int i = b + (t & 63);
    total += wave_sum(i < p.n_slices ? l.of_slice[i] : 0.0);
  }
  const double goal = static_cast<double>(u) * total;
  double passed = 0.0;
  for (int b = 0; b < p.n_slices; b += 64) {
    const int i = b + (t & 63);
    const double x = i < p.n_slices ? l.of_slice[i] : 0.0, upto_x = passed + wave_sums(x);
    const unsigned long long any = __ballot(x > 0.0), over = __ballot(x > 0.0 && upto_x > goal);
    const int src = over ? __ffsll(over) - 1 : any ? 63 - __clzll(any) : -1;
    if (src >= 0) {
      slice = b + src;
      before = of_lane(upto_x - x, src);
    }
    if (over) break;
    passed = of_last_lane(upto_x);
  }
  // ---- the token: neighbours per thread
  constexpr int kEach = kSlice / kDrawThreads;
  const RowAt<T> row(p, r);
  const int at = slice * kSlice + kEach * static_cast<int>(threadIdx.x);
  double weight[kEach], sum = 0.0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) weight[i] = 0.0;
  if (kEach * static_cast<int>(threadIdx.x) < kSlice) {
    float x[kEach / N][N];
#pragma unroll
    for (int v = 0; v < kEach / N; ++v) load16(row.grid, at + v * N, row.skew, p.vocab, x[v]);
    const auto kept_place = [&](int i, Place &a) {   // as in the slices' sums
      const float y = x[i / N][i % N];
      a = place_of(number_of(y), unit);
      return y > -INFINITY && rank_of(key_of(y), at + i - row.skew) <= last && number_of(y) >= least;
    };
    if (w.filtered) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        Place a;
        const bool kept = kept_place(i, a);
        const int b = bin_of(all.top, a.bin);
        if (kept && b < kBins - 1) weight[i] = static_cast<double>(steps_of(a.rest)) * kStep * middle_of(b);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        Place a;
        if (kept_place(i, a) && a.bin - all.top > -1075.0) weight[i] = ldexp(in_octave(a.rest), static_cast<int>(a.bin - all.top));   // (lighter: 0)
      }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += weight[i];
  }
  double run = before + block_scan<kDrawThreads>(sum, l.dwaves) - sum;
  int mine = INT32_MAX, any = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    run += weight[i];
    if (weight[i] > 0.0) {
      any = at + i;
      if (run > goal && mine == INT32_MAX) mine = at + i;
    }
  }
  first_thread(mine != INT32_MAX, &l.i[2]);
  last_thread(any >= 0, &l.i[3]);
  __syncthreads();
  if (static_cast<int>(threadIdx.x) == (l.i[2] != INT32_MAX ? l.i[2] : l.i[3])) {
    const int token = l.i[2] != INT32_MAX ? mine : any;
    p.tokens[r] = token - row.skew;
    if (p.logprob) {
      double one = 0.0;
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (token == at + i) one = weight[i];
      p.logprob[r] = static_cast<float>(log(one / total));
    }
  }
}

// ---- host
int slices_of(int vocab, int skew = 7) { return (vocab + skew + kSlice - 1) / kSlice; }   // (a row may begin 7 places behind an aligned one)

struct Space {
  int n_slices;
  int64_t bins, parts, cuts, listed, lists, bytes;   // offsets; the slices are first
};
Space space_of(int64_t rows, int vocab) {
  Space s;
  const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
  s.n_slices = slices_of(vocab);
  const int64_t all = rows * s.n_slices;
  s.bins = up(all * static_cast<int64_t>(sizeof(Slice)));
  s.parts = s.bins + all * kBins * 8;
  s.cuts = s.parts + all * 2 * kParts * 8;
  s.listed = s.cuts + up(rows * static_cast<int64_t>(sizeof(Cut)));
  s.lists = s.listed + up(all * 4);
  s.bytes = s.lists + all * kListed * static_cast<int64_t>(sizeof(Entry));
  return s;
}

int check_sizes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1) return SDVG_ERR_SHAPE;
  if (vocab > kMostVocab || static_cast<int64_t>(rows) * slices_of(vocab) >= (1 << 23)) return SDVG_ERR_UNSUPPORTED;
  return SDVG_OK;
}

template <typename T>
int launch(const Params &p, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(p.n_rows) * p.n_slices);
  hipLaunchKernelGGL((sample_slices_kernel<T>), grid, dim3(kSliceThreads), 0, s, p);
  SDVG_HIP_CHECK(hipGetLastError());
  if (p.filters) {
    hipLaunchKernelGGL(sample_decide_kernel, dim3(p.n_rows), dim3(kBins), 0, s, p);
    SDVG_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL((sample_collect_kernel<T>), grid, dim3(kSliceThreads), 0, s, p);
    SDVG_HIP_CHECK(hipGetLastError());
  }
  // (a compute unit takes one workgroup of 1024 threads or two of 512: a row is drawn in fewer rounds with the larger one, rows that come in more
  // than one round sooner with the smaller one; 1 row of 262144 tokens 26 and 31 us, 200 of 150001 24 and 30, 777 of 32768 53 and 38)
  if (p.n_rows > 256)
    hipLaunchKernelGGL((sample_draw_kernel<T, kMostDraw / 2>), dim3(p.n_rows), dim3(kMostDraw / 2), 0, s, p);
  else
    hipLaunchKernelGGL((sample_draw_kernel<T, kMostDraw>), dim3(p.n_rows), dim3(kMostDraw), 0, s, p);
  SDVG_HIP_CHECK(hipGetLastError());
  return SDVG_OK;
}
}  // namespace

extern "C" int64_t sdvg_sample_tokens_workspace_bytes(int32_t n_rows, int32_t vocab) {
  const int st = check_sizes(n_rows, vocab);
  return st != SDVG_OK ? st : n_rows == 0 ? 0 : space_of(n_rows, vocab).bytes;
}

extern "C" int sdvg_sample_tokens(const sdvg_sample_args *a, void *workspace, int64_t workspace_bytes, void *stream) {
  if (!a) return SDVG_ERR_NULL;
  const int st = check_sizes(a->n_rows, a->vocab);
  if (st != SDVG_OK) return st;
  if (a->dtype != SDVG_F32 && a->dtype != SDVG_BF16 && a->dtype != SDVG_F16) return SDVG_ERR_UNSUPPORTED;
  if (workspace_bytes < 0) return SDVG_ERR_SHAPE;
  if (a->n_rows > 1 && a->row_stride < a->vocab) return SDVG_ERR_SHAPE;
  if (a->n_rows > 1 && a->row_stride >= int64_t{1} << 40) return SDVG_ERR_UNSUPPORTED;
  if (a->n_rows == 0) return SDVG_OK;
  if (!a->logits || !a->u || !a->tokens || !workspace) return SDVG_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(a->logits) % sdvg::element_bytes(a->dtype) || !sdvg::aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(a->u) | reinterpret_cast<uintptr_t>(a->temperature) | reinterpret_cast<uintptr_t>(a->top_k) |
       reinterpret_cast<uintptr_t>(a->top_p) | reinterpret_cast<uintptr_t>(a->min_p) | reinterpret_cast<uintptr_t>(a->tokens) |
       reinterpret_cast<uintptr_t>(a->logprob)) & 3)
    return SDVG_ERR_ALIGN;
  const Space s = space_of(a->n_rows, a->vocab);
  if (workspace_bytes < s.bytes) return SDVG_ERR_RANGE;
  const int64_t size = sdvg::element_bytes(a->dtype), span = ((a->n_rows > 1 ? (a->n_rows - 1) * a->row_stride : 0) + a->vocab) * size, n4 = int64_t{a->n_rows} * 4;
  for (const void *out : {static_cast<const void *>(a->tokens), static_cast<const void *>(a->logprob)}) {
    if (!out) continue;
    if (!sdvg::disjoint(out, n4, a->logits, span)) return SDVG_ERR_RANGE;
    for (const void *in : {static_cast<const void *>(a->u), static_cast<const void *>(a->temperature), static_cast<const void *>(a->top_k),
                           static_cast<const void *>(a->top_p), static_cast<const void *>(a->min_p)})
      if (in && !sdvg::disjoint(out, n4, in, n4)) return SDVG_ERR_RANGE;
  }
  if (a->logprob && !sdvg::disjoint(a->logprob, n4, a->tokens, n4)) return SDVG_ERR_RANGE;
  char *const at = static_cast<char *>(workspace);
  Params p{static_cast<const char *>(a->logits), a->u, a->temperature, a->top_p, a->min_p, a->top_k, a->tokens, a->logprob,
                 a->all_temperature, a->all_top_p, a->all_min_p, a->all_top_k, a->n_rows > 1 ? a->row_stride : 0, a->n_rows, a->vocab,
                 s.n_slices, 0, reinterpret_cast<Slice *>(at), reinterpret_cast<unsigned long long *>(at + s.bins),
                 reinterpret_cast<Cut *>(at + s.cuts), reinterpret_cast<unsigned long long *>(at + s.parts), reinterpret_cast<int32_t *>(at + s.listed),
                 reinterpret_cast<Entry *>(at + s.lists)};
  if ((reinterpret_cast<uintptr_t>(a->logits) | static_cast<uintptr_t>(p.row_stride * size)) % 16 == 0) p.n_slices = slices_of(a->vocab, 0);
  p.filters = a->top_k || a->top_p || a->min_p || (a->all_top_k > 0 && a->all_top_k < a->vocab) || a->all_top_p < 1.0f || a->all_min_p > 0.0f;
  hipStream_t q = static_cast<hipStream_t>(stream);
  return a->dtype == SDVG_F32 ? launch<float>(p, q) : a->dtype == SDVG_BF16 ? launch<__bf16>(p, q) : launch<_Float16>(p, q);
}
