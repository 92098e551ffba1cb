// Drawing the next tokens: one token per row of logits, with temperature, top-k, top-p and min-p, from given random numbers.
//
// With x = logit / temperature, a token weighs w = exp(x - largest x). The kept tokens are a prefix of the row in the order (larger logit first, of
// equal ones the lower index): the shorter one of what top-k, top-p and min-p leave. The draw is the lowest index at which the sum of kept
// weights, taken in index order, passes u times their total. A token is a whole number that has one right value, so weights and sums are held in 64
// bits, and no sum's order depends on the order in which threads arrive: where those meet they add integers.
//
// What bounds it: the logits are read from memory once (and once more from the caches where a cut has to be found); a launch or a fp64 operation
// per token cost as much. So a row is never sorted. It is cut into slices, a workgroup each:
//   1 slices   the largest logit; a histogram of tokens and their weights over bins of a quarter octave (factor 2^(1/4)) of weight. Where there is no filter the sum of weights alone.
//   2 collect  (filters only) every slice's workgroup adds up the row's histograms, sees in which bins the cuts lie, and writes those bins' tokens to a list.
//   3 draw     a workgroup per row: sorts what of the list the cuts need, then finds the slice with the drawn token from the slices' kept weights, and the token
//              in it.
// A weight in a histogram is an integer in steps of 2^-35 of its bin's upper end, in 64 bits beside the count; without filters it is
// rounded to 2^-34 of its octave. So it is at most 2^-35 off, equal logits have equal weights, and sums of equal weights are exact.
#include <math.h>

#include "paged_kv.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kBins = 256;                 // of weight; the last one has all that is lighter, whose weight does not count (2^-63 of the largest)
constexpr int kCountBits = 14;             // of a slice's bin: tokens below, weight in steps of kStep above
constexpr double kStep = 0x1p-35;
constexpr int kSliceThreads = 256, kMostSlice = 8192, kLeastSlice = 2048;
constexpr int kDrawThreads = 1024, kSorted = 2048;
constexpr int kListMost = 16384;           // tokens of a row's cut bins that are listed; more are looked for in the row again
constexpr int kMostVocab = 1 << 20, kMostSlices = kMostVocab / kLeastSlice + 1;

struct Slice {
  double top;       // floor of the largest x in bins, or in octaves (no filter)
  double sum;       // weights relative to 2^top (no filter)
  float most;       // largest logit; -infinity: none
  int32_t first;    // its lowest index (greedy)
  int32_t nan, pad;
};
// What a row's filters come to, by bins.
struct Cut {
  int32_t from, upto;      // bins in which the last kept token may be
  int32_t k_bin, k_left;   // bin in which top-k ends, tokens it keeps there; 256: nowhere
  int32_t p_on;
  int32_t listed;          // tokens in bins from .. upto and, where it counts, k_bin
  double all;              // weight of all tokens
  double upto_weight[kBins];   // weight of bins 0 .. b, relative to the upper end of bin 0
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
  int32_t n_rows, vocab, slice, n_slices, list_most;
  Slice *slices;           // [row][slice]
  unsigned long long *bins;   // [row][slice][kBins]
  Cut *cuts;               // [row]
  Entry *lists;            // [row][list_most]
};

struct Row {
  double per_bin;          // bins per unit of logit
  float p, m;
  int k;
  bool greedy, filtered;
};
__device__ __forceinline__ Row row_of(const Params &p, int r) {
  Row w;
  const float t = p.temperature ? p.temperature[r] : p.all_temperature;
  w.p = p.top_p ? p.top_p[r] : p.all_top_p;
  w.m = p.min_p ? p.min_p[r] : p.all_min_p;
  w.k = p.top_k ? p.top_k[r] : p.all_top_k;
  if (!(w.p < 1.0f)) w.p = 1.0f;
  if (!(w.m > 0.0f)) w.m = 0.0f;
  if (w.m > 1.0f) w.m = 1.0f;
  if (w.k <= 0 || w.k >= p.vocab) w.k = 0;
  w.greedy = !(t > 0.0f);
  w.filtered = !w.greedy && (w.k > 0 || w.p < 1.0f || w.m > 0.0f);
  w.per_bin = 4.0 * 1.4426950408889634 / static_cast<double>(t);
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

// Order-preserving key; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
// Larger logits first, of equal ones the lower index.
__device__ __forceinline__ unsigned long long rank_of(uint32_t key, uint32_t index) { return static_cast<unsigned long long>(~key) << 32 | index; }
// A logit's place on the scale of bins. +infinity is a number that all others are far from. (The product is rounded by itself: what a fused
// subtraction of its floor would keep beside it is no fraction where the place is a number beyond 2^52.)
__device__ __forceinline__ double place_of(float x, double per_bin) {
#pragma clang fp contract(off)
  return (x == INFINITY ? 0x1p200 : static_cast<double>(x)) * per_bin;
}
__device__ __forceinline__ int bin_of(double top, double floor_x) {
  const double d = top - floor_x;
  return d < kBins - 1 ? static_cast<int>(d) : kBins - 1;
}

// 2^((f - 1) / 4) for 0 <= f < 1: exp's series to the 8th power, 4e-13 off at most.
__device__ __forceinline__ double in_bin(double f) {
  const double y = fma(f, 0.17328679513998632, -0.17328679513998632);
  double s = 1.0 / 40320;
  s = fma(s, y, 1.0 / 5040);
  s = fma(s, y, 1.0 / 720);
  s = fma(s, y, 1.0 / 120);
  s = fma(s, y, 1.0 / 24);
  s = fma(s, y, 1.0 / 6);
  s = fma(s, y, 0.5);
  s = fma(s, y, 1.0);
  return fma(s, y, 1.0);
}
// 2^f for 0 <= f < 1, from the middle, rounded to 2^-34.
__device__ __forceinline__ double in_octave(double f) {
  const double y = fma(f, 0.6931471805599453, -0.34657359027997264);
  double s = 1.0 / 479001600;
  s = fma(s, y, 1.0 / 39916800);
  s = fma(s, y, 1.0 / 3628800);
  s = fma(s, y, 1.0 / 362880);
  s = fma(s, y, 1.0 / 40320);
  s = fma(s, y, 1.0 / 5040);
  s = fma(s, y, 1.0 / 720);
  s = fma(s, y, 1.0 / 120);
  s = fma(s, y, 1.0 / 24);
  s = fma(s, y, 1.0 / 6);
  s = fma(s, y, 0.5);
  s = fma(s, y, 1.0);
  s = fma(s, y, 1.0);
  return fma(s, 1.4142135623730951, 0x1p18) - 0x1p18;
}
// 2^(-b / 4)
__device__ __forceinline__ double end_of_bin(int b) {
  const double q[4] = {1.0, 0.8408964152537145, 0.7071067811865476, 0.5946035575013605};
  return ldexp(q[b & 3], -(b >> 2));
}
__device__ __forceinline__ unsigned long long steps_of(double weight) {   // weight <= 1
  return static_cast<unsigned long long>(__double_as_longlong(fma(weight, 1.0 / kStep, 0x1p52))) & ((1ull << 40) - 1);   // (rounded by the addition)
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_xor(x, d);
    x = y < x ? y : x;
  }
  return x;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}
template <typename V>
__device__ __forceinline__ V wave_scan(V x) {   // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const V y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
// Inclusive sums over a workgroup's threads; `waves` is LDS of a number per wave.
template <int kThreads, typename V>
__device__ __forceinline__ V block_scan(V x, V *waves) {
  const int wave = threadIdx.x >> 6;
  x = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[wave] = x;
  __syncthreads();
  V before = 0;
  for (int w = 0; w < wave; ++w) before += waves[w];
  return before + x;
}

// ---- 1
template <typename T, int kVectors>   // 16-byte vectors per thread
__device__ __forceinline__ void one_slice(const Params &p, int r, int s) {
  constexpr int N = 16 / sizeof(T);
  __shared__ unsigned long long hist[kBins];
  __shared__ double sums[kSliceThreads / 64];
  __shared__ float tops[kSliceThreads / 64];
  __shared__ int firsts[kSliceThreads / 64];
  const Row w = row_of(p, r);
  const RowAt<T> row(p, r);
  float x[kVectors][N];
  float most = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int v = 0; v < kVectors; ++v) load16(row.grid, s * p.slice + (v * kSliceThreads + static_cast<int>(threadIdx.x)) * N, row.skew, p.vocab, x[v]);
  hist[threadIdx.x] = 0;
#pragma unroll
  for (int v = 0; v < kVectors; ++v)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      most = fmaxf(most, x[v][i]);
      nan |= x[v][i] != x[v][i];
    }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  most = wave_max(most);
  if (lane == 0) tops[wave] = most;
  const bool any_nan = __syncthreads_or(nan);
  for (int i = 0; i < kSliceThreads / 64; ++i) most = fmaxf(most, tops[i]);
  Slice out{};
  out.most = most;
  out.nan = any_nan;
  if (!any_nan && most > -INFINITY) {
    if (w.greedy) {
      int first = INT32_MAX;
#pragma unroll
      for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int i = N - 1; i >= 0; --i) {
          const int at = s * p.slice + (v * kSliceThreads + static_cast<int>(threadIdx.x)) * N + i - row.skew;
          if (x[v][i] == most && at < first) first = at;
        }
      first = wave_min(first);
      if (lane == 0) firsts[wave] = first;
      __syncthreads();
      for (int i = 0; i < kSliceThreads / 64; ++i) first = firsts[i] < first ? firsts[i] : first;
      out.first = first;
    } else if (!w.filtered) {
      const double per_octave = 0.25 * w.per_bin;
      out.top = floor(place_of(most, per_octave));
      double sum = 0.0;
#pragma unroll
      for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[v][i] > -INFINITY) {
            const double y = place_of(x[v][i], per_octave), f = floor(y), d = fmax(f - out.top, -2000.0);
            sum += ldexp(in_octave(y - f), static_cast<int>(d));
          }
      sum = wave_sum(sum);
      if (lane == 0) sums[wave] = sum;
      __syncthreads();
      out.sum = 0.0;
      for (int i = 0; i < kSliceThreads / 64; ++i) out.sum += sums[i];
    } else {
      out.top = floor(place_of(most, w.per_bin));
#pragma unroll
      for (int v = 0; v < kVectors; ++v)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[v][i] > -INFINITY) {
            const double y = place_of(x[v][i], w.per_bin), f = floor(y);
            const int b = bin_of(out.top, f);
            const unsigned long long steps = b < kBins - 1 ? steps_of(in_bin(y - f)) : 0;
            atomicAdd(&hist[b], steps << kCountBits | 1);
          }
    }
  }
  if (w.filtered) {
    __syncthreads();
    p.bins[(static_cast<int64_t>(r) * p.n_slices + s) * kBins + threadIdx.x] = hist[threadIdx.x];
  }
  if (threadIdx.x == 0) p.slices[static_cast<int64_t>(r) * p.n_slices + s] = out;
}
template <typename T, int kSlice>
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
// Bins that a slice's are behind the row's.
__device__ __forceinline__ int behind(double top, double slice_top) { return static_cast<int>(fmin(top - slice_top, 1e6)); }

// ---- 2
template <typename T, int kVectors>
__device__ __forceinline__ void collect(const Params &p, int r, int s) {
  constexpr int N = 16 / sizeof(T);
  __shared__ double weight[kBins];
  __shared__ int count[kBins];
  __shared__ double dwaves[kSliceThreads / 64];
  __shared__ int iwaves[kSliceThreads / 64];
  __shared__ int found[3];
  const Row w = row_of(p, r);
  if (!w.filtered) return;
  Whole all = whole_of(p, r);
  if (all.nan || all.most == -INFINITY) return;
  all.top = floor(place_of(all.most, w.per_bin));
  const int b = threadIdx.x;
  // the row's bin b, and what the slices ahead of this one have in it
  unsigned long long steps = 0;
  int n = 0, n_ahead = 0, n_mine = 0;
  const Slice *const slices = p.slices + static_cast<int64_t>(r) * p.n_slices;
  const unsigned long long *const bins = p.bins + static_cast<int64_t>(r) * p.n_slices * kBins;
#pragma unroll 4
  for (int i = 0; i < p.n_slices; ++i) {
    const bool some = slices[i].most > -INFINITY;
    const int off = some ? behind(all.top, slices[i].top) : 0, at = b - off;
    const bool in = some && b < kBins - 1 && at >= 0;
    const unsigned long long h = in ? bins[i * kBins + at] : 0;
    const int c = static_cast<int>(h & ((1u << kCountBits) - 1));
    steps += h >> kCountBits;
    n += c;
    if (i < s) n_ahead += c;
    if (i == s) n_mine = c;
  }
  const double mine = static_cast<double>(steps) * kStep * end_of_bin(b);
  weight[b] = block_scan<kSliceThreads>(mine, dwaves);
  count[b] = block_scan<kSliceThreads>(n, iwaves);
  if (b < 3) found[b] = kBins;
  __syncthreads();
  const double total = weight[kBins - 1];
  // top-k ends in the first bin up to which there are k tokens
  if (w.k > 0 && count[b] >= w.k) atomicMin(&found[0], b);
  __syncthreads();
  const int k_bin = found[0], k_ahead = k_bin > 0 && k_bin < kBins ? count[k_bin - 1] : 0, k_left = k_bin < kBins ? w.k - k_ahead : 0;
  const bool k_inside = k_bin < kBins && count[k_bin] > w.k;
  const bool p_on = w.p < 1.0f;
  int from = kBins, upto = kBins;   // (kBins: all tokens are kept)
  if (p_on) {
    // the weight that top-k leaves is known to within its last bin; the last token of top-p lies in one of these bins
    const double k_low = k_bin == kBins ? total : k_inside ? (k_bin > 0 ? weight[k_bin - 1] : 0.0) + k_left * end_of_bin(k_bin + 1) : weight[k_bin];
    const double k_high = k_bin == kBins ? total : weight[k_bin];
    const double low = w.p * k_low * (1.0 - 1e-9), high = w.p * k_high * (1.0 + 1e-9);
    if (weight[b] >= low) atomicMin(&found[1], b);
    if (weight[b] >= high) atomicMin(&found[2], b);
    __syncthreads();
    from = found[1];
    upto = found[2];
    if (upto > k_bin) upto = k_bin;
    if (from > upto) from = upto;
  } else if (k_bin < kBins) {
    from = upto = k_bin;
  }
  if (w.m > 0.0f) {
    const int m_bin = bin_of(all.top, floor(place_of(all.most, w.per_bin) + 4.0 * log2(static_cast<double>(w.m))));
    if (m_bin < from) from = m_bin;
    if (m_bin < upto) upto = m_bin;
  }
  if (from > kBins - 2)
    from = upto = kBins;
  else if (upto > kBins - 2)
    upto = kBins - 2;
  const bool k_too = p_on && k_inside && k_bin > upto;   // (for the weight that top-p takes a share of)
  // tokens to be listed: of the row, of the slices ahead, of this one
  const bool asked = (b >= from && b <= upto) || (k_too && b == k_bin);
  __syncthreads();
  const int listed = block_scan<kSliceThreads>(asked ? n : 0, iwaves);
  __syncthreads();
  const int ahead = block_scan<kSliceThreads>(asked ? n_ahead : 0, iwaves);
  __syncthreads();
  const int here = block_scan<kSliceThreads>(asked ? n_mine : 0, iwaves);
  __shared__ int sums[3];
  if (b == kSliceThreads - 1) {
    sums[0] = listed;
    sums[1] = ahead;
    sums[2] = here;
  }
  if (s == 0) {
    Cut *const c = p.cuts + r;
    c->upto_weight[b] = weight[b];
    c->upto_count[b] = count[b];
    if (b == kSliceThreads - 1) {
      c->from = from;
      c->upto = upto;
      c->k_bin = k_bin;
      c->k_left = k_left;
      c->p_on = p_on;
      c->listed = listed;
      c->all = total;
    }
  }
  __syncthreads();
  if (sums[0] > p.list_most || sums[2] == 0) return;
  // the tokens themselves; their order in the list does not matter
  const RowAt<T> row(p, r);
  int mine_n = 0;
  float x[kVectors][N];
  uint32_t hit[kVectors];
#pragma unroll
  for (int v = 0; v < kVectors; ++v) load16(row.grid, s * p.slice + (v * kSliceThreads + b) * N, row.skew, p.vocab, x[v]);
#pragma unroll
  for (int v = 0; v < kVectors; ++v) {
    hit[v] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (x[v][i] == -INFINITY) continue;
      const int bin = bin_of(all.top, floor(place_of(x[v][i], w.per_bin)));
      if (bin < kBins - 1 && ((bin >= from && bin <= upto) || (k_too && bin == k_bin))) hit[v] |= 1u << i;
    }
    mine_n += __popc(hit[v]);
  }
  int at = sums[1] + block_scan<kSliceThreads>(mine_n, iwaves) - mine_n;
  Entry *const list = p.lists + static_cast<int64_t>(r) * p.list_most;
#pragma unroll
  for (int v = 0; v < kVectors; ++v)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (hit[v] >> i & 1) {
        if (at < p.list_most) list[at] = Entry{key_of(x[v][i]), static_cast<uint32_t>(s * p.slice + (v * kSliceThreads + b) * N + i - row.skew)};
        ++at;
      }
}
template <typename T, int kSlice>
__global__ __launch_bounds__(kSliceThreads) void sample_collect_kernel(Params p) {
  const int r = blockIdx.x / p.n_slices, s = blockIdx.x - r * p.n_slices;
  collect<T, kSlice * static_cast<int>(sizeof(T)) / 16 / kSliceThreads>(p, r, s);
}

// ---- 3
struct DrawLds {
  unsigned long long ranks[kSorted];
  double upto[kSorted];
  unsigned long long steps[kBins];
  int count[kBins];
  double dwaves[kDrawThreads / 64];
  int iwaves[kDrawThreads / 64];
  double of_slice[kMostSlices];
  unsigned long long cut_steps[kMostSlices];
  unsigned long long low, high;
  double d[2];
  int i[4];
};

// The tokens in the cut bins: from the list, or where it did not hold them from the row.
template <typename T, typename F>
__device__ __forceinline__ void each_candidate(const Params &p, int r, int listed, F &&f) {
  if (listed <= p.list_most) {
    const Entry *const list = p.lists + static_cast<int64_t>(r) * p.list_most;
    for (int i = threadIdx.x; i < listed; i += kDrawThreads) f(list[i].key, list[i].index);
  } else {
    constexpr int N = 16 / sizeof(T);
    const RowAt<T> row(p, r);
    for (int at = threadIdx.x * N; at < row.skew + p.vocab; at += kDrawThreads * N) {
      float x[N];
      load16(row.grid, at, row.skew, p.vocab, x);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (x[i] > -INFINITY) f(key_of(x[i]), static_cast<uint32_t>(at + i - row.skew));
    }
  }
}

struct Reached {
  unsigned long long rank;   // of the last token
  double weight;             // up to it
};
// The last token of bin `bin` (with `n` tokens, weight `before` ahead of it) that is kept: the `left`th one, or (left == 0) the
// first one at which the weight reaches `goal`.
template <typename T>
__device__ Reached resolve(const Params &p, int r, int listed, const Row &w, double top, int bin, int n, double before, int left, double goal, DrawLds &l) {
  unsigned long long low = 0, high = ~0ull;
  const double end = end_of_bin(bin);
  const auto in_it = [&](uint32_t key) { return bin_of(top, floor(place_of(of_key(key), w.per_bin))) == bin; };
  const auto steps_in = [&](uint32_t key) {
    const double y = place_of(of_key(key), w.per_bin);
    return steps_of(in_bin(y - floor(y)));
  };
  const auto weigh = [&](uint32_t key) { return static_cast<double>(steps_in(key)) * kStep * end; };
  while (n > kSorted) {
    // too many to sort: 256 parts of the ranks that there are
    __syncthreads();
    if (threadIdx.x == 0) {
      l.low = ~0ull;
      l.high = 0;
    }
    if (threadIdx.x < kBins) {
      l.steps[threadIdx.x] = 0;
      l.count[threadIdx.x] = 0;
    }
    __syncthreads();
    unsigned long long least = ~0ull, most = 0;
    each_candidate<T>(p, r, listed, [&](uint32_t key, uint32_t index) {
      const unsigned long long rank = rank_of(key, index);
      if (rank < low || rank > high || !in_it(key)) return;
      least = rank < least ? rank : least;
      most = rank > most ? rank : most;
    });
    atomicMin(&l.low, least);
    atomicMax(&l.high, most);
    __syncthreads();
    low = l.low;
    high = l.high;
    int shift = 0;
    while (((high - low) >> shift) >= kBins) ++shift;
    each_candidate<T>(p, r, listed, [&](uint32_t key, uint32_t index) {
      const unsigned long long rank = rank_of(key, index);
      if (rank < low || rank > high || !in_it(key)) return;
      const int part = static_cast<int>((rank - low) >> shift);
      atomicAdd(&l.count[part], 1);
      atomicAdd(&l.steps[part], steps_in(key));
    });
    __syncthreads();
    const int t = threadIdx.x < kBins ? threadIdx.x : kBins - 1;
    const int c = threadIdx.x < kBins ? l.count[t] : 0;
    const double m = threadIdx.x < kBins ? static_cast<double>(l.steps[t]) * kStep * end : 0.0;
    const int c_upto = block_scan<kDrawThreads>(c, l.iwaves);
    const double m_upto = before + block_scan<kDrawThreads>(m, l.dwaves);
    if (threadIdx.x == 0) l.i[0] = static_cast<int>((high - low) >> shift);
    __syncthreads();
    if (c > 0 && (left > 0 ? c_upto >= left : m_upto >= goal)) atomicMin(&l.i[0], static_cast<int>(threadIdx.x));
    __syncthreads();
    const int part = l.i[0];   // (the last one, if rounding leaves none)
    if (static_cast<int>(threadIdx.x) == part) {
      l.i[2] = c;
      l.i[3] = c_upto - c;
      l.d[0] = m_upto - m;
    }
    __syncthreads();
    n = l.i[2];
    if (left > 0) left -= l.i[3];
    before = l.d[0];
    const unsigned long long part_low = low + (static_cast<unsigned long long>(part) << shift);
    const unsigned long long part_high = part_low + ((1ull << shift) - 1);
    low = part_low;
    high = part_high < high ? part_high : high;
  }
  __syncthreads();
  if (threadIdx.x == 0) l.i[0] = 0;
  __syncthreads();
  each_candidate<T>(p, r, listed, [&](uint32_t key, uint32_t index) {
    const unsigned long long rank = rank_of(key, index);
    if (rank < low || rank > high || !in_it(key)) return;
    const int at = atomicAdd(&l.i[0], 1);
    if (at < kSorted) l.ranks[at] = rank;
  });
  __syncthreads();
  n = l.i[0] < kSorted ? l.i[0] : kSorted;
  int size = 64;
  while (size < n) size *= 2;
  for (int i = threadIdx.x; i < size; i += kDrawThreads)
    if (i >= n) l.ranks[i] = ~0ull;
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      __syncthreads();
      for (int i = threadIdx.x; i < size / 2; i += kDrawThreads) {
        const int a = (i / j) * 2 * j + i % j, c = a + j;
        const unsigned long long x = l.ranks[a], y = l.ranks[c];
        if ((x > y) == ((a & k) == 0)) {
          l.ranks[a] = y;
          l.ranks[c] = x;
        }
      }
    }
  __syncthreads();
  // weights in that order, two per thread
  const int a = 2 * threadIdx.x;
  const double x = a < n ? weigh(~static_cast<uint32_t>(l.ranks[a] >> 32)) : 0.0, y = a + 1 < n ? weigh(~static_cast<uint32_t>(l.ranks[a + 1] >> 32)) : 0.0;
  const double sum = before + block_scan<kDrawThreads>(x + y, l.dwaves);
  l.upto[a] = sum - y;
  l.upto[a + 1] = sum;
  if (threadIdx.x == 0) l.i[0] = n - 1;
  __syncthreads();
  if (left > 0) {
    if (threadIdx.x == 0) l.i[0] = left < n ? left - 1 : n - 1;
  } else {
    for (int i = a; i < a + 2; ++i)
      if (i < n && l.upto[i] >= goal) {
        atomicMin(&l.i[0], i);
        break;
      }
  }
  __syncthreads();
  const int at = l.i[0] < 0 ? 0 : l.i[0];
  return Reached{l.ranks[at], l.upto[at]};
}

template <typename T>
__global__ __launch_bounds__(kDrawThreads) void sample_draw_kernel(Params p) {
  constexpr int N = 16 / sizeof(T);
  __shared__ DrawLds l;
  const int r = blockIdx.x;
  const Row w = row_of(p, r);
  const Slice *const slices = p.slices + static_cast<int64_t>(r) * p.n_slices;
  Whole all = whole_of(p, r);
  if (all.nan || all.most == -INFINITY) {
    if (threadIdx.x == 0) {
      p.tokens[r] = -1;
      if (p.logprob) p.logprob[r] = NAN;
    }
    return;
  }
  if (w.greedy) {
    int first = INT32_MAX;
    for (int i = threadIdx.x & 63; i < p.n_slices; i += 64)
      if (slices[i].most == all.most && slices[i].first < first) first = slices[i].first;
    first = wave_min(first);
    if (threadIdx.x == 0) {
      p.tokens[r] = first;
      if (p.logprob) p.logprob[r] = 0.0f;
    }
    return;
  }
  const double unit = w.filtered ? w.per_bin : 0.25 * w.per_bin;   // what the slices' tops are in
  all.top = floor(place_of(all.most, unit));
  // ---- the kept tokens: rank <= last, place >= least
  unsigned long long last = ~0ull;
  double least = -INFINITY;
  if (!w.filtered) {
    for (int i = threadIdx.x; i < p.n_slices; i += kDrawThreads)
      l.of_slice[i] = slices[i].most > -INFINITY ? ldexp(slices[i].sum, static_cast<int>(fmax(slices[i].top - all.top, -2000.0))) : 0.0;
  } else {
    const Cut &c = p.cuts[r];
    const int listed = c.listed;
    if (w.m > 0.0f) least = place_of(all.most, w.per_bin) + 4.0 * log2(static_cast<double>(w.m));
    int end = kBins;   // bin that has the last kept token
    double goal = 0.0;
    const auto weight_ahead = [&](int b) { return b > 0 ? c.upto_weight[b - 1] : 0.0; };
    const auto tokens_in = [&](int b) { return c.upto_count[b] - (b > 0 ? c.upto_count[b - 1] : 0); };
    // top-k's last token is looked for where it can be the last one, and where top-p takes a share of the weight up to it
    double kept = c.all;
    if (c.k_bin < kBins) {
      kept = c.upto_weight[c.k_bin];
      if (c.k_bin <= c.upto || (c.p_on && tokens_in(c.k_bin) > c.k_left)) {
        const Reached at = resolve<T>(p, r, listed, w, all.top, c.k_bin, tokens_in(c.k_bin), weight_ahead(c.k_bin), c.k_left, 0.0, l);
        last = at.rank;
        kept = at.weight;
        end = c.k_bin;
      }
    }
    if (c.p_on && c.from < kBins) {
      goal = static_cast<double>(w.p) * kept;
      int b = c.from;
      while (b < c.upto && c.upto_weight[b] < goal) ++b;
      // (where min-p ends ahead of it, the bin has no token that counts)
      if (b < kBins && tokens_in(b) > 0 && c.upto_weight[b] >= goal * (1.0 - 1e-9)) {
        const Reached at = resolve<T>(p, r, listed, w, all.top, b, tokens_in(b), weight_ahead(b), 0, goal, l);
        if (at.rank < last) last = at.rank;
        if (b < end) end = b;
      }
    }
    if (w.m > 0.0f) {
      const int m_bin = bin_of(all.top, floor(least));
      if (m_bin < end) end = m_bin;
    }
    // ---- the slices' kept weights: all bins ahead of `end`, and what is kept in it
    for (int i = threadIdx.x; i < p.n_slices; i += kDrawThreads) l.cut_steps[i] = 0;
    __syncthreads();
    if (end < kBins - 1) {
      const int skew = RowAt<T>(p, r).skew;
      each_candidate<T>(p, r, listed, [&](uint32_t key, uint32_t index) {
        const double y = place_of(of_key(key), w.per_bin), f = floor(y);
        if (bin_of(all.top, f) != end || rank_of(key, index) > last || y < least) return;
        atomicAdd(&l.cut_steps[(index + skew) / p.slice], steps_of(in_bin(y - f)));
      });
    }
    __syncthreads();
    const unsigned long long *const bins = p.bins + static_cast<int64_t>(r) * p.n_slices * kBins;
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < p.n_slices; i += kDrawThreads / 64) {
      double sum = 0.0;
      if (slices[i].most > -INFINITY) {
        const int off = behind(all.top, slices[i].top);
#pragma unroll
        for (int j = 0; j < kBins / 64; ++j) {
          const int b = 64 * j + lane;
          if (b < kBins - 1 && b + off < end && b + off < kBins - 1) sum += static_cast<double>(bins[i * kBins + b] >> kCountBits) * kStep * end_of_bin(b + off);
        }
      }
      sum = wave_sum(sum);
      if (lane == 0) l.of_slice[i] = sum + (end < kBins - 1 ? static_cast<double>(l.cut_steps[i]) * kStep * end_of_bin(end) : 0.0);
    }
  }
  __syncthreads();
  // ---- the slice
  float u = p.u[r];
  u = u > 0.0f ? (u < 1.0f ? u : 0x1.fffffep-1f) : 0.0f;
  double total = 0.0;
  for (int i = 0; i < p.n_slices; ++i) total += l.of_slice[i];
  const double goal = static_cast<double>(u) * total;
  double before = 0.0, upto = 0.0;
  int slice = 0;
  for (int i = 0; i < p.n_slices; ++i) {
    const double x = l.of_slice[i];
    if (x > 0.0) {   // (the last one that has any, if rounding leaves none)
      slice = i;
      before = upto;
    }
    upto += x;
    if (upto > goal) break;
  }
  // ---- the token: eight neighbours per thread
  const RowAt<T> row(p, r);
  const int at = slice * p.slice + 8 * static_cast<int>(threadIdx.x);
  double weight[8], sum = 0.0;
#pragma unroll
  for (int v = 0; v < 8 / N; ++v) {
    float x[N];
    if (8 * static_cast<int>(threadIdx.x) < p.slice) {
      load16(row.grid, at + v * N, row.skew, p.vocab, x);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double y = place_of(x[i], w.per_bin);
      const bool kept = x[i] > -INFINITY && y >= least && rank_of(key_of(x[i]), at + v * N + i - row.skew) <= last;
      double one = 0.0;   // as in the slices' sums
      if (kept && w.filtered) {
        const double f = floor(y);
        const int b = bin_of(all.top, f);
        if (b < kBins - 1) one = static_cast<double>(steps_of(in_bin(y - f))) * kStep * end_of_bin(b);
      } else if (kept) {
        const double o = 0.25 * y, f = floor(o);
        one = ldexp(in_octave(o - f), static_cast<int>(fmax(f - all.top, -2000.0)));
      }
      weight[v * N + i] = one;
      sum += one;
    }
  }
  const double ahead = before + block_scan<kDrawThreads>(sum, l.dwaves) - sum;
  if (threadIdx.x == 0) {
    l.i[0] = INT32_MAX;
    l.i[1] = -1;
  }
  __syncthreads();
  double run = ahead;
  int mine = INT32_MAX, any = -1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    run += weight[i];
    if (weight[i] > 0.0) {
      any = at + i;
      if (run > goal && mine == INT32_MAX) mine = at + i;
    }
  }
  if (mine != INT32_MAX) atomicMin(&l.i[0], mine);
  if (any >= 0) atomicMax(&l.i[1], any);
  __syncthreads();
  const int token = l.i[0] != INT32_MAX ? l.i[0] : l.i[1];
  if (token >= at && token < at + 8) {
    p.tokens[r] = token - row.skew;
    if (p.logprob) {
      double one = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (token == at + i) one = weight[i];
      p.logprob[r] = static_cast<float>(log(one / total));
    }
  }
}

// ---- host
int slice_of(int64_t rows, int vocab) {
  int s = kMostSlice;
  while (s > kLeastSlice && rows * ((vocab + s - 1) / s) < 512) s /= 2;
  return s;
}
int slices_of(int vocab, int slice) { return (vocab + 7 + slice - 1) / slice; }   // (a row may begin 7 places behind an aligned one)
int list_of(int vocab) { return vocab < kListMost ? vocab : kListMost; }

struct Space {
  int slice, n_slices, list_most;
  int64_t bins, cuts, lists, bytes;   // offsets; the slices are first
};
Space space_of(int64_t rows, int vocab) {
  Space s;
  const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
  s.slice = slice_of(rows, vocab);
  s.n_slices = slices_of(vocab, s.slice);
  s.list_most = list_of(vocab);
  s.bins = up(rows * s.n_slices * static_cast<int64_t>(sizeof(Slice)));
  s.cuts = s.bins + rows * s.n_slices * kBins * 8;
  s.lists = s.cuts + up(rows * static_cast<int64_t>(sizeof(Cut)));
  s.bytes = s.lists + rows * s.list_most * static_cast<int64_t>(sizeof(Entry));
  return s;
}

int check_sizes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1) return SDVG_ERR_SHAPE;
  if (vocab > kMostVocab || static_cast<int64_t>(rows) * slices_of(vocab, kMostSlice) >= (1 << 23)) return SDVG_ERR_UNSUPPORTED;
  return SDVG_OK;
}

template <typename T, int kSlice>
int launch(const Params &p, bool filters, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(p.n_rows) * p.n_slices);
  hipLaunchKernelGGL((sample_slices_kernel<T, kSlice>), grid, dim3(kSliceThreads), 0, s, p);
  SDVG_HIP_CHECK(hipGetLastError());
  if (filters) {
    hipLaunchKernelGGL((sample_collect_kernel<T, kSlice>), grid, dim3(kSliceThreads), 0, s, p);
    SDVG_HIP_CHECK(hipGetLastError());
  }
  hipLaunchKernelGGL((sample_draw_kernel<T>), dim3(p.n_rows), dim3(kDrawThreads), 0, s, p);
  SDVG_HIP_CHECK(hipGetLastError());
  return SDVG_OK;
}
template <typename T>
int launch(const Params &p, bool filters, hipStream_t s) {
  return p.slice == 2048 ? launch<T, 2048>(p, filters, s) : p.slice == 4096 ? launch<T, 4096>(p, filters, s) : launch<T, 8192>(p, filters, s);
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
  const Params p{static_cast<const char *>(a->logits), a->u, a->temperature, a->top_p, a->min_p, a->top_k, a->tokens, a->logprob,
                 a->all_temperature, a->all_top_p, a->all_min_p, a->all_top_k, a->n_rows > 1 ? a->row_stride : 0, a->n_rows, a->vocab, s.slice,
                 s.n_slices, s.list_most, reinterpret_cast<Slice *>(at), reinterpret_cast<unsigned long long *>(at + s.bins),
                 reinterpret_cast<Cut *>(at + s.cuts), reinterpret_cast<Entry *>(at + s.lists)};
  const bool filters = a->top_k || a->top_p || a->min_p || (a->all_top_k > 0 && a->all_top_k < a->vocab) || a->all_top_p < 1.0f || a->all_min_p > 0.0f;
  hipStream_t q = static_cast<hipStream_t>(stream);
  return a->dtype == SDVG_F32 ? launch<float>(p, filters, q) : a->dtype == SDVG_BF16 ? launch<__bf16>(p, filters, q) : launch<_Float16>(p, filters, q);
}
