// Rows of the new tokens of a step: rotary embedding by positions, and the commit into the paged cache with the rotation on
// the way. One kernel does both: for every token the rows of up to three tensors (q rotated, k rotated and / or
// stored, v stored).
//
// Angles: turns = position * freq / (2 pi) in 64 bits, of which only the distance r to the nearest quarter turn
// (|r| <= 1/8) is rounded to 32; sine and cosine of r are exchanged and negated by the quarter. A position of 2^20 times a
// frequency near 1 has 17 bits before the point: in 32 bits 7 would be left behind it.
// A token's 64 sines and cosines are computed once by 64 threads and kept in LDS for all of its rows; with a thread per 16-byte
// chunk, as the pass with tables has it, the angles would cost more vector time than the copy takes from HBM.
#include "paged_kv.h"
#include "row_map.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kThreads = 256;
constexpr int kUnits = 8;             // a row's 128 elements in units of two groups of 8 (the two halves of 8 pairs, or neighbours)
constexpr float kE4m3Max = 448.0f;

struct RowsArg {
  const void *in;
  void *out;
  int64_t in_ts, in_hs, out_ts, out_hs;
};

struct RowsParams {
  RowsArg t[3];               // rotated rows | rows that are stored in k (or a second rotated tensor) | rows that are stored in v
  uint32_t first1, first2, n_rows;  // rows per token: those of t[0] come first, then t[1] from first1 on, t[2] from first2 on
  uint32_t n_tokens;
  const int32_t *positions;   // null: nothing is rotated
  const double *freqs;
  int rotary_units;           // rotary_dim / 16
  float gain;
  const int64_t *slots;       // null: nothing is stored in a cache
  uint32_t n_slots;
  sdvg::FastDiv page;
  int64_t page_stride, token_stride, head_stride;
  const float *scale[2];      // of k and v per head, or null
  sdvg::FastDiv rows;         // by n_rows
};

// Eight elements as floats and back. E: element type.
struct Bf16 {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ void load(const void *p, float *x) {
    const u32x4 v = *static_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(void *p, const float *x) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 f = {x[2 * i], x[2 * i + 1]};
      const bf16x2 b = __builtin_convertvector(f, bf16x2);
      unsigned int w;
      __builtin_memcpy(&w, &b, 4);
      v[i] = w;
    }
    *static_cast<u32x4 *>(p) = v;
  }
};
struct F16 {
  static constexpr int kBytes = 2;
  typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
  static __device__ __forceinline__ void load(const void *p, float *x) {
    const f16x8 v = *static_cast<const f16x8 *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
  }
  static __device__ __forceinline__ void store(void *p, const float *x) {
    f16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<_Float16>(x[i]);
    *static_cast<f16x8 *>(p) = v;
  }
};
struct F32 {
  static constexpr int kBytes = 4;
  typedef __attribute__((ext_vector_type(4))) float f32x4;
  static __device__ __forceinline__ void load(const void *p, float *x) {
    const f32x4 a = static_cast<const f32x4 *>(p)[0], b = static_cast<const f32x4 *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
  static __device__ __forceinline__ void store(void *p, const float *x) {
    static_cast<f32x4 *>(p)[0] = f32x4{x[0], x[1], x[2], x[3]};
    static_cast<f32x4 *>(p)[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
};
struct E4m3 {
  static constexpr int kBytes = 1;
  static __device__ __forceinline__ void store(void *p, const float *x) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = fminf(fmaxf(x[i], -kE4m3Max), kE4m3Max);
      y[i] = x[i] != x[i] ? x[i] : y[i];  // (the clamp would make a number of a NaN)
    }
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    *static_cast<u32x2 *>(p) = u32x2{static_cast<unsigned int>(lo), static_cast<unsigned int>(hi)};
  }
};

// gain * cos and gain * sin of position * freq.
__device__ __forceinline__ void turn(int position, double freq, float gain, float &c, float &s) {
  constexpr double kTurnsPerRadian = 0.15915494309189533577;
  const double quarters = 4.0 * (position * (freq * kTurnsPerRadian));
  const double q = rint(quarters);
  const float r = static_cast<float>(0.5 * (quarters - q));  // of half a turn, |r| <= 1/4
  float sr, cr;
  sincospif(r, &sr, &cr);
  const int n = static_cast<int>(q - 4.0 * floor(0.25 * q));  // quarter 0 .. 3
  c = gain * (n & 1 ? sr : cr);
  s = gain * (n & 1 ? cr : sr);
  if (n == 1 || n == 2) c = -c;
  if (n >= 2) s = -s;
}

// T: type of the rows, C: type of the cache (T where none is written). A workgroup has kTok tokens; 8 threads share a row.
template <typename T, typename C, bool kHalf, int kTok>
__global__ __launch_bounds__(kThreads) void paged_rows_kernel(RowsParams p) {
  __shared__ float cs[kTok][64], sn[kTok][64];
  const uint32_t first = blockIdx.x * kTok;
  const uint32_t n_tok = p.n_tokens - first < kTok ? p.n_tokens - first : kTok;
  if (p.positions) {
    for (uint32_t i = threadIdx.x; i < kTok * 64; i += kThreads) {
      const uint32_t t = i >> 6, pair = i & 63;
      if (t < n_tok && pair < 8u * p.rotary_units) turn(p.positions[first + t], p.freqs[pair], p.gain, cs[t][pair], sn[t][pair]);
    }
    __syncthreads();
  }
  const int u = threadIdx.x & (kUnits - 1);
  for (uint32_t i = threadIdx.x / kUnits; i < n_tok * p.n_rows; i += kThreads / kUnits) {
    const uint32_t t = p.rows.div(i), row = i - t * p.n_rows;
    const int which = row >= p.first2 ? 2 : row >= p.first1 ? 1 : 0;
    const uint32_t head = row - (which == 2 ? p.first2 : which == 1 ? p.first1 : 0);
    const RowsArg &a = p.t[which];
    const bool rotate = p.positions && which < 2 && u < p.rotary_units, store = p.slots && which > 0;
    // the unit's two groups of 8 elements: pairs 8u .. 8u + 7 where it is rotated
    const int g0 = kHalf && u < p.rotary_units ? 8 * u : 16 * u;
    const int g1 = kHalf && u < p.rotary_units ? 8 * (u + p.rotary_units) : 16 * u + 8;
    char *dst;
    if (store) {
      const int64_t slot = p.slots[first + t];
      if (slot < 0 || slot >= p.n_slots) continue;
      const uint32_t page = p.page.div(static_cast<uint32_t>(slot)), place = static_cast<uint32_t>(slot) - page * p.page.d;
      dst = static_cast<char *>(a.out) + (page * p.page_stride + place * p.token_stride + head * p.head_stride) * C::kBytes;
    } else {
      dst = static_cast<char *>(a.out) + (static_cast<int64_t>(first + t) * a.out_ts + head * a.out_hs) * T::kBytes;
    }
    const char *src = static_cast<const char *>(a.in) + (static_cast<int64_t>(first + t) * a.in_ts + head * a.in_hs) * T::kBytes;
    float x[16];
    T::load(src + g0 * T::kBytes, x);
    T::load(src + g1 * T::kBytes, x + 8);
    if (rotate) {
      const float *c = &cs[t][8 * u], *s = &sn[t][8 * u];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float &re = kHalf ? x[j] : x[2 * j], &im = kHalf ? x[8 + j] : x[2 * j + 1];
        const float a0 = re, b0 = im;
        re = __fmaf_rn(a0, c[j], -__fmul_rn(b0, s[j]));
        im = __fmaf_rn(a0, s[j], __fmul_rn(b0, c[j]));
      }
    }
    if (store) {
      if (p.scale[which - 1]) {
        const float scale = p.scale[which - 1][head];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = x[j] / scale;
      }
      C::store(dst + g0 * C::kBytes, x);
      C::store(dst + g1 * C::kBytes, x + 8);
    } else {
      T::store(dst + g0 * T::kBytes, x);
      T::store(dst + g1 * T::kBytes, x + 8);
    }
  }
}

int check_rope(const sdvg_rope_desc *r, int64_t n_tokens) {
  if (r->layout != SDVG_ROPE_INTERLEAVED && r->layout != SDVG_ROPE_HALF) return SDVG_ERR_UNSUPPORTED;
  if (r->rotary_dim < 16 || r->rotary_dim > 128) return SDVG_ERR_SHAPE;
  if (r->rotary_dim & 15) return SDVG_ERR_ALIGN;
  if (!(r->gain - r->gain == 0.f)) return SDVG_ERR_RANGE;  // not finite
  if (n_tokens > 0 && (!r->positions || !r->freqs)) return SDVG_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(r->positions) & 3) || (reinterpret_cast<uintptr_t>(r->freqs) & 7)) return SDVG_ERR_ALIGN;
  return SDVG_OK;
}

// Checks a set of rows (`out`: whether they are written at r->out) and fills its argument.
int check_rows(const sdvg_rows *r, int64_t n_tokens, int size, bool out, RowsArg &a) {
  if (r->n_heads < 1) return SDVG_ERR_SHAPE;
  if (n_tokens > 0 && (!r->in || (out && !r->out))) return SDVG_ERR_NULL;
  int st = sdvg::check_stride(n_tokens, r->in_token_stride, size);
  if (st == SDVG_OK) st = sdvg::check_stride(r->n_heads, r->in_head_stride, size);
  if (st == SDVG_OK && out) st = sdvg::check_stride(n_tokens, r->out_token_stride, size);
  if (st == SDVG_OK && out) st = sdvg::check_stride(r->n_heads, r->out_head_stride, size);
  if (st != SDVG_OK) return st;
  if (!sdvg::aligned16(r->in) || (out && !sdvg::aligned16(r->out))) return SDVG_ERR_ALIGN;
  // (rows of slices of one wide tensor lie between each other, so an overlap is only told by an equal start)
  if (out && n_tokens > 0 && r->in == r->out &&
      ((n_tokens > 1 && r->in_token_stride != r->out_token_stride) || (r->n_heads > 1 && r->in_head_stride != r->out_head_stride)))
    return SDVG_ERR_RANGE;
  a = RowsArg{r->in, r->out, r->in_token_stride, r->in_head_stride, r->out_token_stride, r->out_head_stride};
  return SDVG_OK;
}

template <typename T, typename C, bool kHalf>
int launch_rows(const RowsParams &p, hipStream_t s) {
  // Few tokens: a workgroup each, so that more compute units work on them. Many: 4, which fills the computation of the
  // angles (64 per token) with all threads.
  if (p.n_tokens < 1024) {
    hipLaunchKernelGGL((paged_rows_kernel<T, C, kHalf, 1>), dim3(p.n_tokens), dim3(kThreads), 0, s, p);
  } else {
    hipLaunchKernelGGL((paged_rows_kernel<T, C, kHalf, 4>), dim3((p.n_tokens + 3) / 4), dim3(kThreads), 0, s, p);
  }
  SDVG_HIP_CHECK(hipGetLastError());
  return SDVG_OK;
}
template <typename T, typename C>
int launch_rows(const RowsParams &p, bool half, hipStream_t s) {
  return half ? launch_rows<T, C, true>(p, s) : launch_rows<T, C, false>(p, s);
}

// Rows per token and tokens, checked against what the kernel counts in 32 bits.
int set_rows(RowsParams &p, int64_t h0, int64_t h1, int64_t h2, int64_t n_tokens) {
  const int64_t per_token = h0 + h1 + h2;
  if (per_token > (1 << 24) || n_tokens >= (1 << 26)) return SDVG_ERR_UNSUPPORTED;  // (a grid holds fewer than 2^32 threads)
  p.first1 = static_cast<uint32_t>(h0);
  p.first2 = static_cast<uint32_t>(h0 + h1);
  p.n_rows = static_cast<uint32_t>(per_token);
  p.n_tokens = static_cast<uint32_t>(n_tokens);
  p.rows = sdvg::FastDiv::of(p.n_rows);
  return SDVG_OK;
}

void set_rope(RowsParams &p, const sdvg_rope_desc &r) {
  p.positions = r.positions;
  p.freqs = r.freqs;
  p.rotary_units = r.rotary_dim / 16;
  p.gain = r.gain;
}

}  // namespace

namespace sdvg {

int check_paged_kv(const sdvg_paged_kv *c) {
  if (!c || !c->k || !c->v) return SDVG_ERR_NULL;
  if (c->head_dim != 128) return SDVG_ERR_UNSUPPORTED;
  if (c->dtype != SDVG_BF16 && c->dtype != SDVG_F16 && c->dtype != SDVG_E4M3) return SDVG_ERR_UNSUPPORTED;
  if (c->dtype != SDVG_E4M3 && (c->k_scale || c->v_scale)) return SDVG_ERR_UNSUPPORTED;
  if (c->n_pages < 1 || c->page_tokens < 1 || c->n_kv_heads < 1) return SDVG_ERR_SHAPE;
  if (c->page_tokens & 7) return SDVG_ERR_ALIGN;
  if (int64_t{c->n_pages} * c->page_tokens > INT32_MAX) return SDVG_ERR_UNSUPPORTED;
  if (!aligned16(c->k) || !aligned16(c->v)) return SDVG_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 3) return SDVG_ERR_ALIGN;
  // Rows must not overlap: taken from the smallest stride to the largest, each steps over all that the smaller ones span.
  struct Dim {
    int64_t n, stride;
  } d[3] = {{c->n_pages, c->page_stride}, {c->page_tokens, c->token_stride}, {c->n_kv_heads, c->head_stride}};
  for (const Dim &x : d) {
    const int st = check_stride(x.n, x.stride, element_bytes(c->dtype));
    if (st != SDVG_OK) return st;
  }
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      if (d[j].stride > d[j + 1].stride) {
        const Dim x = d[j];
        d[j] = d[j + 1];
        d[j + 1] = x;
      }
  int64_t span = 128;
  for (const Dim &x : d) {
    if (x.n <= 1) continue;
    if (x.stride < span) return SDVG_ERR_SHAPE;
    span += (x.n - 1) * x.stride;
  }
  return SDVG_OK;
}

int64_t paged_pool_bytes(const sdvg_paged_kv &c) {
  return (rows_span(c.n_pages, c.page_stride, c.page_tokens, c.token_stride) +
          (c.n_kv_heads > 1 ? (c.n_kv_heads - 1) * c.head_stride : 0)) * element_bytes(c.dtype);
}

}  // namespace sdvg

extern "C" int sdvg_rope_positions(const sdvg_rope_desc *rope, const sdvg_rows *x, const sdvg_rows *y, int64_t n_tokens,
                                   int32_t head_dim, int32_t dtype, void *stream) {
  if (!rope || !x) return SDVG_ERR_NULL;
  if (n_tokens < 0) return SDVG_ERR_SHAPE;
  if (head_dim != 128 || (dtype != SDVG_BF16 && dtype != SDVG_F16 && dtype != SDVG_F32)) return SDVG_ERR_UNSUPPORTED;
  const int size = sdvg::element_bytes(dtype);
  RowsParams p{};
  int st = check_rope(rope, n_tokens);
  if (st == SDVG_OK) st = check_rows(x, n_tokens, size, true, p.t[0]);
  if (st == SDVG_OK && y) st = check_rows(y, n_tokens, size, true, p.t[1]);
  if (st == SDVG_OK) st = set_rows(p, x->n_heads, y ? y->n_heads : 0, 0, n_tokens);
  if (st != SDVG_OK || n_tokens == 0) return st;
  set_rope(p, *rope);
  const bool half = rope->layout == SDVG_ROPE_HALF;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == SDVG_BF16  ? launch_rows<Bf16, Bf16>(p, half, s)
         : dtype == SDVG_F16 ? launch_rows<F16, F16>(p, half, s)
                             : launch_rows<F32, F32>(p, half, s);
}

extern "C" int sdvg_paged_commit(const sdvg_paged_kv *cache, const sdvg_rows *k, const sdvg_rows *v, const int64_t *slots,
                                 int64_t n_tokens, int32_t dtype, const sdvg_rope_desc *rope, const sdvg_rows *q,
                                 void *stream) {
  if (!cache || !k || !v) return SDVG_ERR_NULL;
  int st = sdvg::check_paged_kv(cache);
  if (st != SDVG_OK) return st;
  if (n_tokens < 0 || k->n_heads != cache->n_kv_heads || v->n_heads != cache->n_kv_heads) return SDVG_ERR_SHAPE;
  if (dtype != SDVG_BF16 && dtype != SDVG_F16) return SDVG_ERR_UNSUPPORTED;
  if (cache->dtype != dtype && cache->dtype != SDVG_E4M3) return SDVG_ERR_UNSUPPORTED;
  if (q && !rope) return SDVG_ERR_NULL;
  if (n_tokens > 0 && !slots) return SDVG_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(slots) & 7) return SDVG_ERR_ALIGN;
  RowsParams p{};
  if (rope) st = check_rope(rope, n_tokens);
  if (st == SDVG_OK && q) st = check_rows(q, n_tokens, 2, true, p.t[0]);
  if (st == SDVG_OK) st = check_rows(k, n_tokens, 2, false, p.t[1]);
  if (st == SDVG_OK) st = check_rows(v, n_tokens, 2, false, p.t[2]);
  if (st == SDVG_OK) st = set_rows(p, q ? q->n_heads : 0, cache->n_kv_heads, cache->n_kv_heads, n_tokens);
  if (st != SDVG_OK) return st;
  if (n_tokens == 0) return SDVG_OK;
  const int64_t pool = sdvg::paged_pool_bytes(*cache);
  for (const sdvg_rows *r : {k, v}) {
    const int64_t span = sdvg::rows_span(n_tokens, r->in_token_stride, r->n_heads, r->in_head_stride) * 2;
    if (!sdvg::disjoint(r->in, span, cache->k, pool) || !sdvg::disjoint(r->in, span, cache->v, pool)) return SDVG_ERR_RANGE;
  }
  if (rope) set_rope(p, *rope);
  p.t[1].out = cache->k;
  p.t[2].out = cache->v;
  p.slots = slots;
  p.n_slots = static_cast<uint32_t>(cache->n_pages) * static_cast<uint32_t>(cache->page_tokens);
  p.page = sdvg::FastDiv::of(cache->page_tokens);
  p.page_stride = cache->n_pages > 1 ? cache->page_stride : 0;
  p.token_stride = cache->token_stride;
  p.head_stride = cache->n_kv_heads > 1 ? cache->head_stride : 0;
  p.scale[0] = cache->k_scale;
  p.scale[1] = cache->v_scale;
  const bool half = rope && rope->layout == SDVG_ROPE_HALF, e4m3 = cache->dtype == SDVG_E4M3;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == SDVG_BF16) return e4m3 ? launch_rows<Bf16, E4m3>(p, half, s) : launch_rows<Bf16, Bf16>(p, half, s);
  return e4m3 ? launch_rows<F16, E4m3>(p, half, s) : launch_rows<F16, F16>(p, half, s);
}
