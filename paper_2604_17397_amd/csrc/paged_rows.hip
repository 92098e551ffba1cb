// Rows of the new tokens of a step: rotary embedding by positions, and the commit into the paged cache with the rotation on
// the way. One kernel does both: for every token the rows of up to three tensors (q rotated, k rotated and / or
// stored, v stored).
//
// Angles: turns = position * freq / (2 pi) in 64 bits and a rest, of which only the distance r to the nearest quarter turn
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
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kThreads = 256;
constexpr int kUnits = 8;             // threads per row, each with two groups of 8 elements
constexpr int kPass = kThreads / kUnits, kUnroll = 2;  // rows that a workgroup takes at a time, and how many times
constexpr int64_t kMaxTokens = (1 << 26) - 3;  // a grid holds fewer than 2^32 threads, a workgroup has 1 or 4 tokens
constexpr float kE4m3Max = 448.0f;

struct RowsArg {
  const void *in;
  void *out;
  uint32_t in_ts, in_hs, out_ts, out_hs;  // elements, below 2^30
  sdvg::FastDiv heads;
};

struct RowsParams {
  RowsArg t[3];               // rotated rows | rows that are stored in k (or a second rotated tensor) | rows that are stored in v; heads.d 0: none
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
};

// Eight elements as they come from memory (raw), as floats, and back.
template <bool kStream, typename V>
__device__ __forceinline__ void put(void *p, V v) {
  if (kStream)
    __builtin_nontemporal_store(v, static_cast<V *>(p));
  else
    *static_cast<V *>(p) = v;
}
struct Bf16 {
  typedef u32x4 raw;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ raw fetch(const void *p) { return *static_cast<const raw *>(p); }
  static __device__ __forceinline__ void widen(raw v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  template <bool kStream>
  static __device__ __forceinline__ void store(void *p, const float *x) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 f = {x[2 * i], x[2 * i + 1]};
      v[i] = __builtin_bit_cast(unsigned int, __builtin_convertvector(f, bf16x2));
    }
    put<kStream>(p, v);
  }
};
struct F16 {
  typedef __attribute__((ext_vector_type(8))) _Float16 raw;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ raw fetch(const void *p) { return *static_cast<const raw *>(p); }
  static __device__ __forceinline__ void widen(raw v, float *x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
  }
  template <bool kStream>
  static __device__ __forceinline__ void store(void *p, const float *x) {
    raw v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<_Float16>(x[i]);
    put<kStream>(p, v);
  }
};
struct F32 {
  struct raw {
    f32x4 v[2];
  };
  static constexpr int kBytes = 4;
  static __device__ __forceinline__ raw fetch(const void *p) { return raw{{static_cast<const f32x4 *>(p)[0], static_cast<const f32x4 *>(p)[1]}}; }
  static __device__ __forceinline__ void widen(raw v, float *x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v.v[i >> 2][i & 3];
  }
  template <bool kStream>
  static __device__ __forceinline__ void store(void *p, const float *x) {
    put<kStream>(p, f32x4{x[0], x[1], x[2], x[3]});
    put<kStream>(static_cast<f32x4 *>(p) + 1, f32x4{x[4], x[5], x[6], x[7]});
  }
};
struct E4m3 {
  static constexpr int kBytes = 1;
  template <bool kStream>
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
    put<kStream>(p, u32x2{static_cast<unsigned int>(lo), static_cast<unsigned int>(hi)});
  }
};

// gain * cos and gain * sin of position * freq. 1 / (2 pi) has a second number behind its 53 bits, and both products keep what their
// rounding leaves (fma): with products rounded to 64 bits alone an angle near 2^31 was 7e-7 off, 12 steps of fp32, now 1e-15 whatever
// the position. (No difference in the times below.)
__device__ __forceinline__ void turn(int position, double freq, float gain, float &c, float &s) {
  constexpr double kTurnsPerRadian = 0.15915494309189535, kTurnsRest = -9.839338337591243e-18;
  const double p = position, per = freq * kTurnsPerRadian, per_rest = fma(freq, kTurnsPerRadian, -per) + freq * kTurnsRest;
  const double turns = p * per, rest = fma(p, per, -turns) + p * per_rest;
  const double q = rint(4.0 * turns);
  const float r = static_cast<float>(0.5 * (4.0 * turns - q) + 2.0 * rest);  // of half a turn, |r| <= 1/4
  float sr, cr;
  sincospif(r, &sr, &cr);
  const int n = static_cast<int>(q - 4.0 * floor(0.25 * q));  // quarter 0 .. 3
  c = gain * (n & 1 ? sr : cr);
  s = gain * (n & 1 ? cr : sr);
  if (n == 1 || n == 2) c = -c;
  if (n >= 2) s = -s;
}

__device__ __forceinline__ void turn_pair(float &re, float &im, float c, float s) {
  const float a = re, b = im;
  re = __fmaf_rn(a, c, -__fmul_rn(b, s));
  im = __fmaf_rn(a, s, __fmul_rn(b, c));
}
// 8 pairs of which `re` and `im` are the halves; 4 pairs of neighbours.
__device__ __forceinline__ void turn8(float *re, float *im, const float *c, const float *s) {
#pragma unroll
  for (int k = 0; k < 8; ++k) turn_pair(re[k], im[k], c[k], s[k]);
}
__device__ __forceinline__ void turn4(float *x, const float *c, const float *s) {
#pragma unroll
  for (int k = 0; k < 4; ++k) turn_pair(x[2 * k], x[2 * k + 1], c[k], s[k]);
}

// T: type of the rows, C: type of the cache (T where none is written). A workgroup has kTok tokens of one of the tensors
// (blockIdx.y, so that everything about it is scalar); 8 threads share a row. A thread's kUnroll rows are all asked for before
// the angles are computed or the rows before them are turned.
// Bound by HBM from some thousand rows on: 40 + 40 heads x 4680 tokens, bf16, 31.5 us = 6.1 TB/s; 6007 tokens into e4m3 pages, q of 32
// heads beside k and v of 8, 23 us = 5.9 TB/s. Few tokens: 3 us, a launch and two trips to memory. One row at a time per thread with
// the tensor looked up per row, accesses of 16 bytes 16 apart: 44.8 and 30.9 us.
template <typename T, typename C, bool kHalf, int kTok, bool kStream>
__global__ __launch_bounds__(kThreads) void paged_rows_kernel(RowsParams p) {
  __shared__ float cs[kTok][64], sn[kTok][64];
  const uint32_t first = blockIdx.x * kTok;
  const uint32_t n_tok = p.n_tokens - first < kTok ? p.n_tokens - first : kTok;
  const int which = blockIdx.y;
  const RowsArg a = which == 0 ? p.t[0] : which == 1 ? p.t[1] : p.t[2];
  const bool rotate = p.positions && which < 2, store = p.slots && which > 0;
  const int u = threadIdx.x & (kUnits - 1);
  // The thread's two groups of 8 elements: those of pairs 8u .. 8u + 7 in the half layout, otherwise the u-th of both halves, so
  // that the 8 threads of a row touch whole lines with every access (a nontemporal store of parts of one is slow).
  const int units = rotate ? p.rotary_units : 0, c0 = kHalf && u >= units ? u + units : u, c1 = kHalf && u < units ? u + units : u + 8;
  const int g0 = 8 * c0, g1 = 8 * c1;
  const char *src = static_cast<const char *>(a.in) + static_cast<int64_t>(first) * a.in_ts * T::kBytes;
  char *out = static_cast<char *>(a.out) + (store ? 0 : static_cast<int64_t>(first) * a.out_ts * T::kBytes);
  const uint32_t n_rows = n_tok * a.heads.d;

  typename T::raw x[kUnroll][2];
  const auto load = [&](uint32_t base) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const uint32_t i = base + j * kPass;
      if (i >= n_rows) continue;
      const uint32_t t = kTok == 1 ? 0 : a.heads.div(i), head = i - t * a.heads.d;
      const char *row = src + static_cast<uint64_t>(t) * (a.in_ts * T::kBytes) +
                        static_cast<uint64_t>(head) * (a.in_hs * T::kBytes);
      x[j][0] = T::fetch(row + g0 * T::kBytes);
      x[j][1] = T::fetch(row + g1 * T::kBytes);
    }
  };
  load(threadIdx.x / kUnits);
  if (rotate) {
    for (uint32_t i = threadIdx.x; i < kTok * 64; i += kThreads) {
      const uint32_t t = i >> 6, pair = i & 63;
      if (t < n_tok && pair < 8u * p.rotary_units) turn(p.positions[first + t], p.freqs[pair], p.gain, cs[t][pair], sn[t][pair]);
    }
    __syncthreads();
  }
  for (uint32_t base = threadIdx.x / kUnits; base < n_rows; base += kPass * kUnroll) {
    if (base != threadIdx.x / kUnits) load(base);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const uint32_t i = base + j * kPass;
      if (i >= n_rows) continue;
      const uint32_t t = kTok == 1 ? 0 : a.heads.div(i), head = i - t * a.heads.d;
      float y[16];
      T::widen(x[j][0], y);
      T::widen(x[j][1], y + 8);
      if (kHalf) {
        if (u < units) turn8(y, y + 8, &cs[t][8 * u], &sn[t][8 * u]);
      } else {
        if (c0 < 2 * units) turn4(y, &cs[t][4 * c0], &sn[t][4 * c0]);
        if (c1 < 2 * units) turn4(y + 8, &cs[t][4 * c1], &sn[t][4 * c1]);
      }
      if (store) {
        const int64_t slot = p.slots[first + t];
        if (slot < 0 || slot >= p.n_slots) continue;
        const uint32_t s32 = static_cast<uint32_t>(slot), page = p.page.div(s32), place = s32 - page * p.page.d;
        char *row = out + (page * p.page_stride + place * p.token_stride + head * p.head_stride) * C::kBytes;
        if constexpr (C::kBytes == 1) {
          const float *scale = which == 1 ? p.scale[0] : p.scale[1];
          if (scale) {
            const float d = 1.0f / scale[head];
#pragma unroll
            for (int k = 0; k < 16; ++k) y[k] *= d;
          }
        }
        constexpr bool kWhole = kStream && C::kBytes == 2;
        C::template store<kWhole>(row + g0 * C::kBytes, y);
        C::template store<kWhole>(row + g1 * C::kBytes, y + 8);
      } else {
        char *row = out + static_cast<uint64_t>(t) * (a.out_ts * T::kBytes) +
                    static_cast<uint64_t>(head) * (a.out_hs * T::kBytes);
        constexpr bool kWhole = kStream && T::kBytes == 2;
        T::template store<kWhole>(row + g0 * T::kBytes, y);
        T::template store<kWhole>(row + g1 * T::kBytes, y + 8);
      }
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

// Whether rows that one tensor of a launch is written to are, by their start (see below), what another is read from or written to.
bool meet(const sdvg_rows &written, const void *in, const void *out) { return written.out == in || written.out == out; }

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
  if (r->n_heads > (1 << 20)) return SDVG_ERR_UNSUPPORTED;
  const auto step = [](int64_t n, int64_t stride) { return n > 1 ? static_cast<uint32_t>(stride) : 0u; };  // (free where nothing is stepped over)
  a = RowsArg{r->in, r->out, step(n_tokens, r->in_token_stride), step(r->n_heads, r->in_head_stride), step(n_tokens, r->out_token_stride),
              step(r->n_heads, r->out_head_stride), sdvg::FastDiv::of(r->n_heads)};
  return SDVG_OK;
}

template <typename T, typename C, bool kHalf, int kTok, bool kStream>
int launch_rows(const RowsParams &p, hipStream_t s) {
  hipLaunchKernelGGL((paged_rows_kernel<T, C, kHalf, kTok, kStream>),
                     dim3((p.n_tokens + kTok - 1) / kTok, p.t[2].heads.d ? 3 : p.t[1].heads.d ? 2 : 1), dim3(kThreads), 0, s, p);
  SDVG_HIP_CHECK(hipGetLastError());
  return SDVG_OK;
}
template <typename T, typename C, bool kHalf>
int launch_rows(const RowsParams &p, hipStream_t s) {
  // Few tokens: a workgroup each, so that more compute units work on them, and ordinary stores, however many heads they have. Many: 4, which
  // fills the computation of the angles (64 per token) with all threads, and stores as in the pass with tables: ordinary ones up to 4 MiB,
  // which the next kernel finds in the caches. Beyond, 40 + 40 heads x 4680 tokens called in a row 32 us, with ordinary stores 38
  // (what the last call left to be written back meets the next one's reads); the commit of 6007 tokens 22.6 and 23.8.
  const int64_t rows = static_cast<int64_t>(p.n_tokens) * (p.t[0].heads.d + p.t[1].heads.d + p.t[2].heads.d);
  if (p.n_tokens < 1024) return launch_rows<T, C, kHalf, 1, false>(p, s);
  return rows * 128 * T::kBytes <= (4 << 20) ? launch_rows<T, C, kHalf, 4, false>(p, s) : launch_rows<T, C, kHalf, 4, true>(p, s);
}
template <typename T, typename C>
int launch_rows(const RowsParams &p, bool half, hipStream_t s) {
  return half ? launch_rows<T, C, true>(p, s) : launch_rows<T, C, false>(p, s);
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
    const int st = check_stride(x.n, x.stride, element_bytes(c->dtype), int64_t{1} << 40);  // (a pool may be most of the memory)
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
  if (n_tokens >= kMaxTokens) return SDVG_ERR_UNSUPPORTED;
  if (head_dim != 128 || (dtype != SDVG_BF16 && dtype != SDVG_F16 && dtype != SDVG_F32)) return SDVG_ERR_UNSUPPORTED;
  const int size = sdvg::element_bytes(dtype);
  RowsParams p{};
  int st = check_rope(rope, n_tokens);
  if (st == SDVG_OK) st = check_rows(x, n_tokens, size, true, p.t[0]);
  if (st == SDVG_OK && y) st = check_rows(y, n_tokens, size, true, p.t[1]);
  if (st != SDVG_OK || n_tokens == 0) return st;
  if (y && (meet(*x, y->in, y->out) || meet(*y, x->in, nullptr))) return SDVG_ERR_RANGE;
  p.n_tokens = static_cast<uint32_t>(n_tokens);
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
  if (n_tokens >= kMaxTokens || (dtype != SDVG_BF16 && dtype != SDVG_F16)) return SDVG_ERR_UNSUPPORTED;
  if (cache->dtype != dtype && cache->dtype != SDVG_E4M3) return SDVG_ERR_UNSUPPORTED;
  if (q && !rope) return SDVG_ERR_NULL;
  if (n_tokens > 0 && !slots) return SDVG_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(slots) & 7) return SDVG_ERR_ALIGN;
  RowsParams p{};
  if (rope) st = check_rope(rope, n_tokens);
  if (st == SDVG_OK && q) st = check_rows(q, n_tokens, 2, true, p.t[0]);
  if (st == SDVG_OK) st = check_rows(k, n_tokens, 2, false, p.t[1]);
  if (st == SDVG_OK) st = check_rows(v, n_tokens, 2, false, p.t[2]);
  if (st != SDVG_OK || n_tokens == 0) return st;
  p.n_tokens = static_cast<uint32_t>(n_tokens);
  const int64_t pool = sdvg::paged_pool_bytes(*cache);
  const auto apart = [&](const void *rows, int32_t heads, int64_t token_stride, int64_t head_stride) {
    const int64_t span = sdvg::rows_span(n_tokens, token_stride, heads, head_stride) * 2;
    return sdvg::disjoint(rows, span, cache->k, pool) && sdvg::disjoint(rows, span, cache->v, pool);
  };
  for (const sdvg_rows *r : {k, v, q})
    if (r && !apart(r->in, r->n_heads, r->in_token_stride, r->in_head_stride)) return SDVG_ERR_RANGE;
  if (q && (!apart(q->out, q->n_heads, q->out_token_stride, q->out_head_stride) || meet(*q, k->in, v->in))) return SDVG_ERR_RANGE;
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
