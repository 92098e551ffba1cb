// Attention of a few new tokens per request over a paged cache (one decoding or verification step), with the keys of
// long requests split over workgroups and joined.
//
// What bounds it: every cached row of K and V is read once, 512 bytes per key and head in 16 bits, for 4 x 128 FLOP per
// query row; up to some hundred rows per key head the time is the HBM's. So there is no staging through LDS: the matrix
// instructions take both K and V straight from registers as they come from memory.
//
// A wave takes 32 keys per step, and 16 query rows (NT tiles of 16) of a request that share a key head as columns:
//   S^T = K Q^T with v_mfma_f32_16x16x32: lane l holds 8 consecutive dims of key row l % 16, one 16-byte load. The
//     key rows of the two 16-row products are dealt out so that lane l's 8 scores (rows 4 (l / 16) .. + 3 of both) belong to
//     the keys 8 (l / 16) .. + 7 of the step, in order, and to query row l % 16.
//   O^T = V^T P^T: that is the B operand of this product as it is (8 consecutive keys of column l % 16): P never
//     moves between lanes. The A operand wants 8 consecutive keys of one dim per lane, and memory has 8 consecutive dims of one key:
//     lane l loads dims 8 (l % 16) .. + 7 of its 8 keys (a row of 256 bytes per 16 lanes) and transposes this 8 x 8 block among its own
//     registers with 32 v_perm; product d of 8 then has rows 8 m + d of O^T.
// Pages hold multiples of 8 tokens, so such a block of 8 keys lies on one page.
//
// us (kernel and join), TB/s of K and V: one request of 131071 keys, 40 query and 8 key heads, bf16 82 + 6, 6.6 (a read of
// contiguous memory reaches 6.1 to 6.3, with nontemporal loads 6.9 to 7.1; without its arithmetic the kernel takes as long);
// 96 requests of 16 to 16384 keys, f16 190 + 7, 5.9; 24 requests with up to 8 new tokens of 40 heads, window 4096, e4m3 33 + 5, 3.1 (452
// workgroups in one round, which lasts as long as the longest, 24 key tiles; second row tiles of 3 to 8 rows read 22 % of the keys again); one
// request of 936 keys, 12 heads 5.9 + 3 to 4, a chain of latencies: lengths 0.7, page numbers and q 0.6, K and V 1.3, one step 0.5, merge and
// store 0.7, and the launch itself.
#include <math.h>

#include <mutex>
#include <type_traits>

#include "paged_attn_plan.h"
#include "paged_kv.h"
#include "row_map.h"

namespace {

namespace pg = sdvg::paged;

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

constexpr int kJoinThreads = 256;
constexpr int kRows = 16;               // query rows per matrix product
constexpr int kPad = 132;               // floats per row of O in LDS
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What a workgroup needs first, apart from the other arguments: these dwords are preloaded into registers at launch (build.py).
#define FIRST_ARGS                                                                                                    \
  const int32_t *__restrict__ q_start, const int32_t *__restrict__ kv_lens, int32_t n_requests, int32_t n_tokens,     \
      int32_t group, int32_t window, int32_t target, int32_t capacity, uint32_t heads_d, uint32_t heads_m, uint32_t heads_s
struct First {
  const int32_t *q_start, *kv_lens;
  int32_t n_requests, n_tokens, group, window, target;
  int32_t capacity;                   // keys a row of the table can name
  sdvg::FastDiv by_heads;             // workgroups -> items, by (sets of) key heads
};

// What both kernels need of the output. (A launch takes 0.3 us longer per 100 bytes of arguments.)
struct OutParams {
  void *out;
  float *lse, *part_o, *part_ml;      // partial results: O [slot][key head][row][128], (m, l) [slot][key head][row][2]
  const float *v_scale;
  uint32_t o_ts, o_hs;                // elements, below 2^30
  int32_t n_heads;
  sdvg::FastDiv by_group;             // rows -> tokens
};

struct AttnParams {
  const void *q, *k, *v;
  const float *k_scale;
  const int32_t *table;
  int64_t page_stride, token_stride, head_stride;
  uint32_t q_ts, q_hs;                // elements, below 2^30
  int32_t table_stride, table_width, n_pages;
  float scale_log2e;
  sdvg::FastDiv by_page;              // blocks of 8 keys -> pages
  OutParams to;
};

// A workgroup is 4 waves with NT tiles of 16 rows each. HS = 2: two sets of 2 waves have the same rows of neighbouring key heads, whose
// rows of K and V are neighbours in a cache with tokens ahead of heads; read together, they keep more of each visit to a
// memory channel. Two waves per SIMD are what the registers leave room for. (64 rows in two sets of 4 waves with the same keys were
// slower than two workgroups of 32: one request of 131071 keys, 40 to 64 rows, e4m3 101 us and 91.)
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kPerUnit = 2;             // workgroups per compute unit

// ---- the two 16-bit types
// A probability is held as 2^kShift p, p <= 2^kSlack being relative to the running maximum, in the sum as in the product with V. For
// the product it is the sum of two 16-bit numbers, the rounded one and what that rounding leaves, each with its own matrix product:
// rounded once, it was the larger part of the result's error (bf16 2.0e-3 to 2.4e-3 rms, now the 1.65e-3 of the result's own rounding; fp16
// 2.6e-4 and 2.1e-4). us without and with the rest: one request of 131071 keys 87.0, 87.2, 96 requests 196.8, 197.0, 64 x 936 keys 47.8,
// 48.0, one of 936 keys 9.8, 9.8, verification 38.9, 38.8 (16 bits 61.9, 61.3).
// bf16 then has 16 bits and the range of fp32. fp16 has steps of 2^-24 at the least: with 2^13 p, p <= 4, both numbers together have 22 bits
// from 2^-16 of the largest probability down, and a smaller one is off by 2^-38 of the largest at most (many small ones beside one
// large one whose V is small, an attention sink, are what the result then consists of). The maximum is raised more often by it,
// which costs nothing that shows: 96 requests 196.6 us with and without.
struct Bf16 {
  static constexpr float kSlack = 8.0f, kShift = 0.0f, kUnit = 1.0f;   // kUnit = 2^-kShift
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ unsigned pack(float x, float y) {
    const f32x2 f = {x, y};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));
  }
  static __device__ __forceinline__ float first(unsigned w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float second(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
  // elements 2i, 2i + 1 of a dword of four e4m3 numbers (exact in 16 bits)
  static __device__ __forceinline__ unsigned lo8(unsigned w) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  }
  static __device__ __forceinline__ unsigned hi8(unsigned w) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
};
struct F16 {
  static constexpr float kSlack = 2.0f, kShift = 13.0f, kUnit = 0x1p-13f;
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ unsigned pack(float x, float y) {
    const f16x2 h = {static_cast<_Float16>(x), static_cast<_Float16>(y)};
    return __builtin_bit_cast(unsigned, h);
  }
  static __device__ __forceinline__ float first(unsigned w) { return static_cast<float>(__builtin_bit_cast(f16x2, w)[0]); }
  static __device__ __forceinline__ float second(unsigned w) { return static_cast<float>(__builtin_bit_cast(f16x2, w)[1]); }
  static __device__ __forceinline__ unsigned lo8(unsigned w) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
  }
  static __device__ __forceinline__ unsigned hi8(unsigned w) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  }
};
template <typename T>
__device__ __forceinline__ u32x4 widen(u32x2 w) {
  return u32x4{T::lo8(w[0]), T::hi8(w[0]), T::lo8(w[1]), T::hi8(w[1])};
}

// ---- over the 4 lanes that hold one query row (l, l ^ 16, l ^ 32, l ^ 48). A swap of a register with itself leaves the
// pair's two values in its two results.
__device__ __forceinline__ float rows_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum over lanes 0 .. own of a wave: within rows of 16 lanes, then rows to the rows behind them.
__device__ __forceinline__ int scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // last lane of rows 0, 2 to rows 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2, 3
  return x;
}
// 2^x; results below 2^-126 are 0, which a probability beside a largest one of 1 may be.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(scan(x), 63); }

// ---- which part of the work a workgroup has
// Found by every wave for itself: lane i looks at request 64 b + i. Batches of 64 requests at a time.
struct Found {
  pg::Request q;
  int32_t request, tile, piece, pieces, slot, chunk;   // row tile of the request; slot of its first piece; key tiles of a piece
};
template <int kRowTile>
__device__ __forceinline__ pg::Request load_request(const First &p, int r) {
  if (r >= p.n_requests) return pg::Request{0, 0, 0, 0, 0, 0};
  return pg::request_of(p.q_start[r], p.q_start[r + 1], p.kv_lens[r], p.n_tokens, p.group, kRowTile, p.window, p.capacity);
}
// Number `x` among the items (kItems) or among the split row tiles.
template <int kRowTile, int kKeyWaves, bool kItems>
__device__ __forceinline__ bool find(const First &p, int x, Found &f) {
  const int lane = threadIdx.x & 63;
  const pg::Request mine0 = load_request<kRowTile>(p, lane);
  int32_t chunk = INT32_MAX;
  if (p.target > 0) {
    int64_t total = 0, row_tiles = 0;
    for (int b = 0; b < p.n_requests; b += 64) {
      const pg::Request q = b ? load_request<kRowTile>(p, b + lane) : mine0;
      const int64_t w = pg::work_of(q);
      row_tiles += wave_total(q.row_tiles);
      total += wave_total(static_cast<int>(w & 0xffff)) + (static_cast<int64_t>(wave_total(static_cast<int>(w >> 16))) << 16);
    }
    chunk = pg::chunk_of(total, row_tiles, p.target, kKeyWaves);
  }
  // items: the full pieces of all requests come before all others
  int n_full = 0;
  if (kItems && p.target > 0)
    for (int b = 0; b < p.n_requests; b += 64) {
      const pg::Request q = b ? load_request<kRowTile>(p, b + lane) : mine0;
      n_full += wave_total(pg::numbers_of(q, pg::full_pieces(q, chunk), 0, pg::kFull));
    }
  const pg::Range range = !kItems ? pg::kSplit : x < n_full ? pg::kFull : pg::kRest;
  if (range == pg::kRest) x -= n_full;
  int before = 0, slots_before = 0;
  for (int b = 0; b < p.n_requests; b += 64) {
    const pg::Request q = b ? load_request<kRowTile>(p, b + lane) : mine0;
    const int32_t full = pg::full_pieces(q, chunk), pieces = pg::pieces_of(q, chunk, full);
    const int32_t slots = pg::slots_of(q, pieces);
    const int32_t mine = pg::numbers_of(q, full, pieces, range);
    const int upto = scan(mine), slots_upto = scan(slots);  // inclusive
    const int at = x - before - (upto - mine);
    const uint64_t hit = __ballot(at >= 0 && at < mine);
    if (hit) {
      const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      const auto get = [src](int v) { return __builtin_amdgcn_readlane(v, src); };
      f.q = pg::Request{get(q.row0), get(q.n), get(q.len), get(q.first_tile), get(q.tiles), get(q.row_tiles)};
      f.request = b + src;
      f.pieces = get(pieces);
      const pg::Place at_x = pg::place_of(f.q, get(at), get(full), range, p.by_heads.d);
      f.tile = at_x.tile;
      f.piece = at_x.piece;
      f.chunk = chunk;
      f.slot = pg::first_slot(slots_before + get(slots_upto - slots), f.tile, f.pieces);
      // (always so, unless q_start decreases so far that sums leave 32 bits: the workspace is not left even then)
      return f.pieces == 1 || (f.slot >= 0 && f.slot <= pg::max_slots(p.target) - f.pieces);
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    slots_before += __builtin_amdgcn_readlane(slots_upto, 63);
  }
  return false;
}

// T: type of q, of P and of the output. kF8: the cache holds e4m3 numbers.
template <typename T, bool kF8, int NT, int HS>
__global__ __launch_bounds__(kThreads, kPerUnit) void paged_attn_kernel(FIRST_ARGS, AttnParams p) {
  constexpr int kRowTile = kRows * NT, kKeyWaves = kWaves / HS;
  constexpr int kDims = 128 * kRows * HS / kThreads;   // per thread where the workgroup finishes rows
  constexpr int kBytes = kF8 ? 1 : 2;
  __shared__ float o_s[kWaves][kRows][kPad];
  __shared__ float ml_s[kWaves][kRows][2];
  Found f;
  // the key heads of an item are neighbours: together they read whole rows of the cache's tokens
  const First first{q_start, kv_lens, n_requests, n_tokens, group, window, target, capacity, {heads_d, heads_m, heads_s}};
  const int item = first.by_heads.div(blockIdx.x), head0 = (blockIdx.x - item * heads_d) * HS, n_kv_heads = heads_d * HS;
  if (!find<kRowTile, kKeyWaves, true>(first, item, f)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
  const int head = head0 + (HS > 1 ? __builtin_amdgcn_readfirstlane(wave / kKeyWaves) : 0);   // (one for the wave: its addresses stay scalar)
  const int rows = f.q.n * group - f.tile * kRowTile;   // rows of this tile, those past kRowTile included

  // the query rows of this lane: column col of every tile of 16
  u32x4 qf[NT][4];
  int32_t sees[NT], from[NT];   // keys from[..] <= j < sees[..]
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = t * kRows + col;
    const uint32_t all = f.tile * kRowTile + row, i = p.to.by_group.div(all), h = all - i * group;
    sees[t] = from[t] = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[t][s] = u32x4{0, 0, 0, 0};
    if (row < rows) {
      sees[t] = f.q.len - f.q.n + static_cast<int>(i) + 1;
      from[t] = window > 0 && sees[t] > window ? sees[t] - window : 0;
      const uint16_t *src = static_cast<const uint16_t *>(p.q) + (f.q.row0 + static_cast<int64_t>(i)) * p.q_ts +
                            (static_cast<int64_t>(head) * group + h) * p.q_hs;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        // dims of product s in this lane: as K's load has them (below)
        const int d = kF8 ? 64 * (s >> 1) + 16 * quad + 8 * (s & 1) : 32 * s + 8 * quad;
        qf[t][s] = *reinterpret_cast<const u32x4 *>(src + d);
      }
    }
  }
  // tiles in which every row of the workgroup sees every key
  const int last_row = rows < kRowTile ? rows - 1 : kRowTile - 1;
  const int first_i = static_cast<int>(p.to.by_group.div(f.tile * kRowTile)),
            last_i = static_cast<int>(p.to.by_group.div(f.tile * kRowTile + last_row));
  const int all_sees = f.q.len - f.q.n + first_i + 1, last_sees = f.q.len - f.q.n + last_i + 1;
  const int seen_from = window > 0 && all_sees - first_i > window ? all_sees - first_i - window : 0;   // by the request's first token
  const int all_from = window > 0 && last_sees > window ? last_sees - window : 0;

  const float scale = p.scale_log2e * (kF8 && p.k_scale ? p.k_scale[head] : 1.0f);
  f32x4 o[NT][8];
  float m[NT], l[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const pg::KeyTiles keys = pg::key_tiles_of(f.q, f.piece, f.chunk);
  const int begin = keys.begin, end = keys.end;
  const int32_t *table = p.table + static_cast<int64_t>(f.request) * p.table_stride;
  const char *k_head = static_cast<const char *>(p.k) + head * p.head_stride * kBytes,
             *v_head = static_cast<const char *>(p.v) + head * p.head_stride * kBytes;
  // One step's worth of K and V on the way from memory, and where it lies. Loads are issued a step ahead: K's when the
  // scores of the step before are done, V's when its values have been transposed; page numbers two steps ahead, at the start of a
  // step. Loads come back in the order in which they are issued: page numbers that were asked for behind K and V could not be
  // used before both had arrived, and every step took a whole trip to memory.
  struct Place {
    int32_t page;      // -1: not there
    uint32_t token;    // in its page, of the first of the 8 keys
  };
  const auto place_of = [&](uint32_t block) {
    const uint32_t i = p.by_page.div(block);
    const int32_t page = i < static_cast<uint32_t>(p.table_width) ? table[i] : -1;
    return Place{page < p.n_pages ? page : -1, (block - i * p.by_page.d) * 8};
  };
  typedef typename std::conditional<kF8, u32x2, u32x4>::type chunk;  // 8 numbers
  u32x4 kf[2][kF8 ? 2 : 4];
  chunk vf[8];
  // (a page that is not there reads page 0, which is memory of the pool; its keys do not count)
  const auto load_k = [&](const Place &at) {
    const char *row = k_head + ((at.page < 0 ? 0 : at.page) * p.page_stride + (at.token + (col & 3)) * p.token_stride) * kBytes + 16 * quad;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < (kF8 ? 2 : 4); ++s)
        kf[t][s] = *reinterpret_cast<const u32x4 *>(row + 4 * t * p.token_stride * kBytes + 64 * s);
  };
  // (nontemporal: every access takes whole lines, once. K's take half a line each, and the second half of a nontemporal one may be
  // fetched again. One long request, 96 requests, e4m3 verification: 85, 190, 34 us; 92, 206, 36 with neither; 88, 200, 42 with both)
  const auto load_v = [&](const Place &at) {
    const char *row = v_head + ((at.page < 0 ? 0 : at.page) * p.page_stride + at.token * p.token_stride) * kBytes + col * (8 * kBytes);
#pragma unroll
    for (int j = 0; j < 8; ++j) vf[j] = __builtin_nontemporal_load(reinterpret_cast<const chunk *>(row + j * p.token_stride * kBytes));
  };
  Place k_next, v_next;  // of the next step
  // One step; kMore: another one follows.
  const auto step = [&](int tile, int32_t v_page, auto more) {
    constexpr bool kMore = decltype(more)::value;
    const int key0 = tile * pg::kKeyTile;
    Place k_after, v_after;
    if constexpr (kMore) {
      const int after = tile + 2 * kKeyWaves < end ? tile + 2 * kKeyWaves : tile;
      k_after = place_of(after * 4 + (col >> 2));
      v_after = place_of(after * 4 + quad);
    }
    // keys of this lane's block of 8 that a row of the request may see: below .. upto
    const int block0 = key0 + 8 * quad, below = seen_from - block0;
    int upto = f.q.len - block0;
    upto = v_page < 0 ? 0 : upto < 0 ? 0 : upto > 8 ? 8 : upto;
    const bool gaps = __any(upto < 8 || below > 0), masked = gaps || key0 + pg::kKeyTile > all_sees || key0 < all_from;
    u32x4 pf[NT], rest[NT];   // probabilities in 16 bits, and what is left of them
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 k;
          if constexpr (kF8)
            k = widen<T>(u32x2{kf[h][c >> 1][2 * (c & 1)], kf[h][c >> 1][2 * (c & 1) + 1]});
          else
            k = kf[h][c];
          s[h] = T::mfma(k, qf[t][c], s[h]);
        }
      if constexpr (kMore)
        if (t == NT - 1) load_k(k_next);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * scale;
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = block0 + e;
          x[e] = e < upto && key < sees[t] && key >= from[t] ? x[e] : -INFINITY;
        }
      }
      const float high = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      // m is raised only when some row's scores pass it by more than kSlack: numerator and denominator share it, whatever it is
      if (__any(high > m[t] + T::kSlack)) {
        const float top = fmaxf(m[t], rows_max(high));
        const float keep = m[t] == -INFINITY ? 0.f : exp2_of(m[t] - top);
        m[t] = top;
        l[t] *= keep;
#pragma unroll
        for (int d = 0; d < 8; ++d) o[t][d] *= keep;
      }
      const float base = m[t] == -INFINITY ? 0.f : m[t] - T::kShift;   // no key so far: every probability is 2^-inf
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float a = exp2_of(x[2 * c] - base), b = exp2_of(x[2 * c + 1] - base);
        pf[t][c] = T::pack(a, b);
        rest[t][c] = T::pack(a - T::first(pf[t][c]), b - T::second(pf[t][c]));
        l[t] += a + b;
      }
    }
    // V of keys that nobody sees is cleared (0 times anything but a number is no 0)
    if (gaps) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= upto || j < below) vf[j] = chunk{};
    }
    // V^T: dim 2e + h of keys 2c, 2c + 1 from dword e of both
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // (where registers are short nothing moves ahead of its turn: with all of V^T on the way 13 would be spilled, so it takes 229)
      if constexpr (NT == 2 && !kF8) __builtin_amdgcn_sched_barrier(0);
      unsigned w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (kF8)
          w[j] = e & 1 ? T::hi8(vf[j][e >> 1]) : T::lo8(vf[j][e >> 1]);
        else
          w[j] = vf[j][e];
      }
      u32x4 vt[2];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        vt[0][c] = __builtin_amdgcn_perm(w[2 * c + 1], w[2 * c], 0x05040100u);
        vt[1][c] = __builtin_amdgcn_perm(w[2 * c + 1], w[2 * c], 0x07060302u);
      }
      if constexpr (kMore) {
        if (e == 3) {
          load_v(v_next);
          k_next = k_after;
          v_next = v_after;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t][2 * e + h] = T::mfma(vt[h], pf[t], T::mfma(vt[h], rest[t], o[t][2 * e + h]));
    }
  };
  int tile = begin + wave % kKeyWaves;
  if (tile < end) {
    const Place k_at = place_of(tile * 4 + (col >> 2)), v_at = place_of(tile * 4 + quad);
    const int next = tile + kKeyWaves < end ? tile + kKeyWaves : tile;
    k_next = place_of(next * 4 + (col >> 2));
    v_next = place_of(next * 4 + quad);
    load_k(k_at);
    load_v(v_at);
    int32_t page = v_at.page;
    for (; tile + kKeyWaves < end; tile += kKeyWaves) {
      const int32_t page_next = v_next.page;
      step(tile, page, std::true_type{});
      page = page_next;
    }
    step(tile, page, std::false_type{});
  }

  // The waves' results of a tile of 16 rows meet in LDS.
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t * kRows >= rows) break;
    if (t > 0) __syncthreads();
    const float sum = rows_sum(l[t]) * T::kUnit;   // (of p; O stays in units of kUnit until the end)
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // dims 8 (4 quad + i) + d
      float *dst = &o_s[wave][col][8 * (4 * quad + i)];
      *reinterpret_cast<f32x4 *>(dst) = f32x4{o[t][0][i], o[t][1][i], o[t][2][i], o[t][3][i]};
      *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{o[t][4][i], o[t][5][i], o[t][6][i], o[t][7][i]};
    }
    if (quad == 0) {
      ml_s[wave][col][0] = m[t];
      ml_s[wave][col][1] = sum;
    }
    __syncthreads();
    constexpr int kPerRow = 128 / kDims;
    const int r = threadIdx.x / kPerRow, d0 = threadIdx.x % kPerRow * kDims, set = r / kRows, c = r % kRows;
    const int row = t * kRows + c, of_head = head0 + (HS > 1 ? set : 0);
    if (row >= rows) continue;   // (all waves come to the barriers: `rows` is the workgroup's)
    const float(*const ml)[kRows][2] = ml_s + set * kKeyWaves;
    float top = ml[0][c][0], total = 0.f;
    f32x4 acc[kDims / 4] = {};
#pragma unroll
    for (int w = 1; w < kKeyWaves; ++w) top = fmaxf(top, ml[w][c][0]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < kKeyWaves; ++w) {
      const float weight = exp2_of(ml[w][c][0] - base);
      total += weight * ml[w][c][1];
#pragma unroll
      for (int j = 0; j < kDims / 4; ++j)
        acc[j] += weight * *reinterpret_cast<const f32x4 *>(&o_s[set * kKeyWaves + w][c][d0 + 4 * j]);
    }
    if (f.pieces > 1) {
      const int64_t at = (static_cast<int64_t>(f.slot + f.piece) * n_kv_heads + of_head) * kRowTile + row;
#pragma unroll
      for (int j = 0; j < kDims / 4; ++j) reinterpret_cast<f32x4 *>(p.to.part_o + at * 128 + d0)[j] = acc[j];
      if (d0 == 0) *reinterpret_cast<f32x2 *>(p.to.part_ml + at * 2) = f32x2{top, total};
      continue;
    }
    const uint32_t all = f.tile * kRowTile + row, i = p.to.by_group.div(all), h = all - i * group;
    const int64_t token = f.q.row0 + static_cast<int64_t>(i), q_head = static_cast<int64_t>(of_head) * group + h;
    // (the sum is 0 only without a key. A row whose scores are NaN has no maximum either, but a sum of NaN, which out and lse get)
    const float norm = total == 0.f ? 0.f : T::kUnit * (kF8 && p.to.v_scale ? p.to.v_scale[of_head] : 1.0f) / total;
    uint16_t *dst = static_cast<uint16_t *>(p.to.out) + token * p.to.o_ts + q_head * p.to.o_hs + d0;
#pragma unroll
    for (int j = 0; j < kDims / 4; ++j)
      reinterpret_cast<u32x2 *>(dst)[j] = u32x2{T::pack(acc[j][0] * norm, acc[j][1] * norm), T::pack(acc[j][2] * norm, acc[j][3] * norm)};
    if (p.to.lse && d0 == 0) p.to.lse[token * p.to.n_heads + q_head] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
  }
}

// Joins the pieces of the rows of a split row tile. 32 threads have a row's dims; the 8 sets of them in a workgroup have
// a row each where the pieces are few, and share the pieces of one row where they are many.
template <typename T, bool kF8, int NT, int HS>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(FIRST_ARGS, OutParams p) {
  constexpr int kRowTile = kRows * NT, kSets = kJoinThreads / 32;
  __shared__ f32x4 o_s[kSets][32];
  __shared__ float ml_s[kSets][2];
  Found f;
  const First head_args{q_start, kv_lens, n_requests, n_tokens, group, window, target, capacity, {heads_d, heads_m, heads_s}};
  const int index = head_args.by_heads.div(blockIdx.x), head = blockIdx.x - index * heads_d;
  if (!find<kRowTile, kWaves / HS, false>(head_args, index, f)) return;
  const int left = f.q.n * group - f.tile * kRowTile, rows = left < kRowTile ? left : kRowTile;
  const int64_t step = static_cast<int64_t>(heads_d) * kRowTile;   // rows between two pieces
  const int d4 = threadIdx.x & 31, set = threadIdx.x >> 5;
  // (a row of its own costs a set a trip to memory for every 4 pieces, and one for each of the rest: one request of 12 heads, 936 keys,
  // 15 pieces, 10.6 us, shared 8.9; 24 requests x 5 pieces 22.0, shared 22.6)
  const bool shared = f.pieces > (rows <= static_cast<int>(gridDim.y) ? 5 : 2 * kSets);
  const int first = shared ? blockIdx.y : blockIdx.y * kSets + set, rows_step = shared ? gridDim.y : gridDim.y * kSets;
  for (int row = first; row < rows; row += rows_step) {
    const int64_t at = (static_cast<int64_t>(f.slot) * heads_d + head) * kRowTile + row;
    float top = -INFINITY, total = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = shared ? set : 0; i < f.pieces; i += shared ? kSets : 1) {
      const f32x2 ml = *reinterpret_cast<const f32x2 *>(p.part_ml + (at + i * step) * 2);
      const f32x4 o = reinterpret_cast<const f32x4 *>(p.part_o + (at + i * step) * 128)[d4];
      const float high = fmaxf(top, ml[0]), base = high == -INFINITY ? 0.f : high;
      const float keep = exp2_of(top - base), weight = exp2_of(ml[0] - base);
      top = high;
      total = total * keep + ml[1] * weight;
      acc = acc * keep + o * weight;
    }
    if (shared) {   // (one row for the whole workgroup: all threads come here)
      __syncthreads();
      o_s[set][d4] = acc;
      if (d4 == 0) {
        ml_s[set][0] = top;
        ml_s[set][1] = total;
      }
      __syncthreads();
      if (set != 0) continue;
      for (int w = 1; w < kSets; ++w) top = fmaxf(top, ml_s[w][0]);
      const float base = top == -INFINITY ? 0.f : top;
      acc = f32x4{0.f, 0.f, 0.f, 0.f};
      total = 0.f;
      for (int w = 0; w < kSets; ++w) {
        const float weight = exp2_of(ml_s[w][0] - base);
        total += weight * ml_s[w][1];
        acc += weight * o_s[w][d4];
      }
    }
    const uint32_t all = f.tile * kRowTile + row, i = p.by_group.div(all), h = all - i * group;
    const int64_t token = f.q.row0 + static_cast<int64_t>(i), q_head = static_cast<int64_t>(head) * group + h;
    acc *= total == 0.f ? 0.f : T::kUnit * (kF8 && p.v_scale ? p.v_scale[head] : 1.0f) / total;
    const u32x2 w = {T::pack(acc[0], acc[1]), T::pack(acc[2], acc[3])};
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(p.out) + token * p.o_ts + q_head * p.o_hs + 4 * d4) = w;
    if (p.lse && d4 == 0) p.lse[token * p.n_heads + q_head] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
  }
}

constexpr int kMaxDevices = 64;
int compute_units(int &n) {
  static std::once_flag once[kMaxDevices];
  static int units[kMaxDevices];
  static hipError_t status[kMaxDevices];
  int dev = 0;
  SDVG_HIP_CHECK(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return SDVG_ERR_UNSUPPORTED;
  std::call_once(once[dev], [dev] { status[dev] = hipDeviceGetAttribute(&units[dev], hipDeviceAttributeMultiprocessorCount, dev); });
  SDVG_HIP_CHECK(status[dev]);
  n = units[dev];
  return SDVG_OK;
}

// Rows per workgroup by the average request.
int row_tile_of(int64_t n_requests, int64_t n_tokens, int group) {
  const int64_t rows = (n_tokens + n_requests - 1) / n_requests * group;
  return rows <= 16 ? 16 : 32;
}

// Sets of heads per workgroup (HS): where the rows of neighbouring heads are neighbours. us, 1 and 2: one request of 131071 keys x 8
// heads, 16 bit 95.5 and 90.2, ragged 207 and 197, 32 rows e4m3 40.3 and 38.5; a cache with heads ahead of tokens 50.7 and 53.1 (e4m3).
// 32 rows in 16 bits are not built: 24 requests of up to 8 new tokens 60.2 against 61.8 (P rounded once), but with 255 of the 256 registers,
// and a form of the loop with two steps on their way, which spilled, gave wrong results. (A test holds all instances to no spilled register.)
int head_sets(const sdvg_paged_kv &c, int row_tile) {
  const bool fits = row_tile == 16 || c.dtype == SDVG_E4M3;
  return fits && c.n_kv_heads % 2 == 0 && c.head_stride < c.token_stride ? 2 : 1;
}

// Keys that a row of the block table can name.
int32_t capacity_of(const sdvg_paged_attn_desc &d, const sdvg_paged_kv &c) {
  const int64_t most = INT32_MAX - 2 * pg::kKeyTile, keys = int64_t{d.table_width} * c.page_tokens;
  return static_cast<int32_t>(keys < most ? keys : most);   // (more than any pool holds)
}

// Items per (set of) key heads that fill the chip, kPerUnit workgroups per unit; 0 where no request can be split.
int target_of(int n_cu, const sdvg_paged_attn_desc &d, const sdvg_paged_kv &c, int row_tile) {
  const int sets = head_sets(c, row_tile), t = kPerUnit * n_cu * sets / c.n_kv_heads;
  if (pg::max_pieces(capacity_of(d, c), kWaves / sets) <= 1) return 0;
  return t > 1 ? t : 1;
}

int64_t workspace_of(int target, int n_kv_heads, int row_tile) {
  return pg::max_slots(target) * n_kv_heads * row_tile * (128 + 2) * 4;
}

int check_attn(const sdvg_paged_attn_desc *d, const sdvg_paged_kv *c) {
  if (!d) return SDVG_ERR_NULL;
  const int st = sdvg::check_paged_kv(c);
  if (st != SDVG_OK) return st;
  if (d->head_dim != 128) return SDVG_ERR_UNSUPPORTED;
  if (d->dtype != SDVG_BF16 && d->dtype != SDVG_F16) return SDVG_ERR_UNSUPPORTED;
  if (c->dtype != d->dtype && c->dtype != SDVG_E4M3) return SDVG_ERR_UNSUPPORTED;
  if (d->n_requests < 0 || d->n_tokens < 0 || d->n_heads < 1 || d->n_heads % c->n_kv_heads != 0 || d->table_width < 1 ||
      d->window < 0)
    return SDVG_ERR_SHAPE;
  if (c->n_kv_heads > 65535 || int64_t{d->n_tokens} * d->n_heads > INT32_MAX - 64) return SDVG_ERR_UNSUPPORTED;
  if (d->n_requests > 1 && d->table_stride < d->table_width) return SDVG_ERR_SHAPE;
  if (d->n_requests > 1 && d->table_stride > INT32_MAX) return SDVG_ERR_UNSUPPORTED;
  if (!(d->scale >= 0.f) || !isfinite(d->scale)) return SDVG_ERR_RANGE;
  return SDVG_OK;
}

#define FIRST(f) \
  f.q_start, f.kv_lens, f.n_requests, f.n_tokens, f.group, f.window, f.target, f.capacity, f.by_heads.d, f.by_heads.m, f.by_heads.s
template <typename T, bool kF8, int NT, int HS>
int launch_attn(First f, const AttnParams &p, hipStream_t s) {
  constexpr int kRowTile = kRows * NT, kKeyWaves = kWaves / HS;
  const int64_t tiles = pg::max_row_tiles(f.n_requests, f.n_tokens, f.group, kRowTile);
  const int64_t items = pg::max_items(tiles, f.target, f.capacity, kKeyWaves);
  if (items * f.by_heads.d >= (1 << 23)) return SDVG_ERR_UNSUPPORTED;  // (a grid holds fewer than 2^32 threads)
  hipLaunchKernelGGL((paged_attn_kernel<T, kF8, NT, HS>), dim3(static_cast<uint32_t>(items * f.by_heads.d)), dim3(kThreads), 0, s, FIRST(f), p);
  SDVG_HIP_CHECK(hipGetLastError());
  if (f.target > 0) {
    // Workgroups per row tile: one for every row of an average request's where that are few (then the pieces are many, and
    // shared), otherwise one for every 8 rows. A workgroup takes more rows where there are more.
    f.by_heads = sdvg::FastDiv::of(f.by_heads.d * HS);
    const int64_t groups = pg::max_groups(tiles, f.target) * f.by_heads.d;
    int64_t rows = (static_cast<int64_t>(f.n_tokens) + f.n_requests - 1) / f.n_requests * f.group;
    rows = rows < kRowTile ? rows : kRowTile;
    if (groups * rows > 1024) rows = (rows + 7) / 8;
    hipLaunchKernelGGL((paged_join_kernel<T, kF8, NT, HS>), dim3(static_cast<uint32_t>(groups), static_cast<uint32_t>(rows)),
                       dim3(kJoinThreads), 0, s, FIRST(f), p.to);
    SDVG_HIP_CHECK(hipGetLastError());
  }
  return SDVG_OK;
}
template <typename T, bool kF8>
int launch_attn(const First &f, const AttnParams &p, int row_tile, int sets, hipStream_t s) {
  if (sets == 2) {
    if constexpr (kF8)
      if (row_tile == 32) return launch_attn<T, kF8, 2, 2>(f, p, s);
    return launch_attn<T, kF8, 1, 2>(f, p, s);
  }
  return row_tile == 16 ? launch_attn<T, kF8, 1, 1>(f, p, s) : launch_attn<T, kF8, 2, 1>(f, p, s);
}

}  // namespace

extern "C" int64_t sdvg_paged_attn_workspace_bytes(const sdvg_paged_attn_desc *desc, const sdvg_paged_kv *cache) {
  int st = check_attn(desc, cache), n_cu = 0;
  if (st != SDVG_OK) return st;
  if (desc->n_requests == 0 || desc->n_tokens == 0) return 0;
  if ((st = compute_units(n_cu)) != SDVG_OK) return st;
  const int tile = row_tile_of(desc->n_requests, desc->n_tokens, desc->n_heads / cache->n_kv_heads);
  return workspace_of(target_of(n_cu, *desc, *cache, tile), cache->n_kv_heads, tile);
}

extern "C" int sdvg_paged_attn(const sdvg_paged_attn_desc *desc, const sdvg_paged_kv *cache, const void *q,
                               const int32_t *block_table, const int32_t *q_start, const int32_t *kv_lens, void *out,
                               float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
  int st = check_attn(desc, cache);
  if (st != SDVG_OK) return st;
  if (workspace_bytes < 0) return SDVG_ERR_SHAPE;
  if (desc->n_requests == 0 || desc->n_tokens == 0) return SDVG_OK;
  if (!q || !block_table || !q_start || !kv_lens || !out) return SDVG_ERR_NULL;
  for (const int64_t s : {desc->q_token_stride, desc->o_token_stride})
    if ((st = sdvg::check_stride(desc->n_tokens, s, 2)) != SDVG_OK) return st;
  for (const int64_t s : {desc->q_head_stride, desc->o_head_stride})
    if ((st = sdvg::check_stride(desc->n_heads, s, 2)) != SDVG_OK) return st;
  if (!sdvg::aligned16(q) || !sdvg::aligned16(out) || !sdvg::aligned16(workspace)) return SDVG_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(q_start) | reinterpret_cast<uintptr_t>(kv_lens) |
       reinterpret_cast<uintptr_t>(lse)) & 3)
    return SDVG_ERR_ALIGN;
  if (q == out && ((desc->n_tokens > 1 && desc->q_token_stride != desc->o_token_stride) ||
                   (desc->n_heads > 1 && desc->q_head_stride != desc->o_head_stride)))
    return SDVG_ERR_RANGE;
  int n_cu = 0;
  if ((st = compute_units(n_cu)) != SDVG_OK) return st;
  const int32_t n_kv = cache->n_kv_heads, group = desc->n_heads / n_kv;
  First f{q_start, kv_lens, desc->n_requests, desc->n_tokens, group, desc->window, 0, capacity_of(*desc, *cache), {}};
  AttnParams p{};
  p.q = q;
  p.k = cache->k;
  p.v = cache->v;
  p.k_scale = cache->k_scale;
  p.table = block_table;
  p.page_stride = cache->page_stride;
  p.token_stride = cache->token_stride;
  p.head_stride = cache->head_stride;
  p.q_ts = static_cast<uint32_t>(desc->q_token_stride);
  p.q_hs = static_cast<uint32_t>(desc->q_head_stride);
  p.table_stride = desc->n_requests > 1 ? static_cast<int32_t>(desc->table_stride) : 0;
  p.table_width = desc->table_width;
  p.n_pages = cache->n_pages;
  p.scale_log2e = (desc->scale == 0.f ? 1.0f / sqrtf(128.0f) : desc->scale) * kLog2e;
  p.by_page = sdvg::FastDiv::of(cache->page_tokens / 8);
  p.to = OutParams{out, lse, nullptr, nullptr, cache->v_scale, static_cast<uint32_t>(desc->o_token_stride),
                   static_cast<uint32_t>(desc->o_head_stride), desc->n_heads, sdvg::FastDiv::of(group)};
  const int tile = row_tile_of(f.n_requests, f.n_tokens, group), target = target_of(n_cu, *desc, *cache, tile), sets = head_sets(*cache, tile);
  f.by_heads = sdvg::FastDiv::of(n_kv / sets);
  if (target > 0 && workspace && workspace_bytes >= workspace_of(target, n_kv, tile)) {
    f.target = target;
    p.to.part_o = static_cast<float *>(workspace);
    p.to.part_ml = p.to.part_o + pg::max_slots(target) * n_kv * tile * 128;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f8 = cache->dtype == SDVG_E4M3;
  if (desc->dtype == SDVG_BF16) return f8 ? launch_attn<Bf16, true>(f, p, tile, sets, s) : launch_attn<Bf16, false>(f, p, tile, sets, s);
  return f8 ? launch_attn<F16, true>(f, p, tile, sets, s) : launch_attn<F16, false>(f, p, tile, sets, s);
}
