// Attention of a batch over a paged cache where groups of requests share their first keys (a prompt and its continuations): the
// shared keys are read once for all rows of a group, the others as in paged_attn.hip, and a second launch joins both.
//
// What bounds it: the rows of a group that share a key head (new tokens x query heads of the key head, over all its requests) are one
// matrix, so the shared keys cost 4 x 128 FLOP per row and key and 512 bytes per key and key head in 16 bits: the HBM's time below some
// 150 rows per key head, the matrix cores' above.
//
// A workgroup has 128 of these rows, 32 for each of its 4 waves, so that a key is read again for every 128 rows; the last one, where it has no
// more than 64, has two sets of waves with half of every key tile each. K and V tiles of 64 keys lie in LDS, the next
// one on its way while one is used: 16-bit rows are copied there by the load itself, e4m3 rows pass registers, where they
// become 16-bit numbers, once for all waves.
//   S^T = K Q^T with v_mfma_f32_32x32x16: a lane then has 16 scores of one row (lane % 32), keys 8 g + 4 (lane / 32) .. + 3, g = 0 .. 3.
//   O^T = V^T P^T: those are the B operand of this product as they are, if V^T's keys are read in the same order, which the
//     transposing read from LDS does. P goes in as two 16-bit numbers, the rounded one and what that leaves: a third more products than one
//     number takes, for an error that is the result's own rounding.
// The 16-byte chunks of a row are permuted by the row's number (block_attn_index.h has the same), so that no read meets a bank twice.
//
// us of a call (and of kernel and join, traced, when the kernel takes longer than in a loop of calls): 128 requests of one token behind 8191 shared keys,
// 32 query and 8 key heads, f16 86 (79 + 14); 64 behind 65520 keys, 40 / 8 heads, bf16 171 (187 + 15), of which products at the full rate, the second
// number of P counted, would take 104; the rest is the softmax, which two waves of a SIMD do at the same time as often as not, and barriers. Four requests
// of 12 heads behind 936 keys 14.9 (9.6 + 5.8), a chain of latencies. Not kept: key tiles of 32 in a ring of four (these three cases with 90, 202 and 15 us a call, against 83, 170 and 15), the
// scores of a 32-key step ahead of the probabilities of the one before (88, 202; registers spill), row tiles of even size (183 and 181), raised wave priority
// around the products (no difference).
#include "block_attn_index.h"
#include "paged_attn_device.h"
#include "paged_prefix_plan.h"

namespace {

namespace ai = sdvg::attn_index;

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kSharedThreads = 256, kSharedWaves = 4;
constexpr int kTileBytes = pg::kSharedTile * 256;

template <typename T>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (std::is_same<T, Bf16>::value)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Over the two lanes that hold a row (l, l ^ 32).
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_xor(x, d);
    x = y < x ? y : x;
  }
  return __builtin_amdgcn_readfirstlane(x);
}

// 16 bytes per lane from memory to LDS: lane i's to lds + 16 i. In assembly, so that the compiler does not wait for each; the kernel
// waits for all ahead of the barrier that publishes a tile.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(const char *from, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds), "v"(from)
      : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void barrier_after_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void barrier_after_lds() {   // (loads may stay on their way)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- which part of the shared keys a workgroup has
struct FoundShared {
  pg::SharedKeys q;
  pg::Place at;
  pg::SharedPieces pieces;
  int32_t slot, chunk;   // slot of the group's first piece; key tiles of a piece
};
__device__ __forceinline__ pg::SharedKeys load_group(const First &p, const Groups &gr, int g) {
  if (g >= gr.n) return pg::SharedKeys{};
  const int32_t start = pg::clamp(gr.first(g, p.n_requests), 0, p.n_requests), end = pg::clamp(gr.first(g + 1, p.n_requests), start, p.n_requests);
  const int32_t n = gr.lens[g];
  return pg::shared_of(start, end, p.q_start[start], p.q_start[end], n > 0 ? n : 0, p.n_tokens, p.group, p.window, p.capacity);
}
// Item number x (kItems), or the slots of group x. mine0: load_group of this lane.
template <bool kItems>
__device__ __forceinline__ bool find_shared(const First &p, const Groups &gr, const pg::SharedKeys &mine0, int x, FoundShared &f) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0, row_tiles = 0;
  for (int b = 0; b < gr.n; b += 64) {
    const pg::SharedKeys q = b ? load_group(p, gr, b + lane) : mine0;
    const int64_t w = pg::work_of(q);
    row_tiles += wave_total(q.row_tiles);
    total += wave_total(static_cast<int>(w & 0xffff)) + (static_cast<int64_t>(wave_total(static_cast<int>(w >> 16))) << 16);
  }
  f.chunk = pg::shared_chunk(total, row_tiles, gr.shared_target);
  int before = 0;
  for (int b = 0; b < gr.n; b += 64) {
    const pg::SharedKeys q = b ? load_group(p, gr, b + lane) : mine0;
    const pg::SharedPieces n = pg::shared_pieces(q, f.chunk);
    const int32_t mine = pg::shared_items(q, n);
    const int upto = scan(mine), at = x - before - (upto - mine);
    const uint64_t hit = __ballot(kItems ? at >= 0 && at < mine : b + lane == x);
    if (hit) {
      const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      const auto get = [src](int v) { return __builtin_amdgcn_readlane(v, src); };
      f.q = pg::SharedKeys{get(q.request0), get(q.requests), get(q.token0), get(q.tokens), get(q.lo), get(q.hi), get(q.first_tile), get(q.tiles), get(q.row_tiles), get(q.half)};
      f.pieces = pg::SharedPieces{get(n.whole), get(n.half)};
      f.slot = before + get(upto - mine);
      if constexpr (kItems) f.at = pg::shared_place(f.q, f.pieces, get(at));
      return f.slot >= 0 && f.slot <= gr.max_shared - get(mine);
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// Keys that the row of token `token` sees, from and up to: of the request among f's that has the token, whose numbers are clamped as for its own
// keys. A batch of 64 requests at a time, each lane looks for its token among them in 6 steps. (All lanes of the wave come here.)
__device__ __forceinline__ void seen_by(const First &p, const FoundShared &f, int token, int &from, int &sees) {
  const int lane = threadIdx.x & 63;
  sees = 0;
  for (int b = 0; b < f.q.requests; b += 64) {
    const int r = f.q.request0 + (b + lane < f.q.requests ? b + lane : f.q.requests - 1);
    const pg::Rows mine = pg::rows_of(p.q_start[r], p.q_start[r + 1], p.kv_lens[r], p.n_tokens);
    int at = 0;
#pragma unroll
    for (int step = 32; step > 0; step /= 2)
      if (__shfl(mine.row0, at + step) <= token) at += step;
    const pg::Rows q{__shfl(mine.row0, at), __shfl(mine.n, at), __shfl(mine.len, at)};
    if (token >= q.row0 && token - q.row0 < q.n) sees = pg::sees_of(q, token - q.row0);
  }
  from = p.window > 0 && sees > p.window ? sees - p.window : 0;
}

// The shared keys of a row tile. Its waves have 32 rows each; where that leaves two of them without (kHalf), two sets of two waves have the
// same rows and half of every key tile each.
template <typename T, bool kF8, bool kHalf>
__device__ __forceinline__ void attend_shared(const First &first, const Groups &gr, const AttnParams &p, const FoundShared &f, int head, char *lds) {
  constexpr int kRowTile = pg::kSharedRows, kBytes = kF8 ? 1 : 2, kHalves = kHalf ? 1 : 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, hh = lane >> 5;
  const int left = f.q.tokens * first.group - f.at.tile * kRowTile, rows = left < kRowTile ? left : kRowTile;
  const int rw = kHalf ? wave & 1 : wave, set = kHalf ? wave >> 1 : 0;
  const int row = rw * 32 + col;
  const bool any_row = rw * 32 < rows;

  // this lane's row, and the keys it sees
  u32x4 qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) qf[s] = u32x4{0, 0, 0, 0};
  int from = 0, sees = INT32_MAX;
  {
    const uint32_t all = f.at.tile * kRowTile + (row < rows ? row : rows - 1), i = p.to.by_group.div(all), h = all - i * first.group;
    if (row < rows) {
      const uint16_t *src = static_cast<const uint16_t *>(p.q) + (f.q.token0 + static_cast<int64_t>(i)) * p.q_ts +
                            (static_cast<int64_t>(head) * first.group + h) * p.q_hs + 8 * hh;
#pragma unroll
      for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const u32x4 *>(src + 16 * s);
    }
    int a, b;
    seen_by(first, f, f.q.token0 + static_cast<int>(i), a, b);
    if (row < rows) {
      from = a;
      sees = b;
    }
  }
  const int all_sees = wave_min(sees), all_from = -wave_min(-from);
  // keys ahead of `lo` and from `hi` on are seen by no row of the workgroup; what they hold may be anything
  int lo, hi;
  {
    int *const s = reinterpret_cast<int *>(lds);
    const int least = wave_min(row < rows ? from : INT32_MAX), most = -wave_min(row < rows ? -sees : INT32_MAX);
    if (lane == 0) {
      s[wave] = least;
      s[kSharedWaves + wave] = most;
    }
    __syncthreads();
    lo = s[0];
    hi = s[kSharedWaves];
    for (int w = 1; w < kSharedWaves; ++w) {
      lo = s[w] < lo ? s[w] : lo;
      hi = s[kSharedWaves + w] > hi ? s[kSharedWaves + w] : hi;
    }
    __syncthreads();
    lo = __builtin_amdgcn_readfirstlane(lo > f.q.lo ? lo : f.q.lo);
    hi = __builtin_amdgcn_readfirstlane(hi < f.q.hi ? hi : f.q.hi);
  }

  // (scores are compared ahead of their scale, which is positive then; -infinity times 0 would be no number. A scale that is no number makes all scores
  // none, ahead of the masks)
  float scale = p.scale_log2e * (kF8 && p.k_scale ? p.k_scale[head] : 1.0f);
  const uint32_t flip = scale < 0.f ? 0x80008000u : 0u, nan = scale != scale ? 0xffffffffu : 0u;
  if (flip | nan) {
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = (qf[s] ^ flip) | nan;
  }
  scale = fmaxf(fabsf(scale), 0x1p-126f);
  f32x16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  const pg::KeyTiles keys = pg::shared_tiles_of(f.q, f.at, f.chunk);
  const int begin = keys.begin > lo / pg::kSharedTile ? keys.begin : lo / pg::kSharedTile;
  const int last = hi > 0 ? (hi - 1) / pg::kSharedTile + 1 : 0, end = keys.end < last ? keys.end : last;
  const int32_t *table = p.table + static_cast<int64_t>(f.q.request0) * p.table_stride;
  const char *k_head = static_cast<const char *>(p.k) + head * p.head_stride * kBytes,
             *v_head = static_cast<const char *>(p.v) + head * p.head_stride * kBytes;
  const int64_t token_bytes = p.token_stride * kBytes, page_bytes = p.page_stride * kBytes;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds));

  // Pages of a tile's 8 blocks of 8 keys: lane i's is that of block i % 8.
  struct Pages {
    int32_t page;      // -1: not there
    uint32_t token;    // in its page, of the block's first key
  };
  const auto pages_of = [&](int tile) {
    const uint32_t block = tile * 8 + (lane & 7), i = p.by_page.div(block);
    const int32_t page = i < static_cast<uint32_t>(p.table_width) ? table[i] : -1;
    return Pages{page, (block - i * p.by_page.d) * 8};
  };
  const auto there = [&](const Pages &at) { return static_cast<uint32_t>(__ballot(at.page >= 0 && at.page < p.n_pages)) & 0xffu; };
  // Bytes from a head's first row to the first row of block b. (A page that is not there reads page 0, which is memory of the pool; its keys do not count.)
  const auto block_at = [&](const Pages &at, uint32_t valid, int b) {
    const int32_t page = __builtin_amdgcn_readlane(at.page, b);
    const uint32_t token = __builtin_amdgcn_readlane(at.token, b);
    return ((valid >> b) & 1 ? page : 0) * page_bytes + token * token_bytes;
  };
  // 16 bit: a wave copies rows 16 u + 4 wave + lane / 16 (u = 0 .. 3). e4m3: it has rows 32 u + 8 wave + lane / 8 (u = 0, 1) in registers.
  const int in_block = kF8 ? lane >> 3 : 4 * (wave & 1) + (lane >> 4);
  const int64_t k_lane = in_block * token_bytes + (kF8 ? (lane & 7) * 16 : ((lane & 15) ^ ((4 * wave + (lane >> 4)) & 15)) * 16);
  const int64_t v_lane = in_block * token_bytes + (kF8 ? (lane & 7) * 16 : ((lane & 15) ^ (4 * ((lane >> 4) & 3))) * 16);
  u32x4 k_next[kF8 ? 2 : 1], v_next[kF8 ? 2 : 1];
  const auto ask = [&](const Pages &at, uint32_t valid, int slot) {
    if constexpr (kF8) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t base = block_at(at, valid, wave + 4 * u);
        k_next[u] = *reinterpret_cast<const u32x4 *>(k_head + base + k_lane);
        v_next[u] = *reinterpret_cast<const u32x4 *>(v_head + base + v_lane);
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t base = block_at(at, valid, 2 * u + (wave >> 1));
        const uint32_t to = lds0 + slot * (2 * kTileBytes) + (16 * u + 4 * wave) * 256;
        copy16(k_head + base + k_lane, to);
        copy16(v_head + base + v_lane, to + kTileBytes);
      }
    }
  };
  const auto put = [&](int slot) {   // e4m3: what `ask` brought, as 16-bit numbers
    if constexpr (kF8) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = 32 * u + 8 * wave + (lane >> 3), c = 2 * (lane & 7);
        char *const k = lds + slot * (2 * kTileBytes) + r * 256, *const v = k + kTileBytes;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          *reinterpret_cast<u32x4 *>(k + ((c + x) ^ (r & 15)) * 16) = widen<T>(u32x2{k_next[u][2 * x], k_next[u][2 * x + 1]});
          *reinterpret_cast<u32x4 *>(v + ((c + x) ^ (4 * (r & 3))) * 16) = widen<T>(u32x2{v_next[u][2 * x], v_next[u][2 * x + 1]});
        }
      }
    }
  };

  if (begin < end) {
    const auto ahead = [&](int tile) { return pages_of(tile < end ? tile : end - 1); };
    const Pages now = pages_of(begin);
    Pages next = ahead(begin + 1), after = ahead(begin + 2);   // of the next two tiles
    uint32_t valid = there(now);
    ask(now, valid, 0);
    if constexpr (kF8) {
      put(0);
      ask(next, there(next), 0);
    }
    for (int tile = begin; tile < end; ++tile) {
      const int slot = (tile - begin) & 1;
      // this tile has landed, and nobody reads the other slot any more
      if constexpr (kF8)
        barrier_after_lds();
      else
        barrier_after_all();
      const uint32_t valid_next = there(next);
      if constexpr (kF8) {
        if (tile + 1 < end) put(slot ^ 1);
        if (tile + 2 < end) ask(after, there(after), 0);
      } else {
        if (tile + 1 < end) ask(next, valid_next, slot ^ 1);
      }
      next = after;
      after = ahead(tile + 3);
      const int key0 = tile * pg::kSharedTile;
      const bool special = valid != 0xffu || key0 < lo || key0 + pg::kSharedTile > hi;
      if (special) {
        // V of keys that nobody sees is cleared (0 times anything but a number is no 0)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = 16 * u + (threadIdx.x >> 4), key = key0 + r;
          if (key < lo || key >= hi || !((valid >> (r >> 3)) & 1))
            *reinterpret_cast<u32x4 *>(lds + slot * (2 * kTileBytes) + kTileBytes + r * 256 + (threadIdx.x & 15) * 16) = u32x4{0, 0, 0, 0};
        }
        barrier_after_lds();
      }
      if (any_row) {
        // (kHalf: this wave's half of the tile, otherwise both)
        const char *const k_tile = lds + slot * (2 * kTileBytes) + set * (32 * 256), *const v_tile = k_tile + kTileBytes;
        const auto read_k = [&](int c, int kb) { return *reinterpret_cast<const u32x4 *>(k_tile + ai::k_read_offset(lane, c, kb)); };
        const auto read_v = [&](int step, int d) {
          const char *const at = v_tile + ai::v_read_offset(lane, step, d, 0);
          const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at)),
                      b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 8 * 256)));
          return u32x4{a[0], a[1], b[0], b[1]};
        };
        f32x16 s[kHalves];
        u32x4 kf[8], vt[2][4];
#pragma unroll
        for (int c = 0; c < 8; ++c) kf[c] = read_k(c, 0);
#pragma unroll
        for (int kb = 0; kb < kHalves; ++kb) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            s[kb] = mfma32<T>(kf[c], qf[c], s[kb]);
            if (kb + 1 < kHalves)
              kf[c] = read_k(c, kb + 1);
            else if (c < 4)
              vt[0][c] = read_v(0, c);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int first_key = key0 + 32 * set;
        if (special || first_key + 32 * kHalves > all_sees || first_key < all_from) {
#pragma unroll
          for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int in = 32 * kb + 8 * (i >> 2) + 4 * hh + (i & 3), key = first_key + in;
              const bool ok = ((valid >> (4 * set + (in >> 3))) & 1) && key >= lo && key < hi && key >= from && key < sees;
              s[kb][i] = ok ? s[kb][i] : -INFINITY;
            }
        }
        float high = s[0][0];
#pragma unroll
        for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) high = fmaxf(high, s[kb][i]);
        high *= scale;
        // m is raised only when some row's scores pass it by more than kSlack
        if (__any(high > m + T::kSlack)) {
          const float top = fmaxf(m, pair_max(high));
          const float keep = m == -INFINITY ? 0.f : exp2_of(m - top);
          m = top;
          l *= keep;
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d] *= keep;
        }
        const float base = m == -INFINITY ? 0.f : T::kShift - m;
#pragma unroll
        for (int step = 0; step < 2 * kHalves; ++step) {   // 16 keys
          u32x4 pf, rest;   // probabilities in 16 bits, and what is left of them
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int i = 8 * (step & 1) + 2 * c;
            const float a = exp2_of(fmaf(s[step >> 1][i], scale, base)), b = exp2_of(fmaf(s[step >> 1][i + 1], scale, base));
            const unsigned w = T::pack(a, b);
            pf[c] = w;
            rest[c] = T::pack(a - T::first(w), b - T::second(w));
            l += a + b;
          }
          if (step + 1 < 2 * kHalves) {
#pragma unroll
            for (int d = 0; d < 4; ++d) vt[(step + 1) & 1][d] = read_v(step + 1, d);
          }
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d] = mfma32<T>(vt[step & 1][d], rest, o[d]);
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d] = mfma32<T>(vt[step & 1][d], pf, o[d]);
        }
      }
      valid = valid_next;
    }
  }

  // the sets' results meet
  l = pair_sum(l) * T::kUnit;
  if constexpr (kHalf) {
    __syncthreads();
    float *const os = reinterpret_cast<float *>(lds) + rw * 64 * 64, *const ml = reinterpret_cast<float *>(lds) + 2 * 64 * 64 + rw * 128;
    if (set == 1) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) os[(16 * d + i) * 64 + lane] = o[d][i];
      ml[lane] = m;
      ml[64 + lane] = l;
    }
    __syncthreads();
    if (set == 1) return;
    const float other = ml[lane], top = fmaxf(m, other), b = top == -INFINITY ? 0.f : top;
    const float mine = exp2_of(m - b), theirs = exp2_of(other - b);
    m = top;
    l = l * mine + ml[64 + lane] * theirs;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * mine + os[(16 * d + i) * 64 + lane] * theirs;
  }
  if (row >= rows) return;
  const int64_t at = (static_cast<int64_t>(f.slot + f.at.tile * f.pieces.whole + f.at.piece) * gr.by_heads.d + head) * kRowTile + row;
  float *const dst = gr.part_o + at * 128 + 4 * hh;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4 *>(dst + 32 * d + 8 * g) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
  if (hh == 0) *reinterpret_cast<f32x2 *>(gr.part_ml + at * 2) = f32x2{m, l};
}

// Both kinds of workgroups: those that wait for memory and those that keep the matrix cores busy run side by side.
template <typename T, bool kF8, int NT, int HS>
__global__ __launch_bounds__(kThreads, kPerUnit) void paged_prefix_kernel(FIRST_ARGS, Groups gr, AttnParams p) {
  static_assert(kThreads == kSharedThreads && sizeof(float) * kWaves * kRows * (kPad + 2) <= 4 * kTileBytes, "LDS of both kinds");
  __shared__ __attribute__((aligned(16))) char lds[4 * kTileBytes];   // K and V of two tiles
  const First first{q_start, kv_lens, n_requests, n_tokens, group, window, target, capacity, {heads_d, heads_m, heads_s}};
  const pg::Turn turn = pg::turn_of(blockIdx.x, gr.shared_turns, gr.own_turns);
  if (turn.shared) {
    FoundShared f;
    const int item = gr.by_heads.div(turn.block), head = turn.block - item * gr.by_heads.d;
    if (!find_shared<true>(first, gr, load_group(first, gr, threadIdx.x & 63), item, f)) return;
    if (pg::is_half(f.q, f.at.tile))
      attend_shared<T, kF8, true>(first, gr, p, f, head, lds);
    else
      attend_shared<T, kF8, false>(first, gr, p, f, head, lds);
  } else {
    float(*const o_s)[kRows][kPad] = reinterpret_cast<float(*)[kRows][kPad]>(lds);
    attend<T, kF8, NT, HS, true>(first, p, gr, turn.block, o_s, reinterpret_cast<float(*)[kRows][2]>(o_s + kWaves));
  }
}

// Joins the pieces of a request's own keys and those of its group's shared ones. 32 threads have a row's dims; `per` sets of them (1, 2, 4
// or 8) share the pieces of a row.
template <typename T, bool kF8, int NT, int HS>
__global__ __launch_bounds__(kJoinThreads) void paged_prefix_join_kernel(First first, OutParams p, Groups gr, int per) {
  constexpr int kRowTile = kRows * NT, kSets = kJoinThreads / 32;
  __shared__ f32x4 o_s[kSets][32];
  __shared__ float ml_s[kSets][2];
  Found f;
  const int heads = first.by_heads.d, index = first.by_heads.div(blockIdx.x), head = blockIdx.x - index * heads;
  const pg::SharedKeys groups = load_group(first, gr, threadIdx.x & 63);   // (asked for ahead of the requests')
  if (!find<kRowTile, kWaves / HS, false, true>(first, gr, index, f)) return;
  const int left = f.q.n * first.group - f.tile * kRowTile, rows = left < kRowTile ? left : kRowTile;
  FoundShared s{};
  if (f.group >= 0 && !find_shared<false>(first, gr, groups, f.group, s)) s = FoundShared{};   // (no slots)
  const int64_t own_step = static_cast<int64_t>(heads) * kRowTile, shared_step = static_cast<int64_t>(heads) * pg::kSharedRows;
  const int d4 = threadIdx.x & 31, set = threadIdx.x >> 5, sub = set % per, at_once = kSets / per;
  for (int row0 = blockIdx.y * at_once; row0 < rows; row0 += gridDim.y * at_once) {   // (all threads come round as often)
    const int row = row0 + set / per;
    const uint32_t all = f.tile * kRowTile + row, i = p.by_group.div(all), h = all - i * first.group;
    const int64_t own_at = (static_cast<int64_t>(f.slot) * heads + head) * kRowTile + row;
    // its number among the group's rows
    const int64_t among = (static_cast<int64_t>(f.q.row0) - s.q.token0) * first.group + all;
    const bool in = row < rows && among >= 0 && among < static_cast<int64_t>(s.q.tokens) * first.group;
    const int tile = in ? static_cast<int>(among / pg::kSharedRows) : 0;
    const int shared = in && tile < s.q.row_tiles ? (pg::is_half(s.q, tile) ? s.pieces.half : s.pieces.whole) : 0;
    const int64_t shared_at = ((s.slot + static_cast<int64_t>(tile) * s.pieces.whole) * heads + head) * pg::kSharedRows + (among - static_cast<int64_t>(tile) * pg::kSharedRows);
    float top = -INFINITY, total = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const int pieces = row < rows ? f.pieces + shared : 0;
#pragma unroll 4
    for (int j = sub; j < pieces; j += per) {
      const bool own = j < f.pieces;
      const int64_t at = own ? own_at + j * own_step : shared_at + (j - f.pieces) * shared_step;
      const f32x2 ml = *reinterpret_cast<const f32x2 *>((own ? p.part_ml : gr.part_ml) + at * 2);
      const f32x4 o = reinterpret_cast<const f32x4 *>((own ? p.part_o : gr.part_o) + at * 128)[d4];
      const float high = fmaxf(top, ml[0]), base = high == -INFINITY ? 0.f : high;
      const float keep = exp2_of(top - base), weight = exp2_of(ml[0] - base);
      top = high;
      total = total * keep + ml[1] * weight;
      acc = acc * keep + o * weight;
    }
    if (per > 1) {
      __syncthreads();
      o_s[set][d4] = acc;
      if (d4 == 0) {
        ml_s[set][0] = top;
        ml_s[set][1] = total;
      }
      __syncthreads();
      if (sub == 0) {
        for (int w = 1; w < per; ++w) top = fmaxf(top, ml_s[set + w][0]);
        const float base = top == -INFINITY ? 0.f : top;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
        total = 0.f;
        for (int w = 0; w < per; ++w) {
          const float weight = exp2_of(ml_s[set + w][0] - base);
          total += weight * ml_s[set + w][1];
          acc += weight * o_s[set + w][d4];
        }
      }
    }
    if (sub != 0 || row >= rows) continue;
    const int64_t token = f.q.row0 + static_cast<int64_t>(i), q_head = static_cast<int64_t>(head) * first.group + h;
    acc *= total == 0.f ? 0.f : T::kUnit * (kF8 && p.v_scale ? p.v_scale[head] : 1.0f) / total;
    const u32x2 w = {T::pack(acc[0], acc[1]), T::pack(acc[2], acc[3])};
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(p.out) + token * p.o_ts + q_head * p.o_hs + 4 * d4) = w;
    if (p.lse && d4 == 0) p.lse[token * p.n_heads + q_head] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
  }
}

// ---- host
struct Layout {              // of the launch, and of the workspace in rows of 128 + 2 floats
  int own_tile, sets, target, shared_target;
  int64_t own_items, own_slots, shared_slots, own_rows, shared_rows;
  int64_t bytes() const { return (own_rows + shared_rows) * (128 + 2) * 4; }
};
Layout layout_of(int n_cu, const sdvg_paged_attn_desc &d, const sdvg_paged_kv &c, int32_t n_groups) {
  Layout w;
  const int group = d.n_heads / c.n_kv_heads;
  w.own_tile = row_tile_of(d.n_requests, d.n_tokens, group);
  w.sets = head_sets(c, w.own_tile);
  w.target = target_of(n_cu, d, c, w.own_tile);
  // (two workgroups per compute unit, which is what fits; us of a call, 128 x 8191 keys and 64 x 65520: 83 and 170, one per unit 74 and 231, three for two
  // units 76 and 181, four 89 and 181)
  w.shared_target = 2 * n_cu / c.n_kv_heads > 1 ? 2 * n_cu / c.n_kv_heads : 1;
  const int64_t tiles = pg::max_row_tiles(d.n_requests, d.n_tokens, group, w.own_tile);
  w.own_items = pg::max_items(tiles, w.target, capacity_of(d, c), kWaves / w.sets);
  w.own_slots = pg::max_slots(w.target) + tiles;
  w.shared_slots = pg::max_shared_items(pg::max_shared_row_tiles(n_groups, d.n_tokens, group), w.shared_target, capacity_of(d, c));
  w.own_rows = w.own_slots * c.n_kv_heads * w.own_tile;
  w.shared_rows = w.shared_slots * c.n_kv_heads * pg::kSharedRows;
  return w;
}

template <typename T, bool kF8, int NT, int HS>
int launch_prefix(First f, const AttnParams &p, const Groups &gr, hipStream_t s) {
  constexpr int kRowTile = kRows * NT;
  const dim3 grid(static_cast<uint32_t>(gr.shared_turns + gr.own_turns) * pg::kTurn);
  hipLaunchKernelGGL((paged_prefix_kernel<T, kF8, NT, HS>), grid, dim3(kThreads), 0, s, FIRST(f), gr, p);
  SDVG_HIP_CHECK(hipGetLastError());
  f.by_heads = gr.by_heads;
  // the fewer rows, the more sets of threads share a row's pieces
  const int64_t all_rows = static_cast<int64_t>(f.n_tokens) * f.group * f.by_heads.d;
  const int per = all_rows <= 1024 ? 8 : all_rows <= 2048 ? 4 : all_rows <= 4096 ? 2 : 1;
  int64_t rows = (static_cast<int64_t>(f.n_tokens) + f.n_requests - 1) / f.n_requests * f.group;
  rows = ((rows < kRowTile ? rows : kRowTile) * per + 7) / 8;
  const int64_t joins = pg::max_row_tiles(f.n_requests, f.n_tokens, f.group, kRowTile) * f.by_heads.d;
  hipLaunchKernelGGL((paged_prefix_join_kernel<T, kF8, NT, HS>), dim3(static_cast<uint32_t>(joins), static_cast<uint32_t>(rows)),
                     dim3(kJoinThreads), 0, s, f, p.to, gr, per);
  SDVG_HIP_CHECK(hipGetLastError());
  return SDVG_OK;
}
template <typename T, bool kF8>
int launch_prefix(const First &f, const AttnParams &p, const Groups &gr, const Layout &w, hipStream_t s) {
  if (w.sets == 2) {
    if constexpr (kF8)
      if (w.own_tile == 32) return launch_prefix<T, kF8, 2, 2>(f, p, gr, s);
    return launch_prefix<T, kF8, 1, 2>(f, p, gr, s);
  }
  return w.own_tile == 16 ? launch_prefix<T, kF8, 1, 1>(f, p, gr, s) : launch_prefix<T, kF8, 2, 1>(f, p, gr, s);
}

}  // namespace

extern "C" int64_t sdvg_paged_prefix_attn_workspace_bytes(const sdvg_paged_attn_desc *desc, const sdvg_paged_kv *cache, int32_t n_groups) {
  int st = check_attn(desc, cache), n_cu = 0;
  if (st != SDVG_OK) return st;
  if (n_groups < 0) return SDVG_ERR_SHAPE;
  if (desc->n_requests == 0 || desc->n_tokens == 0) return 0;
  if (n_groups == 0) return sdvg_paged_attn_workspace_bytes(desc, cache);
  if ((st = compute_units(n_cu)) != SDVG_OK) return st;
  return layout_of(n_cu, *desc, *cache, n_groups).bytes();
}

extern "C" int sdvg_paged_prefix_attn(const sdvg_paged_attn_desc *desc, const sdvg_paged_kv *cache, const void *q, const int32_t *block_table,
                                      const int32_t *q_start, const int32_t *kv_lens, int32_t n_groups, const int32_t *group_start,
                                      const int32_t *prefix_lens, void *out, float *lse, void *workspace, int64_t workspace_bytes,
                                      void *stream) {
  int st = check_call(desc, cache, q, block_table, q_start, kv_lens, out, lse, workspace, workspace_bytes);
  if (st != SDVG_OK) return st;
  if (n_groups < 0) return SDVG_ERR_SHAPE;
  if (desc->n_requests == 0 || desc->n_tokens == 0) return SDVG_OK;
  if (n_groups > 0 && (!prefix_lens || (!group_start && n_groups > 1))) return SDVG_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(group_start) | reinterpret_cast<uintptr_t>(prefix_lens)) & 3) return SDVG_ERR_ALIGN;
  int n_cu = 0;
  if ((st = compute_units(n_cu)) != SDVG_OK) return st;
  const Layout w = n_groups > 0 ? layout_of(n_cu, *desc, *cache, n_groups) : Layout{};
  if (n_groups == 0 || !workspace || workspace_bytes < w.bytes())
    return sdvg_paged_attn(desc, cache, q, block_table, q_start, kv_lens, out, lse, workspace, workspace_bytes, stream);
  const int32_t n_kv = cache->n_kv_heads;
  const int32_t shared_turns = pg::turns_of(w.shared_slots * n_kv), own_turns = pg::turns_of(w.own_items * (n_kv / w.sets));
  if ((int64_t{shared_turns} + own_turns) * pg::kTurn >= (1 << 23) || w.own_slots * n_kv >= (1 << 23)) return SDVG_ERR_UNSUPPORTED;
  First f = first_of(*desc, *cache, q_start, kv_lens);
  AttnParams p = params_of(*desc, *cache, q, block_table, out, lse);
  f.by_heads = sdvg::FastDiv::of(n_kv / w.sets);
  f.target = w.target;
  Groups gr{group_start, prefix_lens, n_groups, static_cast<int32_t>(w.own_slots), static_cast<int32_t>(w.shared_slots), w.shared_target,
            shared_turns, own_turns, sdvg::FastDiv::of(n_kv), nullptr, nullptr};
  p.to.part_o = static_cast<float *>(workspace);
  gr.part_o = p.to.part_o + w.own_rows * 128;
  p.to.part_ml = gr.part_o + w.shared_rows * 128;
  gr.part_ml = p.to.part_ml + w.own_rows * 2;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f8 = cache->dtype == SDVG_E4M3;
  if (desc->dtype == SDVG_BF16) return f8 ? launch_prefix<Bf16, true>(f, p, gr, w, s) : launch_prefix<Bf16, false>(f, p, gr, w, s);
  return f8 ? launch_prefix<F16, true>(f, p, gr, w, s) : launch_prefix<F16, false>(f, p, gr, w, s);
}
