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
#include "paged_attn_device.h"

namespace {

// T: type of q, of P and of the output. kF8: the cache holds e4m3 numbers.
template <typename T, bool kF8, int NT, int HS>
__global__ __launch_bounds__(kThreads, kPerUnit) void paged_attn_kernel(FIRST_ARGS, AttnParams p) {
  const First first{q_start, kv_lens, n_requests, n_tokens, group, window, target, capacity, {heads_d, heads_m, heads_s}};
  __shared__ float o_s[kWaves][kRows][kPad];
  __shared__ float ml_s[kWaves][kRows][2];
  attend<T, kF8, NT, HS, false>(first, p, Groups{}, blockIdx.x, o_s, ml_s);
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
  if (!find<kRowTile, kWaves / HS, false, false>(head_args, Groups{}, index, f)) return;
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

int64_t workspace_of(int target, int n_kv_heads, int row_tile) {
  return pg::max_slots(target) * n_kv_heads * row_tile * (128 + 2) * 4;
}

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
  int st = check_call(desc, cache, q, block_table, q_start, kv_lens, out, lse, workspace, workspace_bytes), n_cu = 0;
  if (st != SDVG_OK) return st;
  if (desc->n_requests == 0 || desc->n_tokens == 0) return SDVG_OK;
  if ((st = compute_units(n_cu)) != SDVG_OK) return st;
  const int32_t n_kv = cache->n_kv_heads, group = desc->n_heads / n_kv;
  First f = first_of(*desc, *cache, q_start, kv_lens);
  AttnParams p = params_of(*desc, *cache, q, block_table, out, lse);
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
