// How the work of a paged attention launch is cut into workgroups: integer arithmetic on the requests' lengths, which the
// kernels do on the device (lengths are device data) and a host test repeats.
//
// The rows of a request that share a key head (its new tokens x the query heads of the group) are cut into tiles of
// row_tile rows. Work is counted in (row tile, key tile) pairs; `chunk` key tiles at most go to one workgroup ("item"). A request whose keys fit one chunk is
// written by its workgroup; the others leave a partial result per item in a numbered slot, and the join adds up a
// group of consecutive slots per row tile.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define SDVG_PAGED_HD __host__ __device__ inline __attribute__((always_inline))
#else
#define SDVG_PAGED_HD inline
#endif

namespace sdvg {
namespace paged {

constexpr int kKeyTile = 32;   // keys a wave takes per step

// What a request asks for.
struct Request {
  int32_t row0, n;              // first row among all tokens, new tokens
  int32_t len;                  // keys of the last token: positions 0 .. len - 1
  int32_t first_tile, tiles;    // key tiles that any of its rows sees
  int32_t row_tiles;
  int32_t from;                 // keys ahead of this one are another launch's (a prefix that several requests share)
};
SDVG_PAGED_HD int32_t clamp(int32_t x, int32_t lo, int32_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// What a request's numbers name, whatever they are (start, end: q_start[r], q_start[r + 1]): n tokens from row0 on among the batch's n_tokens, the
// last of which sees `len` keys.
struct Rows {
  int32_t row0, n, len;
};
SDVG_PAGED_HD Rows rows_of(int32_t start, int32_t end, int32_t len, int32_t n_tokens) {
  Rows a;
  a.row0 = clamp(start, 0, n_tokens);
  a.n = clamp(end, a.row0, n_tokens) - a.row0;
  a.len = len > 0 ? len : 0;
  return a;
}
// Keys that token row0 + i of them sees, 0 <= i < n (none if not positive).
SDVG_PAGED_HD int32_t sees_of(const Rows &a, int32_t i) { return a.len - a.n + i + 1; }

// capacity: keys that a row of the block table can name.
SDVG_PAGED_HD Request request_of(int32_t start, int32_t end, int32_t len, int32_t n_tokens, int32_t group, int32_t row_tile,
                                 int32_t window, int64_t capacity, int32_t prefix = 0) {
  const Rows rows = rows_of(start, end, len, n_tokens);
  Request q;
  q.row0 = rows.row0;
  q.n = rows.n;
  q.len = rows.len;
  const int64_t first = static_cast<int64_t>(q.len) - q.n + 1 - window;  // of the first token's window
  const int32_t hi = q.len < capacity ? q.len : static_cast<int32_t>(capacity);
  int32_t lo = window > 0 && first > 0 ? static_cast<int32_t>(first) : 0;
  q.from = prefix > 0 ? prefix : 0;
  lo = lo > q.from ? lo : q.from;
  q.first_tile = lo / kKeyTile;
  q.tiles = hi > lo ? static_cast<int32_t>((static_cast<int64_t>(hi) + kKeyTile - 1) / kKeyTile) - q.first_tile : 0;
  q.row_tiles = static_cast<int32_t>((static_cast<int64_t>(q.n) * group + row_tile - 1) / row_tile);
  return q;
}
// (A row tile without keys still is an item: somebody has to write its zeros.)
SDVG_PAGED_HD int64_t work_of(const Request &q) { return static_cast<int64_t>(q.row_tiles) * (q.tiles > 1 ? q.tiles : 1); }

// Key tiles per item at most: total = the sum of work_of over all requests, row_tiles that of theirs, target the items that fill
// the chip with two workgroups per compute unit (<= 0: no split), key_waves the waves that share an item's key tiles, which have
// one each at least.
// Few row tiles: the items are made to fit the chip, so that all run at once and end together; every row tile may add one by rounding
// up. One workgroup per unit is enough for HBM where that rounding is small (up to a quarter of the units: 131071 keys 87 us, with two
// 90; 24 requests x 8 heads x 2000 keys, which is more, 38 and 37).
// Many row tiles: fitting would leave some items much longer than others, so they are made shorter, kFiner rounds of them, and the
// chip fills up again as they end; but not shorter than kRoundChunk (what comes before and after the keys takes as long as some
// 10 key tiles) unless the chip is not filled once, and not shorter than kFilledChunk where the row tiles alone give two thirds of the
// units a workgroup. us with kFilledChunk 24, without, and with 32: 64 requests x 8 heads x 500 keys 25.6, 28.3, 25.6; 32 x 8, 30
// rows, 350 keys 14.2, 20.5, 14.4, lengths of 16 to 500 15.0, 22.4, 15.0; but 64 x 8 x 936 keys 44.9, 43.5, 41.8 and 16 to 1400 keys 43.4, 37.5,
// 54.2. Over 128 batches of one length 3 % better than without, over 128 of unlike lengths 1 %, the worst 1.4 times the best way of all that
// were tried, without 2.1 (profiles/paged_attn_cut_sweep.txt, with the other constants). With fewer row tiles it loses: 40 x 8 x 2000 keys 66, 54.
// Requests of kWhole key tiles on average are not split: 64 x 8 x 120 keys 6.9 us, split 12.2; 250 keys 12.9, 18.4.
constexpr int kFiner = 3, kRoundChunk = 32, kFilledChunk = 24, kWhole = 8;
SDVG_PAGED_HD int64_t ceil_div(int64_t a, int32_t b) {
  if (a <= INT32_MAX) return (static_cast<uint32_t>(a) + static_cast<uint32_t>(b) - 1) / static_cast<uint32_t>(b);  // (the shorter division)
  return (a + b - 1) / b;
}
SDVG_PAGED_HD int32_t chunk_of(int64_t total, int64_t row_tiles, int32_t target, int32_t key_waves) {
  if (target <= 0) return INT32_MAX;
  int64_t c;
  if (4 * row_tiles <= target) {
    const int32_t slots = 8 * row_tiles <= target && target > 1 ? target / 2 : target;
    c = ceil_div(total, slots - static_cast<int32_t>(row_tiles));
  } else {
    const int64_t once = ceil_div(total, target), finer = ceil_div(once, kFiner);
    const int64_t filled = once > kFilledChunk || 3 * row_tiles < target ? once : kFilledChunk;
    const int64_t least = filled < kRoundChunk ? filled : kRoundChunk;
    c = finer > least ? finer : least;
  }
  if (total <= kWhole * row_tiles && c < kWhole) c = kWhole;
  return c > key_waves ? static_cast<int32_t>(c < INT32_MAX ? c : INT32_MAX) : key_waves;
}
// Pieces per row tile: `full` ones of `chunk` key tiles, and one of what is left (of everything where there are no keys). The
// full ones of all requests are started first, so that short ones are left for the end, when the chip runs empty.
SDVG_PAGED_HD int32_t full_pieces(const Request &q, int32_t chunk) {
  return q.tiles >= chunk ? static_cast<int32_t>(static_cast<uint32_t>(q.tiles) / static_cast<uint32_t>(chunk)) : 0;
}
SDVG_PAGED_HD int32_t pieces_of(const Request &q, int32_t chunk, int32_t full) {
  return full + (full == 0 || q.tiles > full * chunk ? 1 : 0);
}

// Items are numbered through all requests, first the full pieces of every request (kFull), then the others (kRest); the join numbers
// the split row tiles (kSplit). How many of a range are a request's, which has `pieces` pieces per row tile, `full` full ones among them:
enum Range { kFull, kRest, kSplit };
// (`join`: a row tile is joined, and has slots, even where its own keys are one piece.)
SDVG_PAGED_HD int32_t numbers_of(const Request &q, int32_t full, int32_t pieces, Range range, bool join = false) {
  return q.row_tiles * (range == kFull ? full : range == kRest ? pieces - full : join || pieces > 1);
}
// Row tile and piece of number i of a request's own. The row tiles of a full piece follow each other where workgroups that read
// the same keys then are on the same XCD (they are dealt out to 8 in turn): where the (sets of) key heads are a multiple of 8. 64 rows x
// 131071 keys x 8 heads, 16 bit, 166 us with the pieces of a row tile in a row, 136 so; with 4 sets of heads (e4m3) 92 and 97.
struct Place {
  int32_t tile, piece;
};
SDVG_PAGED_HD Place place_of(const Request &q, int32_t i, int32_t full, Range range, uint32_t head_sets) {
  if (range != kFull) return Place{i, range == kRest ? full : 0};
  if (q.row_tiles == 1) return Place{0, i};
  if (head_sets % 8 == 0) {
    const int32_t piece = static_cast<uint32_t>(i) / static_cast<uint32_t>(q.row_tiles);
    return Place{i - piece * q.row_tiles, piece};
  }
  const int32_t tile = static_cast<uint32_t>(i) / static_cast<uint32_t>(full);
  return Place{tile, i - tile * full};
}
// Slot of a piece's partial result: slot0 is the number of slots of the requests before.
SDVG_PAGED_HD int32_t slots_of(const Request &q, int32_t pieces, bool join = false) { return join || pieces > 1 ? q.row_tiles * pieces : 0; }
SDVG_PAGED_HD int32_t first_slot(int32_t slot0, int32_t tile, int32_t pieces) { return slot0 + tile * pieces; }
// Key tiles begin .. end - 1 of a piece.
struct KeyTiles {
  int32_t begin, end;
};
SDVG_PAGED_HD KeyTiles key_tiles_of(const Request &q, int32_t piece, int32_t chunk) {
  const int32_t before = piece ? piece * chunk : 0;
  return KeyTiles{q.first_tile + before, q.first_tile + (q.tiles - before < chunk ? q.tiles : before + chunk)};
}

// Bounds for the launch, from what the host knows, with most = kFiner * target >= total / chunk. Items: most full chunks, and one
// more per row tile; no more than `target` where the row tiles are few; and none of a row tile below key_waves key tiles of what a row of
// the block table can name (`capacity` keys; one item where these are kWhole tiles). Slots: a split row tile of t > chunk tiles has ceil(t / chunk) < 2 t / chunk pieces. Groups
// (split row tiles): t > chunk each.
SDVG_PAGED_HD int64_t max_row_tiles(int64_t n_requests, int64_t n_tokens, int32_t group, int32_t row_tile) {
  const int64_t rows = n_tokens * group;
  const int64_t bound = rows / row_tile + n_requests;
  return bound < rows ? bound : rows;
}
SDVG_PAGED_HD int64_t max_pieces(int64_t capacity, int32_t key_waves) { return ceil_div(capacity, kKeyTile) <= kWhole ? 1 : ceil_div(ceil_div(capacity, kKeyTile) + 1, key_waves); }  // (+ 1: a window may begin inside a tile)
SDVG_PAGED_HD int64_t max_items(int64_t row_tiles, int32_t target, int64_t capacity, int32_t key_waves) {
  if (target <= 0) return row_tiles;
  const int64_t by_chunk = 4 * row_tiles <= target ? target : row_tiles + kFiner * static_cast<int64_t>(target);
  const int64_t by_keys = row_tiles * max_pieces(capacity, key_waves);
  return by_chunk < by_keys ? by_chunk : by_keys;
}
SDVG_PAGED_HD int64_t max_groups(int64_t row_tiles, int32_t target) { return row_tiles < kFiner * static_cast<int64_t>(target) ? row_tiles : kFiner * static_cast<int64_t>(target); }
SDVG_PAGED_HD int64_t max_slots(int32_t target) { return 2 * kFiner * static_cast<int64_t>(target); }

}  // namespace paged
}  // namespace sdvg
