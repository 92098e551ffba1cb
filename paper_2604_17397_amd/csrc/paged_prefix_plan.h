// How the keys that groups of requests share are cut into workgroups: integer arithmetic on the groups' rows and keys, which the
// kernels do on the device and a host test repeats. (The requests' own keys are cut as paged_attn_plan.h says.)
//
// The rows of a group that share a key head (the new tokens of all its requests x the query heads of a key head) are cut into tiles
// of kSharedRows rows, the shared keys into pieces of `chunk` key tiles at most; a third more where the last row tile has no more than half
// of the rows, whose key tiles take some three quarters of the time (half the products, the same copies; 64 x 65520 keys of 320 rows 183 us with pieces of one
// length, 174 so). Every item (row tile, piece) leaves a partial result in a numbered slot; a row tile's are consecutive.
#pragma once
#include "paged_attn_plan.h"

namespace sdvg {
namespace paged {

constexpr int kSharedTile = 64;   // keys that a workgroup has in LDS at a time
constexpr int kSharedRows = 128;

struct SharedKeys {
  int32_t request0, requests;     // the group's
  int32_t token0, tokens;         // their new tokens, which are neighbours
  int32_t lo, hi;                 // keys lo .. hi - 1 are shared and may be seen
  int32_t first_tile, tiles;      // key tiles that hold them
  int32_t row_tiles;
  int32_t half;                   // 1: the last of them has at most half of its rows
};
// start, end: the group's first request and the next group's; token0, token1: q_start of the two; n: shared keys.
// (No new token lies among the shared keys, so with a window none sees one ahead of n + 1 - window.)
SDVG_PAGED_HD SharedKeys shared_of(int32_t start, int32_t end, int32_t token0, int32_t token1, int32_t n, int32_t n_tokens, int32_t group,
                                   int32_t window, int64_t capacity) {
  SharedKeys s;
  s.request0 = start;
  s.requests = end - start;
  s.token0 = clamp(token0, 0, n_tokens);
  s.tokens = clamp(token1, s.token0, n_tokens) - s.token0;
  const int64_t first = static_cast<int64_t>(n) + 1 - window;
  s.lo = window > 0 && first > 0 ? static_cast<int32_t>(first) : 0;
  s.hi = n < capacity ? n : static_cast<int32_t>(capacity);
  s.first_tile = s.lo / kSharedTile;
  s.tiles = s.hi > s.lo && s.tokens > 0 ? (s.hi + kSharedTile - 1) / kSharedTile - s.first_tile : 0;
  const int64_t rows = static_cast<int64_t>(s.tokens) * group;
  s.row_tiles = s.tiles > 0 ? static_cast<int32_t>((rows + kSharedRows - 1) / kSharedRows) : 0;
  s.half = s.row_tiles > 0 && rows - (s.row_tiles - int64_t{1}) * kSharedRows <= kSharedRows / 2;
  return s;
}
// In quarters of a (row tile, key tile) pair.
SDVG_PAGED_HD int64_t work_of(const SharedKeys &s) { return (4 * static_cast<int64_t>(s.row_tiles) - s.half) * s.tiles; }

// Key tiles per item at most: total = the sum of work_of over all groups, row_tiles that of theirs, target the items that fill the chip.
// Where the row tiles are few, the items are made to fit the chip once; rounding up adds one per row tile at most.
constexpr int kSharedRounds = 2, kSharedLeast = 8;
SDVG_PAGED_HD int32_t shared_chunk(int64_t total, int64_t row_tiles, int32_t target) {
  int64_t c;
  if (2 * row_tiles <= target) {
    c = ceil_div(total, 4 * (target - static_cast<int32_t>(row_tiles)));
  } else {
    c = ceil_div(total, 4 * kSharedRounds * target);
    if (c < kSharedLeast) c = kSharedLeast;
  }
  return c < 1 ? 1 : c < INT32_MAX / 4 ? static_cast<int32_t>(c) : INT32_MAX / 4;
}
// Pieces of a row tile, of the last one where it is a half; items of a group.
struct SharedPieces {
  int32_t whole, half;
};
SDVG_PAGED_HD int32_t half_chunk(int32_t chunk) { return chunk + (chunk + 2) / 3; }   // (not less than 4 / 3: the items' bound rests on it)
SDVG_PAGED_HD SharedPieces shared_pieces(const SharedKeys &s, int32_t chunk) {
  const uint32_t t = static_cast<uint32_t>(s.tiles), c = static_cast<uint32_t>(chunk), h = static_cast<uint32_t>(half_chunk(chunk));
  return SharedPieces{static_cast<int32_t>((t + c - 1) / c), static_cast<int32_t>((t + h - 1) / h)};
}
SDVG_PAGED_HD int32_t shared_items(const SharedKeys &s, const SharedPieces &n) { return (s.row_tiles - s.half) * n.whole + s.half * n.half; }
SDVG_PAGED_HD bool is_half(const SharedKeys &s, int32_t tile) { return s.half && tile == s.row_tiles - 1; }
// Item i of a group: the row tiles of a piece follow each other, so that workgroups that read the same keys run at the same time. Its
// slot is slot0 (of the groups before) + tile * n.whole + piece.
SDVG_PAGED_HD Place shared_place(const SharedKeys &s, const SharedPieces &n, int32_t i) {
  const int32_t wholes = s.row_tiles - s.half;
  if (i >= wholes * n.whole) return Place{wholes, i - wholes * n.whole};
  const int32_t piece = static_cast<uint32_t>(i) / static_cast<uint32_t>(wholes);
  return Place{i - piece * wholes, piece};
}
SDVG_PAGED_HD KeyTiles shared_tiles_of(const SharedKeys &s, const Place &at, int32_t chunk) {
  const int32_t c = is_half(s, at.tile) ? half_chunk(chunk) : chunk, before = at.piece ? at.piece * c : 0;
  return KeyTiles{s.first_tile + before, s.first_tile + (s.tiles - before < c ? s.tiles : before + c)};
}

// Bounds for the launch from what the host knows: row tiles, and items (and slots). total / (4 chunk) <= target - row_tiles, or
// kSharedRounds * target; and one more per row tile.
SDVG_PAGED_HD int64_t max_shared_row_tiles(int64_t n_groups, int64_t n_tokens, int32_t group) {
  const int64_t rows = n_tokens * group, bound = rows / kSharedRows + n_groups;
  return bound < rows ? bound : rows;
}
SDVG_PAGED_HD int64_t max_shared_items(int64_t row_tiles, int32_t target, int64_t capacity) {
  const int64_t by_chunk = 2 * row_tiles <= target ? target : row_tiles + kSharedRounds * static_cast<int64_t>(target);
  const int64_t by_keys = row_tiles * ceil_div(capacity, kSharedTile);
  return by_chunk < by_keys ? by_chunk : by_keys;
}

// The launch has blocks of both kinds, the shared keys' and the requests' own, in turns of kTurn blocks (one for every compute unit, and
// a multiple of the 8 XCDs, to which a block's number modulo 8 stays the same); what one kind has more comes last. (us of a call: 128 x 8191 shared keys 83, 64 x
// 65520 171, 24 requests of up to 8 tokens 88; in turns of 8 blocks 85, 255, 139, of 64 81, 171, 92, all the shared ones first 95, 176, 83.)
constexpr int kTurn = 256;
struct Turn {
  bool shared;
  int32_t block;   // among those of its kind
};
SDVG_PAGED_HD int32_t turns_of(int64_t blocks) { return static_cast<int32_t>((blocks + kTurn - 1) / kTurn); }
SDVG_PAGED_HD Turn turn_of(int32_t block, int32_t shared_turns, int32_t own_turns) {
  const int32_t turn = block / kTurn, in = block - turn * kTurn, both = shared_turns < own_turns ? shared_turns : own_turns;
  if (turn < 2 * both) return Turn{(turn & 1) == 0, turn / 2 * kTurn + in};
  return Turn{shared_turns > own_turns, (turn - both) * kTurn + in};
}

}  // namespace paged
}  // namespace sdvg
