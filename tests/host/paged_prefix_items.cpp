// The cut of shared keys into items, from the header the kernels use: over all numbers of a launch every (row tile, key tile) pair of every
// group is one item's, no two items share a slot, a row tile's slots follow each other, and the launch's bounds hold.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <set>
#include <utility>
#include <vector>

#include "paged_prefix_plan.h"

namespace pg = sdvg::paged;

static uint64_t state = 88172645463325252ull;
static uint32_t rnd() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return static_cast<uint32_t>(state >> 11);
}
#define CHECK(c)                                                                                                              \
  do {                                                                                                                        \
    if (!(c)) {                                                                                                               \
      printf("line %d: %s (G %d, group %d, row tile %d, window %d, target %d)\n", __LINE__, #c, G, group, row_tile, window, target); \
      exit(1);                                                                                                                \
    }                                                                                                                         \
  } while (0)

static int tokens_of(const pg::SharedKeys &s, int group) { return s.tokens * group; }

static void one(int G, int longest, int most_tokens, int group, int window, int target, int64_t capacity) {
  constexpr int row_tile = pg::kSharedRows, kT = pg::kSharedTile;
  std::vector<int32_t> token(G + 1), n(G);
  for (int g = 0; g < G; ++g) {
    token[g + 1] = token[g] + rnd() % (most_tokens + 1);
    n[g] = rnd() % 8 == 0 ? rnd() % 2 : rnd() % (longest + 1);
  }
  const int tokens = token[G];
  int64_t total = 0, row_tiles = 0;
  std::vector<pg::SharedKeys> q(G);
  for (int g = 0; g < G; ++g) {
    q[g] = pg::shared_of(g, g + 1, token[g], token[g + 1], n[g], tokens, group, window, capacity);
    total += pg::work_of(q[g]);
    row_tiles += q[g].row_tiles;
    CHECK(q[g].token0 == token[g] && q[g].tokens == token[g + 1] - token[g]);
    const int64_t hi = n[g] < capacity ? n[g] : capacity, first = int64_t{n[g]} + 1 - window, lo = window > 0 && first > 0 ? first : 0;
    CHECK(q[g].lo == lo && q[g].hi == hi);
    if (hi > lo && q[g].tokens > 0) {
      CHECK(q[g].first_tile * int64_t{kT} <= lo && (q[g].first_tile + 1) * int64_t{kT} > lo);
      CHECK((q[g].first_tile + int64_t{q[g].tiles}) * kT >= hi && (q[g].first_tile + int64_t{q[g].tiles} - 1) * kT < hi);
      CHECK(int64_t{q[g].row_tiles} * row_tile >= int64_t{q[g].tokens} * group && (q[g].row_tiles - 1ll) * row_tile < int64_t{q[g].tokens} * group);
    } else {
      CHECK(q[g].tiles == 0 && q[g].row_tiles == 0);
    }
  }
  const int32_t chunk = pg::shared_chunk(total, row_tiles, target);
  CHECK(chunk >= 1);
  const int64_t most_row_tiles = pg::max_shared_row_tiles(G, tokens, group), most = pg::max_shared_items(most_row_tiles, target, capacity);
  CHECK(row_tiles <= most_row_tiles);
  std::set<int64_t> slots;
  int64_t items = 0;
  for (int g = 0; g < G; ++g) {
    const pg::SharedPieces pieces = pg::shared_pieces(q[g], chunk);
    const int32_t mine = pg::shared_items(q[g], pieces);
    std::vector<std::vector<int>> seen(q[g].row_tiles, std::vector<int>(q[g].tiles));
    for (int i = 0; i < mine; ++i) {
      const pg::Place at = pg::shared_place(q[g], pieces, i);
      CHECK(at.tile >= 0 && at.tile < q[g].row_tiles && at.piece >= 0 && at.piece < (pg::is_half(q[g], at.tile) ? pieces.half : pieces.whole));
      const int rows = tokens_of(q[g], group) - at.tile * row_tile;
      CHECK(pg::is_half(q[g], at.tile) == (rows <= row_tile / 2));
      const pg::KeyTiles k = pg::shared_tiles_of(q[g], at, chunk);
      CHECK(k.begin < k.end && k.end - k.begin <= (pg::is_half(q[g], at.tile) ? pg::half_chunk(chunk) : chunk));
      for (int t = k.begin; t < k.end; ++t) {
        CHECK(t >= q[g].first_tile && t < q[g].first_tile + q[g].tiles);
        ++seen[at.tile][t - q[g].first_tile];
      }
      const int64_t slot = items + int64_t{at.tile} * pieces.whole + at.piece;
      CHECK(slot < most && slots.insert(slot).second);
    }
    for (const auto &row : seen)
      for (int x : row) CHECK(x == 1);
    items += mine;
  }
  CHECK(items <= most);
}

int main() {
  const int groups[] = {1, 2, 3, 5, 64, 65, 130}, longest[] = {1, 63, 64, 1000, 30000}, most[] = {1, 7, 200}, heads[] = {1, 5, 16};
  for (int G : groups)
    for (int l : longest)
      for (int m : most)
        for (int group : heads)
            for (int window : {0, 1, 100, 1 << 20})
              for (int target : {1, 4, 32, 512}) {
                if (int64_t{G} * l * m > 3000000) continue;
                one(G, l, m, group, window, target, l + 5);
                one(G, l, m, group, window, target, l / 2 + 8);
              }
  // the largest numbers: nothing leaves 64 bits, and what is kept in 32 fits
  const pg::SharedKeys s = pg::shared_of(0, 1, -5, INT32_MAX, INT32_MAX, 1 << 27, 16, 0, INT32_MAX - 64);
  if (s.row_tiles != (1 << 24) || s.half || s.tiles <= 0 || pg::work_of(s) != (int64_t{1} << 26) * s.tiles || pg::shared_chunk(pg::work_of(s), s.row_tiles, 512) < 1) return 1;
  // every block of both kinds has its turn, once
  for (int shared : {0, 1, 2, 5, 40})
    for (int own : {1, 2, 7, 40}) {
      std::set<std::pair<bool, int>> turns;
      for (int b = 0; b < (shared + own) * pg::kTurn; ++b) {
        const pg::Turn t = pg::turn_of(b, shared, own);
        if (t.block < 0 || t.block >= (t.shared ? shared : own) * pg::kTurn || t.block % 8 != b % 8 || !turns.insert({t.shared, t.block}).second) return 1;
      }
    }
  printf("ok\n");
  return 0;
}
