// The cut of the keys behind shared prefixes, from the header the kernels use: over all numbers of a launch every (row tile, key tile) pair behind
// a request's prefix is one item's, every item of every row tile has a slot of its own, the join names every row tile once with the
// slots that its items wrote, and the launch's bounds hold (blocks, slots of the workspace, joins).
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <set>
#include <utility>
#include <vector>

#include "paged_prefix_plan.h"

namespace pg = sdvg::paged;

static uint64_t state = 2463534242ull * 7919;
static uint32_t rnd() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return static_cast<uint32_t>(state >> 11);
}
#define CHECK(c)                                                                                                            \
  do {                                                                                                                      \
    if (!(c)) {                                                                                                             \
      printf("line %d: %s (R %d, group %d, row tile %d, window %d, target %d, sets %d)\n", __LINE__, #c, R, group, row_tile, \
             window, target, sets);                                                                                         \
      exit(1);                                                                                                              \
    }                                                                                                                       \
  } while (0)

static long split = 0, whole = 0, empty = 0, most_of_slots = 0;

static void one(int R, int longest_prefix, int longest, int most_new, int group, int row_tile, int window, int target, int key_waves, int sets) {
  std::vector<int32_t> start(R + 1), len(R), prefix(R);
  for (int r = 0; r < R; ++r) {
    const int n = rnd() % (most_new + 1);
    start[r + 1] = start[r] + n;
    // groups of some requests; some share nothing, some lengths end inside the prefix
    prefix[r] = r && rnd() % 4 ? prefix[r - 1] : rnd() % 5 ? static_cast<int>(rnd() % (longest_prefix + 1)) : 0;
    len[r] = rnd() % 16 == 0 ? rnd() % 3 : prefix[r] + n + rnd() % (longest + 1);
  }
  const int tokens = start[R];
  if (tokens == 0) return;
  const int64_t capacity = longest_prefix + longest + most_new + 31 - (rnd() % 4 ? 0 : longest / 2);
  const int t = pg::max_pieces(capacity, key_waves) <= 1 ? 0 : target;   // as the launch has it: no split where a table names few keys
  std::vector<pg::Request> q(R);
  std::vector<int32_t> full(R), pieces(R);
  int64_t total = 0, row_tiles = 0;
  for (int r = 0; r < R; ++r) {
    q[r] = pg::request_of(start[r], start[r + 1], len[r], tokens, group, row_tile, window, capacity, prefix[r]);
    const int64_t hi = std::min<int64_t>(len[r], capacity), n = start[r + 1] - start[r], lo = std::max<int64_t>(prefix[r], window > 0 ? std::max<int64_t>(0, len[r] - n + 1 - window) : 0);
    if (hi > lo) {
      CHECK(q[r].first_tile == lo / pg::kKeyTile && q[r].first_tile + q[r].tiles == (hi + pg::kKeyTile - 1) / pg::kKeyTile);
    } else {
      CHECK(q[r].tiles == 0);
    }
    CHECK(q[r].from == prefix[r]);
    total += pg::work_of(q[r]);
    row_tiles += q[r].row_tiles;
  }
  const int32_t chunk = pg::chunk_of(total, row_tiles, t, key_waves);
  int32_t count[3] = {0, 0, 0};
  int64_t n_slots = 0;
  for (int r = 0; r < R; ++r) {
    full[r] = pg::full_pieces(q[r], chunk);
    pieces[r] = pg::pieces_of(q[r], chunk, full[r]);
    for (int k = 0; k < 3; ++k) count[k] += pg::numbers_of(q[r], full[r], pieces[r], static_cast<pg::Range>(k), true);
    n_slots += pg::slots_of(q[r], pieces[r], true);
  }
  // what the launch has room for, from what the host knows
  const int64_t tiles = pg::max_row_tiles(R, tokens, group, row_tile), blocks = pg::max_items(tiles, t, capacity, key_waves), slots_there = pg::max_slots(t) + tiles;
  CHECK(row_tiles <= tiles && count[pg::kFull] + int64_t{count[pg::kRest]} <= blocks && n_slots <= slots_there && count[pg::kSplit] == row_tiles);
  if (2 * n_slots > slots_there) ++most_of_slots;
  struct Found {
    int r;
    pg::Place at;
    int32_t slot;
  };
  const auto find = [&](int32_t x, pg::Range range) {
    int32_t slot0 = 0;
    for (int r = 0;; ++r) {
      CHECK(r < R);
      const int32_t mine = pg::numbers_of(q[r], full[r], pieces[r], range, true);
      if (x < mine) {
        const pg::Place at = pg::place_of(q[r], x, full[r], range, sets);
        return Found{r, at, pg::first_slot(slot0, at.tile, pieces[r])};
      }
      x -= mine;
      slot0 += pg::slots_of(q[r], pieces[r], true);
    }
  };
  std::vector<std::vector<uint8_t>> seen(R);
  std::vector<std::vector<std::vector<int32_t>>> slots(R);
  for (int r = 0; r < R; ++r) {
    seen[r].resize(static_cast<size_t>(q[r].row_tiles) * std::max(q[r].tiles, 1));
    slots[r].resize(q[r].row_tiles);
  }
  std::set<int32_t> taken;
  for (int32_t x = 0; x < count[pg::kFull] + count[pg::kRest]; ++x) {
    const bool among_full = x < count[pg::kFull];
    const Found f = find(among_full ? x : x - count[pg::kFull], among_full ? pg::kFull : pg::kRest);
    const pg::Request &a = q[f.r];
    CHECK(f.at.tile >= 0 && f.at.tile < a.row_tiles && f.at.piece >= 0 && f.at.piece < pieces[f.r]);
    const pg::KeyTiles keys = pg::key_tiles_of(a, f.at.piece, chunk);
    CHECK(keys.begin >= a.first_tile && keys.end <= a.first_tile + a.tiles && keys.end - keys.begin <= chunk);
    if (a.tiles == 0) {
      CHECK(keys.begin == keys.end && pieces[f.r] == 1 && !seen[f.r][f.at.tile]++);
      ++empty;
    } else {
      CHECK(keys.begin < keys.end);
      for (int k = keys.begin; k < keys.end; ++k) CHECK(!seen[f.r][static_cast<size_t>(f.at.tile) * a.tiles + k - a.first_tile]++);
    }
    const int32_t slot = f.slot + f.at.piece;
    CHECK(slot >= 0 && slot < slots_there && f.slot <= slots_there - pieces[f.r] && taken.insert(slot).second);
    slots[f.r][f.at.tile].push_back(slot);
  }
  for (int r = 0; r < R; ++r)
    for (uint8_t s : seen[r]) CHECK(s == 1);
  std::set<std::pair<int, int>> joined;
  for (int32_t x = 0; x < count[pg::kSplit]; ++x) {
    const Found f = find(x, pg::kSplit);
    CHECK(f.at.tile >= 0 && f.at.tile < q[f.r].row_tiles && joined.insert({f.r, f.at.tile}).second);
    std::vector<int32_t> &have = slots[f.r][f.at.tile];
    std::sort(have.begin(), have.end());
    CHECK(static_cast<int>(have.size()) == pieces[f.r]);
    for (int i = 0; i < pieces[f.r]; ++i) CHECK(have[i] == f.slot + i);
    ++(pieces[f.r] > 1 ? split : whole);
  }
}

int main() {
  for (int R : {1, 2, 5, 63, 64, 65, 200})
    for (int longest_prefix : {0, 40, 5000})
      for (int longest : {0, 33, 700, 9000})
        for (int group : {1, 5, 40})
          for (int row_tile : {16, 32})
            for (int window : {0, 17, 4096})
              for (int target : {1, 7, 64, 512})
                for (int sets : {1, 8}) {
                  one(R, longest_prefix, longest, 1, group, row_tile, window, target, 4, sets);
                  one(R, longest_prefix, longest, 9, group, row_tile, window, target, 2, sets);
                }
  if (split < 1000 || whole < 1000 || empty < 1000 || most_of_slots < 20) return printf("too few of a kind: %ld, %ld, %ld, %ld\n", split, whole, empty, most_of_slots), 1;
  printf("ok\n");
  return 0;
}
