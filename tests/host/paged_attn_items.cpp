// The numbering of paged attention's workgroups, from the header the kernels use: over all numbers of a launch every (row tile, key tile)
// pair is one item's, the pieces of split row tiles have slots of their own, and the join's numbers name each split row tile once,
// with the slots that its items wrote.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <set>
#include <vector>

#include "paged_attn_plan.h"

namespace pg = sdvg::paged;

static uint64_t state = 1181783497276652981ull;
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

static long split_launches = 0, tiles_inner = 0;

static void one(int R, int longest, int most_new, int group, int row_tile, int window, int target, int key_waves, int sets) {
  std::vector<int32_t> start(R + 1), len(R);
  for (int r = 0; r < R; ++r) {
    const int n = rnd() % (most_new + 1);
    start[r + 1] = start[r] + n;
    len[r] = rnd() % 16 == 0 ? rnd() % 3 : n + rnd() % (longest + 1);
  }
  const int tokens = start[R];
  if (tokens == 0) return;
  const int64_t capacity = longest + most_new + 31;
  std::vector<pg::Request> q(R);
  std::vector<int32_t> full(R), pieces(R);
  int64_t total = 0, row_tiles = 0;
  for (int r = 0; r < R; ++r) {
    q[r] = pg::request_of(start[r], start[r + 1], len[r], tokens, group, row_tile, window, capacity);
    total += pg::work_of(q[r]);
    row_tiles += q[r].row_tiles;
  }
  const int32_t chunk = pg::chunk_of(total, row_tiles, target, key_waves);
  int32_t count[3] = {0, 0, 0};
  for (int r = 0; r < R; ++r) {
    full[r] = pg::full_pieces(q[r], chunk);
    pieces[r] = pg::pieces_of(q[r], chunk, full[r]);
    for (int k = 0; k < 3; ++k) count[k] += pg::numbers_of(q[r], full[r], pieces[r], static_cast<pg::Range>(k));
  }
  // what number x of a range is: (request, row tile, piece, first slot)
  struct Found {
    int r;
    pg::Place at;
    int32_t slot;
  };
  const auto find = [&](int32_t x, pg::Range range) {
    int32_t slot0 = 0;
    for (int r = 0;; ++r) {
      CHECK(r < R);
      const int32_t mine = pg::numbers_of(q[r], full[r], pieces[r], range);
      if (x < mine) {
        const pg::Place at = pg::place_of(q[r], x, full[r], range, sets);
        return Found{r, at, pg::first_slot(slot0, at.tile, pieces[r])};
      }
      x -= mine;
      slot0 += pg::slots_of(q[r], pieces[r]);
    }
  };
  std::vector<std::vector<uint8_t>> seen(R);   // [row tile][key tile], and whether a row tile without keys is somebody's
  for (int r = 0; r < R; ++r) seen[r].resize(static_cast<size_t>(q[r].row_tiles) * std::max(q[r].tiles, 1));
  std::vector<std::vector<std::vector<int32_t>>> slots(R);
  for (int r = 0; r < R; ++r) slots[r].resize(q[r].row_tiles);
  std::set<int32_t> taken;
  for (int32_t x = 0; x < count[pg::kFull] + count[pg::kRest]; ++x) {
    const bool among_full = x < count[pg::kFull];
    const Found f = find(among_full ? x : x - count[pg::kFull], among_full ? pg::kFull : pg::kRest);
    const pg::Request &a = q[f.r];
    CHECK(f.at.tile >= 0 && f.at.tile < a.row_tiles && f.at.piece >= 0 && f.at.piece < pieces[f.r]);
    const pg::KeyTiles keys = pg::key_tiles_of(a, f.at.piece, chunk);
    CHECK(keys.begin >= a.first_tile && keys.end <= a.first_tile + a.tiles && keys.end - keys.begin <= chunk);
    CHECK(among_full ? keys.end - keys.begin == chunk : keys.end - keys.begin < chunk);
    if (a.tiles == 0) {
      CHECK(keys.begin == keys.end && pieces[f.r] == 1 && !seen[f.r][f.at.tile]++);
    } else {
      CHECK(keys.begin < keys.end);
      for (int k = keys.begin; k < keys.end; ++k) CHECK(!seen[f.r][static_cast<size_t>(f.at.tile) * a.tiles + k - a.first_tile]++);
    }
    if (pieces[f.r] > 1) {
      const int32_t slot = f.slot + f.at.piece;
      CHECK(slot >= 0 && slot < pg::max_slots(target) && taken.insert(slot).second);
      slots[f.r][f.at.tile].push_back(slot);
    }
  }
  for (int r = 0; r < R; ++r)
    for (uint8_t s : seen[r]) CHECK(s == 1);
  std::set<std::pair<int, int>> joined;
  for (int32_t x = 0; x < count[pg::kSplit]; ++x) {
    const Found f = find(x, pg::kSplit);
    CHECK(f.at.tile >= 0 && f.at.tile < q[f.r].row_tiles && pieces[f.r] > 1 && joined.insert({f.r, f.at.tile}).second);
    std::vector<int32_t> &have = slots[f.r][f.at.tile];
    std::sort(have.begin(), have.end());
    CHECK(static_cast<int>(have.size()) == pieces[f.r]);
    for (int i = 0; i < pieces[f.r]; ++i) CHECK(have[i] == f.slot + i);
  }
  for (int r = 0; r < R; ++r)
    for (int t = 0; t < q[r].row_tiles; ++t) CHECK(pieces[r] == 1 || joined.count({r, t}));
  if (count[pg::kSplit]) {
    ++split_launches;
    if (sets % 8 == 0) ++tiles_inner;
  }
}

int main() {
  for (int R : {1, 2, 5, 63, 64, 65, 200})
    for (int longest : {0, 31, 33, 700, 9000})
      for (int group : {1, 3, 8, 40})
        for (int row_tile : {16, 32})
          for (int window : {0, 17, 4096})
            for (int target : {0, 1, 7, 64, 512})
              for (int sets : {1, 4, 8, 16}) {
                one(R, longest, 1, group, row_tile, window, target, 4, sets);
                one(R, longest, 9, group, row_tile, window, target, 2, sets);
              }
  if (split_launches < 1000 || tiles_inner < 500) return printf("too few launches were split: %ld, %ld\n", split_launches, tiles_inner), 1;
  printf("ok\n");
  return 0;
}
