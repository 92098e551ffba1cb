// The cut of paged attention launches into items, from the header the kernels use: for many batches of lengths every (row tile,
// key tile) pair is one item's, the launch's bounds hold, and no two pieces share a slot.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "paged_attn_plan.h"

namespace pg = sdvg::paged;

static uint64_t state = 88172645463325252ull;
static uint32_t rnd() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return static_cast<uint32_t>(state >> 11);
}
#define CHECK(c)                                                                             \
  do {                                                                                       \
    if (!(c)) {                                                                              \
      printf("line %d: %s (R %d, group %d, row tile %d, window %d, target %d)\n", __LINE__, #c, R, group, row_tile, window, target); \
      exit(1);                                                                               \
    }                                                                                        \
  } while (0)

static void one(int R, int longest, int most_new, int group, int row_tile, int window, int target, int64_t capacity, int key_waves) {
  std::vector<int32_t> start(R + 1), len(R);
  int tokens = 0;
  for (int r = 0; r < R; ++r) {
    start[r] = tokens;
    const int n = rnd() % (most_new + 1);
    tokens += n;
    len[r] = n + rnd() % (longest + 1);
    if (rnd() % 16 == 0) len[r] = rnd() % 3;      // shorter than its own new tokens, or empty
  }
  start[R] = tokens;
  if (tokens == 0) return;
  int64_t total = 0;
  std::vector<pg::Request> q(R);
  for (int r = 0; r < R; ++r) {
    q[r] = pg::request_of(start[r], start[r + 1], len[r], tokens, group, row_tile, window, capacity);
    CHECK(q[r].row0 == start[r] && q[r].n == start[r + 1] - start[r]);
    CHECK(int64_t{q[r].row_tiles} * row_tile >= int64_t{q[r].n} * group && int64_t{q[r].row_tiles - 1} * row_tile < int64_t{q[r].n} * group);
    total += pg::work_of(q[r]);
    // every key that some row sees lies in the tiles
    const int64_t hi = len[r] < capacity ? len[r] : capacity, first = int64_t{len[r]} - q[r].n + 1 - window;
    const int64_t lo = window > 0 && first > 0 ? first : 0;
    if (hi > lo) CHECK(q[r].first_tile * 32ll <= lo && (q[r].first_tile + int64_t{q[r].tiles}) * 32 >= hi && (q[r].first_tile + int64_t{q[r].tiles} - 1) * 32 < hi);
    else CHECK(q[r].tiles == 0);
  }
  int64_t items = 0, slots = 0, groups = 0, row_tiles = 0, all_row_tiles = 0;
  for (const pg::Request &x : q) all_row_tiles += x.row_tiles;
  const int32_t chunk = pg::chunk_of(total, all_row_tiles, target, key_waves);
  for (int r = 0; r < R; ++r) {
    const int full = pg::full_pieces(q[r], chunk), n = pg::pieces_of(q[r], chunk, full);
    CHECK(int64_t{full} * chunk <= q[r].tiles && (n == full || n == full + 1) && (n > full || int64_t{full} * chunk == q[r].tiles));
    row_tiles += q[r].row_tiles;
    items += int64_t{q[r].row_tiles} * n;
    if (n > 1) {
      slots += int64_t{q[r].row_tiles} * n;
      groups += q[r].row_tiles;
    }
    CHECK(n >= 1 && int64_t{n} * chunk >= q[r].tiles && (n == 1 || int64_t{n - 1} * chunk < q[r].tiles));
  }
  if (4 * row_tiles <= target) CHECK(items <= target);
  CHECK(row_tiles <= pg::max_row_tiles(R, tokens, group, row_tile));
  const int64_t bound = pg::max_row_tiles(R, tokens, group, row_tile);
  CHECK(items <= pg::max_items(bound, target, capacity, key_waves));
  if (pg::max_pieces(capacity, key_waves) == 1) CHECK(groups == 0);
  CHECK(slots <= pg::max_slots(target > 0 ? target : 0));
  CHECK(groups <= (target > 0 ? pg::max_groups(row_tiles, target) : 0));
}

int main() {
  const int groups[] = {1, 2, 3, 5, 8, 16, 40}, rows[] = {16, 32, 64}, windows[] = {0, 1, 17, 4096}, targets[] = {0, 1, 7, 64, 128, 1024};
  int n = 0;
  for (int R : {1, 2, 5, 63, 64, 65, 300})
    for (int longest : {0, 1, 31, 33, 2000, 200000})
      for (int group : groups)
        for (int row_tile : rows)
          for (int window : windows)
            for (int target : targets) {
              one(R, longest, 1, group, row_tile, window, target, INT32_MAX - 64, 4);
              one(R, longest, 9, group, row_tile, window, target, n % 3 ? INT32_MAX - 64 : longest / 2 + 8, 1 << n % 3);
              one(R, longest, 2, group, row_tile, window, target, (longest + 9) / 8 * 8, 2);
              ++n;
            }
  // out of range: clamped
  const pg::Request q = pg::request_of(-5, 9, -3, 4, 2, 16, 0, 100);
  if (q.row0 != 0 || q.n != 4 || q.len != 0 || q.tiles != 0 || q.row_tiles != 1) return printf("clamp\n"), 1;
  const pg::Request e = pg::request_of(7, 3, 50, 4, 2, 16, 0, 100);
  if (e.row0 != 4 || e.n != 0 || e.row_tiles != 0) return printf("clamp end\n"), 1;
  const pg::Request f = pg::request_of(0, 1, INT32_MAX, 1, 1, 16, 0, INT32_MAX - 64);
  if (f.tiles != (INT32_MAX - 64 + 31) / 32) return printf("longest\n"), 1;
  printf("ok\n");
  return 0;
}
