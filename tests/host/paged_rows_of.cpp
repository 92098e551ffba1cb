// What a request's numbers in q_start and kv_lens name, from the header the kernels use, against the same in 64 bits: every token has
// clamped neighbours, and the keys that it sees are those that both kernels of an attention take.
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include "paged_prefix_plan.h"

namespace pg = sdvg::paged;

int main() {
  const int32_t odd[] = {INT32_MIN, INT32_MIN + 1, -900, -3, -1, 0, 1, 2, 3, 63, 64, 700, 900, INT32_MAX - 1, INT32_MAX};
  long n = 0;
  for (int32_t tokens : {1, 2, 64, 700, INT32_MAX - 64})
    for (int32_t start : odd)
      for (int32_t end : odd)
        for (int32_t len : odd) {
          const pg::Rows a = pg::rows_of(start, end, len, tokens);
          const int64_t row0 = std::min<int64_t>(std::max<int64_t>(start, 0), tokens), last = std::min<int64_t>(std::max<int64_t>(end, row0), tokens);
          if (a.row0 != row0 || a.n != last - row0 || a.len != std::max<int64_t>(len, 0)) return printf("rows of %d, %d, %d, %d\n", start, end, len, tokens), 1;
          for (int64_t i : {int64_t{0}, int64_t{1}, int64_t{a.n} / 2, int64_t{a.n} - 2, int64_t{a.n} - 1}) {
            if (i < 0 || i >= a.n) continue;
            if (pg::sees_of(a, static_cast<int32_t>(i)) != int64_t{a.len} - a.n + i + 1) return printf("keys of %d, %d, %d, %d\n", start, end, len, tokens), 1;
            ++n;
          }
          // the same rows and keys for the request's own keys, and the same rows for its group of one
          for (int32_t prefix : {0, 64, 700}) {
            const pg::Request q = pg::request_of(start, end, len, tokens, 1, 16, 0, 1 << 20, prefix);
            const pg::SharedKeys s = pg::shared_of(0, 1, start, end, prefix, tokens, 1, 0, 1 << 20);
            if (q.row0 != a.row0 || q.n != a.n || q.len != a.len || s.token0 != a.row0 || s.tokens != a.n) return printf("request of %d, %d, %d, %d\n", start, end, len, tokens), 1;
          }
        }
  if (n < 1000) return 1;
  printf("ok\n");
  return 0;
}
