// Plan of one step over the paged cache: block tables, slots, positions and row ranges of all requests from their
// lengths, in one launch without a meeting between workgroups.
//
// All outputs follow from two prefix sums over the requests (new tokens, pages taken). Every workgroup
// has a few consecutive requests and sums what lies before them itself: reading 3 x 4 bytes of every earlier request from
// L2 is cheaper than a second launch or a hand-over in memory up to some thousand requests. A chain of latencies (lengths, sums, page,
// store): 2.9 us for one request, 4.1 for 200 with up to 8 tokens each, 4.5 for 48 prompts (112000 tokens, 1.4 MB written).
#include "row_map.h"
#include "sdvg_common.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxGroups = 1024;   // workgroups along the requests; each takes n_requests / kMaxGroups, rounded up
constexpr int kSegmentTokens = kThreads;  // new tokens of a request per workgroup, by the average (prompts of up to 4680 tokens 4.5 us; 4 times as many 5.1)
constexpr int kMaxSegments = 64;

struct PlanParams {
  sdvg_page_plan_args a;
  sdvg::FastDiv page;     // by page_tokens
  int per_group;          // requests per workgroup
};

// What one request asks for.
struct Ask {
  int64_t cached, fresh;  // tokens
  int64_t need, take;     // pages: of the whole request, and of those the ones to come from the free list
  int64_t held;
};
__device__ __forceinline__ Ask ask_of(const PlanParams &p, int r) {
  Ask q;
  const int c = p.a.cached[r], n = p.a.new_tokens[r];
  q.cached = c > 0 ? c : 0;
  q.fresh = n > 0 ? n : 0;
  int64_t len = q.cached + q.fresh;
  len = len < INT32_MAX ? len : INT32_MAX;
  q.need = (len + p.a.page_tokens - 1) / p.a.page_tokens;
  if (q.need > p.a.table_width) q.need = p.a.table_width;
  if (p.a.held) {
    q.held = p.a.held[r] > 0 ? p.a.held[r] : 0;
    q.take = q.need > q.held ? q.need - q.held : 0;
  } else {
    q.held = q.need;
    q.take = 0;
  }
  return q;
}

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

__global__ __launch_bounds__(kThreads) void page_plan_kernel(PlanParams p) {
  __shared__ int64_t part[2][kThreads / 64];
  const sdvg_page_plan_args &a = p.a;
  const int first = blockIdx.x * p.per_group, seg = blockIdx.y, n_seg = gridDim.y;
  const bool writer = seg == 0;  // of everything but the tokens

  // tokens and pages asked for by the requests before this workgroup's
  int64_t tokens = 0, pages = 0;
  for (int r = threadIdx.x; r < first; r += kThreads) {
    const Ask q = ask_of(p, r);
    tokens += q.fresh;
    pages += q.take;
  }
  tokens = wave_sum(tokens);
  pages = wave_sum(pages);
  if ((threadIdx.x & 63) == 0) {
    part[0][threadIdx.x >> 6] = tokens;
    part[1][threadIdx.x >> 6] = pages;
  }
  __syncthreads();
  tokens = pages = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    tokens += part[0][w];
    pages += part[1][w];
  }
  tokens = tokens < a.max_tokens ? tokens : a.max_tokens;  // those that have rows

  const int64_t next = a.held && a.next_free && *a.next_free > 0 ? *a.next_free : 0;
  if (writer && first == 0 && threadIdx.x == 0) a.q_start[0] = 0;
  const int last = first + p.per_group < a.n_requests ? first + p.per_group : a.n_requests;
  for (int r = first; r < last; ++r) {
    Ask q = ask_of(p, r);
    if (q.fresh > a.max_tokens - tokens) q.fresh = a.max_tokens - tokens;
    const int64_t base = next + pages;   // place in the free list of this request's first page
    int32_t *row = a.block_table + r * a.table_stride;
    // a page of this request, wherever it comes from: -1 if there is none
    const auto page_at = [&](int64_t j) -> int32_t {
      if (j < q.held) return j < a.table_width ? row[j] : -1;
      const int64_t at = base + (j - q.held);
      return j < q.need && at < a.n_free ? a.free_pages[at] : -1;
    };
    if (writer) {
      for (int64_t j = q.held + threadIdx.x; j < q.need; j += kThreads) row[j] = page_at(j);
      if (threadIdx.x == 0) {
        a.q_start[r + 1] = static_cast<int32_t>(tokens + q.fresh);
        const int64_t len = q.cached + q.fresh;
        a.kv_lens[r] = static_cast<int32_t>(len < INT32_MAX ? len : INT32_MAX);
        if (a.held) {
          int64_t left = a.n_free - base;  // pages the list still has for this request
          left = left < 0 ? 0 : left < q.take ? left : q.take;
          a.held_out[r] = static_cast<int32_t>(q.held + left);
        }
      }
    }
    for (int64_t i = seg * kThreads + threadIdx.x; i < q.fresh; i += n_seg * kThreads) {
      const int64_t at = q.cached + i;
      const bool fits = at < INT32_MAX;
      const uint32_t pos = static_cast<uint32_t>(fits ? at : 0), j = p.page.div(pos);
      const int32_t page = fits && j < static_cast<uint32_t>(a.table_width) ? page_at(j) : -1;
      a.positions[tokens + i] = static_cast<int32_t>(pos);
      a.slots[tokens + i] = page < 0 ? -1 : static_cast<int64_t>(page) * a.page_tokens + (pos - j * p.page.d);
    }
    tokens += q.fresh;
    pages += q.take;
  }
  if (last < a.n_requests) return;
  // the last workgroups also know the totals
  if (writer && threadIdx.x == 0 && a.held) {
    const int64_t total = next + pages;
    *a.next_free_out = static_cast<int32_t>(total < INT32_MAX ? total : INT32_MAX);
  }
  for (int64_t t = tokens + seg * kThreads + threadIdx.x; t < a.max_tokens; t += n_seg * kThreads) {
    a.positions[t] = 0;
    a.slots[t] = -1;
  }
}

struct Range {
  const void *p;
  int64_t bytes;
};
bool overlap(const Range &x, const Range &y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
  return x.p && y.p && x.bytes > 0 && y.bytes > 0 && a < b + y.bytes && b < a + x.bytes;
}
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

extern "C" int sdvg_page_plan(const sdvg_page_plan_args *args, void *stream) {
  if (!args) return SDVG_ERR_NULL;
  sdvg_page_plan_args a = *args;
  const int64_t R = a.n_requests, M = a.max_tokens;
  if (R < 0 || M < 0 || a.page_tokens < 1 || a.table_width < 1 || a.n_free < 0) return SDVG_ERR_SHAPE;
  if (M > INT32_MAX) return SDVG_ERR_UNSUPPORTED;
  if (a.page_tokens & 7) return SDVG_ERR_ALIGN;
  if (a.table_stride < a.table_width) return SDVG_ERR_SHAPE;
  if (!a.q_start || (R > 0 && (!a.cached || !a.new_tokens || !a.block_table || !a.kv_lens))) return SDVG_ERR_NULL;
  if (M > 0 && (!a.positions || !a.slots)) return SDVG_ERR_NULL;
  if (a.held) {
    if ((R > 0 && !a.held_out) || !a.next_free_out || (a.n_free > 0 && !a.free_pages)) return SDVG_ERR_NULL;
  } else {
    a.free_pages = a.next_free = nullptr;
    a.held_out = a.next_free_out = nullptr;
    a.n_free = 0;
  }
  for (const void *p : {static_cast<const void *>(a.cached), static_cast<const void *>(a.new_tokens),
                        static_cast<const void *>(a.free_pages), static_cast<const void *>(a.held),
                        static_cast<const void *>(a.next_free), static_cast<const void *>(a.block_table),
                        static_cast<const void *>(a.q_start), static_cast<const void *>(a.kv_lens),
                        static_cast<const void *>(a.positions), static_cast<const void *>(a.held_out),
                        static_cast<const void *>(a.next_free_out)})
    if (!aligned(p, 4)) return SDVG_ERR_ALIGN;
  if (!aligned(a.slots, 8)) return SDVG_ERR_ALIGN;
  const int64_t table = R > 0 ? ((R - 1) * a.table_stride + a.table_width) * 4 : 0;
  const Range in[] = {{a.cached, R * 4}, {a.new_tokens, R * 4}, {a.free_pages, int64_t{a.n_free} * 4}, {a.held, R * 4},
                      {a.next_free, 4}};
  const Range out[] = {{a.block_table, table}, {a.q_start, (R + 1) * 4}, {a.kv_lens, R * 4},  {a.positions, M * 4},
                       {a.held_out, R * 4},    {a.next_free_out, 4},     {a.slots, M * 8}};
  for (const Range &x : out) {
    for (const Range &y : in)
      if (overlap(x, y)) return SDVG_ERR_RANGE;
    for (const Range &y : out)
      if (&x != &y && overlap(x, y)) return SDVG_ERR_RANGE;
  }
  PlanParams p{a, sdvg::FastDiv::of(a.page_tokens), 1};
  p.per_group = R > kMaxGroups ? static_cast<int>((R + kMaxGroups - 1) / kMaxGroups) : 1;
  const int64_t groups = R > 0 ? (R + p.per_group - 1) / p.per_group : 1;
  // as if the new tokens were spread evenly over the workgroups; a request with many more only takes more turns
  int64_t segments = (M + groups * kSegmentTokens - 1) / (groups * kSegmentTokens);
  segments = segments < 1 ? 1 : segments > kMaxSegments ? kMaxSegments : segments;
  hipLaunchKernelGGL(page_plan_kernel, dim3(static_cast<uint32_t>(groups), static_cast<uint32_t>(segments)), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), p);
  SDVG_HIP_CHECK(hipGetLastError());
  return SDVG_OK;
}
