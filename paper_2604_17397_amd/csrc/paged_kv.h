// What the paged cache's entry points share: types of its elements on the device, checks of its descriptor.
#pragma once
#include "sdvg_common.h"

namespace sdvg {

// The checks every entry point makes of a paged cache (paged_rows.hip).
int check_paged_kv(const sdvg_paged_kv *c);

// Bytes from the first to one past the last element of either pool of a checked cache.
int64_t paged_pool_bytes(const sdvg_paged_kv &c);

inline int element_bytes(int dtype) { return dtype == SDVG_F32 ? 4 : dtype == SDVG_E4M3 ? 1 : 2; }

inline bool disjoint(const void *x, int64_t x_bytes, const void *y, int64_t y_bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
  return a >= b + static_cast<uintptr_t>(y_bytes) || b >= a + static_cast<uintptr_t>(x_bytes);
}

// One stride in elements of `size` bytes over rows of 128, below `most`: status of its check. Strides of dimensions of one
// entry are free.
inline int check_stride(int64_t n, int64_t stride, int size, int64_t most = int64_t{1} << 30) {
  if (n <= 1) return SDVG_OK;
  if (stride < 128) return SDVG_ERR_SHAPE;
  if ((stride * size) & 15) return SDVG_ERR_ALIGN;
  return stride >= most ? SDVG_ERR_UNSUPPORTED : SDVG_OK;
}

// Elements from the first to one past the last of [n0][n1][128].
inline int64_t rows_span(int64_t n0, int64_t s0, int64_t n1, int64_t s1) {
  return (n0 > 1 ? (n0 - 1) * s0 : 0) + (n1 > 1 ? (n1 - 1) * s1 : 0) + 128;
}

}  // namespace sdvg
