// Paged K/V caches (focus_paged_kv): the host's checks and the row addresses shared
// by the kernels that fill, read and cut them.
#pragma once

#include "common.h"

namespace focus {

inline bool pieces16(int64_t elements, int64_t elt) { return elements * elt % 16 == 0; }

// Whether rows of `row` elements at counts x strides from one another do not overlap:
// each stride at least what the smaller ones span (dimensions of one element aside).
template <int N>
inline bool disjoint_rows(int64_t row, const int64_t (&strides)[N], const int64_t (&counts)[N]) {
  int64_t span = row;
  bool used[N] = {};
  for (int k = 0; k < N; ++k) {
    int at = -1;
    for (int i = 0; i < N; ++i)
      if (!used[i] && (at < 0 || strides[i] < strides[at])) at = i;
    used[at] = true;
    if (counts[at] <= 1) continue;
    if (strides[at] < span) return false;
    if (strides[at] > (int64_t{1} << 62) / counts[at]) return false;
    span = strides[at] * counts[at];
  }
  return true;
}

// Checks of a cache's description; E_OK for batch 0 whatever the pointers.
inline focus_status check_paged(const focus_paged_kv& c) {
  const int64_t es = elt_bytes(c.dtype);
  if (es == 0) return FOCUS_E_DTYPE;
  if (c.n_kv_heads <= 0 || c.head_dim <= 0 || c.n_pages < 0 || c.batch < 0 || c.max_pages < 0) return FOCUS_E_ARG;
  if (c.head_dim > 256 || !pieces16(c.head_dim, es)) return FOCUS_E_UNSUPPORTED;
  if (c.page_rows < 8 || c.page_rows > 1024 || (c.page_rows & (c.page_rows - 1))) return FOCUS_E_UNSUPPORTED;
  if ((int64_t)c.max_pages * c.page_rows > INT32_MAX / 2 || c.n_pages > INT32_MAX) return FOCUS_E_SHAPE;
  if (c.page_stride < c.head_dim || c.row_stride < c.head_dim || c.head_stride < c.head_dim ||
      !pieces16(c.page_stride, es) || !pieces16(c.row_stride, es) || !pieces16(c.head_stride, es) ||
      !disjoint_rows<3>(c.head_dim, {c.page_stride, c.row_stride, c.head_stride}, {c.n_pages, c.page_rows, c.n_kv_heads}))
    return FOCUS_E_ARG;
  if (c.row_stride > INT32_MAX) return FOCUS_E_SHAPE;
  if (c.weight && c.weight_rows < (int64_t)c.max_pages * c.page_rows) return FOCUS_E_SHAPE;
  if (c.batch == 0) return FOCUS_OK;
  if (!c.length || (c.max_pages > 0 && !c.table) || (c.n_pages > 0 && (!c.k || !c.v))) return FOCUS_E_NULL;
  if (!aligned16(c.k) || !aligned16(c.v) || (reinterpret_cast<uintptr_t>(c.table) & 3u) ||
      (reinterpret_cast<uintptr_t>(c.length) & 3u) || (reinterpret_cast<uintptr_t>(c.weight) & 3u))
    return FOCUS_E_ARG;
  return FOCUS_OK;
}

// log2 of a checked page_rows.
inline int page_shift(const focus_paged_kv& c) { return __builtin_ctz((unsigned)c.page_rows); }

// Rows of sequence b, clipped to what its table holds.
__device__ inline int paged_length(const focus_paged_kv& c, int b) {
  const int64_t cap = (int64_t)c.max_pages * c.page_rows, n = c.length[b];
  return (int)(n < 0 ? 0 : n > cap ? cap : n);
}

// Page of row r (inside the table) of sequence b; -1 for one outside the pool.
__device__ inline int64_t page_of(const focus_paged_kv& c, int b, int r, int shift) {
  const int64_t p = c.table[(int64_t)b * c.max_pages + (r >> shift)];
  return p >= 0 && p < c.n_pages ? p : -1;
}

// First element of head g of a row in page p.
__device__ inline int64_t row_at(const focus_paged_kv& c, int64_t p, int r, int g) {
  return p * c.page_stride + (int64_t)(r & (c.page_rows - 1)) * c.row_stride + (int64_t)g * c.head_stride;
}

// Inclusive prefix over the wave of a sum or, for values from 0 up, a maximum (DPP: rows of
// 16 lanes, then their last lanes' values).
template <typename Op>
__device__ inline int wave_prefix(int x, Op op) {
#define FOCUS_STEP(ctrl, rows) x = op(x, __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, true))
  FOCUS_STEP(0x111, 0xf);
  FOCUS_STEP(0x112, 0xf);
  FOCUS_STEP(0x114, 0xf);
  FOCUS_STEP(0x118, 0xf);
  FOCUS_STEP(0x142, 0xa);
  FOCUS_STEP(0x143, 0xc);
#undef FOCUS_STEP
  return x;
}
__device__ inline int wave_scan(int x) {
  return wave_prefix(x, [](int a, int b) { return a + b; });
}
__device__ inline int wave_max(int x) {
  return __builtin_amdgcn_readlane(wave_prefix(x, [](int a, int b) { return max(a, b); }), 63);
}

}  // namespace focus
