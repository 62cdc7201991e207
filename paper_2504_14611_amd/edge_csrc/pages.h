// Shared by the kernels that work on a paged cache: where a key stands, and the checks of the cache's description.
#pragma once

#include "edge_common.h"

namespace edge {

// x / by for 0 <= x < 2^31 and 1 <= by <= 2^30: with 2^(l-1) < by <= 2^l and mul = ceil(2^(31+l) / by) the error
// mul * by - 2^(31+l) is below 2^l, so that x * mul / 2^(31+l) is never a
// whole number too large; mul is below 2^32, being at most 2^32 - 2^(33-l) + 1 or, of a power of two, 2^31.
struct Divide {
  unsigned mul, shift;
};
inline Divide divide_by(int by) {
  int l = 0;
  while ((1 << l) < by) ++l;
  return {(unsigned)(((1ull << (31 + l)) + by - 1) / by), (unsigned)(31 + l)};
}
__device__ inline int divide(int x, Divide d) { return (int)((uint64_t)(unsigned)x * d.mul >> d.shift); }

struct Pool {  // keys or values: strides in elements
  char *at;
  int64_t page, head, slot;
  float *scale;
  int64_t scale_page, scale_head, scale_slot;
};

struct Pages {
  int pages, page_size, kv_heads, dim;
  Divide by_page;
  Pool k, v;
  int sequences, width;
  const int *table;
  int64_t table_stride;
  const int *row_start, *key_count;
};

// The page of key j >= 0 of sequence u, or -1 where the key is absent.
__device__ inline int page_of(const Pages &p, int u, int j, int *slot) {
  const int i = divide(j, p.by_page);
  *slot = j - i * p.page_size;
  if (i >= p.width) return -1;
  const int page = p.table[u * p.table_stride + i];
  return (unsigned)page < (unsigned)p.pages ? page : -1;
}

inline Pages pages_of(const jdob_edge_cache &c, int sequences, int width, const int *table, int64_t table_stride,
                      const int *row_start, const int *key_count) {
  return {c.num_pages, c.page_size, c.num_kv_heads, c.head_dim, divide_by(c.page_size),
          {(char *)c.k, c.k_page_stride, c.k_head_stride, c.k_slot_stride, c.k_scale, c.k_scale_page_stride,
           c.k_scale_head_stride, c.k_scale_slot_stride},
          {(char *)c.v, c.v_page_stride, c.v_head_stride, c.v_slot_stride, c.v_scale, c.v_scale_page_stride,
           c.v_scale_head_stride, c.v_scale_slot_stride},
          sequences, width, table, table_stride, row_start, key_count};
}

// Sizes and types; nothing else of the description is read where no row or key is.
inline int cache_check_sizes(const jdob_edge_cache &c, int sequences, int width) {
  if (c.num_pages < 0 || c.page_size < 1 || c.num_kv_heads < 1 || c.head_dim < 1 || (c.bits8 != 0 && c.bits8 != 1) ||
      sequences < 0 || width < 0)
    return JDOB_ERR_INVALID_ARG;
  if (c.dtype != JDOB_EDGE_BF16 && c.dtype != JDOB_EDGE_F16) return JDOB_ERR_UNSUPPORTED;
  if (c.page_size > JDOB_EDGE_MAX_PAGE_SIZE || c.num_kv_heads > 1024 || c.head_dim > JDOB_EDGE_MAX_HEAD_DIM ||
      c.head_dim % 8 || sequences > JDOB_EDGE_MAX_SEQUENCES)
    return JDOB_ERR_UNSUPPORTED;
  return JDOB_OK;
}

// Whether slots, heads or pages with such strides share elements: each of the three that there is more than one of
// has to pass over what the smaller ones span.
inline bool slots_overlap(const jdob_edge_cache &c, int width, int64_t page, int64_t head, int64_t slot) {
  int64_t stride[3] = {page, head, slot}, count[3] = {c.num_pages, c.num_kv_heads, c.page_size};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] < stride[i]) {
        const int64_t s = stride[i], n = count[i];
        stride[i] = stride[j], count[i] = count[j];
        stride[j] = s, count[j] = n;
      }
  int64_t span = width;  // elements from the first to behind the last
  for (int i = 0; i < 3; ++i) {
    if (count[i] < 2) continue;
    if (stride[i] < span || stride[i] > INT64_MAX / 4 / count[i]) return true;
    span += stride[i] * (count[i] - 1);
  }
  return false;
}

// Arrays, strides and the table.  Keys that share elements could not be written apart and are refused for reading, too.
inline int cache_check_arrays(const jdob_edge_cache &c, int width, const int *table, int64_t table_stride,
                              const int *row_start, const int *key_count) {
  if (!row_start || !key_count || (width > 0 && !table) || table_stride < width) return JDOB_ERR_INVALID_ARG;
  if (c.num_pages == 0) return JDOB_OK;
  if (!c.k || !c.v || (c.bits8 && (!c.k_scale || !c.v_scale))) return JDOB_ERR_INVALID_ARG;
  if (slots_overlap(c, c.head_dim, c.k_page_stride, c.k_head_stride, c.k_slot_stride) ||
      slots_overlap(c, c.head_dim, c.v_page_stride, c.v_head_stride, c.v_slot_stride))
    return JDOB_ERR_INVALID_ARG;
  if (c.bits8 && (slots_overlap(c, 1, c.k_scale_page_stride, c.k_scale_head_stride, c.k_scale_slot_stride) ||
                  slots_overlap(c, 1, c.v_scale_page_stride, c.v_scale_head_stride, c.v_scale_slot_stride)))
    return JDOB_ERR_INVALID_ARG;
  return JDOB_OK;
}

}  // namespace edge
