// New rows' keys and values into the pages of a cache, and back.
//
//   write, 8 bits:  s = max|x| / 127,  c = round(x / s);   read:  x = c s
//
// A key or a value of a row, up to 128 elements, belongs to 8 or 16 lanes of 8 elements each, so that the largest
// |x| takes three or four lane exchanges and no LDS.
#include "pages.h"

namespace edge {
namespace {

struct RowsParams {
  Pages c;
  int rows;
  char *k, *v;
  int64_t k_stride, k_head, v_stride, v_head;
};

constexpr int CACHE_THREADS = 256;

// Where a row's key stands; all L lanes of a group bring the same row.  page: -1 where it stands nowhere, -2 where
// the row belongs to no sequence.
struct Place {
  int page, slot;
};

template <int L>
__device__ inline Place place_of(const RowsParams &p, int row) {
  const int n = p.c.sequences, lane = threadIdx.x % WAVE, in = lane % L;
  // The last sequence that starts at or before the row: every step the group's lanes look at L starts.  The steps'
  // sizes depend on the number of sequences alone, so that all groups of the wave take them together.
  int u = 0;
  for (int size = n; size > 1;) {
    size = (size + L - 1) / L;
    const int at = u + in * size;
    const unsigned long long before = __ballot(at < n && p.c.row_start[at < n ? at : 0] <= row);
    const int hits = __builtin_popcountll(before >> (lane / L * L) & ((1ull << L) - 1));
    u += (hits > 0 ? hits - 1 : 0) * size;
  }
  int64_t begin = p.c.row_start[u], end = p.c.row_start[u + 1], keys = p.c.key_count[u];
  end = end < p.rows ? end : p.rows;
  if (row < begin || row >= end) return {-2, 0};
  const int64_t key = (keys > 0 ? keys : 0) - end + row;
  Place at = {-1, 0};
  if (key >= 0) at.page = page_of(p.c, u, (int)key, &at.slot);
  return at;
}

// A workgroup takes 256 / L rows of one head.
template <typename T, bool BITS8, int L>
__global__ __launch_bounds__(CACHE_THREADS) void write_kernel(RowsParams p) {
  constexpr int ROWS = CACHE_THREADS / L;
  const int head = block_index() % p.c.kv_heads, e = threadIdx.x % L * 8;
  const int64_t row = (int64_t)(block_index() / p.c.kv_heads) * ROWS + threadIdx.x / L;
  if (block_index() / p.c.kv_heads * (int64_t)ROWS >= p.rows) return;
  const bool in = row < p.rows && e < p.c.dim;
  typedef typename Raw<T, 8>::type Vec;
  Vec k = {}, v = {};
  if (in) {
    k = *(const Vec *)((const T *)p.k + row * p.k_stride + head * p.k_head + e);
    v = *(const Vec *)((const T *)p.v + row * p.v_stride + head * p.v_head + e);
  }
  const Place at = place_of<L>(p, row < p.rows ? (int)row : 0);
  const bool stands = in && at.page >= 0;
  auto put = [&](const Vec &x, const Pool &to) {
    const int64_t spot = at.page * to.page + head * to.head + at.slot * to.slot + e;
    if constexpr (!BITS8) {
      if (stands) *(Vec *)((T *)to.at + spot) = x;
    } else {
      // the largest |x| by its bit pattern, which orders like the value and puts NaN above all else
      float f[8];
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = (float)x[i];
        const unsigned a = __float_as_uint(f[i]) & 0x7fffffffu;
        m = a > m ? a : m;
      }
#pragma unroll
      for (int d = L / 2; d > 0; d >>= 1) {
        const unsigned a = __shfl_xor(m, d);
        m = a > m ? a : m;
      }
      const bool finite = m < 0x7f800000u;
      const float scale = __uint_as_float(m) / 127.0f;
      Raw<int8_t, 8>::type c;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = fminf(fmaxf(rintf(f[i] / scale), -127.0f), 127.0f);
        c[i] = finite && scale > 0.0f ? (int8_t)(int)y : (int8_t)0;
      }
      if (stands) {
        *(Raw<int8_t, 8>::type *)((int8_t *)to.at + spot) = c;
        if (e == 0)
          to.scale[at.page * to.scale_page + head * to.scale_head + at.slot * to.scale_slot] =
              finite ? scale : __uint_as_float(0x7fc00000u);
      }
    }
  };
  put(k, p.c.k);
  put(v, p.c.v);
}

template <typename T, bool BITS8, int L>
__global__ __launch_bounds__(CACHE_THREADS) void read_kernel(RowsParams p) {
  constexpr int ROWS = CACHE_THREADS / L;
  const int head = block_index() % p.c.kv_heads, e = threadIdx.x % L * 8;
  const int64_t row = (int64_t)(block_index() / p.c.kv_heads) * ROWS + threadIdx.x / L;
  if (block_index() / p.c.kv_heads * (int64_t)ROWS >= p.rows) return;
  const Place at = place_of<L>(p, row < p.rows ? (int)row : 0);
  if (row >= p.rows || e >= p.c.dim || at.page == -2) return;
  typedef typename Raw<T, 8>::type Vec;
  auto get = [&](const Pool &from, T *to) {
    const int64_t spot = at.page * from.page + head * from.head + at.slot * from.slot + e;
    Vec x = {};
    if constexpr (!BITS8) {
      if (at.page >= 0) x = *(const Vec *)((const T *)from.at + spot);
    } else if (at.page >= 0) {
      const Raw<int8_t, 8>::type c = *(const Raw<int8_t, 8>::type *)((const int8_t *)from.at + spot);
      const float scale = from.scale[at.page * from.scale_page + head * from.scale_head + at.slot * from.scale_slot];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (T)((float)c[i] * scale);
    }
    *(Vec *)to = x;
  };
  get(p.c.k, (T *)p.k + row * p.k_stride + head * p.k_head + e);
  get(p.c.v, (T *)p.v + row * p.v_stride + head * p.v_head + e);
}

template <typename T, bool BITS8, int L>
int rows_launch(const RowsParams &p, bool write, hipStream_t stream) {
  constexpr int ROWS = CACHE_THREADS / L;
  const int64_t blocks = ((int64_t)p.rows + ROWS - 1) / ROWS * p.c.kv_heads;
  if (blocks > MAX_BLOCKS) return JDOB_ERR_UNSUPPORTED;
  return launch(write ? write_kernel<T, BITS8, L> : read_kernel<T, BITS8, L>, blocks, CACHE_THREADS, stream, p);
}

template <typename T>
int rows_dispatch(const RowsParams &p, bool bits8, bool write, hipStream_t stream) {
  if (p.c.dim <= 64)
    return bits8 ? rows_launch<T, true, 8>(p, write, stream) : rows_launch<T, false, 8>(p, write, stream);
  return bits8 ? rows_launch<T, true, 16>(p, write, stream) : rows_launch<T, false, 16>(p, write, stream);
}

int cache_rows(const jdob_edge_cache_rows_args *a, bool write, void *hip_stream) {
  if (!a) return JDOB_ERR_INVALID_ARG;
  const int sizes = cache_check_sizes(a->cache, a->num_sequences, a->table_width);
  if (sizes != JDOB_OK) return sizes;
  if (a->rows < 0) return JDOB_ERR_INVALID_ARG;
  if (a->rows > JDOB_EDGE_MAX_ROWS) return JDOB_ERR_UNSUPPORTED;
  if (a->rows == 0 || a->num_sequences == 0) return JDOB_OK;
  const int code = cache_check_arrays(a->cache, a->table_width, a->table, a->table_stride, a->row_start, a->key_count);
  if (code != JDOB_OK) return code;
  if (!a->k || !a->v) return JDOB_ERR_INVALID_ARG;
  const int64_t d = a->cache.head_dim, g = a->cache.num_kv_heads;
  if (a->k_stride < 0 || a->k_head_stride < 0 || a->v_stride < 0 || a->v_head_stride < 0) return JDOB_ERR_INVALID_ARG;
  // rows and heads that are written at once must not share elements
  if (!write && ((a->rows > 1 && (a->k_stride < d || a->v_stride < d)) ||
                 (g > 1 && (a->k_head_stride < d || a->v_head_stride < d))))
    return JDOB_ERR_INVALID_ARG;
  const RowsParams p = {pages_of(a->cache, a->num_sequences, a->table_width, a->table, a->table_stride, a->row_start,
                                 a->key_count),
                        a->rows, (char *)a->k, (char *)a->v, a->k_stride, a->k_head_stride, a->v_stride, a->v_head_stride};
  hipStream_t stream = (hipStream_t)hip_stream;
  return a->cache.dtype == JDOB_EDGE_BF16 ? rows_dispatch<__bf16>(p, a->cache.bits8, write, stream)
                                          : rows_dispatch<_Float16>(p, a->cache.bits8, write, stream);
}

}  // namespace
}  // namespace edge

extern "C" int jdob_edge_cache_write(const jdob_edge_cache_rows_args *a, void *hip_stream) {
  return edge::cache_rows(a, true, hip_stream);
}

extern "C" int jdob_edge_cache_read(const jdob_edge_cache_rows_args *a, void *hip_stream) {
  return edge::cache_rows(a, false, hip_stream);
}
