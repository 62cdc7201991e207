// New rows' keys and values into the pages of a cache, and back.
//
//   write, 8 bits:  s = max|x| / 127,  c = round(x / s);   read:  x = c s
//
// A key or a value of a row, up to 128 elements, belongs to 8 or 16 lanes of 8 elements each, so that the largest
// |x| takes three or four lane exchanges and no barrier; a workgroup takes neighbouring rows of one head, which stand
// side by side on a page.
//
// Bound: HBM.  131,072 8-bit rows of 8 heads of 128 read back in 162 us (805 MB, 5.0 TB/s; a large copy moves 4.9; with
// one block of rows a workgroup 198); 16,192 rows written in 8 bits in 26 us (101 MB, 3.9 TB/s; lane exchanges without
// LDS change nothing there) and read back in 19; 32 rows written in 3.5 us, a launch.
#include <type_traits>

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

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef int8_t Codes __attribute__((ext_vector_type(8)));

// Where a row's key stands.  page: -1 where it stands nowhere, -2 where the row belongs to no sequence.
struct Place {
  int page, slot;
};

// Looks up rows that a group of L lanes brings alike.  Rows in ascending order share a look at row_start as long as they
// belong to one sequence.
template <int L>
struct Places {
  const RowsParams &p;
  int u;
  int64_t begin, end, keys;

  __device__ Places(const RowsParams &p) : p(p), u(0), begin(0), end(-1), keys(0) {}

  __device__ void search(int row) {
    const int n = p.c.sequences, lane = threadIdx.x % WAVE, in = lane % L;
    // The last sequence that starts at or before the row: every step the group's lanes look at L starts.  The steps'
    // sizes depend on the number of sequences alone, so that all groups of the wave take them together.
    u = 0;
    for (int size = n; size > 1;) {
      size = (size + L - 1) / L;
      const int at = u + in * size;
      const unsigned long long before = __ballot(at < n && p.c.row_start[at < n ? at : 0] <= row);
      const int hits = __builtin_popcountll(before >> (lane / L * L) & ((1ull << L) - 1));
      u += (hits > 0 ? hits - 1 : 0) * size;
    }
    begin = p.c.row_start[u], end = p.c.row_start[u + 1], keys = p.c.key_count[u];
    end = end < p.rows ? end : p.rows;
    keys = keys > 0 ? keys : 0;
  }

  __device__ Place find(int row) {
    if (__any(row < begin || row >= end)) search(row);
    if (row < begin || row >= end) return {-2, 0};
    const int64_t key = keys - end + row;
    Place at = {-1, 0};
    if (key >= 0) at.page = page_of(p.c, u, (int)key, &at.slot);
    return at;
  }
};

// The codes of a row of which each of L lanes holds eight elements, and its scale.
template <typename T, int L>
__device__ inline u32x2 codes_of(const typename Raw<T, 8>::type &x, float *scale) {
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
  const bool finite = m < 0x7f800000u, some = finite && m > 0;
  const float s = __uint_as_float(m) / 127.0f, r = some ? 1.0f / s : 0.0f;
  *scale = finite ? s : __uint_as_float(0x7fc00000u);
  // x / s is x r, put right by what it leaves of x: the same code as by a division for all values of 16 bits (every
  // mantissa of x and of the largest value tried; below 1/256 of it x has code 0 either way) where what is left is a
  // binary32 number.  A division takes ten instructions for the three: 32 prompts took 38 us to write.
  u32x2 c = {0, 0};
  const bool small = sizeof(T) == 2 && !__is_same(T, _Float16) && m < 0x12800000u;  // 2^-90
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = f[i] * r;
    // adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves it in the low bits
    const float y = __builtin_fmaf(__builtin_fmaf(-q, s, f[i]), r, q) + 0x1.8p23f;
    c[i / 4] |= (__float_as_uint(y) & 0xffu) << (i % 4 * 8);
  }
  if (__any(small && some)) {
    u32x2 d = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      d[i / 4] |= ((unsigned)(int)fminf(fmaxf(rintf(f[i] / s), -127.0f), 127.0f) & 0xffu) << (i % 4 * 8);
    c[0] = small ? d[0] : c[0];
    c[1] = small ? d[1] : c[1];
  }
  c[0] = some ? c[0] : 0;
  c[1] = some ? c[1] : 0;
  return c;
}

// A workgroup takes 256 / L rows of one head.
template <typename T, bool BITS8, int L>
__global__ __launch_bounds__(CACHE_THREADS) void write_kernel(RowsParams p) {
  constexpr int ROWS = CACHE_THREADS / L;
  typedef typename Raw<T, 8>::type Vec;
  const int head = block_index() % p.c.kv_heads, e = threadIdx.x % L * 8;
  const int64_t first = (int64_t)(block_index() / p.c.kv_heads) * ROWS, row = first + threadIdx.x / L;
  if (first >= p.rows) return;
  const bool in = row < p.rows && e < p.c.dim;
  Vec x[2] = {};
  if (in) {
    x[0] = *(const Vec *)((const T *)p.k + row * p.k_stride + head * p.k_head + e);
    x[1] = *(const Vec *)((const T *)p.v + row * p.v_stride + head * p.v_head + e);
  }
  Places<L> places(p);
  const Place at = places.find(row < p.rows ? (int)row : p.rows - 1);
  const bool stands = in && at.page >= 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Pool &to = i ? p.c.v : p.c.k;
    const int64_t spot = at.page * to.page + head * to.head + at.slot * to.slot + e;
    if constexpr (!BITS8) {
      if (stands) *(Vec *)((T *)to.at + spot) = x[i];
    } else {
      float scale;
      const u32x2 c = codes_of<T, L>(x[i], &scale);
      if (stands) {
        *(Raw<int8_t, 8>::type *)((int8_t *)to.at + spot) = __builtin_bit_cast(Codes, c);
        if (e == 0) to.scale[at.page * to.scale_page + head * to.scale_head + at.slot * to.scale_slot] = scale;
      }
    }
  }
}

// A workgroup takes B times 256 / L rows of one head.
template <typename T, bool BITS8, int L, int B>
__global__ __launch_bounds__(CACHE_THREADS) void read_kernel(RowsParams p) {
  constexpr int ROWS = CACHE_THREADS / L;
  typedef typename Raw<T, 8>::type Vec;
  const int head = block_index() % p.c.kv_heads, e = threadIdx.x % L * 8;
  const int64_t row0 = (int64_t)(block_index() / p.c.kv_heads) * (B * ROWS) + threadIdx.x / L;
  if (block_index() / p.c.kv_heads * (int64_t)(B * ROWS) >= p.rows) return;
  Places<L> places(p);
  Place at[B];
#pragma unroll
  for (int b = 0; b < B; ++b) at[b] = places.find(row0 + b * ROWS < p.rows ? (int)(row0 + b * ROWS) : p.rows - 1);
  typedef typename std::conditional<BITS8, Codes, Vec>::type In;
  In x[B][2];
  float scale[B][2];
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const Pool &from = i ? p.c.v : p.c.k;
      const int64_t spot = at[b].page * from.page + head * from.head + at[b].slot * from.slot + e;
      x[b][i] = In{};
      if (at[b].page < 0 || e >= p.c.dim) continue;
      if constexpr (BITS8) {
        x[b][i] = __builtin_bit_cast(Codes, *(const Raw<int8_t, 8>::type *)((const int8_t *)from.at + spot));
        scale[b][i] = from.scale[at[b].page * from.scale_page + head * from.scale_head + at[b].slot * from.scale_slot];
      } else {
        x[b][i] = *(const Vec *)((const T *)from.at + spot);
      }
    }
#pragma unroll
  for (int b = 0; b < B; ++b) {
    const int64_t row = row0 + b * ROWS;
    if (row >= p.rows || e >= p.c.dim || at[b].page == -2) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      T *const to = i ? (T *)p.v + row * p.v_stride + head * p.v_head : (T *)p.k + row * p.k_stride + head * p.k_head;
      Vec y;
      if constexpr (BITS8) {
        const float s = at[b].page < 0 ? 0.0f : scale[b][i];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = (T)((float)x[b][i][j] * s);
      } else {
        y = x[b][i];
      }
      *(Vec *)(to + e) = y;
    }
  }
}

template <typename T, bool BITS8, int L>
int rows_launch(const RowsParams &p, bool write, hipStream_t stream) {
  constexpr int ROWS = CACHE_THREADS / L, B = 4;
  auto blocks = [&](int b) { return ((int64_t)p.rows + b * ROWS - 1) / (b * ROWS) * p.c.kv_heads; };
  // More rows a workgroup keep more loads of a read under way, but leave few workgroups for few rows (131,072 rows as above).
  // A write has no use for them: 131,072 8-bit rows of one sequence took 190 us for 178, of 256 sequences 190 for 201.
  const bool more = !write && blocks(B) >= 2048;
  const int64_t n = blocks(more ? B : 1);
  if (n > MAX_BLOCKS) return JDOB_ERR_UNSUPPORTED;
  return launch(write  ? write_kernel<T, BITS8, L>
                : more ? read_kernel<T, BITS8, L, B>
                       : read_kernel<T, BITS8, L, 1>,
                n, CACHE_THREADS, stream, p);
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
  if (!write && (pieces_overlap(a->rows, a->k_stride, g, a->k_head_stride, d) ||
                 pieces_overlap(a->rows, a->v_stride, g, a->v_head_stride, d)))
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
