// Causal attention of sequences' newest rows over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - max),  keys j that are there and j <= m - n + i
//
// With 8 bits k_j and v_j are codes times a scale of the key: scores are multiplied by the key's scale, p by the
// value's, and the codes go into the products as they are.
//
// The rows of all heads that read one key head stand together as columns, 16 or 32 for a workgroup; its waves take
// tiles of 32 keys in turn, and the tiles are dealt over workgroups, whose partial results a second kernel joins.  One
// pass over the keys: a running maximum and sum per column, the output rescaled when the maximum grows.
//
// Keys and values come straight into the registers that the matrix units read; LDS is only used to join the waves.
// The products are formed transposed, 16 x 16 at a time: S^T = K Q^T leaves a column in a lane (four times: lane
// group g = lane / 16 holds keys 4 g .. 4 g + 3 of every 16), O^T = V^T P^T takes the lane's own p as its second
// operand.  Which key or element stands at which place of the summed dimension is free as long as both operands
// agree: a lane's 8 elements of a key are any 8 that the query's lane has too, and V's operand, 8 keys of one
// element a lane, is cut out of 8 rows' pieces that the lane loads side by side.
//
// Bound: HBM, at 5 to 5.8 TB/s where there are keys enough (a large copy moves 4.9; what the last cache keeps from pass
// to pass helps).  Kernels alone: 32 rows of 32 heads after 15 to 8191 keys 89 us, one after 131,071 8-bit keys 48,
// 256 rows of 64 heads after 511 to 4095 8-bit keys 248; the join 5 to 6.  A tile of 32 8-bit keys of 128 takes 390
// vector and 110 scalar instructions a wave (half of them turn codes into bfloat16) and 24 products, 1.4 us where a wave
// has a SIMD to itself: few keys are bound by that and by the launch (one key 6.4 us, 512 keys 10.7).  Tiles of 64 keys
// took more registers and as long a key; eight waves a workgroup took 0.8 us off 512 keys and put 0.4 on one.
#include <type_traits>

#include "pages.h"

namespace edge {
namespace {

struct PagedParams {
  Pages c;
  int group, max_queries, tile_columns;  // group: heads of a key head
  float scale;  // times log2(e)
  int64_t query_rows;
  const char *q;
  char *out;
  int64_t q_stride, q_head, out_stride, out_head;  // elements
  int tiles;          // tiles of columns of a sequence
  int shares;         // of the keys, besides one for each sequence (0: keys are not split)
  Divide by_heads, by_tiles, by_group;  // of key heads, tiles and heads of a key head
  float *part;        // [share][tile][key head][columns of a tile][dim + 4]
};

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

template <typename T>
struct Mma16;
template <>
struct Mma16<__bf16> {
  typedef bf16x8 frag;
  __device__ static f32x4 m16(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma16<_Float16> {
  typedef f16x8 frag;
  __device__ static f32x4 m16(frag a, frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// A sequence's rows and keys, kept within the arrays whatever the index arrays hold.
struct Newest {
  int row, rows, keys;  // the first row, rows, the keys as counted
  int last;             // keys that the table has room for
};

__device__ inline Newest newest(const PagedParams &p, int u) {
  const int most = (int)p.query_rows;
  int at = p.c.row_start[u], end = p.c.row_start[u + 1];
  at = at < 0 ? 0 : at < most ? at : most;
  end = end < at ? at : end < most ? end : most;
  const int keys = p.c.key_count[u] > 0 ? p.c.key_count[u] : 0;
  const int64_t room = (int64_t)p.c.width * p.c.page_size;
  return {at, end - at, keys, (int)(keys < room ? keys : room)};
}

// Sequences of very different lengths: each has a share for every so many keys, as few as p.shares and one more for each
// sequence's end allow.  Every wave forms the shares' list from the lengths.
struct Share {
  Newest q;
  int u, index, count;  // the sequence, which of its shares, how many it has
  int first;            // the sequence's first share in the list
};
constexpr int SHARE_UNIT = 128, LEAST_KEYS = 256;

__device__ inline int units_of(const Newest &q) { return (q.last >> 7) + ((q.last & 127) != 0); }

// The share at place `at` of the list, or with `of_sequence` the first of sequence `at`; false where there is none.
__device__ inline bool share_of(const PagedParams &p, int at, bool of_sequence, Share *s) {
  const int lane = threadIdx.x % WAVE, n = p.c.sequences;
  double units = 0.0;  // (exact)
  for (int u = lane; u < n; u += WAVE) {
    const Newest q = newest(p, u);
    units += q.rows ? units_of(q) : 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) units += __shfl_xor(units, d);
  const int each = __builtin_amdgcn_readfirstlane((int)fmax(ceil(units / p.shares), (double)LEAST_KEYS / SHARE_UNIT));  // units, to 2^24
  int before = 0;
  for (int u0 = 0; u0 < n; u0 += WAVE) {
    Newest q = {0, 0, 0, 0};
    if (u0 + lane < n) q = newest(p, u0 + lane);
    const int mine = !q.rows ? 0 : q.last ? (units_of(q) + each - 1) / each : 1;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) {
      const int x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    const unsigned long long found = of_sequence ? at < u0 + WAVE ? 1ull << (at - u0) : 0 : __ballot(before + upto > at);
    if (found) {
      const int l = __builtin_ctzll(found);
      *s = {{__builtin_amdgcn_readlane(q.row, l), __builtin_amdgcn_readlane(q.rows, l), __builtin_amdgcn_readlane(q.keys, l),
             __builtin_amdgcn_readlane(q.last, l)},
            u0 + l, 0, __builtin_amdgcn_readlane(mine, l), before + __builtin_amdgcn_readlane(upto - mine, l)};
      s->index = of_sequence ? 0 : at - s->first;
      return s->count > 0;
    }
    before += __builtin_amdgcn_readlane(upto, WAVE - 1);
  }
  return false;
}

// Which elements of a key's or value's row a lane holds, for heads padded to DP.
// Keys: product j takes 8 elements of lane group g from key_element(j, g) on.
// Values: product i's row m is element value_element(i, m).
template <int DP, bool BITS8>
__device__ constexpr int key_element(int j, int g) {
  return !BITS8 || j * 32 + 32 > DP / 64 * 64 ? j * 32 + g * 8 : j / 2 * 64 + g * 16 + j % 2 * 8;
}
template <int DP>
__device__ constexpr int value_element(int i, int m) {
  return DP != 96 ? m * (DP / 16) + i : i < 4 ? m * 4 + i : 64 + m * 2 + i - 4;
}

// 32 keys and values as a lane holds them.
template <int DP, bool BITS8>
struct Tile {
  static constexpr int KW = DP / (BITS8 ? 16 : 8);                             // words of a key
  static constexpr int VW = BITS8 ? (DP == 128 ? 2 : DP == 96 ? 2 : 1) : DP / 32;  // words of a value
  unsigned k[2][KW], v[8][VW];
  f32x4 k_scale[2], v_scale[2];
};

// A stretch of memory from `at` on: what is read from behind its end is zero and does not touch memory.  Both are the
// same for all lanes of the wave.
__device__ inline __amdgpu_buffer_rsrc_t window(const void *at, int bytes) {
  const uint64_t a = (uint64_t)at;
  const uint64_t same = (uint64_t)__builtin_amdgcn_readfirstlane((unsigned)(a >> 32)) << 32 |
                        (unsigned)__builtin_amdgcn_readfirstlane((unsigned)a);
  return __builtin_amdgcn_make_buffer_rsrc((void *)same, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
template <int BYTES>
__device__ inline void window_load(unsigned *to, __amdgpu_buffer_rsrc_t w, unsigned offset) {
  if constexpr (BYTES == 16) {
    const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(w, offset, 0, 0));
    to[0] = x[0], to[1] = x[1], to[2] = x[2], to[3] = x[3];
  } else if constexpr (BYTES == 8) {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(w, offset, 0, 0));
    to[0] = x[0], to[1] = x[1];
  } else if constexpr (BYTES == 4) {
    *to = __builtin_amdgcn_raw_buffer_load_b32(w, offset, 0, 0);
  } else {
    *to = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(w, offset, 0, 0);
  }
}

constexpr int TILE_KEYS = 32;
constexpr int64_t NO_TILE = INT64_MAX / 2;  // behind any key
constexpr unsigned FLAT = 0x70000000u;      // bytes from a head's first row or scale on that Anywhere's windows cover

__device__ const u32x4 paged_zeros = {0, 0, 0, 0};

// A wave's keys of one head whatever the page's size and the arrays' alignment: every lane looks up its own keys' pages,
// RUN keys from a multiple of RUN on at once (pages of a multiple of RUN keys).  WINDOW: through one window over each of
// the arrays (FLAT: they are small enough), with offsets of 32 bits for addresses of 64 (32 users' tokens after up to 8191
// 8-bit keys on pages of 20: 89 us and 106; three after 91,511 on pages of 7, a key at once: 118 and 342).
template <typename T, int DP, bool BITS8, int RUN, bool WINDOW>
struct Anywhere {
  typedef typename std::conditional<BITS8, int8_t, unsigned short>::type E;
  const PagedParams &p;
  int u, head, until, l16, g;  // until: keys from there on are not read
  int64_t tile;                // to be looked up next
  int step;
  struct Spot {
    int page, slot;  // page: -1 where there is none
  };
  struct Spots {  // of a tile: the lane's key of each half, and its runs of values
    Spot key[2], run[2][4 / RUN];
  } next, after;

  __device__ Anywhere(const PagedParams &p, int u, int head, int until, int tile, int step)
      : p(p), u(u), head(head), until(until), l16(threadIdx.x % 16), g(threadIdx.x % WAVE / 16), tile(tile), step(step) {}

  __device__ Spot spot(int64_t j) const {
    const int i = divide(j < until ? (int)j : 0, p.c.by_page);  // (key 0 is there to be looked up if any is)
    const int page = p.c.table[u * p.c.table_stride + i];
    return {j < until && (unsigned)page < (unsigned)p.c.pages ? page : -1, (int)j - i * p.c.page_size};
  }

  // The tile that was looked up last is the next one to be loaded; looks up another and returns its first key.
  __device__ int64_t find() {
    next = after;
    const int64_t first = tile * TILE_KEYS;
    tile += step;
    if (first >= until) return NO_TILE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      after.key[h] = spot(first + h * 16 + l16);
#pragma unroll
      for (int r = 0; r < 4 / RUN; ++r) after.run[h][r] = spot(first + h * 16 + g * 4 + r * RUN);
    }
    return first;
  }

  // Whether the lane's value h, r of the next tile is there.  (A run that the last key is part of may end behind it.)
  __device__ bool there(int64_t first, int h, int r) const {
    return next.run[h][r / RUN].page >= 0 && (RUN == 1 || first + h * 16 + g * 4 + r < until);
  }
  __device__ unsigned gone(int64_t first) const {
    unsigned bits = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) bits |= there(first, h, r) ? 0 : 1u << (h * 4 + r);
    return bits;
  }

  static constexpr int N = BITS8 ? 4 : 2, SZ = sizeof(E);  // elements a word
  // Offsets that lie behind an array's end, also when a row's and an element's are added.
  static constexpr unsigned NO_ROW = 0x80000000u, NO_ELEMENT = FLAT;

  __device__ static __amdgpu_buffer_rsrc_t all(const Pool &x, int head) {
    return window(x.at + head * x.head * SZ, FLAT);
  }

  // A lane's row of keys or values: an address, or a distance from the head's first row.
  struct Row {
    const E *at;
    unsigned offset;
    bool have;
  };
  __device__ Row row(const Pool &x, Spot at, int more) const {
    if constexpr (WINDOW)
      return {nullptr, at.page < 0 ? NO_ROW : (unsigned)at.page * (unsigned)(x.page * SZ) + (unsigned)(at.slot + more) * (unsigned)(x.slot * SZ), true};
    return {(const E *)x.at + at.page * x.page + head * x.head + (at.slot + more) * x.slot, 0, at.page >= 0};
  }

  template <int M>
  __device__ void piece(unsigned *to, const Pool &x, const Row &row, int e) const {
    if constexpr (WINDOW) {
      window_load<M * SZ>(to, all(x, head), row.offset + (e < p.c.dim ? (unsigned)e * SZ : NO_ELEMENT));
    } else {
      typedef typename Raw<E, M>::type V;
      const V v = *(const V *)(row.have && e < p.c.dim ? (const void *)(row.at + e) : (const void *)&paged_zeros);
      if constexpr (sizeof v < sizeof(unsigned)) {
        *to = __builtin_bit_cast(unsigned short, v);
      } else {
        __builtin_memcpy(to, &v, sizeof v);
      }
    }
  }

  __device__ void scales(f32x4 (&to)[2], const Pool &x) const {
    const auto w = window(x.scale + head * x.scale_head, FLAT);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const Spot at = next.run[h][r / RUN];
        const int slot = at.slot + r % RUN;
        if constexpr (WINDOW) {
          unsigned v;
          window_load<4>(&v, w, at.page < 0 ? NO_ROW : (unsigned)at.page * (unsigned)(x.scale_page * 4) + (unsigned)slot * (unsigned)(x.scale_slot * 4));
          to[h][r] = __uint_as_float(v);
        } else {
          const float *const v = x.scale + at.page * x.scale_page + head * x.scale_head + slot * x.scale_slot;
          to[h][r] = *(at.page >= 0 ? v : (const float *)&paged_zeros);
        }
      }
  }

  // (What stands behind the last key in its run is on its page: read, and seen by nobody.)
  __device__ void load_keys(Tile<DP, BITS8> &t, int64_t first) const {
    if (first >= until) return;  // (it will not be taken)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Row k = row(p.c.k, next.key[h], 0);
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) piece<8>(t.k[h] + j * 8 / N, p.c.k, k, key_element<DP, BITS8>(j, g));
      if constexpr (!WINDOW) __builtin_amdgcn_sched_barrier(0);  // (all addresses at once would take more registers than there are)
    }
    if constexpr (BITS8) scales(t.k_scale, p.c.k);
  }

  __device__ void load_values(Tile<DP, BITS8> &t, int64_t first) const {
    if (first >= until) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const Row v = row(p.c.v, next.run[h][r / RUN], r % RUN);
        unsigned *const to = t.v[h * 4 + r];
        if constexpr (DP == 96) {
          piece<4>(to, p.c.v, v, l16 * 4);
          piece<2>(to + 4 / N, p.c.v, v, 64 + l16 * 2);
        } else {
          piece<DP / 16>(to, p.c.v, v, l16 * (DP / 16));
        }
        if constexpr (!WINDOW) __builtin_amdgcn_sched_barrier(0);
      }
    if constexpr (BITS8) scales(t.v_scale, p.c.v);
  }
};

__device__ inline int64_t of_lane(int64_t x, int lane) {
  return (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}

// The same where 16 keys that start at a multiple of 16 stand side by side on one page, and their rows at multiples of
// 16 bytes: the pages of 64 tiles are looked up at once, a tile a lane, and tiles without any are passed over; a lane's
// offsets within the 16 rows stay the same from tile to tile, and rows behind the last key, or of a page that is not
// there, are kept out by the end of a window.
template <typename T, int DP, bool BITS8>
struct InPages {
  typedef typename std::conditional<BITS8, int8_t, unsigned short>::type E;
  static constexpr int SZ = sizeof(E), NK = BITS8 ? (DP + 32) / 64 : DP / 32, NV = DP == 96 ? 2 : 1;
  static constexpr unsigned BEHIND = 0x80000000u;  // behind any window's end
  const PagedParams &p;
  int u, head, until;
  unsigned k_at[NK], v_at[4][NV];
  // Where the halves' 16 rows start, in bytes from the head's first; below zero: a page that is not there.
  struct Spots {
    int64_t k[2], v[2], k_scale[2], v_scale[2];
  } next, after, lanes;  // lanes: of the tiles tile, tile + step, ...
  int64_t tile;
  int step;
  unsigned long long left;  // those of them that are still to come
  const char *k, *v, *k_scale, *v_scale;  // of the head

  __device__ InPages(const PagedParams &p, int u, int head, int until, int tile, int step)
      : p(p), u(u), head(head), until(until), tile(tile), step(step) {
    look();
    k = p.c.k.at + head * p.c.k.head * SZ;
    v = p.c.v.at + head * p.c.v.head * SZ;
    k_scale = (const char *)(p.c.k.scale + head * p.c.k.scale_head);
    v_scale = (const char *)(p.c.v.scale + head * p.c.v.scale_head);
    const int l16 = threadIdx.x % 16, g = threadIdx.x % WAVE / 16, dim = p.c.dim;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int e = key_element<DP, BITS8>(BITS8 ? 2 * i : i, g);
      k_at[i] = e < dim ? (unsigned)(l16 * p.c.k.slot + e) * SZ : BEHIND;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const unsigned row = (unsigned)((g * 4 + r) * p.c.v.slot);
      if constexpr (DP == 96) {
        v_at[r][0] = l16 * 4 < dim ? (row + l16 * 4) * SZ : BEHIND;
        v_at[r][1] = 64 + l16 * 2 < dim ? (row + 64 + l16 * 2) * SZ : BEHIND;
      } else {
        v_at[r][0] = l16 * (DP / 16) < dim ? (row + l16 * (DP / 16)) * SZ : BEHIND;
      }
    }
  }

  __device__ void look() {
    const int64_t first = (tile + (int64_t)(threadIdx.x % WAVE) * step) * TILE_KEYS;
    bool any = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int page = -1, slot = 0;
      if (first + h * 16 < until) page = page_of(p.c, u, (int)first + h * 16, &slot);
      any |= page >= 0;
      auto spot = [&](int64_t by_page, int64_t by_slot, int size) { return page < 0 ? -1 : (page * by_page + slot * by_slot) * size; };
      lanes.k[h] = spot(p.c.k.page, p.c.k.slot, SZ);
      lanes.v[h] = spot(p.c.v.page, p.c.v.slot, SZ);
      if constexpr (BITS8) {
        lanes.k_scale[h] = spot(p.c.k.scale_page, 1, 4);
        lanes.v_scale[h] = spot(p.c.v.scale_page, 1, 4);
      }
    }
    left = __ballot(any);
  }

  // The tile that was looked up last is the next one to be loaded; looks up another and returns its first key.
  __device__ int64_t find() {
    next = after;
#pragma unroll
    for (int h = 0; h < 2; ++h) after.k[h] = after.v[h] = after.k_scale[h] = after.v_scale[h] = -1;
    while (!left) {
      if ((tile + (int64_t)WAVE * step) * TILE_KEYS >= until) return NO_TILE;
      tile += (int64_t)WAVE * step;
      look();
    }
    const int l = __builtin_ctzll(left);
    left &= left - 1;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      after.k[h] = of_lane(lanes.k[h], l);
      after.v[h] = of_lane(lanes.v[h], l);
      if constexpr (BITS8) {
        after.k_scale[h] = of_lane(lanes.k_scale[h], l);
        after.v_scale[h] = of_lane(lanes.v_scale[h], l);
      }
    }
    return (tile + (int64_t)l * step) * TILE_KEYS;
  }

  __device__ unsigned gone(int64_t) const { return (next.k[0] < 0 ? 0xfu : 0) | (next.k[1] < 0 ? 0xf0u : 0); }

  // The 16 rows as far as there are any (the last key's tile ends with it).
  __device__ __amdgpu_buffer_rsrc_t rows_of(const char *x, int64_t at, int slot, int64_t first, int h) const {
    const int64_t behind = until - (first + h * 16);
    const int rows = behind < 16 ? (int)behind : 16;
    return window(x + at, at < 0 ? 0 : ((rows - 1) * slot + p.c.dim) * SZ);
  }
  // (all 16 scales are on the page, those behind the last key among them)
  __device__ f32x4 scales_of(const char *x, int64_t at) const {
    unsigned w[4];
    window_load<16>(w, window(x + at, at < 0 ? 0 : 64), threadIdx.x % WAVE / 16 * 16);
    return (f32x4){__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
  }

  __device__ void load_keys(Tile<DP, BITS8> &t, int64_t first) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto w = rows_of(k, next.k[h], (int)p.c.k.slot, first, h);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        if constexpr (!BITS8) {
          window_load<16>(t.k[h] + i * 4, w, k_at[i]);
        } else if (i * 64 + 64 <= DP) {
          window_load<16>(t.k[h] + i * 4, w, k_at[i]);
        } else {
          window_load<8>(t.k[h] + i * 4, w, k_at[i]);
        }
      }
      if constexpr (BITS8) t.k_scale[h] = scales_of(k_scale, next.k_scale[h]);
    }
  }

  __device__ void load_values(Tile<DP, BITS8> &t, int64_t first) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto w = rows_of(v, next.v[h], (int)p.c.v.slot, first, h);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        unsigned *const to = t.v[h * 4 + r];
        if constexpr (DP == 96) {
          window_load<4 * SZ>(to, w, v_at[r][0]);
          window_load<2 * SZ>(to + SZ, w, v_at[r][1]);
        } else {
          window_load<DP / 16 * SZ>(to, w, v_at[r][0]);
        }
      }
      if constexpr (BITS8) t.v_scale[h] = scales_of(v_scale, next.v_scale[h]);
    }
  }
};

// The running state of 16 columns in a wave: lanes l % 16 + 16 g hold column l % 16.
template <int DP>
struct State16 {
  float top, sum;       // the maximum so far (of q.k; -inf: nothing seen yet), the sum of this lane's keys
  f32x4 out[DP / 16];   // out[i][r]: element value_element(i, 4 g + r)
};

__device__ inline float base_of(float top) { return top == -INFINITY ? 0.0f : top; }

// What the four lanes of a column hold, put together.
__device__ inline float column_max(float x) {
  const unsigned a = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const unsigned c = __float_as_uint(fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1])));
  const auto d = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  return fmaxf(__uint_as_float(d[0]), __uint_as_float(d[1]));
}
__device__ inline float column_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

constexpr float GROWTH = 8.0f;  // the maximum may lag behind by this much (p up to 2^8) before out is rescaled

// Values near the end of bfloat16's range, or scales of 8-bit ones, times p to 2^8, and their sums pass binary32.  A wave
// that finds such a sum takes its keys once more, with p LOW times as large in that sum's column: 2^31 keys, p to 2^-32 and
// values to 2^128 do not.  (Weights below 2^-86 of the largest, and elements of the column below 2^-86, may lose bits
// there.)  What is joined has been divided by its sum.  32 users' tokens take 95.5 us for 95.2 without.
constexpr float LOW = 0x1p-40f;

// Eight codes as elements of T, exactly.
template <typename T>
__device__ inline typename Mma16<T>::frag of_codes(unsigned lo, unsigned hi) {
  typename Mma16<T>::frag f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = (T)(float)(int8_t)(lo >> 8 * i);
    f[i + 4] = (T)(float)(int8_t)(hi >> 8 * i);
  }
  return f;
}

// p goes into its product as two parts of 16 bits, the rounded one and what it left: bounded by memory, the second
// product costs nothing (32 users' tokens 95 us with one part or two), and the output's error against 64 bits is that
// of its own rounding (1.6e-3 in bfloat16; 2.3e-3 with one part).  With 8 bits the parts are bfloat16 ones of p times the
// value's scale.
template <typename T, bool BITS8>
using Weight = typename std::conditional<BITS8, __bf16, T>::type;

// Parts of binary16 end at 2^-25.  There p is made 2^LIFT times as large, below 2^16 still, and where some p of a tile is
// below SMALL, so that its parts hold fewer than 16 bits, what they leave of p goes through the products again, AGAIN
// times as large, until that is 1 / END: what is lost of a weight is then below 2^-25 2^-60 2^-7 of the largest, which
// 2^31 keys with values to 2^16 cannot make a binary16 output show.  (Nothing at all would be left of p below 2^-25
// otherwise, while the sum has it.)  32 users' tokens take 96 us for 95 without, 104 where all tiles go through again;
// binary32 products, an eighth of the rate, took 100 for all (four rows of 64 heads of 16 users 135 for 130, one tile 6.8
// for 5.7).
template <typename T, bool BITS8>
constexpr bool LIFTED = !BITS8 && __is_same(T, _Float16);
constexpr float LIFT = 7.0f, SMALL = 0x1p-9f, AGAIN = 0x1p20f, END = 0x1p-60f;

// Scores of the columns with 32 keys: column c's with key 16 h + 4 g + r in sc[c][h][r].
template <typename T, int DP, bool BITS8, int CT>
__device__ inline void scores(f32x4 (&sc)[CT][2], const typename Mma16<T>::frag (&q)[CT][DP / 32], const Tile<DP, BITS8> &t) {
  typedef typename Mma16<T>::frag frag;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int c = 0; c < CT; ++c) sc[c][h] = (f32x4){};
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
      frag k;
      if constexpr (BITS8) {
        k = of_codes<T>(t.k[h][2 * j], t.k[h][2 * j + 1]);
      } else {
        k = __builtin_bit_cast(frag, (u32x4){t.k[h][4 * j], t.k[h][4 * j + 1], t.k[h][4 * j + 2], t.k[h][4 * j + 3]});
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) sc[c][h] = Mma16<T>::m16(k, q[c][j], sc[c][h]);
    }
    if constexpr (BITS8) {
#pragma unroll
      for (int c = 0; c < CT; ++c) sc[c][h] *= t.k_scale[h];
    }
  }
}

// p times 2^lift of a column's scores relative to its maximum, which is raised first where it lags; the sum goes on.
template <int DP>
__device__ inline void softmax(State16<DP> &s, f32x4 (&sc)[2], float scale, float lift) {
  float top = -INFINITY;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[h][r]);
  top = column_max(top);
  // (false where neither has seen anything: -inf - -inf is NaN)
  const bool grows = (top - s.top) * scale > GROWTH;
  if (__any(grows)) {
    // a column's own scores decide for it: what other columns see does not change its roundings
    const float next = grows ? top : s.top;
    const float f = s.top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((s.top - next) * scale);
    s.top = next;
    s.sum *= f;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) s.out[i] *= f;
  }
  // The difference first: sc * scale - top * scale with the product rounded puts all p of a wave off by the same factor, but
  // another one in another wave, whose keys are weighed against these by exp(scale (top - top')).
  const float base = base_of(s.top);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sc[h][r] = __builtin_amdgcn_exp2f((sc[h][r] - base) * scale + lift);
      s.sum += sc[h][r];
    }
}

// Element i of the lane's piece of its eight 16-bit values.
template <int DP>
__device__ inline u32x4 value_words(const Tile<DP, false> &t, int i) {
  u32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const unsigned a = t.v[2 * e][i / 2], b = t.v[2 * e + 1][i / 2];
    x[e] = i % 2 ? a >> 16 | (b & 0xffff0000u) : (a & 0xffffu) | b << 16;
  }
  return x;
}

// The values' sums with weights p, which are used up.
template <typename T, int DP, bool BITS8, int CT>
__device__ inline void weighted(State16<DP> (&s)[CT], f32x4 (&p)[CT][2], const Tile<DP, BITS8> &t) {
  typedef Weight<T, BITS8> P;
  typedef typename Mma16<P>::frag frag;
  float least = 0.0f;  // of the lane's p that are not zero
  if constexpr (LIFTED<T, BITS8>) {
    unsigned x = ~0u;  // (the bits of 0 become the largest of all, those of a NaN)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const unsigned y = __float_as_uint(p[c][h][r]) - 1;
          x = y < x ? y : x;
        }
    least = __uint_as_float(x);
  }
  float back = 1.0f;
  for (;;) {
    frag w[CT], rest[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = BITS8 ? p[c][h][r] * t.v_scale[h][r] : p[c][h][r], left = x - (float)(P)x;
          w[c][h * 4 + r] = (P)x;
          rest[c][h * 4 + r] = (P)left;
          if constexpr (LIFTED<T, BITS8>) p[c][h][r] = (left - (float)(P)left) * AGAIN;
        }
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      frag v;
      if constexpr (BITS8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (P)(float)(int8_t)(t.v[e][i / 4] >> 8 * (i % 4));
      } else {
        v = __builtin_bit_cast(frag, value_words(t, i));
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        s[c].out[i] = Mma16<P>::m16(v, w[c], s[c].out[i]);
        s[c].out[i] = Mma16<P>::m16(v, rest[c], s[c].out[i]);
      }
      if (i % 2) __builtin_amdgcn_sched_barrier(0);  // (all operands at once would take more registers than there are)
    }
    if (!LIFTED<T, BITS8> || back == END || !__any(least < SMALL)) break;
    // (out, at most 2^31 2^15 2^16, is enlarged with p: in a sum of its own it would take registers that are not there)
    least *= AGAIN;
    back *= 1.0f / AGAIN;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) s[c].out[i] *= AGAIN;
  }
  if (LIFTED<T, BITS8> && back < 1.0f) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) s[c].out[i] *= back;
  }
}

// Takes infinities and NaN out of 16-bit values; the elements of the columns that see them become NaN.  seen[c]: 1 for
// each of the lane's keys that column c sees.
template <typename T, int DP, int CT>
__device__ inline void take_non_finite(State16<DP> (&s)[CT], Tile<DP, false> &t, const typename Mma16<T>::frag (&seen)[CT]) {
  // two values a word: an exponent of ones carries into the sign's place
  constexpr unsigned EXP = __is_same(T, __bf16) ? 0x7f807f80u : 0x7c007c00u, ONE = __is_same(T, __bf16) ? 0x00800080u : 0x04000400u;
  constexpr unsigned UNIT = __is_same(T, __bf16) ? 0x3f80u : 0x3c00u;
  unsigned bad = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int w = 0; w < Tile<DP, false>::VW; ++w) bad |= ((t.v[e][w] & EXP) + ONE) & 0x80008000u;
  if (!__any(bad != 0)) return;
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) {
    u32x4 x = value_words(t, i);  // (from here on: 1 where a value is not finite)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = ((((x[e] & EXP) + ONE) & 0x80008000u) >> 15) * UNIT;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const f32x4 n = Mma16<T>::m16(__builtin_bit_cast(typename Mma16<T>::frag, x), seen[c], (f32x4){});
#pragma unroll
      for (int r = 0; r < 4; ++r) s[c].out[i][r] = n[r] > 0.0f ? __uint_as_float(0x7fc00000u) : s[c].out[i][r];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int w = 0; w < Tile<DP, false>::VW; ++w) {
      const unsigned m = ((t.v[e][w] & EXP) + ONE) & 0x80008000u;
      t.v[e][w] &= ~((m << 1) - (m >> 15));
    }
}

// Waves that a SIMD is to have room for: as many as leave them registers for all that a tile takes.  (On pages of 20 keys 24
// users' binary16 drafts of heads of 96 take 22.4 us with three waves and 24.8 with two, 32 users' tokens over 8 bits 90 and 102.)
constexpr int waves_a_simd(int dp, bool bits8, int ct, int aligned) {
  if (aligned != 16) return aligned == -4 && (dp < 128 || bits8) ? 3 : aligned > 0 && bits8 && dp == 128 ? 1 : 2;
  if (ct == 2) return 2;
  return dp == 64 ? 4 : bits8 || dp == 96 ? 3 : 2;
}

// ALIGNED: 16 (InPages), 4 or 1 (Anywhere; negative: through windows).
template <typename T, int DP, bool BITS8, int CT, int ALIGNED, int WAVES>
__global__ __launch_bounds__(WAVES *WAVE, waves_a_simd(DP, BITS8, CT, ALIGNED)) void paged_kernel(PagedParams p) {
  typedef typename Mma16<T>::frag frag;
  constexpr int THREADS = WAVES * WAVE, COLUMNS = 16 * CT, PITCH = DP + 4;
  __shared__ __align__(16) float mix[WAVES * COLUMNS * PITCH];
  __shared__ float tops[WAVES][COLUMNS], sums[WAVES][COLUMNS];
  const int lane = threadIdx.x % WAVE, wave = wave_index(), l16 = lane % 16, g = lane / 16;
  const int a = block_index(), b = divide(a, p.by_heads), c0 = divide(b, p.by_tiles);
  const int kv = a - b * p.c.kv_heads, tile = b - c0 * p.tiles, column0 = tile * COLUMNS;
  Share share;
  if (p.shares) {
    if (!share_of(p, c0, false, &share)) return;
  } else {
    if (c0 >= p.c.sequences) return;
    share = {newest(p, c0), c0, 0, 1, 0};
  }
  const Newest &q = share.q;
  const int u = share.u, rows = q.rows < p.max_queries ? q.rows : p.max_queries, columns = rows * p.group;
  if (column0 >= columns) return;
  const int shift = q.keys - q.rows;  // row i sees keys 0 .. shift + i
  const int first_row = divide(column0, p.by_group);
  const int last_row = divide((column0 + COLUMNS < columns ? column0 + COLUMNS : columns) - 1, p.by_group);
  // what the tile's last row does not see is not read
  const int until = shift + last_row + 1 < q.last ? shift + last_row + 1 : q.last;
  frag qf[CT][DP / 32];
  int limit[CT];
  State16<DP> s[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int column = column0 + c * 16 + l16;
    const bool have = column < columns;
    const int row = divide(have ? column : column0, p.by_group), head = kv * p.group + (have ? column : column0) - row * p.group;
    limit[c] = have ? shift + row : -1;
    const T *const qrow = (const T *)p.q + (q.row + row) * p.q_stride + head * p.q_head;
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
      const int e = key_element<DP, BITS8>(j, g);
      qf[c][j] = frag{};
      if (have && e < p.c.dim) qf[c][j] = *(const typename Raw<T, 8>::type *)(qrow + e);
    }
  }
  const int first_limit = shift + first_row;
  typedef typename std::conditional<ALIGNED == 16, InPages<T, DP, BITS8>, Anywhere<T, DP, BITS8, ALIGNED % 4 ? 1 : 4, (ALIGNED < 0)>>::type Cache;
  // Whether it is for the second time; then tops holds what the columns' p are multiplied by for their sums of values.
  bool again = false;
  for (;;) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      s[c].top = -INFINITY;
      s[c].sum = 0.0f;
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) s[c].out[i] = (f32x4){};
    }
    // A share's waves take every so many tiles, so that pages that are not there are missing from all shares alike.
    // (where the first tile stands is not the compiler's to know: it would keep what follows from it for the second time)
    int from = share.index * WAVES + wave;
    asm volatile("" : "+v"(from));
    Cache cache(p, u, kv, until, __builtin_amdgcn_readfirstlane(from), share.count * WAVES);
    Tile<DP, BITS8> t;
    int64_t first = cache.find(), second = cache.find();
    cache.load_keys(t, first);
    cache.load_values(t, first);
    // A tile's registers are loaded again as soon as they have been read: the next keys come while p and the values' sums
    // are formed, the next values while the next scores are, and the page of the tile behind them is looked up.
    while (first < until) {
      const unsigned gone = cache.gone(first);
      f32x4 sc[CT][2];
      scores<T, DP, BITS8, CT>(sc, qf, t);
      const int64_t third = cache.find();
      cache.load_keys(t, second);
      __builtin_amdgcn_sched_barrier(0);
      if (first + TILE_KEYS - 1 > first_limit || first + TILE_KEYS > until || __any(gone != 0)) {
        // some column does not see some key
        frag saw[CT];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int64_t key = first + h * 16 + g * 4 + r;
            const bool there = key < until && !(gone >> (h * 4 + r) & 1);
            bool good = true;
            if constexpr (BITS8) {
              // p = 0 of a column that does not see a value times a scale that is not finite would be NaN; whoever sees
              // it has no finite output
              good = fabsf(t.v_scale[h][r]) < INFINITY;
              t.v_scale[h][r] = good ? t.v_scale[h][r] : 0.0f;
            }
#pragma unroll
            for (int c = 0; c < CT; ++c) {
              const bool seen = there && key <= limit[c];
              sc[c][h][r] = seen ? sc[c][h][r] : -INFINITY;
              saw[c][h * 4 + r] = (T)(seen ? 1.0f : 0.0f);
              if (!good && seen) s[c].sum = __uint_as_float(0x7fc00000u);
            }
          }
        if constexpr (!BITS8) take_non_finite<T, DP, CT>(s, t, saw);  // (likewise)
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) softmax<DP>(s[c], sc[c], p.scale, LIFTED<T, BITS8> ? LIFT : 0.0f);
      if (again) {
#pragma unroll
        for (int c = 0; c < CT; ++c) sc[c][0] *= tops[wave][c * 16 + l16], sc[c][1] *= tops[wave][c * 16 + l16];
      }
      weighted<T, DP, BITS8, CT>(s, sc, t);
      cache.load_values(t, second);
      __builtin_amdgcn_sched_barrier(0);
      first = second;
      second = third;
    }
    if constexpr (LIFTED<T, BITS8>) break;  // (2^31 keys, p to 2^15 and values to 2^16 stay within binary32)
    if (again) break;
    unsigned long long bad[CT], any = 0;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      float z = 0.0f;  // NaN with any sum that is not finite
#pragma unroll
      for (int i = 0; i < DP / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) z = __builtin_fmaf(s[c].out[i][r], 0.0f, z);
      any |= bad[c] = __ballot(z != z);
    }
    if (!any) break;
    again = true;
#pragma unroll
    for (int c = 0; c < CT; ++c)  // (the column's four lanes write the same)
      tops[wave][c * 16 + l16] = (bad[c] >> l16 | bad[c] >> (l16 + 16) | bad[c] >> (l16 + 32) | bad[c] >> (l16 + 48)) & 1 ? LOW : 1.0f;
  }
  float even[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) even[c] = again ? 1.0f / tops[wave][c * 16 + l16] : 1.0f;
  lanes_meet();
  // The waves' results: each column's maximum and sum, then outputs relative to them, whose sums pass no value.
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    s[c].sum = column_sum(s[c].sum);
    if (g == 0) {
      tops[wave][c * 16 + l16] = s[c].top;
      sums[wave][c * 16 + l16] = s[c].sum;
    }
  }
  __syncthreads();
  auto top_of = [&](int c) {
    float top = tops[0][c];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w][c]);
    return top;
  };
  auto sum_of = [&](int c, float top) {
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += sums[w][c] * __builtin_amdgcn_exp2f((tops[w][c] - base_of(top)) * p.scale);
    return sum;
  };
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int col = c * 16 + l16;
    const float top = top_of(col), sum = sum_of(col, top);
    const float f = __builtin_amdgcn_exp2f((s[c].top - base_of(top)) * p.scale) * (sum > 0.0f ? 1.0f / sum : sum) * even[c];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        mix[(wave * COLUMNS + c * 16 + l16) * PITCH + value_element<DP>(i, 4 * g + r)] = s[c].out[i][r] * f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < COLUMNS * (DP / 4); i += THREADS) {
    const int c = i / (DP / 4), at = i % (DP / 4) * 4, col = column0 + c;
    if (col >= columns || at >= p.c.dim) continue;
    f32x4 y = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) y += *(const f32x4 *)(mix + (w * COLUMNS + c) * PITCH + at);
    if (share.count == 1) {
      const float z[4] = {y[0], y[1], y[2], y[3]};
      const int row = divide(col, p.by_group);
      store_f32<T, 4>((T *)p.out + (q.row + row) * p.out_stride + (kv * p.group + col - row * p.group) * p.out_head + at, z);
    } else {
      const int pitch = p.c.dim + 4;
      float *const part = p.part + ((((int64_t)c0 * p.tiles + tile) * p.c.kv_heads + kv) * COLUMNS + c) * pitch;
      *(f32x4 *)(part + at) = y;
      if (at == 0) {
        const float top = top_of(c);
        part[p.c.dim] = top, part[p.c.dim + 1] = sum_of(c, top);
      }
    }
  }
}

// EACH waves put one column's partial results together, in workgroups of four waves or EACH.  by_tiles stands for the
// columns of a sequence here.
template <typename T, int EACH>
__global__ __launch_bounds__((EACH < 4 ? 4 : EACH) * WAVE) void paged_join_kernel(PagedParams p) {
  // halves of 32 lanes, which hold four elements each, take shares in turn, MORE of them at once
  constexpr int WAVES = EACH < 4 ? 4 : EACH, HALVES = 2 * EACH, MORE = 8;
  __shared__ __align__(16) float mix[WAVES][128];
  __shared__ float sums[WAVES];
  const int lane = threadIdx.x % WAVE, wave = wave_index(), l32 = lane % 32;
  const int64_t a0 = (int64_t)block_index() * (WAVES / EACH) + wave / EACH;
  const int a = a0 < MAX_BLOCKS ? (int)a0 : MAX_BLOCKS;
  const int b = divide(a, p.by_heads), u = divide(b, p.by_tiles);
  const int kv = a - b * p.c.kv_heads, col = b - u * (p.max_queries * p.group), tile = col / p.tile_columns;
  Share share = {};
  // (whole waves, and with EACH > 1 whole workgroups, have nothing to do)
  const bool some = u < p.c.sequences && share_of(p, u, true, &share) && share.count > 1 &&
                    col < (share.q.rows < p.max_queries ? share.q.rows : p.max_queries) * p.group;
  if (!some) return;
  const int64_t pitch = p.c.dim + 4, step = (int64_t)p.tiles * p.c.kv_heads * p.tile_columns * pitch;
  const float *const part = p.part + ((((int64_t)share.first * p.tiles + tile) * p.c.kv_heads + kv) * p.tile_columns + col % p.tile_columns) * pitch;
  // A running maximum again: everything of a share is read at once.  y stays the weighted mean, which passes no value.
  float top = -INFINITY, sum = 0.0f;
  f32x4 y = {0, 0, 0, 0};
  const int at = l32 * 4 < p.c.dim ? l32 * 4 : 0;
  for (int i0 = wave % EACH * 2 + lane / 32; __any(i0 < share.count); i0 += HALVES * MORE) {
    f32x4 x[MORE];
    float tops[MORE], parts[MORE], high = top;
#pragma unroll
    for (int i = 0; i < MORE; ++i) {
      const bool have = i0 + i * HALVES < share.count;
      const float *const from = part + (have ? i0 + i * HALVES : 0) * step;
      x[i] = *(const f32x4 *)(from + at);
      tops[i] = have ? from[p.c.dim] : -INFINITY;
      parts[i] = from[p.c.dim + 1];
    }
#pragma unroll
    for (int i = 0; i < MORE; ++i) high = fmaxf(high, tops[i]);
    const float base = base_of(high), before = sum * __builtin_amdgcn_exp2f((top - base) * p.scale);
    top = high;
    sum = before;
#pragma unroll
    for (int i = 0; i < MORE; ++i) {
      const bool have = i0 + i * HALVES < share.count;  // (others are repeated, and may hold anything)
      parts[i] = have ? parts[i] * __builtin_amdgcn_exp2f((tops[i] - base) * p.scale) : 0.0f;
      sum += parts[i];
    }
    const float f = sum > 0.0f ? 1.0f / sum : sum;
    y *= before * f;
#pragma unroll
    for (int i = 0; i < MORE; ++i) {
      const bool have = i0 + i * HALVES < share.count;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += have ? parts[i] * f * x[i][j] : 0.0f;
    }
  }
  // the two halves', then the waves' results
  auto both = [&](float top2, float sum2, f32x4 y2) {
    const float high = fmaxf(top, top2), base = base_of(high);
    sum *= __builtin_amdgcn_exp2f((top - base) * p.scale);
    sum2 *= __builtin_amdgcn_exp2f((top2 - base) * p.scale);
    const float both = sum + sum2, f = both > 0.0f ? 1.0f / both : both;
    top = high;
    y = y * (sum * f) + y2 * (sum2 * f);
    sum = both;
  };
  f32x4 other;
#pragma unroll
  for (int i = 0; i < 4; ++i) other[i] = __shfl_xor(y[i], 32);
  both(__shfl_xor(top, 32), __shfl_xor(sum, 32), other);
  if constexpr (EACH > 1) {
    __shared__ float tops[WAVES];
    if (lane < 32) *(f32x4 *)(mix[wave] + l32 * 4) = y;
    if (lane == 0) tops[wave] = top, sums[wave] = sum;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < EACH; ++w) both(tops[w], sums[w], *(const f32x4 *)(mix[w] + l32 * 4));
  }
  if (lane >= 32 || l32 * 4 >= p.c.dim) return;
  const float z[4] = {y[0], y[1], y[2], y[3]};
  const int row = divide(col, p.by_group);
  store_f32<T, 4>((T *)p.out + (share.q.row + row) * p.out_stride + (kv * p.group + col - row * p.group) * p.out_head + l32 * 4, z);
}

// ------------------------------------------------------------------ host side

int paged_check_sizes(const jdob_edge_attend_paged_args *a) {
  if (!a || a->num_heads < 1 || a->max_queries < 0 || a->max_keys < 0 || a->query_rows < 0 || !(a->scale > 0.0f) ||
      !isfinite(a->scale))
    return JDOB_ERR_INVALID_ARG;
  const int code = cache_check_sizes(a->cache, a->num_sequences, a->table_width);
  if (code != JDOB_OK) return code;
  if (a->num_heads % a->cache.num_kv_heads) return JDOB_ERR_INVALID_ARG;
  if (a->num_heads > 1024 || a->query_rows > JDOB_EDGE_MAX_ROWS) return JDOB_ERR_UNSUPPORTED;
  return JDOB_OK;
}

bool has_work(const jdob_edge_attend_paged_args *a) {
  return a->num_sequences > 0 && a->query_rows > 0 && a->max_queries > 0;
}

struct PagedPlan {
  int64_t tiles;
  int queries, columns, shares;  // columns: of a tile
  int64_t list;                  // of shares (or sequences) that there may be
};

// `in_pages`: InPages reads the cache.
PagedPlan paged_plan(const jdob_edge_attend_paged_args *a, bool in_pages) {
  const int64_t queries = a->max_queries < a->query_rows ? a->max_queries : a->query_rows;  // no sequence has more
  const int64_t room = (int64_t)a->table_width * a->cache.page_size, n = a->num_sequences;
  const int64_t keys = a->max_keys < room ? a->max_keys : room;
  const int64_t all = queries * (a->num_heads / a->cache.num_kv_heads);
  // Keys that are read once for 32 columns, not twice: 16 users' 4 rows of 64 heads after up to 16,383 8-bit keys take 84 us
  // so and 106 by 16 columns, after up to 4095 34 and 40.  By 16 columns, where waves need half the registers, if there
  // are few keys (4 users, up to 1023 keys: 14 us and 17) or InPages does not read them: there are no kernels for 32 of
  // those (through windows 24 users' drafts on pages of 20 keys would take the same 23 us, 16 users' 4 rows of 64 heads after
  // up to 4095 8-bit keys 44 for 57).
  const int columns = all <= 16 || !in_pages || n * keys * a->cache.num_kv_heads <= 1 << 17 ? 16 : 32;
  const int64_t tiles = (all + columns - 1) / columns, layers = tiles * a->cache.num_kv_heads;
  const int64_t groups = layers * n, most = n * ((keys + LEAST_KEYS - 1) / LEAST_KEYS);
  // How many shares: few sequences' fill the chip once, two workgroups a compute unit, with half a share a sequence lost
  // at its end (one of 131,072 8-bit keys, 8 key heads: 53 us, with 128 shares a head 61); many, whose lengths may be
  // anything, are dealt twice as finely (32 of 15 to 8191 keys: 98 us, 114 as for few; 64 of up to 8191: 121 and 134;
  // but 64 of 2047 each 58 and 52).
  int64_t shares = groups <= 128 ? (512 - groups / 2) / layers : 1024 / layers;
  shares = shares < 1 ? 1 : shares < most ? shares : most;
  // Not at all where the join, a launch of 5 us, costs more than it gives: 512 keys take 11 us in one workgroup and 14 in
  // two; many sequences fill the chip, and one of 8192 keys among them ends 100 us after the others at most.  Forming the
  // list takes two looks at every 64 sequences.
  if (keys <= 512 || (groups >= 2048 && keys <= 8192) || n > 1024) shares = 0;
  return {tiles, (int)queries, columns, (int)shares, n + shares};
}

template <typename T, int DP, bool BITS8>
int paged(const PagedParams &p, int aligned, int64_t blocks, hipStream_t stream) {
  constexpr int WAVES = 4;
  return launch(p.tile_columns == 32 ? paged_kernel<T, DP, BITS8, 2, 16, WAVES>
                : aligned == 16      ? paged_kernel<T, DP, BITS8, 1, 16, WAVES>
                : aligned == -4      ? paged_kernel<T, DP, BITS8, 1, -4, WAVES>
                : aligned == -1      ? paged_kernel<T, DP, BITS8, 1, -1, WAVES>
                : aligned == 4       ? paged_kernel<T, DP, BITS8, 1, 4, WAVES>
                                     : paged_kernel<T, DP, BITS8, 1, 1, WAVES>,
                blocks, WAVES * WAVE, stream, p);
}

// Whether InPages can read the cache; 16 rows have to stay within a window, whose offsets pass 2^31 nowhere.
bool in_pages(const jdob_edge_cache &c) {
  const int64_t unit = c.bits8 ? 16 : 8;
  auto pool = [&](const void *at, int64_t page, int64_t head, int64_t slot, int64_t scale_slot) {
    return (uintptr_t)at % 16 == 0 && page % unit == 0 && head % unit == 0 && slot % unit == 0 && slot < (1 << 24) &&
           (!c.bits8 || scale_slot == 1);
  };
  // (8-bit keys are read 16 elements at once up to 64, and beyond 96 to 128)
  return c.page_size % 16 == 0 && pool(c.k, c.k_page_stride, c.k_head_stride, c.k_slot_stride, c.k_scale_slot_stride) &&
         pool(c.v, c.v_page_stride, c.v_head_stride, c.v_slot_stride, c.v_scale_slot_stride) &&
         (!c.bits8 || c.head_dim % 16 == 0 || (c.head_dim > 64 && c.head_dim <= 96));
}

// Whether windows cover the cache's arrays, and rows start at multiples of four bytes: elements from a head's first row to
// the last of its rows' ends, with strides as checked.
bool flat(const jdob_edge_cache &c) {
  const int64_t pages = c.num_pages > 0 ? c.num_pages - 1 : 0, slots = c.page_size - 1, unit = c.bits8 ? 4 : 2;
  auto spans = [&](int64_t page, int64_t slot, int64_t size) {
    return page < FLAT && slot < FLAT && pages * page + slots * slot + JDOB_EDGE_MAX_HEAD_DIM < FLAT / size;
  };
  auto rows = [&](const void *at, int64_t page, int64_t head, int64_t slot) {
    return (uintptr_t)at % 4 == 0 && (page | head | slot) % unit == 0 && spans(page, slot, c.bits8 ? 1 : 2);
  };
  return rows(c.k, c.k_page_stride, c.k_head_stride, c.k_slot_stride) &&
         rows(c.v, c.v_page_stride, c.v_head_stride, c.v_slot_stride) &&
         (!c.bits8 || (spans(c.k_scale_page_stride, c.k_scale_slot_stride, 4) && spans(c.v_scale_page_stride, c.v_scale_slot_stride, 4)));
}

template <typename T, bool BITS8>
int paged(PagedParams p, const PagedPlan &f, int aligned, hipStream_t stream) {
  const int64_t each = (int64_t)f.queries * p.group, all = each * p.c.sequences * p.c.kv_heads;
  const int64_t blocks = f.list * p.c.kv_heads * f.tiles;
  // (tiles are fewer than columns, whose numbers within a sequence are divided)
  if (each >= 1 << 30 || blocks > MAX_BLOCKS || (f.shares && all > MAX_BLOCKS)) return JDOB_ERR_UNSUPPORTED;
  p.by_heads = divide_by(p.c.kv_heads), p.by_tiles = divide_by((int)f.tiles), p.by_group = divide_by(p.group);
  const int code = p.c.dim <= 64   ? paged<T, 64, BITS8>(p, aligned, blocks, stream)
                   : p.c.dim <= 96 ? paged<T, 96, BITS8>(p, aligned, blocks, stream)
                                   : paged<T, 128, BITS8>(p, aligned, blocks, stream);
  if (code != JDOB_OK || !f.shares) return code;
  p.by_tiles = divide_by((int)each);
  // few columns of many shares
  if (f.shares >= 16 * p.c.sequences) return launch(paged_join_kernel<T, 8>, all, 8 * WAVE, stream, p);
  return launch(paged_join_kernel<T, 1>, (all + 3) / 4, 4 * WAVE, stream, p);
}

}  // namespace
}  // namespace edge

extern "C" int64_t jdob_edge_attend_paged_workspace(const jdob_edge_attend_paged_args *a) {
  using namespace edge;
  if (paged_check_sizes(a) != JDOB_OK) return -1;
  if (!has_work(a)) return 0;
  // (whether InPages reads the cache follows from its arrays, too)
  int64_t most = 0;
  for (bool in : {false, true}) {
    const PagedPlan f = paged_plan(a, in);
    const int64_t columns = f.shares ? f.list * a->cache.num_kv_heads * f.tiles * f.columns : 0;
    most = columns > most ? columns : most;
  }
  return most * (a->cache.head_dim + 4) * (int64_t)sizeof(float);
}

extern "C" int jdob_edge_attend_paged(const jdob_edge_attend_paged_args *a, void *hip_stream) {
  using namespace edge;
  int code = paged_check_sizes(a);
  if (code != JDOB_OK || !has_work(a)) return code;
  code = cache_check_arrays(a->cache, a->table_width, a->table, a->table_stride, a->query_start, a->key_count);
  if (code != JDOB_OK) return code;
  if (!a->q || !a->out || a->q_stride < 0 || a->q_head_stride < 0) return JDOB_ERR_INVALID_ARG;
  // rows and heads of out that are written at once must not share elements
  if (a->out_stride < 0 || a->out_head_stride < 0 ||
      pieces_overlap(a->query_rows, a->out_stride, a->num_heads, a->out_head_stride, a->cache.head_dim))
    return JDOB_ERR_INVALID_ARG;
  const int64_t need = jdob_edge_attend_paged_workspace(a);
  if (need > 0 && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return JDOB_ERR_INVALID_ARG;
  const bool in = in_pages(a->cache);
  const int run = a->cache.page_size % 4 == 0 ? 4 : 1, aligned = in ? 16 : flat(a->cache) ? -run : run;
  const PagedPlan f = paged_plan(a, in);
  const PagedParams p = {pages_of(a->cache, a->num_sequences, a->table_width, a->table, a->table_stride, a->query_start,
                                  a->key_count),
                         a->num_heads / a->cache.num_kv_heads, f.queries, f.columns,
                         log2_scale(a->scale), a->query_rows, (const char *)a->q, (char *)a->out, a->q_stride,
                         a->q_head_stride, a->out_stride, a->out_head_stride, (int)f.tiles, f.shares, {}, {}, {},
                         (float *)a->workspace};
  hipStream_t stream = (hipStream_t)hip_stream;
  if (a->cache.dtype == JDOB_EDGE_BF16)
    return a->cache.bits8 ? paged<__bf16, true>(p, f, aligned, stream) : paged<__bf16, false>(p, f, aligned, stream);
  return a->cache.bits8 ? paged<_Float16, true>(p, f, aligned, stream) : paged<_Float16, false>(p, f, aligned, stream);
}
