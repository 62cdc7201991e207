// Causal attention of sequences' newest rows over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - max),  keys j that are there and j <= m - n + i
//
// With 8 bits k_j and v_j are codes times a scale of the key: scores are multiplied by the key's scale, p by the
// value's, and the codes go into the products as they are.
//
// The rows of all heads that read one key head stand together as columns, 16 or 32 for a workgroup; its waves take
// 32 keys in turn, and the keys are split over workgroups, whose partial results a second kernel joins.  One pass
// over the keys: a running maximum and sum per column, the output rescaled when the maximum grows.
//
// Keys and values come straight into the registers that the matrix units read; LDS is only used to join the waves.
// The products are formed transposed, 16 x 16 at a time: S^T = K Q^T leaves a column in a lane (four times: lane
// group g = lane / 16 holds keys 4 g .. 4 g + 3 of every 16), O^T = V^T P^T takes the lane's own p as its second
// operand.  Which key or element stands at which place of the summed dimension is free as long as both operands
// agree: a lane's 8 elements of a key are any 8 that the query's lane has too, and V's operand, 8 keys of one
// element a lane, is cut out of 8 rows' pieces that the lane loads side by side.
#include <type_traits>

#include "pages.h"

namespace edge {
namespace {

struct PagedParams {
  Pages c;
  int heads, group, max_queries, tile_columns;
  float scale;  // times log2(e)
  int64_t query_rows;
  const char *q;
  char *out;
  int64_t q_stride, q_head, out_stride, out_head;  // elements
  int splits, each;   // splits of the keys, keys of one
  int tiles;          // tiles of columns of a sequence
  float *part;        // [sequence][key head][tile][split][columns of a tile][dim + 4]
};

typedef short s16x8 __attribute__((ext_vector_type(8)));
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
  int64_t row;
  int rows, keys;  // the keys as counted
  int last;        // keys that the table has room for
};

__device__ inline Newest newest(const PagedParams &p, int u) {
  int64_t at = p.c.row_start[u], end = p.c.row_start[u + 1];
  at = at < 0 ? 0 : at < p.query_rows ? at : p.query_rows;
  end = end < at ? at : end < p.query_rows ? end : p.query_rows;
  const int keys = p.c.key_count[u] > 0 ? p.c.key_count[u] : 0;
  const int64_t room = (int64_t)p.c.width * p.c.page_size;
  return {at, (int)(end - at), keys, (int)(keys < room ? keys : room)};
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
  unsigned gone;  // a bit for each of the lane's 8 keys that is absent
};

// A wave's keys of one head, and where the lane's are found: key by key, whatever the page's size and the arrays' alignment.
template <typename T, int DP, bool BITS8>
struct Anywhere {
  const PagedParams &p;
  int u, head, until, lane_key, g;  // until: keys from there on are not read

  __device__ Anywhere(const PagedParams &p, int u, int head, int until)
      : p(p), u(u), head(head), until(until), lane_key(threadIdx.x % 16), g(threadIdx.x % WAVE / 16) {}

  template <typename E, int N>
  __device__ static void piece(unsigned *to, const E *row, int e, bool have) {
    typename Raw<E, N>::type x = {};
    if (have) x = *(const typename Raw<E, N>::type *)(row + e);
    if constexpr (sizeof x < sizeof(unsigned)) {
      *to = __builtin_bit_cast(unsigned short, x);
    } else {
      __builtin_memcpy(to, &x, sizeof x);
    }
  }

  __device__ void find(int64_t) {}
  __device__ void load(Tile<DP, BITS8> &t, int64_t first) const {
    typedef typename std::conditional<BITS8, int8_t, unsigned short>::type E;
    constexpr int N = BITS8 ? 4 : 2;  // elements a word
    const int dim = p.c.dim;
    t.gone = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t key = first + h * 16 + lane_key;
      int slot = 0;
      const int page = key < until ? page_of(p.c, u, (int)key, &slot) : -1;
      const E *const row = (const E *)p.c.k.at + page * p.c.k.page + head * p.c.k.head + slot * p.c.k.slot;
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) {
        const int e = key_element<DP, BITS8>(j, g);
        piece<E, 8>(t.k[h] + j * 8 / N, row, e, page >= 0 && e < dim);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t key = first + h * 16 + g * 4 + r;
        int slot = 0;
        const int page = key < until ? page_of(p.c, u, (int)key, &slot) : -1;
        const E *const row = (const E *)p.c.v.at + page * p.c.v.page + head * p.c.v.head + slot * p.c.v.slot;
        unsigned *const to = t.v[h * 4 + r];
        const int m = lane_key;
        if constexpr (DP == 96) {
          piece<E, 4>(to, row, m * 4, page >= 0 && m * 4 < dim);
          piece<E, 2>(to + 4 / N, row, 64 + m * 2, page >= 0 && 64 + m * 2 < dim);
        } else {
          piece<E, DP / 16>(to, row, m * (DP / 16), page >= 0 && m * (DP / 16) < dim);
        }
        if constexpr (BITS8) {
          t.k_scale[h][r] = t.v_scale[h][r] = 0.0f;
          if (page >= 0) {
            t.k_scale[h][r] = p.c.k.scale[page * p.c.k.scale_page + head * p.c.k.scale_head + slot * p.c.k.scale_slot];
            t.v_scale[h][r] = p.c.v.scale[page * p.c.v.scale_page + head * p.c.v.scale_head + slot * p.c.v.scale_slot];
          }
        }
        t.gone |= page < 0 ? 1u << (h * 4 + r) : 0;
      }
    }
  }
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

// The same where 16 keys that start at a multiple of 16 stand side by side on one page, and their rows at multiples of
// 16 bytes: the page is looked up once for all lanes, a lane's offsets within the 16 rows stay the same from tile to
// tile, and rows behind the last key, or of a page that is not there, are kept out by the end of a window.
template <typename T, int DP, bool BITS8>
struct InPages {
  typedef typename std::conditional<BITS8, int8_t, unsigned short>::type E;
  static constexpr int SZ = sizeof(E), NK = BITS8 ? (DP + 32) / 64 : DP / 32, NV = DP == 96 ? 2 : 1;
  static constexpr unsigned BEHIND = 0x80000000u;  // behind any window's end
  const PagedParams &p;
  int u, head, until;
  unsigned k_at[NK], v_at[4][NV];
  struct Spot {
    int page[2], slot[2];
  } spot;  // of the next tile

  __device__ InPages(const PagedParams &p, int u, int head, int until) : p(p), u(u), head(head), until(until) {
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

  __device__ void find(int64_t first) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      spot.page[h] = -1;
      spot.slot[h] = 0;
      if (first + h * 16 < until)
        spot.page[h] = __builtin_amdgcn_readfirstlane(page_of(p.c, u, (int)first + h * 16, &spot.slot[h]));
    }
  }

  __device__ void load(Tile<DP, BITS8> &t, int64_t first) const {
    t.gone = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int page = spot.page[h], slot = spot.slot[h];
      const int64_t behind = until - (first + h * 16);
      const int rows = page < 0 ? 0 : behind < 16 ? (int)behind : 16;  // (a page only where there are keys)
      const E *const k = (const E *)p.c.k.at + page * p.c.k.page + head * p.c.k.head + slot * p.c.k.slot;
      const E *const v = (const E *)p.c.v.at + page * p.c.v.page + head * p.c.v.head + slot * p.c.v.slot;
      const auto kw = window(k, rows ? (int)((rows - 1) * p.c.k.slot + p.c.dim) * SZ : 0);
      const auto vw = window(v, rows ? (int)((rows - 1) * p.c.v.slot + p.c.dim) * SZ : 0);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        if constexpr (BITS8) {
          if (i * 64 + 64 <= DP) {
            window_load<16>(t.k[h] + i * 4, kw, k_at[i]);
          } else {
            window_load<8>(t.k[h] + i * 4, kw, k_at[i]);
          }
        } else {
          window_load<16>(t.k[h] + i * 4, kw, k_at[i]);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        unsigned *const to = t.v[h * 4 + r];
        if constexpr (DP == 96) {
          window_load<4 * SZ>(to, vw, v_at[r][0]);
          window_load<2 * SZ>(to + SZ, vw, v_at[r][1]);
        } else {
          window_load<DP / 16 * SZ>(to, vw, v_at[r][0]);
        }
      }
      if constexpr (BITS8) {
        // (all 16 are on the page, those behind the last key among them)
        const float *const ks = p.c.k.scale + page * p.c.k.scale_page + head * p.c.k.scale_head + slot;
        const float *const vs = p.c.v.scale + page * p.c.v.scale_page + head * p.c.v.scale_head + slot;
        unsigned w[2][4];
        window_load<16>(w[0], window(ks, rows ? 64 : 0), threadIdx.x % WAVE / 16 * 16);
        window_load<16>(w[1], window(vs, rows ? 64 : 0), threadIdx.x % WAVE / 16 * 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) t.k_scale[h][r] = __uint_as_float(w[0][r]), t.v_scale[h][r] = __uint_as_float(w[1][r]);
      }
      t.gone |= page < 0 ? 0xfu << (h * 4) : 0;
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
// Up to here (log2 units) sc * scale - top * scale may be formed with one rounding of top * scale: it puts p
// off by at most a factor of two, the same for all of a column, which its sum takes back.
constexpr float NEAR = 0x1p24f;

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

// Scores of the columns with 32 keys, softmax, and the values' sums.  Of the tile's keys the lane's column c sees
// 0 .. sees[c] that are there; MASKED: some column of the tile does not see some key.
template <typename T, int DP, bool BITS8, int CT, bool MASKED>
__device__ inline void attend_tile(State16<DP> (&s)[CT], const typename Mma16<T>::frag (&q)[CT][DP / 32],
                                   const Tile<DP, BITS8> &t, const int (&sees)[CT], float scale) {
  typedef typename Mma16<T>::frag frag;
  const int g = threadIdx.x % WAVE / 16;
  f32x4 sc[CT][2];
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
  // p in the type of its product: with 8 bits in two bfloat16 parts, whose range holds p times any scale
  typedef typename std::conditional<BITS8, __bf16, T>::type P;
  typedef typename Mma16<P>::frag pfrag;
  pfrag p[CT], rest[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    auto seen = [&](int h, int r) { return h * 16 + g * 4 + r <= sees[c] && !(t.gone >> (h * 4 + r) & 1); };
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (MASKED) sc[c][h][r] = seen(h, r) ? sc[c][h][r] : -INFINITY;
        top = fmaxf(top, sc[c][h][r]);
      }
    top = column_max(top);
    // (false where neither has seen anything: -inf - -inf is NaN)
    const bool grows = (top - s[c].top) * scale > GROWTH;
    if (__any(grows)) {
      // a column's own scores decide for it: what other columns see does not change its roundings
      const float next = grows ? top : s[c].top;
      const float f = s[c].top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((s[c].top - next) * scale);
      s[c].top = next;
      s[c].sum *= f;
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) s[c].out[i] *= f;
    }
    const float base = base_of(s[c].top) * scale;
    const bool far = !(fabsf(base) < NEAR);
    if (__any(far)) {
      // the difference first, again column by column
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[c][h][r] = far ? (sc[c][h][r] - s[c].top) * scale : sc[c][h][r] * scale - base;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[c][h][r] = sc[c][h][r] * scale - base;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = __builtin_amdgcn_exp2f(sc[c][h][r]);
        s[c].sum += x;
        if constexpr (BITS8) {
          // (what a column does not see may have any scale)
          x *= MASKED && !seen(h, r) ? 0.0f : t.v_scale[h][r];
        }
        p[c][h * 4 + r] = (P)x;
        if constexpr (BITS8) rest[c][h * 4 + r] = (P)(x - (float)p[c][h * 4 + r]);
      }
  }
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) {
    pfrag v;
    if constexpr (BITS8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (P)(float)(int8_t)(t.v[e][i / 4] >> 8 * (i % 4));
    } else {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned a = t.v[2 * e][i / 2], b = t.v[2 * e + 1][i / 2];
        w[e] = i % 2 ? a >> 16 | (b & 0xffff0000u) : (a & 0xffffu) | b << 16;
      }
      v = __builtin_bit_cast(pfrag, w);
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      s[c].out[i] = Mma16<P>::m16(v, p[c], s[c].out[i]);
      if constexpr (BITS8) s[c].out[i] = Mma16<P>::m16(v, rest[c], s[c].out[i]);
    }
  }
}

// Takes infinities and NaN out of the lane's 16-bit values, and says whether the wave had any.
template <typename T, int DP>
__device__ inline bool clear_non_finite(Tile<DP, false> &t) {
  constexpr unsigned EXP = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int w = 0; w < Tile<DP, false>::VW; ++w) {
      unsigned &x = t.v[e][w];
      const bool lo = (x & EXP) == EXP, hi = (x >> 16 & EXP) == EXP;
      bad |= lo || hi;
      x &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
    }
  return __any(bad);
}

// Adds the infinities and NaN of 16-bit values first .. first + 31 to the columns that see them.  Rare, and slow.
template <typename T, int DP, int CT>
__device__ inline void add_non_finite(const PagedParams &p, State16<DP> (&s)[CT], int u, int head, int first, int until,
                                      const int (&sees)[CT]) {
  constexpr unsigned EXP = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
  const int g = threadIdx.x % WAVE / 16;
  for (int j = 0; j < 32 && first + j < until; ++j) {
    int slot = 0;
    const int page = page_of(p.c, u, first + j, &slot);
    if (page < 0) continue;
    const T *const row = (const T *)p.c.v.at + page * p.c.v.page + head * p.c.v.head + slot * p.c.v.slot;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = value_element<DP>(i, 4 * g + r);
        const T x = e < p.c.dim ? row[e] : (T)0.0f;
        const unsigned bits = __builtin_bit_cast(unsigned short, x);
#pragma unroll
        for (int c = 0; c < CT; ++c)
          if ((bits & EXP) == EXP && j <= sees[c]) s[c].out[i][r] += (float)x;
      }
  }
}

constexpr int PAGED_WAVES = 4, TILE_KEYS = 32;

template <typename T, int DP, bool BITS8, int CT, bool IN_PAGES>
__global__ __launch_bounds__(PAGED_WAVES *WAVE, CT == 1 ? 2 : 1) void paged_kernel(PagedParams p) {
  typedef typename Mma16<T>::frag frag;
  constexpr int THREADS = PAGED_WAVES * WAVE, COLUMNS = 16 * CT, PITCH = DP + 4;
  __shared__ __align__(16) float mix[PAGED_WAVES * COLUMNS * PITCH];
  __shared__ float tops[PAGED_WAVES][COLUMNS], sums[PAGED_WAVES][COLUMNS];
  const int lane = threadIdx.x % WAVE, wave = wave_index(), l16 = lane % 16, g = lane / 16;
  const int kv = block_index() % p.c.kv_heads, split = block_index() / p.c.kv_heads % p.splits;
  const int tile = block_index() / p.c.kv_heads / p.splits % p.tiles, u = block_index() / p.c.kv_heads / p.splits / p.tiles;
  if (u >= p.c.sequences) return;
  const Newest q = newest(p, u);
  const int rows = q.rows < p.max_queries ? q.rows : p.max_queries;
  const int64_t columns = (int64_t)rows * p.group, column0 = (int64_t)tile * COLUMNS;
  if (column0 >= columns) return;
  const int shift = q.keys - q.rows;  // row i sees keys 0 .. shift + i
  const int first_row = (int)(column0 / p.group);
  const int last_row = (int)((column0 + COLUMNS < columns ? column0 + COLUMNS : columns) - 1) / p.group;
  // this split's keys; the last split takes what the others leave (max_keys may be too small)
  const int64_t from = (int64_t)split * p.each;
  int64_t until = split + 1 < p.splits && from + p.each < q.last ? from + p.each : q.last;
  if (from >= until && split > 0) return;
  // what the tile's last row does not see is not read (and what it sees is there, or is no part of a column's output)
  until = shift + last_row + 1 < until ? shift + last_row + 1 : until;
  frag qf[CT][DP / 32];
  int limit[CT];
  State16<DP> s[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int64_t column = column0 + c * 16 + l16;
    const bool have = column < columns;
    const int row = have ? (int)(column / p.group) : 0, head = kv * p.group + (have ? (int)(column % p.group) : 0);
    limit[c] = have ? shift + row : -1;
    const T *const qrow = (const T *)p.q + (q.row + row) * p.q_stride + head * p.q_head;
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
      const int e = key_element<DP, BITS8>(j, g);
      qf[c][j] = frag{};
      if (have && e < p.c.dim) qf[c][j] = *(const typename Raw<T, 8>::type *)(qrow + e);
    }
    s[c].top = -INFINITY;
    s[c].sum = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) s[c].out[i] = (f32x4){};
  }
  const int first_limit = shift + first_row;
  typedef typename std::conditional<IN_PAGES, InPages<T, DP, BITS8>, Anywhere<T, DP, BITS8>>::type Cache;
  constexpr int STEP = PAGED_WAVES * TILE_KEYS;
  Cache cache(p, u, kv, (int)until);
  int64_t first = from + wave * TILE_KEYS;  // passes 2^31 behind the longest sequence's end
  Tile<DP, BITS8> even, odd;
  // Takes the tile at `first`, while the next one is loaded and the page of the one behind that is looked up.
  auto take = [&](Tile<DP, BITS8> &now, Tile<DP, BITS8> &next) {
    cache.load(next, first + STEP);
    cache.find(first + 2 * STEP);
    __builtin_amdgcn_sched_barrier(0);
    int sees[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) sees[c] = (int)((limit[c] < until ? limit[c] : until - 1) - first);
    if (first + TILE_KEYS - 1 <= first_limit && first + TILE_KEYS <= until && !__any(now.gone != 0)) {
      attend_tile<T, DP, BITS8, CT, false>(s, qf, now, sees, p.scale);
    } else {
      if constexpr (!BITS8) {
        // p = 0 of a column that does not see a value times an infinity would be NaN
        if (clear_non_finite<T, DP>(now)) add_non_finite<T, DP, CT>(p, s, u, kv, (int)first, (int)until, sees);
      }
      attend_tile<T, DP, BITS8, CT, true>(s, qf, now, sees, p.scale);
    }
    first += STEP;
  };
  cache.find(first);
  cache.load(even, first);
  cache.find(first + STEP);
  while (first < until) {
    take(even, odd);
    if (first >= until) break;
    take(odd, even);
  }
  // the waves' results: each column's maximum, then sums and outputs relative to it
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    s[c].sum = column_sum(s[c].sum);
    if (g == 0) {
      tops[wave][c * 16 + l16] = s[c].top;
      sums[wave][c * 16 + l16] = s[c].sum;
    }
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < PAGED_WAVES; ++w) top = fmaxf(top, tops[w][c * 16 + l16]);
    const float f = __builtin_amdgcn_exp2f((s[c].top - base_of(top)) * p.scale);
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        mix[(wave * COLUMNS + c * 16 + l16) * PITCH + value_element<DP>(i, 4 * g + r)] = s[c].out[i][r] * f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < COLUMNS * (DP / 4); i += THREADS) {
    const int c = i / (DP / 4), at = i % (DP / 4) * 4;
    const int64_t col = column0 + c;
    if (col >= columns || at >= p.c.dim) continue;
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < PAGED_WAVES; ++w) top = fmaxf(top, tops[w][c]);
    f32x4 y = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < PAGED_WAVES; ++w) {
      sum += sums[w][c] * __builtin_amdgcn_exp2f((tops[w][c] - base_of(top)) * p.scale);
      y += *(const f32x4 *)(mix + (w * COLUMNS + c) * PITCH + at);
    }
    if (p.splits == 1) {
      const float f = sum > 0.0f ? 1.0f / sum : sum;
      const float z[4] = {y[0] * f, y[1] * f, y[2] * f, y[3] * f};
      T *const out = (T *)p.out + (q.row + col / p.group) * p.out_stride + (kv * p.group + col % p.group) * p.out_head;
      store_f32<T, 4>(out + at, z);
    } else {
      const int64_t group = ((int64_t)u * p.c.kv_heads + kv) * p.tiles + tile, pitch = p.c.dim + 4;
      float *const part = p.part + ((group * p.splits + split) * COLUMNS + c) * pitch;
      *(f32x4 *)(part + at) = y;
      if (at == 0) part[p.c.dim] = top, part[p.c.dim + 1] = sum;
    }
  }
}

constexpr int MAX_SPLITS = 256, JOIN_THREADS = 256;

// A workgroup puts one column's partial results together.
template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void paged_join_kernel(PagedParams p) {
  __shared__ float weight[MAX_SPLITS], mix[8][128];
  const int columns_each = p.max_queries * p.group;
  const int kv = block_index() % p.c.kv_heads, col = block_index() / p.c.kv_heads % columns_each;
  const int u = block_index() / p.c.kv_heads / columns_each, tile = col / p.tile_columns;
  if (u >= p.c.sequences) return;
  const Newest q = newest(p, u);
  const int rows = q.rows < p.max_queries ? q.rows : p.max_queries;
  if (col >= rows * p.group) return;
  const int64_t pitch = p.c.dim + 4, step = p.tile_columns * pitch;
  const float *const part =
      p.part + (((int64_t)u * p.c.kv_heads + kv) * p.tiles + tile) * p.splits * step + col % p.tile_columns * pitch;
  const int used = q.last > 0 ? (q.last - 1) / p.each + 1 : 1, splits = used < p.splits ? used : p.splits;
  const int t = threadIdx.x, lane = t % WAVE;
  // every wave for itself: the maximum, the weights, their sum
  float tops[MAX_SPLITS / WAVE], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < MAX_SPLITS / WAVE; ++i) {
    tops[i] = i * WAVE + lane < splits ? part[(i * WAVE + lane) * step + p.c.dim] : -INFINITY;
    top = fmaxf(top, tops[i]);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float base = base_of(top);
#pragma unroll
  for (int i = 0; i < MAX_SPLITS / WAVE; ++i)
    if (i * WAVE + lane < splits) {
      const float w = __builtin_amdgcn_exp2f((tops[i] - base) * p.scale);
      sum += w * part[(i * WAVE + lane) * step + p.c.dim + 1];
      if (t < WAVE) weight[i * WAVE + lane] = w;
    }
  sum = wave_sum(sum);
  __syncthreads();
  const int at = t % 32 * 4, g = t / 32;
  f32x4 y = {0, 0, 0, 0};
  if (at < p.c.dim) {
#pragma unroll 4
    for (int i = g; i < splits; i += 8) y += *(const f32x4 *)(part + i * step + at) * weight[i];
    *(f32x4 *)(mix[g] + at) = y;
  }
  __syncthreads();
  if (t < p.c.dim) {
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) z += mix[i][t];
    T *const out = (T *)p.out + (q.row + col / p.group) * p.out_stride + (kv * p.group + col % p.group) * p.out_head;
    out[t] = (T)(z * (sum > 0.0f ? 1.0f / sum : sum));
  }
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
  int queries, columns, splits, each;  // columns: of a tile
};

PagedPlan paged_plan(const jdob_edge_attend_paged_args *a) {
  const int64_t queries = a->max_queries < a->query_rows ? a->max_queries : a->query_rows;  // no sequence has more
  const int64_t room = (int64_t)a->table_width * a->cache.page_size;
  const int64_t keys = a->max_keys < room ? a->max_keys : room;
  const int64_t all = queries * (a->num_heads / a->cache.num_kv_heads);
  const int columns = all <= 16 ? 16 : 32;
  const int64_t tiles = (all + columns - 1) / columns, groups = tiles * a->cache.num_kv_heads * a->num_sequences;
  // about four workgroups for each place that the chip has for one (two a compute unit), whose sequences may be
  // of very different lengths, but no fewer than 512 keys each
  int64_t each = groups < 2048 ? (keys * groups + 2047) / 2048 : keys;
  each = each < 512 ? 512 : (each + 127) & ~127;
  int64_t splits = (keys + each - 1) / each;
  if (splits > MAX_SPLITS) {
    each = ((keys + MAX_SPLITS - 1) / MAX_SPLITS + 127) & ~127;
    splits = (keys + each - 1) / each;
  }
  return {tiles, (int)queries, columns, (int)(splits < 1 ? 1 : splits), (int)(each < INT32_MAX ? each : INT32_MAX)};
}

template <typename T, int DP, bool BITS8>
int paged(const PagedParams &p, int columns, bool in_pages, int64_t blocks, hipStream_t stream) {
  if (columns == 16)
    return launch(in_pages ? paged_kernel<T, DP, BITS8, 1, true> : paged_kernel<T, DP, BITS8, 1, false>, blocks,
                  PAGED_WAVES * WAVE, stream, p);
  return launch(in_pages ? paged_kernel<T, DP, BITS8, 2, true> : paged_kernel<T, DP, BITS8, 2, false>, blocks,
                PAGED_WAVES * WAVE, stream, p);
}

// Whether a pool's rows can be read as InPages reads them; 16 rows have to stay within a window, whose offsets pass
// 2^31 nowhere.
bool in_pages(const Pool &x, bool bits8) {
  const int64_t unit = bits8 ? 16 : 8;
  return (uintptr_t)x.at % 16 == 0 && x.page % unit == 0 && x.head % unit == 0 && x.slot % unit == 0 && x.slot < (1 << 24) &&
         (!bits8 || x.scale_slot == 1);
}

template <typename T, bool BITS8>
int paged(const PagedParams &p, const PagedPlan &f, hipStream_t stream) {
  // (8-bit keys are read 16 elements at once up to 64, and beyond 96 to 128)
  const bool in = p.c.page_size % 16 == 0 && in_pages(p.c.k, BITS8) && in_pages(p.c.v, BITS8) &&
                  (!BITS8 || p.c.dim % 16 == 0 || (p.c.dim > 64 && p.c.dim <= 96));
  const int64_t groups = (int64_t)p.c.sequences * p.c.kv_heads * f.tiles;
  const int64_t all = (int64_t)p.c.sequences * p.c.kv_heads * f.queries * p.group;
  // (each factor is below 2^31, and tiles are fewer than columns)
  if (f.tiles > MAX_BLOCKS || groups > MAX_BLOCKS || groups * f.splits > MAX_BLOCKS || (f.splits > 1 && all > MAX_BLOCKS))
    return JDOB_ERR_UNSUPPORTED;
  const int64_t blocks = groups * f.splits;
  const int code = p.c.dim <= 64   ? paged<T, 64, BITS8>(p, f.columns, in, blocks, stream)
                   : p.c.dim <= 96 ? paged<T, 96, BITS8>(p, f.columns, in, blocks, stream)
                                   : paged<T, 128, BITS8>(p, f.columns, in, blocks, stream);
  if (code != JDOB_OK || f.splits == 1) return code;
  return launch(paged_join_kernel<T>, all, JOIN_THREADS, stream, p);
}

}  // namespace
}  // namespace edge

extern "C" int64_t jdob_edge_attend_paged_workspace(const jdob_edge_attend_paged_args *a) {
  using namespace edge;
  if (paged_check_sizes(a) != JDOB_OK) return -1;
  if (!has_work(a)) return 0;
  const PagedPlan f = paged_plan(a);
  if (f.splits == 1) return 0;
  return (int64_t)a->num_sequences * a->cache.num_kv_heads * f.tiles * f.splits * f.columns * (a->cache.head_dim + 4) *
         (int64_t)sizeof(float);
}

extern "C" int jdob_edge_attend_paged(const jdob_edge_attend_paged_args *a, void *hip_stream) {
  using namespace edge;
  int code = paged_check_sizes(a);
  if (code != JDOB_OK || !has_work(a)) return code;
  code = cache_check_arrays(a->cache, a->table_width, a->table, a->table_stride, a->query_start, a->key_count);
  if (code != JDOB_OK) return code;
  if (!a->q || !a->out || a->q_stride < 0 || a->q_head_stride < 0) return JDOB_ERR_INVALID_ARG;
  // rows and heads of out that are written at once must not share elements
  if ((a->query_rows > 1 && a->out_stride < a->cache.head_dim) || (a->num_heads > 1 && a->out_head_stride < a->cache.head_dim) ||
      a->out_stride < 0 || a->out_head_stride < 0)
    return JDOB_ERR_INVALID_ARG;
  const int64_t need = jdob_edge_attend_paged_workspace(a);
  if (need > 0 && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return JDOB_ERR_INVALID_ARG;
  const PagedPlan f = paged_plan(a);
  const PagedParams p = {pages_of(a->cache, a->num_sequences, a->table_width, a->table, a->table_stride, a->query_start,
                                  a->key_count),
                         a->num_heads, a->num_heads / a->cache.num_kv_heads, f.queries, f.columns,
                         a->scale * 1.44269504088896f, a->query_rows, (const char *)a->q, (char *)a->out, a->q_stride,
                         a->q_head_stride, a->out_stride, a->out_head_stride, f.splits, f.each, (int)f.tiles,
                         (float *)a->workspace};
  hipStream_t stream = (hipStream_t)hip_stream;
  if (a->cache.dtype == JDOB_EDGE_BF16)
    return a->cache.bits8 ? paged<__bf16, true>(p, f, stream) : paged<__bf16, false>(p, f, stream);
  return a->cache.bits8 ? paged<_Float16, true>(p, f, stream) : paged<_Float16, false>(p, f, stream);
}
