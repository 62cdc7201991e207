// Causal attention of packed sequences of different lengths with grouped heads.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - max),  j <= m - n + i
//
// One pass over the keys: a running maximum and sum per row, the output rescaled when the maximum
// grows.  The products are formed transposed: S^T = K Q^T puts one query row in one lane (twice: the
// two halves of a wave hold other keys of it), so maxima and sums are the lane's own but for one
// exchange, and the lane's p are, without any movement, the second operand of O^T = V^T P^T; V's
// columns come from LDS by transposing reads whose order of keys is that of p.
//
// Two kernels.  `prompt_kernel`: many rows, each wave 32 of them, all waves of a workgroup share the
// staged keys.  `few_kernel`: few rows after a long history, where the rows of all heads that read
// one key head stand together as 32 columns, each wave takes other keys, and the keys are split
// over workgroups, whose partial results `join_kernel` puts together.
//
// p is rounded to dtype for its product with v, its sum is not.  Against 64 bits that makes the output's error
// 2.0e-3 with prompts and 2.3e-3 with tokens where its own rounding to bfloat16 alone makes 1.6e-3 and 1.7e-3.
// With p in two parts, the rounded one and what it left, the errors are those; a prompt of 16,384 rows then takes
// 1.49 ms for 1.02, ragged prompts 214 us for 184, tokens 136 us for 131.
//
// Measured (kernel alone): 16,384 rows with 16 heads of 128 1.02-1.09 ms (1.0-1.08 PFLOP/s); 32 prompts of
// 40 to 1000 rows 180-220 us (their rows, keys and values move in 69 us, their products take 60 at a
// library's rate); one row of 32 heads after 131,071 keys 109 us (4.9 TB/s) and 10 us for the join.
// Many rows are bound by instructions: the matrix units are busy 58 % of the time (27 % with the short
// prompts, whose tiles' beginnings cost as much as their products), the vector units for p nearly as
// long, in turn within a wave and only by chance at once in two.  Few rows are bound by HBM.
#include "edge_common.h"

namespace edge {
namespace {

struct AttendParams {
  int sequences, heads, kv_heads, group, dim, max_queries;
  float scale;  // times log2(e)
  int64_t query_rows, key_rows;
  const char *q, *k, *v;
  char *out;
  int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head, out_stride, out_head;  // elements
  const int *query_start;
  const int64_t *key_start;
  const int *key_count;
  int splits, each;   // few: splits of the keys, keys of one
  int tiles;          // few: tiles of 32 columns of a sequence; prompt: tiles of rows of all
  float *part;        // few: [sequence][key head][tile][split][32 columns][dim + 2]
};

template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
  typedef bf16x8 frag;
  __device__ static f32x16 m32(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<_Float16> {
  typedef f16x8 frag;
  __device__ static f32x16 m32(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

typedef short s16x4 __attribute__((ext_vector_type(4)));

// A sequence's rows and keys, kept within the arrays whatever the index arrays hold.
struct Sequence {
  int64_t row, key;
  int rows, keys;
};

__device__ inline Sequence sequence(const AttendParams &p, int u) {
  int64_t at = p.query_start[u], end = p.query_start[u + 1];
  at = at < 0 ? 0 : at < p.query_rows ? at : p.query_rows;
  end = end < at ? at : end < p.query_rows ? end : p.query_rows;
  int64_t key = p.key_start[u], count = p.key_count[u];
  key = key < 0 ? 0 : key < p.key_rows ? key : p.key_rows;
  count = count < 0 ? 0 : count < p.key_rows - key ? count : p.key_rows - key;
  return {at, key, (int)(end - at), (int)count};
}

__device__ const u32x4 attend_zeros = {0, 0, 0, 0};

// Staged keys or values: rows of DP elements, 16-byte chunks exchanged within the row so that what LDS
// serves at once (256 bytes) falls on different banks.  Keys are read 16 bytes a lane, equal chunks of
// rows 0-3, 12-15, 20-23 and 24-27 at once, then of the others; values 8 bytes a lane, four rows' equal
// 64 bytes at once.  (With keys exchanged by r & 7 and values by twice that, every read took twice its
// time.)
template <int DP>
__device__ inline int key_swap(int r) {
  return DP == 128 ? r & 15 : DP == 96 ? r >> 2 & 3 : r >> 1 & 7;
}
template <int DP>
__device__ inline int value_swap(int r) {
  return DP == 128 ? (r & 3) << 2 : DP == 96 ? 0 : (r >> 1 & 1) << 2;
}
template <int DP>
__device__ inline int key_spot(int r, int c) {
  return r * (DP * 2) + ((c ^ key_swap<DP>(r)) << 4);
}
template <int DP>
__device__ inline int value_spot(int r, int c) {
  return r * (DP * 2) + ((c ^ value_swap<DP>(r)) << 4);
}

// Stages keys first .. first + COUNT - 1 of `count` by THREADS threads, of which this is number `t` and
// its wave's first is t0: zeros behind the last key.  Behind `dim`, where queries are zero and the output
// is not stored, stand zeros, or unless `careful` any of the row's own elements (their product with zero
// is zero but for infinities and NaN).  DIRECT: memory to LDS, without registers between.
template <typename T, int DP, bool DIRECT, bool VALUES, int COUNT, int THREADS>
__device__ inline void stage(char *dst, const T *base, int64_t stride, int64_t first, int count, int dim, bool careful,
                             int t, int t0) {
  constexpr int CH = DP / 8;
  static_assert(COUNT * CH % THREADS == 0, "whole rounds");
  const T *const tile = base + first * stride;
  auto each = [&](auto one) {
#pragma unroll
    for (int i = 0; i < COUNT * CH / THREADS; ++i) {
      const int slot = i * THREADS + t, r = slot / CH;
      one(i * THREADS, r, (slot % CH) ^ (VALUES ? value_swap<DP>(r) : key_swap<DP>(r)));
    }
  };
  const unsigned to = lds_address(dst) + t0 * 16;
  if constexpr (!DIRECT) {
    each([&](int s0, int r, int c) {
      u32x4 x = {0, 0, 0, 0};
      if (first + r < count && c * 8 < dim)
        x = __builtin_bit_cast(u32x4, *(const typename Raw<unsigned short, 8>::type *)(tile + r * stride + c * 8));
      *(u32x4 *)(dst + (s0 + t) * 16) = x;
    });
  } else if (first + COUNT <= count && !careful) {
    each([&](int s0, int r, int c) {
      load_to_lds(tile, (unsigned)r * (unsigned)(stride * 2) + (c * 8 < dim ? c * 16 : 0), to + s0 * 16);
    });
  } else {
    each([&](int s0, int r, int c) {
      const bool in = first + r < count && c * 8 < dim;
      load_to_lds(in ? (const void *)(tile + r * stride + c * 8) : (const void *)&attend_zeros, to + s0 * 16);
    });
  }
}

// The running state of 32 rows in a wave: lane l and l + 32 hold row l % 32.
template <int DP>
struct State {
  float top, sum;           // the maximum so far (of q.k; -inf: nothing seen yet), this half's sum
  f32x16 out[DP / 32];      // out[d][e]: column 32 d + 8 (e / 4) + 4 half + e % 4

  __device__ void clear();
  __device__ bool has_nan() const {
    bool bad = sum != sum;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) bad |= out[d][e] != out[d][e];
    return bad;
  }
};

__device__ inline float other_half(float x) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(threadIdx.x % WAVE < 32 ? both[1] : both[0]);
}

// What a row's scores are taken relative to: its maximum, or 0 where it has seen nothing (masked scores
// are -inf, and -inf - -inf would be NaN).
__device__ inline float base_of(float top) { return top == -INFINITY ? 0.0f : top; }

template <int DP>
__device__ void State<DP>::clear() {
  top = -INFINITY;
  sum = 0.0f;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) out[d] = (f32x16){};
}

constexpr float GROWTH = 8.0f;  // the maximum may lag behind by this much (p up to 2^8) before out is rescaled
// Up to here (log2 units) sc * scale - top * scale may be formed with one rounding of top * scale: it puts p
// off by at most a factor of two, the same for all of a row, which its sum takes back.
constexpr float NEAR = 0x1p24f;

// Scores of 32 rows with KT * 32 staged keys, softmax, and the values' sums.  The lane's row sees the
// tile's keys 0 .. sees; MASKED: some key of the tile lies behind that for some row.
// LDS is read well before its use, a group at a time: left to itself the compiler reads each operand
// right before its product and waits for it.
template <typename T, int DP, int KT, bool MASKED, int GROUP = 4>
__device__ inline void attend_tile(State<DP> &s, const typename Mma<T>::frag (&q)[DP / 16], const char *keys,
                                   const char *values, int sees, float scale) {
  typedef typename Mma<T>::frag frag;
  const int lane = threadIdx.x % WAVE, l32 = lane % 32, half = lane / 32, l16 = lane % 16, g16 = lane / 16;
  constexpr int N = KT * DP / 16, G = N % GROUP == 0 ? GROUP : 3;  // operands in all, and in a group
  static_assert(N % G == 0, "whole groups");
  f32x16 sc[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) sc[t] = (f32x16){};
  frag kf[2][G];
  auto fetch_keys = [&](int g) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int t = (g * G + i) % KT, c = (g * G + i) / KT;
      kf[g & 1][i] = *(const frag *)(keys + key_spot<DP>(t * 32 + l32, c * 2 + half));
    }
  };
  fetch_keys(0);
#pragma unroll
  for (int g = 0; g < N / G; ++g) {
    if (g + 1 < N / G) fetch_keys(g + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int t = (g * G + i) % KT, c = (g * G + i) / KT;
      sc[t] = Mma<T>::m32(kf[g & 1][i], q[c], sc[t]);
    }
  }
  // columns 32 d .. 32 d + 31 of 16 keys: the transposing reads give a lane four keys of one column
  struct Pair { s16x4 lo, hi; };
  auto fetch = [&](Pair (&vf)[DP / 32], int b) {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      const int c = d * 4 + (g16 % 2) * 2 + l16 % 4 / 2, r = b * 16 + half * 4 + l16 / 4;
      vf[d].lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4 *)(values + value_spot<DP>(r, c) + l16 % 2 * 8));
      vf[d].hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4 *)(values + value_spot<DP>(r + 8, c) + l16 % 2 * 8));
    }
  };
  Pair vf[2][DP / 32];
  fetch(vf[0], 0);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (MASKED) {
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        sc[t][e] = t * 32 + 8 * (e / 4) + 4 * half + e % 4 <= sees ? sc[t][e] : -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[t][e]);
  top = fmaxf(top, other_half(top));
  // (false where neither has seen anything: -inf - -inf is NaN)
  const bool grows = (top - s.top) * scale > GROWTH;
  if (__any(grows)) {
    // a row's own scores decide for it: what other rows of the wave see does not change its roundings
    const float next = grows ? top : s.top;
    // (nothing has been seen yet: out is zero, or holds infinities that are to stay)
    const float f = s.top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((s.top - next) * scale);
    s.top = next;
    s.sum *= f;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) s.out[d] *= f;
  }
  float times = scale, base = base_of(s.top) * scale;
  const bool far = !(fabsf(base) < NEAR);
  if (__any(far)) {
    // the difference first, again row by row
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[t][e] = far ? (sc[t][e] - s.top) * scale : sc[t][e];
    times = far ? 1.0f : times;
    base = far ? 0.0f : base;
  }
  frag p[KT * 2];
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = __builtin_amdgcn_exp2f(sc[t][e] * times - base);
      s.sum += x;
      p[t * 2 + e / 8][e % 8] = (T)x;
    }
#pragma unroll
  for (int b = 0; b < KT * 2; ++b) {
    if (b + 1 < KT * 2) fetch(vf[(b + 1) & 1], b + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) s.out[d] = Mma<T>::m32(__builtin_bit_cast(frag, vf[b & 1][d]), p[b], s.out[d]);
  }
}

// Whether the wave finds an infinity or a NaN among KEYS staged values.
template <typename T, int DP, int KEYS>
__device__ inline bool any_non_finite(const char *values) {
  const int lane = threadIdx.x % WAVE;
  constexpr unsigned EXP = sizeof(T) == 2 && __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
  bool bad = false;
  for (int i = lane; i < KEYS * DP / 8; i += WAVE) {
    const u32x4 x = *(const u32x4 *)(values + i * 16);
#pragma unroll
    for (int c = 0; c < 4; ++c) bad |= (x[c] & EXP) == EXP || (x[c] >> 16 & EXP) == EXP;
  }
  return __any(bad);
}

// Replaces the staged values' infinities and NaN by zeros after adding them to the rows that see them
// (their products with p = 0 of rows that do not would be NaN).  Rare, and slow.
template <typename T, int DP, int KEYS>
__device__ inline void take_non_finite(State<DP> &s, char *values, int sees) {
  constexpr unsigned EXP = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
  const int half = threadIdx.x % WAVE / 32;
  for (int r = 0; r < KEYS; ++r)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int at = 32 * d + 8 * (e / 4) + 4 * half + e % 4;
        const T x = *(const T *)(values + value_spot<DP>(r, at / 8) + at % 8 * 2);
        const unsigned bits = __builtin_bit_cast(unsigned short, x);
        if ((bits & EXP) == EXP && r <= sees) s.out[d][e] += (float)x;
      }
}

template <typename T, int DP, int KEYS, int THREADS>
__device__ inline void clear_non_finite(char *values, int t) {
  constexpr unsigned EXP = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
  for (int i = t; i < KEYS * DP; i += THREADS) {
    unsigned short *x = (unsigned short *)values + i;
    if ((*x & EXP) == EXP) *x = 0;
  }
}

// Eight elements of a query row, zeros behind `dim`.
template <typename T>
__device__ inline typename Mma<T>::frag query(const T *row, int c, int dim, bool have) {
  typename Mma<T>::frag f = {};
  if (have && c * 8 < dim) f = *(const typename Raw<T, 8>::type *)(row + c * 8);
  return f;
}

// ------------------------------------------------------------------ many rows

constexpr int PROMPT_WAVES = 4, PROMPT_ROWS = 32 * PROMPT_WAVES, PROMPT_KEYS = 64;

__device__ inline int64_t lane_of(int64_t x, int lane) {
  return (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}

// Which sequence and which of its tiles a tile index stands for: the sequences' tiles follow each
// other.  False behind the last one.
__device__ inline bool find_tile(const AttendParams &p, int tile, int *t, Sequence *q) {
  const int lane = threadIdx.x % WAVE;
  int before = 0;
  for (int u0 = 0; u0 < p.sequences; u0 += WAVE) {
    Sequence mine = {0, 0, 0, 0};
    if (u0 + lane < p.sequences) mine = sequence(p, u0 + lane);
    const int n = (mine.rows + PROMPT_ROWS - 1) / PROMPT_ROWS;
    int upto = n;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) {
      const int x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    const unsigned long long past = __ballot(before + upto > tile);
    if (past) {
      const int l = __builtin_ctzll(past);
      *q = {lane_of(mine.row, l), lane_of(mine.key, l), __builtin_amdgcn_readlane(mine.rows, l),
            __builtin_amdgcn_readlane(mine.keys, l)};
      *t = before + __builtin_amdgcn_readlane(upto, l) - 1 - tile;  // the last rows see most: first
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, WAVE - 1);
  }
  return false;
}

template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(PROMPT_WAVES *WAVE, 2) void prompt_kernel(AttendParams p) {
  typedef typename Mma<T>::frag frag;
  constexpr int THREADS = PROMPT_WAVES * WAVE, BYTES = PROMPT_KEYS * DP * 2;
  // two buffers of keys and values; the waves' rows (32 each) come in through the second
  __shared__ __align__(16) char room[4 * BYTES];
  static_assert(2 * BYTES >= PROMPT_ROWS * DP * 2, "room for the rows");
  const int lane = threadIdx.x % WAVE, wave = wave_index(), l32 = lane % 32, half = lane / 32;
  // Workgroups go to the chip's eight dies in turn: heads that read one key head should share a die's cache.
  const int kv = block_index() % p.heads % p.kv_heads, head = kv * p.group + block_index() % p.heads / p.kv_heads;
  const int tile = block_index() / p.heads;
  int t;
  Sequence q;
  if (!find_tile(p, tile, &t, &q)) return;
  const int row0 = t * PROMPT_ROWS, wave_row = row0 + wave * 32, mine = wave_row + l32;
  const int shift = q.keys - q.rows;  // row i sees keys 0 .. shift + i
  const T *const k = (const T *)p.k + q.key * p.k_stride + kv * p.k_head;
  const T *const v = (const T *)p.v + q.key * p.v_stride + kv * p.v_head;
  const int last_row = (row0 + PROMPT_ROWS < q.rows ? row0 + PROMPT_ROWS : q.rows) - 1;
  const int seen = shift + last_row + 1;  // keys that some row of the workgroup sees
  const int tiles = seen > 0 ? (seen - 1) / PROMPT_KEYS + 1 : 0;  // (counts of keys go up to 2^31 - 1)
  // tiles that all rows of the workgroup see
  const int whole = shift + row0 < 0 ? 0 : (shift + row0 + 1) / PROMPT_KEYS;
  // the last key that the wave's last row sees (-1: it has no rows, or they see nothing)
  const int wave_last = wave_row + 31 < last_row ? wave_row + 31 : last_row;
  const int wave_any = wave_row <= last_row ? shift + wave_last : -1;
  const int limit = shift + (mine < last_row ? mine : last_row);
  bool careful = false;
  auto keys = [&](int kt) { return room + (kt & 1) * 2 * BYTES; };
  auto values = [&](int kt) { return room + ((kt & 1) * 2 + 1) * BYTES; };
  auto load = [&](int kt) {
    stage<T, DP, DIRECT, false, PROMPT_KEYS, THREADS>(keys(kt), k, p.k_stride, (int64_t)kt * PROMPT_KEYS, q.keys, p.dim,
                                                      careful, threadIdx.x, wave * WAVE);
    stage<T, DP, DIRECT, true, PROMPT_KEYS, THREADS>(values(kt), v, p.v_stride, (int64_t)kt * PROMPT_KEYS, q.keys, p.dim,
                                                     careful, threadIdx.x, wave * WAVE);
  };
  auto advance = [&](int kt) {
    wait_loads<0>();
    barrier();
    if (kt + 1 < tiles) load(kt + 1);
  };
  // The wave's rows come through its corner of the second buffers and leave through the same corner of all:
  // a lane a row, straight from and to memory, took 128 us for 32 prompts' 272 MB of them.
  char *const corner = room + wave * 32 * DP * 2;
  frag qf[DP / 16];
  if constexpr (DIRECT) {
    const int valid = last_row - wave_row + 1;  // (rows behind them are copies)
    const T *const rows = (const T *)p.q + (q.row + wave_row) * p.q_stride + head * p.q_head;
    const unsigned to = lds_address(corner + 2 * BYTES);
#pragma unroll
    for (int i = 0; i < 32 * DP / 8 / WAVE; ++i) {
      const int slot = i * WAVE + lane, r = slot / (DP / 8), c = (slot % (DP / 8)) ^ key_swap<DP>(r);
      const T *const from = rows + (int64_t)(r < valid ? r : valid - 1) * p.q_stride + c * 8;
      load_to_lds(c * 8 < p.dim ? (const void *)from : (const void *)&attend_zeros, to + i * WAVE * 16);
    }
    if (tiles > 0) load(0);
    if (tiles > 0) {
      wait_loads<2 * BYTES / 16 / THREADS>();
    } else {
      wait_loads<0>();
    }
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) qf[c] = *(const frag *)(corner + 2 * BYTES + key_spot<DP>(l32, c * 2 + half));
  } else {
    if (tiles > 0) load(0);
    const T *const qrow = (const T *)p.q + (q.row + (mine < q.rows ? mine : 0)) * p.q_stride + head * p.q_head;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) qf[c] = query<T>(qrow, c * 2 + half, p.dim, mine < q.rows);
  }
  State<DP> s;
  s.clear();
  int kt = 0;
  for (; kt < whole; ++kt) {
    advance(kt);
    if (wave_row <= last_row)
      attend_tile<T, DP, PROMPT_KEYS / 32, false>(s, qf, keys(kt), values(kt), 0, p.scale);
  }
  for (; kt < tiles; ++kt) {
    advance(kt);
    const int first = kt * PROMPT_KEYS;
    if (first > wave_any) continue;  // the wave's rows see nothing of this tile
    attend_tile<T, DP, PROMPT_KEYS / 32, true>(s, qf, keys(kt), values(kt), limit - first, p.scale);
  }
  // A NaN may come from a value that its row does not see (p = 0 times an infinity): once more, with care.
  if (__syncthreads_or(mine < q.rows && s.has_nan())) {
    careful = true;
    s.clear();
    if (tiles > 0) load(0);
    for (kt = 0; kt < tiles; ++kt) {
      advance(kt);
      const int first = kt * PROMPT_KEYS;
      char *const v_now = values(kt);
      if (any_non_finite<T, DP, PROMPT_KEYS>(v_now)) {  // the same for all waves
        take_non_finite<T, DP, PROMPT_KEYS>(s, v_now, limit - first);
        __syncthreads();
        clear_non_finite<T, DP, PROMPT_KEYS, THREADS>(v_now, threadIdx.x);
        __syncthreads();
      }
      attend_tile<T, DP, PROMPT_KEYS / 32, true>(s, qf, keys(kt), v_now, limit - first, p.scale);
    }
  }
  const float sum = s.sum + other_half(s.sum), f = sum > 0.0f ? 1.0f / sum : sum;
  __syncthreads();  // the last keys and values have been read
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y[4] = {s.out[d][4 * e] * f, s.out[d][4 * e + 1] * f, s.out[d][4 * e + 2] * f, s.out[d][4 * e + 3] * f};
      store_f32<T, 4>((T *)(corner + key_spot<DP>(l32, d * 4 + e) + half * 8), y);
    }
  lanes_meet();
  T *const out = (T *)p.out + (q.row + wave_row) * p.out_stride + head * p.out_head;
#pragma unroll
  for (int i = 0; i < 32 * DP / 8 / WAVE; ++i) {
    const int slot = i * WAVE + lane, r = slot / (DP / 8), c = slot % (DP / 8);
    if (wave_row + r < q.rows && c * 8 < p.dim)
      *(typename Raw<T, 8>::type *)(out + r * p.out_stride + c * 8) = *(const frag *)(corner + key_spot<DP>(r, c));
  }
}

// ------------------------------------------------------------------ few rows

constexpr int FEW_WAVES = 2, FEW_COLUMNS = 32, FEW_KEYS = 32;

// A workgroup takes 32 columns (rows times the heads of one key head) and `each` keys of them; its
// waves take 32 keys in turn, each staged in the wave's own two buffers, so that no wave waits for
// another before the end.  (Heads to 64 leave registers for two waves a SIMD, if the compiler is told to.)
template <typename T, int DP, bool DIRECT>
__global__ __launch_bounds__(FEW_WAVES *WAVE, DP == 64 ? 2 : 1) void few_kernel(AttendParams p) {
  typedef typename Mma<T>::frag frag;
  constexpr int THREADS = FEW_WAVES * WAVE, BYTES = FEW_KEYS * DP * 2, CORNER = 4 * BYTES;
  constexpr int LOADS = 2 * BYTES / (WAVE * 16), MIX = FEW_WAVES * 32 * (DP + 4) * 4;
  __shared__ __align__(16) char room[FEW_WAVES * CORNER > MIX ? FEW_WAVES * CORNER : MIX];
  __shared__ float tops[FEW_WAVES][32], sums[FEW_WAVES][32];
  const int lane = threadIdx.x % WAVE, wave = wave_index(), l32 = lane % 32, half = lane / 32;
  const int kv = block_index() % p.kv_heads, split = block_index() / p.kv_heads % p.splits;
  const int tile = block_index() / p.kv_heads / p.splits % p.tiles, u = block_index() / p.kv_heads / p.splits / p.tiles;
  if (u >= p.sequences) return;
  const Sequence q = sequence(p, u);
  const int rows = q.rows < p.max_queries ? q.rows : p.max_queries;
  const int columns = rows * p.group, column = tile * FEW_COLUMNS + l32;
  if (tile * FEW_COLUMNS >= columns) return;
  // this split's keys; the last split takes what the others leave (max_keys may be too small)
  const int64_t from = (int64_t)split * p.each;
  const int64_t until = split + 1 < p.splits && from + p.each < q.keys ? from + p.each : q.keys;
  if (from >= until && split > 0) return;
  const bool have = column < columns;
  const int row = have ? column / p.group : 0, head = kv * p.group + (have ? column % p.group : 0);
  const int shift = q.keys - q.rows, limit = have ? shift + row : -1;
  const T *const qrow = (const T *)p.q + (q.row + row) * p.q_stride + head * p.q_head;
  frag qf[DP / 16];
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) qf[c] = query<T>(qrow, c * 2 + half, p.dim, have);
  const T *const k = (const T *)p.k + q.key * p.k_stride + kv * p.k_head;
  const T *const v = (const T *)p.v + q.key * p.v_stride + kv * p.v_head;
  const int first_limit = shift + tile * FEW_COLUMNS / p.group;  // of the tile's first row
  State<DP> s;
  char *const corner = room + wave * CORNER;
  auto keys_of = [&](bool careful) {
    s.clear();
    auto load = [&](int b, int64_t first) {
      stage<T, DP, DIRECT, false, FEW_KEYS, WAVE>(corner + b * 2 * BYTES, k, p.k_stride, first, q.keys, p.dim, careful, lane, 0);
      stage<T, DP, DIRECT, true, FEW_KEYS, WAVE>(corner + (b * 2 + 1) * BYTES, v, p.v_stride, first, q.keys, p.dim, careful,
                                                 lane, 0);
    };
    int64_t first = from + wave * FEW_KEYS;  // passes 2^31 behind the longest sequence's end
    int b = 0;
    if (first < until) load(0, first);
    for (; first < until; first += FEW_WAVES * FEW_KEYS, b ^= 1) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the other buffer has been read
      if (first + FEW_WAVES * FEW_KEYS < until) {
        load(b ^ 1, first + FEW_WAVES * FEW_KEYS);
        if constexpr (DIRECT) wait_loads<LOADS>();
      } else if constexpr (DIRECT) {
        wait_loads<0>();
      }
      const char *const keys = corner + b * 2 * BYTES;
      char *const values = corner + (b * 2 + 1) * BYTES;
      // keys behind `until` are the next split's (or none)
      const int64_t last = limit < until - 1 ? limit : until - 1;
      if (first + FEW_KEYS - 1 <= first_limit && first + FEW_KEYS <= until && !careful) {
        attend_tile<T, DP, 1, false>(s, qf, keys, values, 0, p.scale);
        continue;
      }
      if (careful && any_non_finite<T, DP, FEW_KEYS>(values)) {
        take_non_finite<T, DP, FEW_KEYS>(s, values, (int)(last - first));
        // the wave's own values: its lanes run together, their LDS accesses in order
        lanes_meet();
        clear_non_finite<T, DP, FEW_KEYS, WAVE>(values, lane);
        lanes_meet();
      }
      attend_tile<T, DP, 1, true>(s, qf, keys, values, (int)(last - first), p.scale);
    }
  };
  keys_of(false);
  // A NaN may come from a value that its row does not see (p = 0 times an infinity): once more, with care.
  if (__any(have && s.has_nan())) keys_of(true);
  // the waves' results: each column's maximum, then sums and outputs relative to it
  s.sum += other_half(s.sum);
  if (half == 0) {
    tops[wave][l32] = s.top;
    sums[wave][l32] = s.sum;
  }
  __syncthreads();  // also: the staged keys have been read
  float top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) top = fmaxf(top, tops[w][l32]);
  const float base = base_of(top);
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) sum += sums[w][l32] * __builtin_amdgcn_exp2f((tops[w][l32] - base) * p.scale);
  const float f = __builtin_amdgcn_exp2f((s.top - base) * p.scale);
  float *const mix = (float *)room;  // [wave][column][DP + 4]
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 y = {s.out[d][4 * e] * f, s.out[d][4 * e + 1] * f, s.out[d][4 * e + 2] * f, s.out[d][4 * e + 3] * f};
      *(f32x4 *)(mix + (wave * 32 + l32) * (DP + 4) + 32 * d + 8 * e + 4 * half) = y;
    }
  __syncthreads();  // also: the waves' maxima and sums have been read
  if (wave == 0 && half == 0) sums[0][l32] = sum, tops[0][l32] = top;
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * (DP / 4); i += THREADS) {
    const int c = i / (DP / 4), at = i % (DP / 4) * 4, col = tile * FEW_COLUMNS + c;
    if (col >= columns || at >= p.dim) continue;
    f32x4 y = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) y += *(const f32x4 *)(mix + (w * 32 + c) * (DP + 4) + at);
    if (p.splits == 1) {
      const float g = sums[0][c] > 0.0f ? 1.0f / sums[0][c] : sums[0][c];
      const float z[4] = {y[0] * g, y[1] * g, y[2] * g, y[3] * g};
      T *const out = (T *)p.out + (q.row + col / p.group) * p.out_stride + (kv * p.group + col % p.group) * p.out_head;
      store_f32<T, 4>(out + at, z);
    } else {
      const int64_t group = ((int64_t)u * p.kv_heads + kv) * p.tiles + tile, pitch = p.dim + 4;
      float *const part = p.part + ((group * p.splits + split) * 32 + c) * pitch;
      *(f32x4 *)(part + at) = y;
      if (at == 0) part[p.dim] = tops[0][c], part[p.dim + 1] = sums[0][c];
    }
  }
}

constexpr int MAX_SPLITS = 256, JOIN_THREADS = 256;

// A workgroup puts one column's partial results together.
template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(AttendParams p) {
  __shared__ float weight[MAX_SPLITS], mix[8][128];
  const int columns_each = p.max_queries * p.group;
  const int kv = block_index() % p.kv_heads, col = block_index() / p.kv_heads % columns_each;
  const int u = block_index() / p.kv_heads / columns_each, tile = col / FEW_COLUMNS;
  if (u >= p.sequences) return;
  const Sequence q = sequence(p, u);
  const int rows = q.rows < p.max_queries ? q.rows : p.max_queries;
  if (col >= rows * p.group) return;
  const int64_t pitch = p.dim + 4, step = 32 * pitch;
  const float *const part = p.part + (((int64_t)u * p.kv_heads + kv) * p.tiles + tile) * p.splits * step + col % FEW_COLUMNS * pitch;
  const int used = q.keys > 0 ? (q.keys - 1) / p.each + 1 : 1, splits = used < p.splits ? used : p.splits;
  const int t = threadIdx.x, lane = t % WAVE;
  // every wave for itself: the maximum, the weights, their sum
  float tops[MAX_SPLITS / WAVE], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < MAX_SPLITS / WAVE; ++i) {
    tops[i] = i * WAVE + lane < splits ? part[(i * WAVE + lane) * step + p.dim] : -INFINITY;
    top = fmaxf(top, tops[i]);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float base = base_of(top);
#pragma unroll
  for (int i = 0; i < MAX_SPLITS / WAVE; ++i)
    if (i * WAVE + lane < splits) {
      const float w = __builtin_amdgcn_exp2f((tops[i] - base) * p.scale);
      sum += w * part[(i * WAVE + lane) * step + p.dim + 1];
      if (t < WAVE) weight[i * WAVE + lane] = w;
    }
  sum = wave_sum(sum);
  __syncthreads();
  const int at = t % 32 * 4, g = t / 32;
  f32x4 y = {0, 0, 0, 0};
  if (at < p.dim) {
#pragma unroll 4
    for (int i = g; i < splits; i += 8) y += *(const f32x4 *)(part + i * step + at) * weight[i];
    *(f32x4 *)(mix[g] + at) = y;
  }
  __syncthreads();
  if (t < p.dim) {
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) z += mix[i][t];
    T *const out = (T *)p.out + (q.row + col / p.group) * p.out_stride + (kv * p.group + col % p.group) * p.out_head;
    out[t] = (T)(z * (sum > 0.0f ? 1.0f / sum : sum));
  }
}

// ------------------------------------------------------------------ host side

int attend_check(const jdob_edge_attend_args *a, bool sizes_only) {
  if (!a || a->num_sequences < 0 || a->num_heads < 1 || a->num_kv_heads < 1 || a->num_heads % a->num_kv_heads ||
      a->head_dim < 1 || a->max_queries < 0 || a->max_keys < 0 || a->query_rows < 0 || a->key_rows < 0 ||
      !(a->scale > 0.0f) || !isfinite(a->scale))
    return JDOB_ERR_INVALID_ARG;
  if (a->dtype != JDOB_EDGE_BF16 && a->dtype != JDOB_EDGE_F16) return JDOB_ERR_UNSUPPORTED;
  if (a->head_dim > JDOB_EDGE_MAX_HEAD_DIM || a->head_dim % 8 || a->num_heads > 1024 ||
      a->num_sequences > JDOB_EDGE_MAX_SEQUENCES || a->query_rows > JDOB_EDGE_MAX_ROWS)
    return JDOB_ERR_UNSUPPORTED;
  if (sizes_only || a->num_sequences == 0 || a->query_rows == 0 || a->max_queries == 0) return JDOB_OK;
  if (!a->q || !a->out || !a->query_start || !a->key_start || !a->key_count || (a->key_rows > 0 && (!a->k || !a->v)))
    return JDOB_ERR_INVALID_ARG;
  if (a->q_stride < 0 || a->q_head_stride < 0 || a->k_stride < 0 || a->k_head_stride < 0 || a->v_stride < 0 ||
      a->v_head_stride < 0 || a->out_stride < 0 || a->out_head_stride < 0)
    return JDOB_ERR_INVALID_ARG;
  // rows and heads of out that are written at once must not share elements
  if ((a->query_rows > 1 && a->out_stride < a->head_dim) || (a->num_heads > 1 && a->out_head_stride < a->head_dim))
    return JDOB_ERR_INVALID_ARG;
  const int64_t need = jdob_edge_attend_workspace(a);
  if (need > 0 && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need))
    return JDOB_ERR_INVALID_ARG;
  return JDOB_OK;
}

struct FewPlan {
  bool few;
  int tiles, splits, each;
};

FewPlan few_plan(const jdob_edge_attend_args *a) {
  const int64_t columns = (int64_t)a->max_queries * (a->num_heads / a->num_kv_heads);
  const int64_t tiles = (columns + FEW_COLUMNS - 1) / FEW_COLUMNS;
  const int64_t groups = tiles * a->num_kv_heads * a->num_sequences;
  // Many rows take prompt_kernel, whose workgroups stage each key once for 128 rows of one head, unless
  // that gives the chip too few workgroups for the keys there are: 64 rows of 32 heads after 20,000 keys
  // (32 workgroups) take 369 us there and 100 us here.
  const int64_t prompts = (a->query_rows / PROMPT_ROWS + a->num_sequences) * a->num_heads;
  const bool long_keys = prompts < 256 && a->max_keys >= 1024 && columns <= 4096;
  if ((columns > 128 && !long_keys) || groups > (1 << 24)) return {false, 0, 0, 0};
  // about four workgroups for each place that the chip has for one (two a compute unit), whose
  // sequences may be of very different lengths, but no fewer than 512 keys each
  int64_t each = (a->max_keys * groups + 2047) / 2048;
  each = each > a->max_keys ? a->max_keys : each;
  each = each < 512 ? 512 : (each + 63) & ~63;
  int64_t splits = (a->max_keys + each - 1) / each;
  if (splits > MAX_SPLITS) {
    each = (((int64_t)a->max_keys + MAX_SPLITS - 1) / MAX_SPLITS + 63) & ~63;
    splits = (a->max_keys + each - 1) / each;
  }
  return {true, (int)tiles, (int)(splits < 1 ? 1 : splits), (int)(each < INT32_MAX ? each : INT32_MAX)};
}

template <typename T, int DP>
int attend(AttendParams p, bool few, bool direct, hipStream_t stream) {
  if (few) {
    const int64_t groups = (int64_t)p.sequences * p.kv_heads * p.tiles;
    const int64_t columns = (int64_t)p.sequences * p.kv_heads * p.max_queries * p.group;
    if (groups * p.splits > MAX_BLOCKS || columns > MAX_BLOCKS) return JDOB_ERR_UNSUPPORTED;
    const int code = direct ? launch(few_kernel<T, DP, true>, groups * p.splits, FEW_WAVES * WAVE, stream, p)
                            : launch(few_kernel<T, DP, false>, groups * p.splits, FEW_WAVES * WAVE, stream, p);
    if (code != JDOB_OK || p.splits == 1) return code;
    return launch(join_kernel<T>, columns, JOIN_THREADS, stream, p);
  }
  const int64_t blocks = (int64_t)p.tiles * p.heads;
  if (blocks > MAX_BLOCKS) return JDOB_ERR_UNSUPPORTED;
  return direct ? launch(prompt_kernel<T, DP, true>, blocks, PROMPT_WAVES * WAVE, stream, p)
                : launch(prompt_kernel<T, DP, false>, blocks, PROMPT_WAVES * WAVE, stream, p);
}

template <typename T>
int attend(const AttendParams &p, bool few, bool direct, hipStream_t stream) {
  if (p.dim <= 64) return attend<T, 64>(p, few, direct, stream);
  return p.dim <= 96 ? attend<T, 96>(p, few, direct, stream) : attend<T, 128>(p, few, direct, stream);
}

}  // namespace
}  // namespace edge

extern "C" int64_t jdob_edge_attend_workspace(const jdob_edge_attend_args *a) {
  using namespace edge;
  if (attend_check(a, true) != JDOB_OK) return -1;
  if (a->num_sequences == 0 || a->query_rows == 0 || a->max_queries == 0) return 0;
  const FewPlan f = few_plan(a);
  if (!f.few || f.splits == 1) return 0;
  return (int64_t)a->num_sequences * a->num_kv_heads * f.tiles * f.splits * 32 * (a->head_dim + 4) * (int64_t)sizeof(float);
}

extern "C" int jdob_edge_attend(const jdob_edge_attend_args *a, void *hip_stream) {
  using namespace edge;
  const int code = attend_check(a, false);
  if (code != JDOB_OK || a->num_sequences == 0 || a->query_rows == 0 || a->max_queries == 0) return code;
  const FewPlan f = few_plan(a);
  AttendParams p = {a->num_sequences, a->num_heads, a->num_kv_heads, a->num_heads / a->num_kv_heads, a->head_dim,
                    a->max_queries, a->scale * 1.44269504088896f, a->query_rows, a->key_rows,
                    (const char *)a->q, (const char *)a->k, (const char *)a->v, (char *)a->out,
                    a->q_stride, a->q_head_stride, a->k_stride, a->k_head_stride, a->v_stride, a->v_head_stride,
                    a->out_stride, a->out_head_stride, a->query_start, a->key_start, a->key_count,
                    f.splits, f.each, f.tiles, (float *)a->workspace};
  // every sequence's rows fill whole tiles but for one
  if (!f.few) p.tiles = (int)(a->query_rows / PROMPT_ROWS + a->num_sequences);
  const bool direct = (uintptr_t)a->q % 16 == 0 && a->q_stride % 8 == 0 && a->q_head_stride % 8 == 0 &&
                      (uintptr_t)a->k % 16 == 0 && (uintptr_t)a->v % 16 == 0 && a->k_stride % 8 == 0 &&
                    a->k_head_stride % 8 == 0 && a->v_stride % 8 == 0 && a->v_head_stride % 8 == 0 && a->k_stride < (1 << 24) && a->v_stride < (1 << 24);
  hipStream_t stream = (hipStream_t)hip_stream;
  return a->dtype == JDOB_EDGE_BF16 ? attend<__bf16>(p, f.few, direct, stream) : attend<_Float16>(p, f.few, direct, stream);
}
