// The shared projection of all users' rows beside each row's low-rank adapter.
//
//   out = x W^T + gain_a ((x A_a^T) B_a^T),  a = the row's adapter (or none)
//
// `down_kernel` forms the low-rank rows gain_a (x A_a^T) in the workspace.  Then either kernel forms
// x W^T and adds the low-rank rows times B_a^T before it stores: `stream_kernel` for few rows, where
// reading W is all that counts, `tile_kernel` for many, where the products are.
//
// Measured (kernel alone): x A^T of 8192 x 4096 with rank 16 22-25 us (3 TB/s of x), of 32 rows with
// 32 adapters 11 us; W streamed past 32 rows, 4096 x 4096, 9.8 us (3.4 TB/s); tiles at 8192 x 4096 x 4096
// 235 us in a graph (1.17 PFLOP/s; a library's product 178 us), with 32 adapters 242 at least and 278 in the
// middle of single launches; 6007 x 4096 x 14336 in 8 bits 357 us in a graph (1.97 POP/s; a library's 1.87),
// with 16 adapters 396 and 439.  The matrix units are busy 61 % (54 %) of the large
// tiles' time, at clocks that the load lowers to about 2.1 GHz; LDS is busy a quarter of it, without
// conflicts.  What is left is the slices' two barriers, the loads' issue behind them, and the tiles'
// beginnings and ends (one workgroup a compute unit).
#include "edge_common.h"

namespace edge {
namespace {

struct ProjectParams {
  int rows, in_dim, out_dim;
  const char *x, *w;               // rows of x and W
  int64_t x_pitch, w_pitch;        // bytes
  const float *x_scale, *w_scale;  // 8 bits only
  int num_adapters, max_rank;      // num_adapters 0: x W^T alone
  const void *down, *up;
  const float *gain;
  const int *rank, *row_adapter;
  // The low-rank rows, gain and scales applied, zeros behind the adapter's rank; slabs = ranks / 32.
  // stream_kernel: binary32 [rows][32 slabs].  tile_kernel: [slab][rows][64] of dtype, the rows' 32
  // values rounded, then what the rounding left of each.  binary16 holds neither large values nor what is
  // left of small ones: there 16 ranks' values of a row are divided by a power of two that brings the
  // largest of them to [2^14, 2^15), v_scale [slab][rows][2] (so 22 bits are left of any that is not more
  // than 2^17 times smaller than the largest).
  void *v;
  float *v_scale;
  int slabs, split;                // split: v is in two parts
  void *out;
  int64_t out_stride;
};

// 16-bit products: eight elements of A and of B a lane.
template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
  typedef bf16x8 frag;
  __device__ static f32x4 m16(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  __device__ static f32x16 m32(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<_Float16> {
  typedef f16x8 frag;
  __device__ static f32x4 m16(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  __device__ static f32x16 m32(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// Products of x and W: 16 bytes a lane of either, 16-bit or 8-bit.
template <typename T, bool X8>
struct Main {
  typedef f32x16 acc;
  __device__ static acc mma(u32x4 a, u32x4 b, acc c) {
    typedef typename Mma<T>::frag frag;
    return Mma<T>::m32(__builtin_bit_cast(frag, a), __builtin_bit_cast(frag, b), c);
  }
};
template <typename T>
struct Main<T, true> {
  typedef i32x16 acc;
  __device__ static acc mma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a),
                                                 __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// 131072 products of two codes are at most 2^31 (all of them -128), which wraps around to -2^31; no sum is as
// low as that itself, and with fewer products none is as high.
__device__ inline bool may_wrap(const ProjectParams &p) { return p.in_dim == 131072; }

template <int N>
struct Count {
  static constexpr int value = N;
};

// The adapter of a row: -1 for none.
__device__ inline int adapter_of(const ProjectParams &p, int row) {
  const int a = p.row_adapter[row];
  return (unsigned)a < (unsigned)p.num_adapters ? a : -1;
}

__device__ inline int rank_of(const ProjectParams &p, int a) {
  const int r = p.rank ? p.rank[a] : p.max_rank;
  return r < 0 ? 0 : r < p.max_rank ? r : p.max_rank;
}

// 16 bytes of a row from byte `at` on, zeros from `len` on.
template <bool X8>
__device__ inline u32x4 chunk(const char *row, int at, int len) {
  if (at + 16 <= len) return *(const typename Raw<unsigned, 4>::type *)(row + at);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 16; j += X8 ? 1 : 2)
    if (at + j < len)
      v[j / 4] |= (unsigned)(X8 ? *(const unsigned char *)(row + at + j) : *(const unsigned short *)(row + at + j))
                  << (j % 4 * 8);
  return v;
}

// ------------------------------------------------------------------ rows through registers and LDS

constexpr int SLICE = 128;  // bytes of the inner dimension taken at a time: 64 or 128 elements

// Where 16-byte chunk c of row r of a slice stands in LDS: rows of 128 bytes, chunks exchanged within
// the row so that eight rows' equal chunks fall on different banks.
__device__ inline int spot(int r, int c) { return r * SLICE + ((c ^ (r & 7)) << 4); }

// A wave's slices of ROWS rows.  The matrix units want equal lanes in equal rows, memory wants
// neighbouring lanes in neighbouring bytes (a lane a row makes each lane's 16 bytes a request of
// their own, and W came at 2.5 TB/s): eight lanes load a row's 128 bytes, and the wave's own corner of
// LDS hands them to the lanes that need them.
template <int ROWS>
struct Rows {
  const char *at[ROWS / 8];
  // rows first.., clamped to `last`
  __device__ Rows(const char *base, int64_t pitch, int first, int last) {
    const int lane = threadIdx.x % WAVE;
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i) {
      const int row = first + i * 8 + lane / 8;
      at[i] = base + (row < last ? row : last) * pitch + lane % 8 * 16;
    }
  }
  __device__ void load(u32x4 (&r)[ROWS / 8], int slice) const {
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i) r[i] = *(const typename Raw<unsigned, 4>::type *)(at[i] + slice * SLICE);
  }
  // the last slice, of `len` bytes
  template <bool X8>
  __device__ void load_part(u32x4 (&r)[ROWS / 8], int slice, int len) const {
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i)
      r[i] = chunk<X8>(at[i] + slice * SLICE, 0, len - (int)(threadIdx.x % 8) * 16);
  }
  __device__ static void put(char *corner, const u32x4 (&r)[ROWS / 8]) {
    const int lane = threadIdx.x % WAVE;
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i) *(u32x4 *)(corner + spot(i * 8 + lane / 8, lane % 8)) = r[i];
  }
};

// ------------------------------------------------------------------ v = gain x A^T

// Eight elements of a row from element k on, zeros from `len` on.
template <typename T>
__device__ inline typename Mma<T>::frag eight(const T *row, int k, int len) {
  typename Mma<T>::frag f;
  if (k + 8 <= len) return *(const typename Raw<T, 8>::type *)(row + k);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = k + i < len ? row[k + i] : (T)0.0f;
  return f;
}

constexpr int DOWN_ROWS = 32, DOWN_WAVES = 8;

// A workgroup takes 32 rows, each of its waves one contiguous part of the inner dimension, RC * 16
// ranks at a time.  Of the adapters among its rows it takes every gridDim.z-th.  8-bit rows become
// 16-bit ones on their way into LDS (both 16-bit types hold them exactly): a slice of them is 64
// elements too.
template <typename T, bool X8, int RC>
__global__ __launch_bounds__(DOWN_WAVES *WAVE) void down_kernel(ProjectParams p) {
  constexpr int DEPTH = RC == 4 ? 2 : RC == 2 && X8 ? 3 : 4, RANKS = RC * 16, CORNER = (RANKS + DOWN_ROWS) * SLICE, SUMS = RC * 2 * WAVE * 16;
  __shared__ __align__(16) char room[DOWN_WAVES * (CORNER > SUMS ? CORNER : SUMS)];
  const int lane = threadIdx.x % WAVE, wave = wave_index();
  const int row0 = (int)block_index() * DOWN_ROWS, m = lane % 16, q = lane / 16;
  if (row0 >= p.rows) return;
  char *const corner = room + wave * CORNER;
  // x: eight lanes a row and eight elements a lane
  const char *xr[DOWN_ROWS / 8];
#pragma unroll
  for (int i = 0; i < DOWN_ROWS / 8; ++i) {
    const int row = row0 + i * 8 + lane / 8;
    xr[i] = p.x + (row < p.rows ? row : p.rows - 1) * p.x_pitch + lane % 8 * (X8 ? 8 : 16);
  }
  typedef typename Raw<unsigned, X8 ? 2 : 4>::type xword;
  const int full = p.in_dim / 64;  // whole slices; the wave's are those from lo to hi
  const int lo = full * wave / DOWN_WAVES, hi = full * (wave + 1) / DOWN_WAVES;
  const int mine = lane < DOWN_ROWS && row0 + lane < p.rows ? adapter_of(p, row0 + lane) : -1;
  unsigned long long left = __ballot(mine >= 0);
  for (int n = 0; left; ++n) {
    const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
    const unsigned long long these = __ballot(mine == a);
    left &= ~these;
    if (n % (int)gridDim.z != (int)blockIdx.z) continue;
    const int rank = rank_of(p, a);
    const float gain = p.gain[a];
    const char *const down = (const char *)p.down + (int64_t)a * p.max_rank * p.in_dim * 2;
    for (int r0 = 0; r0 < p.slabs * 32; r0 += RANKS) {
      f32x4 acc[RC][2];
#pragma unroll
      for (int c = 0; c < RC; ++c) acc[c][0] = acc[c][1] = (f32x4){0, 0, 0, 0};
      if (r0 < rank) {
        // ranks behind the last are its copies here, and zeros in v
        const Rows<RANKS> ar(down, (int64_t)p.in_dim * 2, r0, rank - 1);
        u32x4 av[DEPTH][RANKS / 8];
        xword xv[DEPTH][DOWN_ROWS / 8];
        auto load = [&](int d, int s) {
          ar.load(av[d], s);
#pragma unroll
          for (int i = 0; i < DOWN_ROWS / 8; ++i) xv[d][i] = *(const xword *)(xr[i] + s * (X8 ? 64 : 128));
        };
        auto multiply = [&](int d) {
          lanes_meet();
          Rows<RANKS>::put(corner, av[d]);
#pragma unroll
          for (int i = 0; i < DOWN_ROWS / 8; ++i) {
            char *const to = corner + RANKS * SLICE + spot(i * 8 + lane / 8, lane % 8);
            if constexpr (X8) {
              typedef signed char c8 __attribute__((ext_vector_type(8)));
              typedef unsigned u2 __attribute__((ext_vector_type(2)));
              const c8 c = __builtin_bit_cast(c8, (u2)xv[d][i]);
              typename Mma<T>::frag f;
#pragma unroll
              for (int e = 0; e < 8; ++e) f[e] = (T)(float)c[e];
              *(typename Mma<T>::frag *)to = f;
            } else {
              *(u32x4 *)to = xv[d][i];
            }
          }
          lanes_meet();
          typedef typename Mma<T>::frag frag;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            frag xf[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) xf[j] = *(const frag *)(corner + RANKS * SLICE + spot(j * 16 + m, k * 4 + q));
#pragma unroll
            for (int c = 0; c < RC; ++c) {
              const frag af = *(const frag *)(corner + spot(c * 16 + m, k * 4 + q));
#pragma unroll
              for (int j = 0; j < 2; ++j) acc[c][j] = Mma<T>::m16(af, xf[j], acc[c][j]);
            }
          }
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
          if (lo + d < hi) load(d, lo + d);
        for (int s = lo; s < hi; s += DEPTH) {
#pragma unroll
          for (int d = 0; d < DEPTH; ++d) {
            if (s + d >= hi) break;
            multiply(d);
            if (s + d + DEPTH < hi) load(d, s + d + DEPTH);
          }
        }
        if (full * 64 < p.in_dim && wave == 0) {
          const int rest = p.in_dim - full * 64;
          ar.template load_part<false>(av[0], full, rest * 2);
#pragma unroll
          for (int i = 0; i < DOWN_ROWS / 8; ++i) {
            const u32x4 v = chunk<X8>(xr[i] + full * (X8 ? 64 : 128), 0, (rest - lane % 8 * 8) * (X8 ? 1 : 2));
#pragma unroll
            for (int e = 0; e < (X8 ? 2 : 4); ++e) xv[0][i][e] = v[e];
          }
          multiply(0);
        }
      }
      __syncthreads();  // the waves' corners have been read
#pragma unroll
      for (int c = 0; c < RC; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j) *(f32x4 *)(room + wave * SUMS + ((c * 2 + j) * WAVE + lane) * 16) = acc[c][j];
      __syncthreads();
      // entry e = (chunk of ranks, half of the rows): a lane's four consecutive ranks of one row
      for (int e = wave; e < RC * 2; e += DOWN_WAVES) {
        f32x4 s = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < DOWN_WAVES; ++i) s += *(const f32x4 *)(room + i * SUMS + (e * WAVE + lane) * 16);
        const int local = (e % 2) * 16 + m, r = r0 + e / 2 * 16 + q * 4, row = row0 + local;
        if (!(these >> local & 1) || r >= p.slabs * 32) continue;
        s *= X8 ? gain * p.x_scale[row] : gain;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = r + i < rank ? s[i] : 0.0f;
        if (p.split) {
          T *const dst = (T *)p.v + ((int64_t)(r / 32) * p.rows + row) * 64 + r % 32;
          if constexpr (__is_same(T, _Float16)) {
            // the lanes that hold the row's other ranks of these 16 are here, too
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(s[i]) < INFINITY ? fabsf(s[i]) : 0.0f);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const int e = __builtin_amdgcn_frexp_expf(top) - 15, down_by = e < -126 ? -126 : e;
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = ldexpf(s[i], -down_by);
            if (q == 0) p.v_scale[((int64_t)(r / 32) * p.rows + row) * 2 + r / 16 % 2] = ldexpf(1.0f, down_by);
          }
          float high[4], low[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            high[i] = (float)(T)s[i];
            low[i] = fabsf(high[i]) < INFINITY ? s[i] - high[i] : 0.0f;
          }
          store_f32<T, 4>(dst, high);
          store_f32<T, 4>(dst + 32, low);
        } else {
          *(f32x4 *)((float *)p.v + (int64_t)row * p.slabs * 32 + r) = s;
        }
      }
      __syncthreads();  // the sums have been read
    }
  }
}

// ------------------------------------------------------------------ few rows: W streams through

// Products of 16 rows of W with 16 of x: 16 bytes a lane of either, 16-bit or 8-bit.
template <typename T, bool X8>
struct Small {
  typedef f32x4 acc;
  __device__ static acc mma(u32x4 a, u32x4 b, acc c) {
    typedef typename Mma<T>::frag frag;
    return Mma<T>::m16(__builtin_bit_cast(frag, a), __builtin_bit_cast(frag, b), c);
  }
};
template <typename T>
struct Small<T, true> {
  typedef i32x4 acc;
  __device__ static acc mma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// One row's low-rank part of one column: v . B's row, whole eights of either in registers as far as
// RANKS goes, which are loaded long before they are used.
template <typename T, int RANKS>
struct LowRank {
  int rank = 0;
  const float *v;
  const T *b;
  f32x4 vf[RANKS / 4];
  typename Mma<T>::frag bf[RANKS / 8];

  __device__ void load(const ProjectParams &p, int row, int col) {
    const int a = row < p.rows && col < p.out_dim ? adapter_of(p, row) : -1;
    if (a < 0) return;
    rank = rank_of(p, a);
    v = (const float *)p.v + (int64_t)row * p.slabs * 32;  // zeros from the rank to a multiple of 32
    b = (const T *)p.up + ((int64_t)a * p.out_dim + col) * p.max_rank;
#pragma unroll
    for (int r = 0; r < RANKS; r += 8)
      if (r + 8 <= rank) {
        bf[r / 8] = *(const typename Raw<T, 8>::type *)(b + r);
        vf[r / 4] = *(const f32x4 *)(v + r);
        vf[r / 4 + 1] = *(const f32x4 *)(v + r + 4);
      }
  }
  __device__ float value() const {
    float y = 0.0f;
#pragma unroll
    for (int r = 0; r < RANKS; r += 8)
      if (r + 8 <= rank)
#pragma unroll
        for (int k = 0; k < 8; ++k) y += vf[r / 4 + k / 4][k % 4] * (float)bf[r / 8][k];
    for (int r = rank < RANKS ? rank & ~7 : RANKS; r < rank; r += 8) {
      const typename Mma<T>::frag f = eight<T>(b, r, rank);
#pragma unroll
      for (int k = 0; k < 8; ++k) y += v[r + k] * (float)f[k];
    }
    return y;
  }
};

// A workgroup takes 16 columns and all rows (NT * 16); each wave takes one contiguous part of the inner
// dimension, and their sums meet in LDS.  DW slices of W and DX of x are under way (W comes from
// memory, x from the cache that all workgroups share).
template <typename T, bool X8, int NT, int WAVES, int DW, int DX>
__global__ __launch_bounds__(WAVES *WAVE) void stream_kernel(ProjectParams p) {
  typedef typename Small<T, X8>::acc acc_t;
  static_assert(DW % DX == 0, "rings");
  constexpr int THREADS = WAVES * WAVE, OUTPUTS = NT * 256, EACH = (OUTPUTS + THREADS - 1) / THREADS;
  constexpr int CORNER = (1 + NT) * 16 * SLICE;
  __shared__ __align__(16) char room[WAVES * CORNER];
  const int lane = threadIdx.x % WAVE, wave = wave_index(), m = lane % 16, q = lane / 16;
  const int col0 = blockIdx.x * 16, len = p.in_dim * (X8 ? 1 : 2);
  const Rows<16> wr(p.w, p.w_pitch, col0, p.out_dim - 1);
  const Rows<NT * 16> xr(p.x, p.x_pitch, 0, p.rows - 1);
  const int full = len / SLICE;  // whole slices; the wave's are those from lo to hi
  const int lo = full * wave / WAVES, hi = full * (wave + 1) / WAVES;
  u32x4 w[DW][2], x[DX][NT * 2];
#pragma unroll
  for (int d = 0; d < DW; ++d)
    if (lo + d < hi) wr.load(w[d], lo + d);
#pragma unroll
  for (int d = 0; d < DX; ++d)
    if (lo + d < hi) xr.load(x[d], lo + d);
  // the thread's outputs: row (e * THREADS + threadIdx.x) / 16, column col0 + threadIdx.x % 16
  LowRank<T, 16> low[EACH];
  if (p.num_adapters > 0) {
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      low[e].load(p, (e * THREADS + (int)threadIdx.x) / 16, col0 + threadIdx.x % 16);
  }
  acc_t acc[NT] = {};
  char *const corner = room + wave * CORNER;
  auto multiply = [&](const u32x4 (&wv)[2], const u32x4 (&xv)[NT * 2]) {
    lanes_meet();
    Rows<16>::put(corner, wv);
    Rows<NT * 16>::put(corner + 16 * SLICE, xv);
    lanes_meet();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 wf = *(const u32x4 *)(corner + spot(m, h * 4 + q));
#pragma unroll
      for (int t = 0; t < NT; ++t)
        acc[t] = Small<T, X8>::mma(wf, *(const u32x4 *)(corner + 16 * SLICE + spot(t * 16 + m, h * 4 + q)), acc[t]);
    }
  };
  for (int s = lo; s < hi; s += DW) {
#pragma unroll
    for (int d = 0; d < DW; ++d) {
      if (s + d >= hi) break;
      multiply(w[d], x[d % DX]);
      if (s + d + DW < hi) wr.load(w[d], s + d + DW);
      if (s + d + DX < hi) xr.load(x[d % DX], s + d + DX);
    }
  }
  if (full * SLICE < len && wave == 0) {
    wr.template load_part<X8>(w[0], full, len - full * SLICE);
    xr.template load_part<X8>(x[0], full, len - full * SLICE);
    multiply(w[0], x[0]);
  }
  __syncthreads();  // the waves' corners have been read
#pragma unroll
  for (int t = 0; t < NT; ++t) *(acc_t *)(room + ((wave * NT + t) * WAVE + lane) * 16) = acc[t];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int o = e * THREADS + threadIdx.x, row = o / 16, c = o % 16;
    if (o >= OUTPUTS || row >= p.rows || col0 + c >= p.out_dim) continue;
    auto part = [&](int w) { return (*(const acc_t *)(room + ((w * NT + row / 16) * WAVE + c / 4 * 16 + row % 16) * 16))[c % 4]; };
    auto sum = part(0);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += part(w);
    float y = (float)sum;
    if constexpr (X8) {
      if (may_wrap(p) && sum == INT32_MIN) y = -y;
      y *= p.x_scale[row] * p.w_scale[col0 + c];
    }
    if (p.num_adapters > 0) y += low[e].value();
    ((T *)p.out)[row * p.out_stride + col0 + c] = (T)y;
  }
}

// ------------------------------------------------------------------ many rows: tiles

__device__ const u32x4 edge_zeros = {0, 0, 0, 0};

// The same for a tile, whose 32 rows' equal chunks are read together: LDS serves rows 0-3, 12-15, 20-23
// and 24-27 at once, then the others, and its banks take 256 bytes, two rows.
__device__ inline int tile_spot(int r, int c) { return r * SLICE + ((c ^ (r >> 1 & 7)) << 4); }

// Stages COUNT rows' slice (bytes [at, at + 128) of rows first.., clamped to `last`) at dst.  DIRECT:
// memory to LDS, without registers between; needs chunks that lie within the row or behind it.
template <bool X8, bool DIRECT, int COUNT, int THREADS>
__device__ inline void stage(char *dst, const char *base, int64_t pitch, int first, int last, int at, int len) {
  static_assert(COUNT * 8 % THREADS == 0, "whole rounds");
  const char *const tile = base + first * pitch + at;
  auto each = [&](auto one) {
#pragma unroll
    for (int i = 0; i < COUNT * 8 / THREADS; ++i) {
      const int slot = i * THREADS + threadIdx.x, r = slot / 8, c = (slot % 8) ^ (r >> 1 & 7);
      one(i * THREADS, first + r < last ? r : last - first, c * 16);
    }
  };
  const unsigned to = lds_address(dst) + wave_index() * WAVE * 16;
  if constexpr (!DIRECT) {
    each([&](int s0, int r, int byte) {
      *(u32x4 *)(dst + (s0 + threadIdx.x) * 16) = chunk<X8>(tile + r * pitch + byte, 0, len - at - byte);
    });
  } else if (at + SLICE <= len) {
    each([&](int s0, int r, int byte) { load_to_lds(tile, (unsigned)r * (unsigned)pitch + byte, to + s0 * 16); });
  } else {
    each([&](int s0, int r, int byte) {
      load_to_lds(at + byte < len ? tile + r * pitch + byte : (const char *)&edge_zeros, to + s0 * 16);
    });
  }
}

// The low-rank part of one row's 16 columns first + 8 (e / 4) + e % 4.  The first eight ranks' B are
// loaded before the main loop, from all adapters' corners of memory, and used behind it.
template <typename T>
struct RowLow {
  typedef typename Mma<T>::frag frag;
  int rank = 0, first, out_dim, pitch;
  const float *v;
  const T *b;
  f32x4 vf[2];
  frag bf[16];

  __device__ const T *row_of(int e) const {
    const int col = first + 8 * (e / 4) + e % 4;
    return b + (int64_t)(col < out_dim ? col : out_dim - 1) * pitch;
  }
  __device__ void load(const ProjectParams &p, int row, int col) {
    const int a = p.num_adapters > 0 && row < p.rows ? adapter_of(p, row) : -1;
    if (a < 0) return;
    rank = rank_of(p, a);
    first = col;
    out_dim = p.out_dim;
    pitch = p.max_rank;
    v = (const float *)p.v + (int64_t)row * p.slabs * 32;  // zeros from the rank to a multiple of 32
    b = (const T *)p.up + (int64_t)a * p.out_dim * p.max_rank;
    if (rank < 8) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) vf[i] = *(const f32x4 *)(v + 4 * i);
#pragma unroll
    for (int e = 0; e < 16; ++e) bf[e] = *(const typename Raw<T, 8>::type *)row_of(e);
  }
  __device__ float value(int e) const {
    float y = 0.0f;
    if (rank >= 8)
#pragma unroll
      for (int k = 0; k < 8; ++k) y += vf[k / 4][k % 4] * (float)bf[e][k];
    for (int r = rank < 8 ? 0 : 8; r < rank; r += 8) {
      const frag f = eight<T>(row_of(e), r, rank);
#pragma unroll
      for (int k = 0; k < 8; ++k) y += v[r + k] * (float)f[k];
    }
    return y;
  }
};

template <typename T, bool X8, bool DIRECT, int BM, int BN, int WM, int WN, int STAGES>
struct Tile {
  static constexpr int THREADS = WM * WN * WAVE;
  static constexpr int FM = BM / WM / 32, FN = BN / WN / 32;  // 32x32 tiles a wave: rows, columns
  static constexpr int STAGE = (BM + BN) * SLICE;             // bytes
  static constexpr int LOADS = STAGE / 16 / THREADS;          // a thread's, each stage
  static constexpr int ROW_LOADS = BM * 8 / THREADS;          // of them for rows
  static constexpr int OUT = BM * BN * 2;
  static constexpr int ROOM = STAGES * STAGE > OUT ? STAGES * STAGE : OUT;
};

// One workgroup: BM rows by BN columns, WM x WN waves.  W's rows are the products' first operand,
// so a lane holds four consecutive columns of one row.  A wave reads its operands a quarter of a slice
// ahead, those of the next slice's first quarter before it multiplies the last of this one, so that the
// barrier between them leaves the matrix units work; behind it the slice's buffer takes the slice after
// the next.  Behind the slices of the inner dimension come those of the low-rank part: for each
// adapter among the tile's rows, 32 ranks at a time, the rows' two-part v and the columns' B twice.
// Their product is added to the adapter's own rows only (zeros times an infinity are not zero), so
// other rows' v may be anything.  ROWWISE: few rows with many adapters, where each output's low-rank
// part is computed by itself.
template <typename T, bool X8, bool DIRECT, int BM, int BN, int WM, int WN, int STAGES, bool ROWWISE>
__global__ __launch_bounds__(WM *WN *WAVE, 2) void tile_kernel(ProjectParams p) {
  typedef Tile<T, X8, DIRECT, BM, BN, WM, WN, STAGES> K;
  typedef typename Mma<T>::frag frag;
  constexpr bool SMALL = K::FM * K::FN == 1, SCALED = __is_same(T, _Float16);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  __shared__ __align__(16) char room[K::ROOM];
  __shared__ int ids[BM], list[BM], listed;
  const int lane = threadIdx.x % WAVE, wave = wave_index();
  const int wm = wave / WN, wn = wave % WN, l32 = lane % 32, half = lane / 32;
  const int tiles_m = (p.rows + BM - 1) / BM, tiles_n = (p.out_dim + BN - 1) / BN;
  // Workgroups go to the chip's eight dies in turn: each die takes a contiguous run of tiles, in
  // groups of eight tiles of rows, so that what its cache holds serves several tiles.
  const int total = tiles_m * tiles_n, die = block_index() % 8, slot = block_index() / 8;
  if (block_index() >= (unsigned)total) return;
  const int tile = die * (total / 8) + (die < total % 8 ? die : total % 8) + slot;
  const int group = tile / (8 * tiles_n), high = tiles_m - group * 8 < 8 ? tiles_m - group * 8 : 8;
  const int in_group = tile - group * 8 * tiles_n;
  const int row0 = (group * 8 + in_group % high) * BM, col0 = in_group / high * BN;
  const int len = p.in_dim * (X8 ? 1 : 2), slices = (len + SLICE - 1) / SLICE;

  // the dies start at different places of the inner dimension and do not all ask for the same ones
  const int turn = slices * die / 8;
  auto buffer = [&](int t) { return room + t % STAGES * K::STAGE; };
  auto place = [&](int t) { return (t + turn < slices ? t + turn : t + turn - slices) * SLICE; };
  auto load = [&](int t) {
    char *const buf = buffer(t);
    const int at = place(t);
    stage<X8, DIRECT, BM, K::THREADS>(buf, p.x, p.x_pitch, row0, p.rows - 1, at, len);
    stage<X8, DIRECT, BN, K::THREADS>(buf + BM * SLICE, p.w, p.w_pitch, col0, p.out_dim - 1, at, len);
  };
  // slice n of the low-rank part, which is slice slices + n of all
  auto load_low = [&](int n) {
    char *const buf = buffer(slices + n);
    const int a = __builtin_amdgcn_readfirstlane(list[n / p.slabs]), slab = n % p.slabs;
    stage<false, true, BM, K::THREADS>(buf, (const char *)p.v + (int64_t)slab * p.rows * SLICE, SLICE, row0,
                                       p.rows - 1, 0, SLICE);
    const int left = rank_of(p, a) - slab * 32;
    const T *const up = (const T *)p.up + ((int64_t)a * p.out_dim + col0) * p.max_rank + slab * 32;
    const bool direct = (left % 8 == 0 || left >= 32) && p.max_rank % 8 == 0 && (uintptr_t)p.up % 16 == 0;
    const unsigned to = lds_address(buf + BM * SLICE) + wave * WAVE * 16;
#pragma unroll
    for (int i = 0; i < BN * 8 / K::THREADS; ++i) {
      const int e = i * K::THREADS + threadIdx.x, c = e / 8, r = ((e % 8) ^ (c >> 1 & 7)) % 4 * 8;
      const bool in = col0 + c < p.out_dim && r < left;
      const T *const from = up + (in ? (int64_t)c * p.max_rank + r : 0);
      if (direct) {
        load_to_lds(in ? (const void *)from : (const void *)&edge_zeros, to + i * K::THREADS * 16);
      } else {
        frag f = {};
        if (in) f = eight<T>(from, 0, left - r);
        *(frag *)(buf + BM * SLICE + e * 16) = f;
      }
    }
  };
  typename Main<T, X8>::acc acc[K::FM][K::FN] = {};
#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < slices) load(s);
  RowLow<T> low;
  if constexpr (ROWWISE) {
    static_assert(K::FM == 1 && K::FN == 1, "a row a lane");
    low.load(p, row0 + wm * 32 + l32, col0 + wn * 32 + 4 * half);
  }
  int behind = 0;  // slices of the low-rank part
  if (!ROWWISE && p.num_adapters > 0) {
    for (int r0 = wave * WAVE; r0 < BM; r0 += K::THREADS) {
      const int r = r0 + lane, a = r < BM && row0 + r < p.rows ? adapter_of(p, row0 + r) : -1;
      if (r < BM) ids[r] = a;
    }
    __syncthreads();
    if (wave == 0) {  // the adapters, each once
      int n = 0;
      for (int r0 = 0; r0 < BM; r0 += WAVE) {
        int a = r0 + lane < BM ? ids[r0 + lane] : -1;
        for (int i = 0; i < n; ++i) a = a == list[i] ? -1 : a;
        unsigned long long left = __ballot(a >= 0);
        while (left) {
          const int b = __builtin_amdgcn_readlane(a, __builtin_ctzll(left));
          left &= ~__ballot(a == b);
          if (lane == 0) list[n] = b;
          ++n;
        }
        lanes_meet();
      }
      if (lane == 0) listed = n;
    }
    __syncthreads();
    behind = __builtin_amdgcn_readfirstlane(listed) * p.slabs;
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
      if (s >= slices && s - slices < behind) load_low(s - slices);
  }
  auto load_any = [&](int t) {
    if (t < slices) {
      load(t);
    } else if (t - slices < behind) {
      load_low(t - slices);
    }
  };
  u32x4 xf[2][K::FM], wf[2][K::FN];
  auto fetch = [&](int t, int k) {  // 32 bytes of the inner dimension
    const char *const buf = buffer(t);
#pragma unroll
    for (int i = 0; i < K::FM; ++i)
      xf[k & 1][i] = *(const u32x4 *)(buf + tile_spot((wm * K::FM + i) * 32 + l32, k * 2 + half));
#pragma unroll
    for (int j = 0; j < K::FN; ++j)
      wf[k & 1][j] = *(const u32x4 *)(buf + BM * SLICE + tile_spot((wn * K::FN + j) * 32 + l32, k * 2 + half));
  };
  auto multiply = [&](int k, int i0, int i1) {
#pragma unroll
    for (int i = 0; i < K::FM; ++i)
      if (i >= i0 && i < i1)
#pragma unroll
        for (int j = 0; j < K::FN; ++j) acc[i][j] = Main<T, X8>::mma(wf[k & 1][j], xf[k & 1][i], acc[i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int HALF = K::FM / 2;
  // rows of slice t, then columns
  auto load_rows = [&](int t) {
    if (t < slices) stage<X8, DIRECT, BM, K::THREADS>(buffer(t), p.x, p.x_pitch, row0, p.rows - 1, place(t), len);
  };
  auto load_columns = [&](int t) {
    if (t < slices) {
      stage<X8, DIRECT, BN, K::THREADS>(buffer(t) + BM * SLICE, p.w, p.w_pitch, col0, p.out_dim - 1, place(t), len);
    } else if (t - slices < behind) {
      load_low(t - slices);
    }
  };
  // slice t has landed: of the loads after it those of STAGES - 2 slices and of `rows` are under way
  auto landed = [&](int t) {
    if (DIRECT && t + STAGES - 1 < slices) {
      wait_loads<(STAGES - 2) * K::LOADS + K::ROW_LOADS>();
    } else {
      wait_loads<0>();
    }
    barrier();
  };
  if constexpr (SMALL) {
    // A wave's one product a quarter would not cover the reads of the next: it reads a whole slice while it
    // multiplies the one before, and passes one barrier a slice.
    u32x4 xs[2][4], ws[2][4];
    auto multiply_slice = [&](auto set) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        acc[0][0] = Main<T, X8>::mma(ws[decltype(set)::value][k], xs[decltype(set)::value][k], acc[0][0]);
    };
    auto step = [&](int t, auto set, auto other) {
      // slice t has landed and the one before it has been read, by all waves
      if (DIRECT && t + STAGES - 2 < slices) {
        wait_loads<(STAGES - 2) * K::LOADS>();
      } else {
        wait_loads<0>();
      }
      barrier();
      if (t > 0) load_any(t + STAGES - 1);
      const char *const buf = buffer(t);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        xs[decltype(set)::value][k] = *(const u32x4 *)(buf + tile_spot(wm * 32 + l32, k * 2 + half));
        ws[decltype(set)::value][k] = *(const u32x4 *)(buf + BM * SLICE + tile_spot(wn * 32 + l32, k * 2 + half));
      }
      __builtin_amdgcn_sched_barrier(0);
      if (t > 0) multiply_slice(other);
      __builtin_amdgcn_sched_barrier(0);
    };
    int t = 0;
    for (; t + 1 < slices; t += 2) {
      step(t, Count<0>(), Count<1>());
      step(t + 1, Count<1>(), Count<0>());
    }
    if (t < slices) {
      step(t, Count<0>(), Count<1>());
      multiply_slice(Count<0>());
    } else {
      multiply_slice(Count<1>());
    }
  } else {
    wait_loads<0>();
    barrier();
    fetch(0, 0);
    for (int t = 0; t < slices; ++t) {
      fetch(t, 1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(0, 0, K::FM);
      fetch(t, 2);
      __builtin_amdgcn_sched_barrier(0);
      multiply(1, 0, K::FM);
      fetch(t, 3);
      __builtin_amdgcn_sched_barrier(0);
      multiply(2, 0, HALF);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      barrier();  // the slice has been read by all waves: its buffer is free
      load_rows(t + STAGES);
      multiply(2, HALF, K::FM);
      landed(t + 1);
      load_columns(t + STAGES);
      if (t + 1 < slices) fetch(t + 1, 0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(3, 0, K::FM);
    }
  }

  // to binary32, with the scales of 8-bit rows and columns
  f32x16 sum[K::FM][K::FN];
#pragma unroll
  for (int i = 0; i < K::FM; ++i) {
    float xs = 1.0f;
    if constexpr (X8) {
      const int row = row0 + (wm * K::FM + i) * 32 + l32;
      xs = p.x_scale[row < p.rows ? row : p.rows - 1];
    }
#pragma unroll
    for (int j = 0; j < K::FN; ++j) {
      if constexpr (X8) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int col = col0 + (wn * K::FN + j) * 32 + 8 * (e / 4) + 4 * half + e % 4;
          sum[i][j][e] = (float)acc[i][j][e] * (xs * p.w_scale[col < p.out_dim ? col : p.out_dim - 1]);
        }
        if (may_wrap(p)) {
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[i][j][e] = acc[i][j][e] == INT32_MIN ? -sum[i][j][e] : sum[i][j][e];
        }
      } else {
        sum[i][j] = acc[i][j];
      }
    }
  }
  for (int n = 0; n < behind; ++n) {
    f32x2 times[K::FM];  // the powers of two that ranks 0-15 and 16-31 of the slab were divided by
    if constexpr (SCALED) {
#pragma unroll
      for (int i = 0; i < K::FM; ++i) {
        const int row = row0 + (wm * K::FM + i) * 32 + l32;
        times[i] = ((const f32x2 *)p.v_scale)[(int64_t)(n % p.slabs) * p.rows + (row < p.rows ? row : p.rows - 1)];
      }
#pragma unroll
      for (int i = 0; i < K::FM; ++i) asm volatile("" : "+v"(times[i]));  // here, before further loads are under way
    }
    if (SMALL || n > 0) {
      wait_loads<0>();
      barrier();
      load_any(slices + n + STAGES - 1);
    }
    const char *const buf = buffer(slices + n);
    const int a = __builtin_amdgcn_readfirstlane(list[n / p.slabs]);
#pragma unroll
    for (int i = 0; i < K::FM; ++i) {
      const int r = (wm * K::FM + i) * 32 + l32;
      const bool mine = ids[r] == a;
      if (!__any(mine)) continue;
      frag v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = *(const frag *)(buf + tile_spot(r, k * 2 + half));
#pragma unroll
      for (int j = 0; j < K::FN; ++j) {
        auto up = [&](int k) { return *(const frag *)(buf + BM * SLICE + tile_spot((wn * K::FN + j) * 32 + l32, k * 2 + half)); };
        if constexpr (SCALED) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {  // 16 ranks: the rounded values, and what the rounding left
            f32x16 more = {};
            more = Mma<T>::m32(up(k), v[k], more);
            more = Mma<T>::m32(up(k + 2), v[k + 2], more);
            if (mine) sum[i][j] += more * times[i][k];
          }
        } else {
          f32x16 more = {};
#pragma unroll
          for (int k = 0; k < 4; ++k) more = Mma<T>::m32(up(k), v[k], more);
          if (mine) sum[i][j] += more;
        }
      }
    }
  }
  if constexpr (ROWWISE) {
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[0][0][e] += low.value(e);
  }
  wait_loads<0>();
  __syncthreads();  // all slices have been read

  // The tile goes through LDS, so that rows are stored in runs of 16 bytes a lane: chunks of eight
  // columns, exchanged within the row so that 32 rows' equal chunks fall on different banks.
  constexpr int CHUNKS = BN / 8, SWAP = CHUNKS < 32 ? CHUNKS - 1 : 31;
#pragma unroll
  for (int i = 0; i < K::FM; ++i) {
    const int r = (wm * K::FM + i) * 32 + l32;
#pragma unroll
    for (int j = 0; j < K::FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = (wn * K::FN + j) * 4 + e;
        const float y[4] = {sum[i][j][4 * e], sum[i][j][4 * e + 1], sum[i][j][4 * e + 2], sum[i][j][4 * e + 3]};
        store_f32<T, 4>((T *)(room + r * (BN * 2) + ((c ^ (r & SWAP)) << 4) + half * 8), y);
      }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < BM * CHUNKS; e += K::THREADS) {
    const int r = e / CHUNKS, c = e % CHUNKS, col = col0 + c * 8;
    if (row0 + r >= p.rows || col >= p.out_dim) continue;
    const typename Mma<T>::frag y = *(const typename Mma<T>::frag *)(room + r * (BN * 2) + ((c ^ (r & SWAP)) << 4));
    T *const dst = (T *)p.out + (row0 + r) * p.out_stride + col;
    if (col + 8 <= p.out_dim) {
      *(typename Raw<T, 8>::type *)dst = y;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < p.out_dim) dst[i] = y[i];
    }
  }
}

// ------------------------------------------------------------------ host side

// Up to here W streams through.  64 rows of 4096 (calls in a graph, without adapters) through 1024 columns take
// 12.1 us so and 23.9 by tiles of 64 x 64 (8 bits: 8.1 and 14.2), through 4096 columns 14.5 and 24.3 (11.1 and
// 14.7).  The rule looks at rows alone: through 14336 columns, where x passes 896 workgroups, tiles would be
// the faster ones from 33 rows on (64 rows: 53 and 30, 8 bits 31 and 16).
constexpr int STREAM_ROWS = 64;

int project_check(const jdob_edge_project_args *a, bool sizes_only) {
  if (!a || a->rows < 0 || a->in_dim < 1 || a->out_dim < 1 || a->num_adapters < 0 ||
      (a->bits8 != 0 && a->bits8 != 1))
    return JDOB_ERR_INVALID_ARG;
  if (a->num_adapters > 0 && a->max_rank < 1) return JDOB_ERR_INVALID_ARG;
  if (a->dtype != JDOB_EDGE_BF16 && a->dtype != JDOB_EDGE_F16) return JDOB_ERR_UNSUPPORTED;
  if (a->num_adapters > 0 && a->max_rank > JDOB_EDGE_MAX_RANK) return JDOB_ERR_UNSUPPORTED;
  if (a->rows > JDOB_EDGE_MAX_ROWS || a->in_dim > JDOB_EDGE_MAX_PROJECT_DIM ||
      a->out_dim > JDOB_EDGE_MAX_PROJECT_DIM || (a->bits8 && a->in_dim > 131072))
    return JDOB_ERR_UNSUPPORTED;
  // the smallest tiles have to fit a grid
  if ((int64_t)((a->rows + 63) / 64) * ((a->out_dim + 63) / 64) > MAX_BLOCKS) return JDOB_ERR_UNSUPPORTED;
  if (sizes_only || a->rows == 0) return JDOB_OK;
  if (!a->x || !a->weight || !a->out || a->x_stride < a->in_dim || a->weight_stride < a->in_dim ||
      a->out_stride < a->out_dim || (a->bits8 && (!a->x_scale || !a->weight_scale)))
    return JDOB_ERR_INVALID_ARG;
  if (a->num_adapters > 0) {
    if (!a->down || !a->up || !a->gain || !a->row_adapter || !a->workspace ||
        (uintptr_t)a->workspace % 16 || a->workspace_bytes < jdob_edge_project_workspace(a))
      return JDOB_ERR_INVALID_ARG;
  }
  return JDOB_OK;
}

template <typename T, bool X8>
int launch_down(const ProjectParams &p, hipStream_t stream) {
  const int groups = (p.rows + DOWN_ROWS - 1) / DOWN_ROWS;
  // Few rows may all have adapters of their own: up to 128 rows those are dealt to several workgroups.  Beyond,
  // a workgroup takes all of its 32 rows' adapters one after the other: through 4096 x 4096 with 64 adapters of
  // rank 16, 128 rows take 40 us, 129 rows 127 and 512 rows 82.
  const int layers = groups <= 4 ? (p.num_adapters < 32 ? p.num_adapters : 32) : 1;
  constexpr int threads = DOWN_WAVES * WAVE;
  if (p.max_rank <= 16) return launch(down_kernel<T, X8, 1>, groups, threads, stream, p, layers);
  if (p.max_rank <= 32) return launch(down_kernel<T, X8, 2>, groups, threads, stream, p, layers);
  return launch(down_kernel<T, X8, 4>, groups, threads, stream, p, layers);
}

template <typename T, bool X8, int NT, int WAVES, int DW, int DX>
int launch_stream(const ProjectParams &p, hipStream_t stream) {
  return launch(stream_kernel<T, X8, NT, WAVES, DW, DX>, (p.out_dim + 15) / 16, WAVES * WAVE, stream, p);
}

template <typename T, bool X8, bool DIRECT, int BM, int BN, int WM, int WN, int STAGES, bool ROWWISE = false>
int launch_tile(const ProjectParams &p, hipStream_t stream) {
  const int64_t tiles = (int64_t)((p.rows + BM - 1) / BM) * ((p.out_dim + BN - 1) / BN);
  return launch(tile_kernel<T, X8, DIRECT, BM, BN, WM, WN, STAGES, ROWWISE>, tiles, WM * WN * WAVE, stream, p);
}

// Few rows with many adapters: the low-rank part output by output.  Through 4096 x 4096 with rank 16, in
// slices and so (calls in a graph): 128 rows with 8 adapters 36.1 and 38.1 us, with 16 38.5 and 38.3, with 64
// 54.7 and 40.4; 512 rows with 64 84.3 and 81.9.  (It counts the adapters that there are, not those that the
// rows have, which the host does not know.)
bool rowwise(int rows, int num_adapters) { return rows <= 512 && num_adapters * 8 >= rows; }

template <typename T, bool X8>
int project(const ProjectParams &p, hipStream_t stream) {
  if (p.num_adapters > 0) {
    const int code = launch_down<T, X8>(p, stream);
    if (code != JDOB_OK) return code;
  }
  if (p.rows <= 16) return launch_stream<T, X8, 1, 8, 4, 4>(p, stream);
  if (p.rows <= 32) return launch_stream<T, X8, 2, 8, 4, 4>(p, stream);
  if (p.rows <= STREAM_ROWS) return launch_stream<T, X8, 4, 8, 4, 2>(p, stream);
  const bool direct = (uintptr_t)p.x % 16 == 0 && (uintptr_t)p.w % 16 == 0 && p.x_pitch % 16 == 0 &&
                      p.w_pitch % 16 == 0 && p.x_pitch < (1 << 22) && p.w_pitch < (1 << 22) &&
                      p.in_dim * (X8 ? 1 : 2) % 16 == 0;
  const bool rw = rowwise(p.rows, p.num_adapters);
  if (!direct)
    return rw ? launch_tile<T, X8, false, 64, 64, 2, 2, 2, true>(p, stream)
              : launch_tile<T, X8, false, 128, 128, 2, 2, 2>(p, stream);
  if (rw) return launch_tile<T, X8, true, 64, 64, 2, 2, 4, true>(p, stream);
  // The tile that takes least time by a count of rounds, of 256 workgroups with tiles of 256 x 256 (one a compute
  // unit) and of 512 with the others (two).  Measured at 8192 x 4096 x 4096, a slice of 128 bytes takes a round
  // 1.84 us with 256 x 256 (8 bits: 2.10), 1.08 with 128 x 128 (1.23) and 0.43 with 64 x 64 (0.45); the rule
  // takes 256 x 256 as equal in both types.
  auto rounds = [&](int side, int at_once) {
    const int64_t tiles = (int64_t)((p.rows + side - 1) / side) * ((p.out_dim + side - 1) / side);
    return (double)((tiles + at_once - 1) / at_once);
  };
  const double t256 = 1.86 * rounds(256, 256), t128 = (X8 ? 1.4 : 1.1) * rounds(128, 512), t64 = 0.47 * rounds(64, 512);
  if (t64 <= t128 && t64 <= t256) return launch_tile<T, X8, true, 64, 64, 2, 2, 4>(p, stream);
  if (t128 <= t256) return launch_tile<T, X8, true, 128, 128, 2, 2, 2>(p, stream);
  return launch_tile<T, X8, true, 256, 256, 2, 4, 2>(p, stream);
}

}  // namespace
}  // namespace edge

extern "C" int64_t jdob_edge_project_workspace(const jdob_edge_project_args *a) {
  using namespace edge;
  if (project_check(a, true) != JDOB_OK) return -1;
  if (a->num_adapters == 0 || a->rows == 0) return 0;
  // 32 ranks of a row: binary32, or two 16-bit parts; two scales
  return (int64_t)a->rows * ((a->max_rank + 31) / 32) * (a->dtype == JDOB_EDGE_F16 ? 136 : 128);
}

extern "C" int jdob_edge_project(const jdob_edge_project_args *a, void *hip_stream) {
  using namespace edge;
  const int code = project_check(a, false);
  if (code != JDOB_OK || a->rows == 0) return code;
  const int size = a->bits8 ? 1 : 2, slabs = (a->max_rank + 31) / 32;
  const bool split = a->rows > STREAM_ROWS && !rowwise(a->rows, a->num_adapters);
  const ProjectParams p = {a->rows, a->in_dim, a->out_dim, (const char *)a->x, (const char *)a->weight,
                     a->x_stride * size, a->weight_stride * size, a->x_scale, a->weight_scale,
                     a->num_adapters, a->max_rank, a->down, a->up, a->gain, a->rank,
                     a->row_adapter, a->workspace, (float *)((char *)a->workspace + (int64_t)a->rows * slabs * 128),
                     slabs, split, a->out, a->out_stride};
  hipStream_t stream = (hipStream_t)hip_stream;
  if (a->dtype == JDOB_EDGE_BF16)
    return a->bits8 ? project<__bf16, true>(p, stream) : project<__bf16, false>(p, stream);
  return a->bits8 ? project<_Float16, true>(p, stream) : project<_Float16, false>(p, stream);
}
