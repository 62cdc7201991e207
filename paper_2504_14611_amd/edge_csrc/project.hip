// The shared projection of all users' rows beside each row's low-rank adapter.
//
//   out = x W^T + gain_a ((x A_a^T) B_a^T),  a = the row's adapter (or none)
//
// Two kernels.  `down_kernel` forms the low-rank rows v = x A_a^T (binary32, in the workspace);
// `tile_kernel` forms x W^T tile by tile and, before it stores a tile, multiplies the v of the
// tile's rows with the B of each adapter among them onto the same accumulators.
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
  float *v;                        // [splits][rows][rank_pad] partial low-rank rows
  int rank_pad, splits, split_len; // split_len: elements of the inner dimension, a multiple of 32
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

// The adapter of a row: -1 for none.
__device__ inline int adapter_of(const ProjectParams &p, int row) {
  const int a = p.row_adapter[row];
  return (unsigned)a < (unsigned)p.num_adapters ? a : -1;
}

__device__ inline int rank_of(const ProjectParams &p, int a) {
  const int r = p.rank ? p.rank[a] : p.max_rank;
  return r < 0 ? 0 : r < p.max_rank ? r : p.max_rank;
}

// ------------------------------------------------------------------ v = x A^T

// Eight elements of a row from element k on, zeros from `len` on.
template <typename T>
__device__ inline typename Mma<T>::frag eight(const T *row, int k, int len) {
  typename Mma<T>::frag f;
  if (k + 8 <= len) return *(const typename Raw<T, 8>::type *)(row + k);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = k + i < len ? row[k + i] : (T)0.0f;
  return f;
}

// The same of a row of 8-bit integers, which both 16-bit types hold exactly.
template <typename T>
__device__ inline typename Mma<T>::frag eight(const int8_t *row, int k, int len) {
  typename Mma<T>::frag f;
  if (k + 8 <= len) {
    const typename Raw<int8_t, 8>::type c = *(const typename Raw<int8_t, 8>::type *)(row + k);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (T)(float)c[i];
    return f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = k + i < len ? (T)(float)row[k + i] : (T)0.0f;
  return f;
}

constexpr int DOWN_ROWS = 32, DOWN_WAVES = 4;

// A workgroup takes 32 rows and one split of the inner dimension, each wave a quarter of the split;
// RC * 16 ranks at a time.  Of the adapters among its rows it takes every gridDim.z-th.
template <typename T, typename X, int RC>
__global__ __launch_bounds__(DOWN_WAVES *WAVE) void down_kernel(ProjectParams p) {
  __shared__ float part[DOWN_WAVES][RC * 2][WAVE][4];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int row0 = blockIdx.x * DOWN_ROWS, m = lane % 16, q = lane / 16;
  const int lo = blockIdx.y * p.split_len;
  const int hi = lo + p.split_len < p.in_dim ? lo + p.split_len : p.in_dim;
  const X *xr[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = row0 + j * 16 + m;
    xr[j] = (const X *)(p.x + (row < p.rows ? row : p.rows - 1) * p.x_pitch);
  }
  const int mine = lane < DOWN_ROWS && row0 + lane < p.rows ? adapter_of(p, row0 + lane) : -1;
  unsigned long long left = __ballot(mine >= 0);
  for (int n = 0; left; ++n) {
    const int a = __shfl(mine, __builtin_ctzll(left));
    const unsigned long long these = __ballot(mine == a);
    left &= ~these;
    if (n % (int)gridDim.z != (int)blockIdx.z) continue;
    const int rank = rank_of(p, a);
    const T *const down = (const T *)p.down + (int64_t)a * p.max_rank * p.in_dim;
    for (int r0 = 0; r0 < rank; r0 += RC * 16) {
      f32x4 acc[RC][2];
#pragma unroll
      for (int c = 0; c < RC; ++c) acc[c][0] = acc[c][1] = (f32x4){0, 0, 0, 0};
      for (int k = lo + wave * 32 + q * 8; k < ((hi + 31) & ~31); k += DOWN_WAVES * 32) {
        typename Mma<T>::frag xf[2], af[RC];
#pragma unroll
        for (int j = 0; j < 2; ++j) xf[j] = eight<T>(xr[j], k, hi);
#pragma unroll
        for (int c = 0; c < RC; ++c) {
          const int r = r0 + c * 16 + m;
          af[c] = eight<T>(down + (int64_t)(r < rank ? r : 0) * p.in_dim, k, r < rank ? hi : 0);
        }
#pragma unroll
        for (int c = 0; c < RC; ++c)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[c][j] = Mma<T>::m16(af[c], xf[j], acc[c][j]);
      }
      __syncthreads();  // the previous round's sums have been read
#pragma unroll
      for (int c = 0; c < RC; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j) *(f32x4 *)part[wave][c * 2 + j][lane] = acc[c][j];
      __syncthreads();
      // entry e = (chunk of ranks, half of the rows): lane's four consecutive ranks of one row
      for (int e = wave; e < RC * 2; e += DOWN_WAVES) {
        f32x4 s = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < DOWN_WAVES; ++i) s += *(const f32x4 *)part[i][e][lane];
        const int local = (e % 2) * 16 + m, r = r0 + e / 2 * 16 + q * 4;
        if ((these >> local & 1) && r < p.rank_pad) {
          float *dst = p.v + ((int64_t)blockIdx.y * p.rows + row0 + local) * p.rank_pad + r;
          *(f32x4 *)dst = s;
        }
      }
    }
  }
}

// v of one row and rank, times the adapter's gain (and the row's scale of 8-bit rows)
template <bool X8>
__device__ inline float low_rank(const ProjectParams &p, int row, int a, int r) {
  float s = 0.0f;
  for (int i = 0; i < p.splits; ++i) s += p.v[((int64_t)i * p.rows + row) * p.rank_pad + r];
  s *= p.gain[a];
  return X8 ? s * p.x_scale[row] : s;
}

// ------------------------------------------------------------------ out = x W^T + v B^T

__device__ const u32x4 edge_zeros = {0, 0, 0, 0};

constexpr int SLICE = 128;  // bytes of the inner dimension staged at a time: 64 or 128 elements

// Where 16-byte chunk c of row r of a staged slice stands: rows of 128 bytes, chunks exchanged
// within the row so that eight rows' equal chunks fall on different LDS banks.
__device__ inline int spot(int r, int c) { return r * SLICE + ((c ^ (r & 7)) << 4); }

template <typename T, bool X8, bool FAST, int BM, int BN, int WM, int WN>
struct Tile {
  static constexpr int WAVES = WM * WN, THREADS = WAVES * WAVE;
  static constexpr int FM = BM / WM / 32, FN = BN / WN / 32;  // 32x32 tiles a wave: rows, columns
  static constexpr int STAGE = (BM + BN) * SLICE;

  // Stages `count` rows' slice (bytes [at, at + 128) of rows first.., clamped to `last`) at dst.
  template <int COUNT>
  __device__ static void stage(char *dst, const char *base, int64_t pitch, int first, int last,
                               int at, int len) {
#pragma unroll
    for (int i = 0; i < COUNT * 8 / THREADS; ++i) {
      const int slot = i * THREADS + threadIdx.x, r = slot / 8, c = (slot % 8) ^ (r & 7);
      const int row = first + r < last ? first + r : last;
      const int byte = at + c * 16;
      const char *src = base + row * pitch + byte;
      if constexpr (FAST) {
        // rows are whole multiples of 16 bytes: a chunk lies within the row or behind it
        const char *from = byte < len ? src : (const char *)&edge_zeros;
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) unsigned *)from,
            (__attribute__((address_space(3))) unsigned *)(dst + (i * THREADS + (threadIdx.x & ~63)) * 16),
            16, 0, 0);
      } else {
        u32x4 v = {0, 0, 0, 0};
        if (byte + 16 <= len) {
          v = *(const typename Raw<unsigned, 4>::type *)src;
        } else if (byte < len) {
          constexpr int E = X8 ? 1 : 2;
          unsigned char b[16];
#pragma unroll
          for (int j = 0; j < 16 / E; ++j) {
            const bool in = byte + j * E < len;
            if constexpr (X8) {
              b[j] = in ? (unsigned char)src[j] : 0;
            } else {
              const unsigned short h = in ? ((const unsigned short *)src)[j] : 0;
              b[2 * j] = (unsigned char)h;
              b[2 * j + 1] = (unsigned char)(h >> 8);
            }
          }
          __builtin_memcpy(&v, b, 16);
        }
        *(u32x4 *)(dst + slot * 16) = v;
      }
    }
  }
};

// One workgroup: BM rows by BN columns, WM x WN waves.  W's rows are the products' first operand,
// so a lane holds four consecutive columns of one row.
template <typename T, bool X8, bool FAST, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *WAVE) void tile_kernel(ProjectParams p) {
  typedef Tile<T, X8, FAST, BM, BN, WM, WN> K;
  __shared__ __align__(16) char buf0[K::STAGE], buf1[K::STAGE];
  __shared__ int ids[BM];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int wm = wave / WN, wn = wave % WN, l32 = lane % 32, half = lane / 32;
  const int tiles_n = (p.out_dim + BN - 1) / BN;
  const int row0 = (int)blockIdx.x / tiles_n * BM, col0 = (int)blockIdx.x % tiles_n * BN;
  const int len = p.in_dim * (X8 ? 1 : 2), slices = (len + SLICE - 1) / SLICE;

  auto stage = [&](char *buf, int s) {
    K::template stage<BM>(buf, p.x, p.x_pitch, row0, p.rows - 1, s * SLICE, len);
    K::template stage<BN>(buf + BM * SLICE, p.w, p.w_pitch, col0, p.out_dim - 1, s * SLICE, len);
  };
  typename Main<T, X8>::acc acc[K::FM][K::FN] = {};
  auto multiply = [&](const char *buf) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // 32 bytes of the inner dimension each
      u32x4 xf[K::FM], wf[K::FN];
#pragma unroll
      for (int i = 0; i < K::FM; ++i)
        xf[i] = *(const u32x4 *)(buf + spot((wm * K::FM + i) * 32 + l32, k * 2 + half));
#pragma unroll
      for (int j = 0; j < K::FN; ++j)
        wf[j] = *(const u32x4 *)(buf + BM * SLICE + spot((wn * K::FN + j) * 32 + l32, k * 2 + half));
#pragma unroll
      for (int i = 0; i < K::FM; ++i)
#pragma unroll
        for (int j = 0; j < K::FN; ++j) acc[i][j] = Main<T, X8>::mma(wf[j], xf[i], acc[i][j]);
    }
  };
  stage(buf0, 0);
  for (int s = 0; s < slices; s += 2) {
    __syncthreads();
    if (s + 1 < slices) stage(buf1, s + 1);
    multiply(buf0);
    if (s + 1 < slices) {
      __syncthreads();
      if (s + 2 < slices) stage(buf0, s + 2);
      multiply(buf1);
    }
  }

  // to binary32, with the scales of 8-bit rows and columns
  f32x16 sum[K::FM][K::FN];
#pragma unroll
  for (int i = 0; i < K::FM; ++i)
#pragma unroll
    for (int j = 0; j < K::FN; ++j) {
      if constexpr (X8) {
        const int row = row0 + (wm * K::FM + i) * 32 + l32;
        const float xs = p.x_scale[row < p.rows ? row : p.rows - 1];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int col = col0 + (wn * K::FN + j) * 32 + 8 * (e / 4) + 4 * half + e % 4;
          sum[i][j][e] = (float)acc[i][j][e] * (xs * p.w_scale[col < p.out_dim ? col : p.out_dim - 1]);
        }
      } else {
        sum[i][j] = acc[i][j];
      }
    }

  if (p.num_adapters > 0) {
    // For each adapter among the tile's rows, 32 ranks at a time: the rows' v (zeros for rows of
    // other adapters) as two 16-bit parts whose sum is v to 16 (22) bits, and the columns' B.
    // The product is added to the adapter's own rows only: zeros times an infinity are not zero.
    char *const vbuf = buf0, *const bbuf = buf0 + BM * SLICE;
    __syncthreads();
    for (int r = threadIdx.x; r < BM; r += K::THREADS)
      ids[r] = row0 + r < p.rows ? adapter_of(p, row0 + r) : -1;
    __syncthreads();
    int done = 0;  // rows before it belong to adapters that have been applied
    while (true) {
      while (done < BM) {
        const int a = ids[done];
        bool seen = a < 0;
        for (int r = 0; r < done && !seen; ++r) seen = ids[r] == a;
        if (!seen) break;
        ++done;
      }
      if (done >= BM) break;
      const int a = ids[done++], rank = rank_of(p, a);
      const T *const up = (const T *)p.up + (int64_t)a * p.out_dim * p.max_rank;
      for (int r0 = 0; r0 < rank; r0 += 32) {
        __syncthreads();
        for (int e = threadIdx.x; e < BM * 32; e += K::THREADS) {
          const int r = e / 32, k = e % 32;
          const float v = ids[r] == a && r0 + k < rank ? low_rank<X8>(p, row0 + r, a, r0 + k) : 0.0f;
          const T high = (T)v, low = (T)(v - (float)high);
          *(T *)(vbuf + spot(r, k / 8) + k % 8 * 2) = high;
          *(T *)(vbuf + spot(r, 4 + k / 8) + k % 8 * 2) = low;
        }
        for (int e = threadIdx.x; e < BN * 32; e += K::THREADS) {
          const int c = e / 32, k = e % 32;
          const bool in = col0 + c < p.out_dim && r0 + k < rank;
          *(T *)(bbuf + spot(c, k / 8) + k % 8 * 2) =
              in ? up[(int64_t)(col0 + c) * p.max_rank + r0 + k] : (T)0.0f;
        }
        __syncthreads();
        typedef typename Mma<T>::frag frag;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < K::FN; ++j) {
            const frag b = *(const frag *)(bbuf + spot((wn * K::FN + j) * 32 + l32, k * 2 + half));
#pragma unroll
            for (int i = 0; i < K::FM; ++i) {
              const int r = (wm * K::FM + i) * 32 + l32;
              const frag h = *(const frag *)(vbuf + spot(r, k * 2 + half));
              const frag l = *(const frag *)(vbuf + spot(r, 4 + k * 2 + half));
              const f32x16 more = Mma<T>::m32(b, l, Mma<T>::m32(b, h, (f32x16){}));
              if (ids[r] == a) sum[i][j] += more;
            }
          }
      }
    }
  }

  T *const out = (T *)p.out;
#pragma unroll
  for (int i = 0; i < K::FM; ++i) {
    const int row = row0 + (wm * K::FM + i) * 32 + l32;
    if (row >= p.rows) continue;
#pragma unroll
    for (int j = 0; j < K::FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = col0 + (wn * K::FN + j) * 32 + 8 * e + 4 * half;
        T *dst = out + row * p.out_stride + col;
        float y[4] = {sum[i][j][4 * e], sum[i][j][4 * e + 1], sum[i][j][4 * e + 2], sum[i][j][4 * e + 3]};
        if (col + 4 <= p.out_dim) {
          store_f32<T, 4>(dst, y);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (col + c < p.out_dim) dst[c] = (T)y[c];
        }
      }
  }
}

// ------------------------------------------------------------------ host side

struct DownPlan {
  int rank_pad, splits, split_len;
};

// Splits of the inner dimension for v: enough workgroups for the chip at few rows, none shorter
// than 256 elements.
DownPlan down_plan(int rows, int in_dim, int max_rank) {
  const int groups = (rows + DOWN_ROWS - 1) / DOWN_ROWS;
  int splits = 512 / groups;
  const int most = (in_dim + 255) / 256;
  splits = splits < 1 ? 1 : splits > most ? most : splits;
  splits = splits > 16 ? 16 : splits;
  const int each = (in_dim + splits - 1) / splits, len = (each + 31) & ~31;
  return {(max_rank + 15) & ~15, (in_dim + len - 1) / len, len};
}

int project_check(const jdob_edge_project_args *a, bool sizes_only) {
  if (!a || a->rows < 0 || a->in_dim < 1 || a->out_dim < 1 || a->num_adapters < 0 ||
      (a->bits8 != 0 && a->bits8 != 1))
    return JDOB_ERR_INVALID_ARG;
  if (a->num_adapters > 0 && a->max_rank < 1) return JDOB_ERR_INVALID_ARG;
  if (a->dtype != JDOB_EDGE_BF16 && a->dtype != JDOB_EDGE_F16) return JDOB_ERR_UNSUPPORTED;
  if (a->num_adapters > 0 && a->max_rank > JDOB_EDGE_MAX_RANK) return JDOB_ERR_UNSUPPORTED;
  if (a->in_dim > (1 << 20) || a->out_dim > (1 << 20) || (a->bits8 && a->in_dim > 131072))
    return JDOB_ERR_UNSUPPORTED;
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

template <typename T, typename X>
int launch_down(const ProjectParams &p, hipStream_t stream) {
  const int groups = (p.rows + DOWN_ROWS - 1) / DOWN_ROWS;
  // few rows may all have adapters of their own: those are dealt to several workgroups
  const dim3 grid((unsigned)groups, (unsigned)p.splits, groups <= 4 ? 8 : 1);
  constexpr int threads = DOWN_WAVES * WAVE;
  if (p.max_rank <= 16) return launch(down_kernel<T, X, 1>, grid, threads, stream, p);
  if (p.max_rank <= 32) return launch(down_kernel<T, X, 2>, grid, threads, stream, p);
  return launch(down_kernel<T, X, 4>, grid, threads, stream, p);
}

template <typename T, bool X8, bool FAST, int BM, int BN, int WM, int WN>
int launch_tile(const ProjectParams &p, hipStream_t stream) {
  const int64_t tiles = (int64_t)((p.rows + BM - 1) / BM) * ((p.out_dim + BN - 1) / BN);
  if (tiles > 0x7fffffff) return JDOB_ERR_UNSUPPORTED;
  return launch(tile_kernel<T, X8, FAST, BM, BN, WM, WN>, dim3((unsigned)tiles), WM * WN * WAVE,
                stream, p);
}

template <typename T, bool X8>
int project(const ProjectParams &p, hipStream_t stream) {
  if (p.num_adapters > 0) {
    const int code = X8 ? launch_down<T, int8_t>(p, stream) : launch_down<T, T>(p, stream);
    if (code != JDOB_OK) return code;
  }
  const bool fast = (uintptr_t)p.x % 16 == 0 && (uintptr_t)p.w % 16 == 0 && p.x_pitch % 16 == 0 &&
                    p.w_pitch % 16 == 0 && p.in_dim * (X8 ? 1 : 2) % 16 == 0;
  if (!fast) return launch_tile<T, X8, false, 128, 128, 2, 2>(p, stream);
  return launch_tile<T, X8, true, 128, 128, 2, 2>(p, stream);
}

}  // namespace
}  // namespace edge

extern "C" int64_t jdob_edge_project_workspace(const jdob_edge_project_args *a) {
  using namespace edge;
  if (project_check(a, true) != JDOB_OK) return -1;
  if (a->num_adapters == 0 || a->rows == 0) return 0;
  const DownPlan d = down_plan(a->rows, a->in_dim, a->max_rank);
  return (int64_t)d.splits * a->rows * d.rank_pad * (int64_t)sizeof(float);
}

extern "C" int jdob_edge_project(const jdob_edge_project_args *a, void *hip_stream) {
  using namespace edge;
  const int code = project_check(a, false);
  if (code != JDOB_OK || a->rows == 0) return code;
  const int size = a->bits8 ? 1 : 2;
  ProjectParams p = {a->rows, a->in_dim, a->out_dim, (const char *)a->x, (const char *)a->weight,
                     a->x_stride * size, a->weight_stride * size, a->x_scale, a->weight_scale,
                     a->num_adapters, a->max_rank, a->down, a->up, a->gain, a->rank,
                     a->row_adapter, (float *)a->workspace, 0, 0, 0, a->out, a->out_stride};
  if (a->num_adapters > 0) {
    const DownPlan d = down_plan(a->rows, a->in_dim, a->max_rank);
    p.rank_pad = d.rank_pad;
    p.splits = d.splits;
    p.split_len = d.split_len;
  }
  hipStream_t stream = (hipStream_t)hip_stream;
  if (a->dtype == JDOB_EDGE_BF16)
    return a->bits8 ? project<__bf16, true>(p, stream) : project<__bf16, false>(p, stream);
  return a->bits8 ? project<_Float16, true>(p, stream) : project<_Float16, false>(p, stream);
}
