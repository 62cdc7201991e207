// RMS norm of rows with the residual's addition, in the rows' type or in 8 bits with scales.
//
//   h = x + r,  y_i = h_i w_i / sqrt(mean(h^2) + eps),  s = max|y| / 127,  q_i = round(y_i / s)
//
// Bound: HBM.  A row is read once, kept in registers as binary32 through both reductions (the sum
// of squares, then the largest |y|) and written once, so the bytes moved are the operator's own.
// A row belongs to TPR threads with NV vectors of 16 bytes each.  8191 bfloat16 rows of 4096 with a
// residual, in 8 bits: 42 us back to back, 5.5 TB/s (a large copy moves 4.8 TB/s; part of these rows stays
// in the last cache from pass to pass); 32 rows: 4.8 us, a launch.
#include "edge_common.h"

namespace edge {
namespace {

struct NormParams {
  int rows, dim;
  float eps;
  const void *x, *residual, *weight;
  void *sum, *out;
  int8_t *q;
  float *scale;
  int64_t x_stride, residual_stride, sum_stride, out_stride, q_stride;
};

// The reductions over a row's threads: within the wave by lane exchanges, then over the row's waves
// through LDS (`part`: one word a wave).
template <int TPR>
__device__ inline float row_sum(float x, float *part) {
  x = wave_sum(x);
  if constexpr (TPR > WAVE) {
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int i = 0; i < TPR / WAVE; ++i) x += part[i];
  }
  return x;
}

template <int TPR>
__device__ inline unsigned row_max(unsigned x, unsigned *part) {
  x = wave_max(x);
  if constexpr (TPR > WAVE) {
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int i = 0; i < TPR / WAVE; ++i) x = part[i] > x ? part[i] : x;
  }
  return x;
}

constexpr int norm_threads(int tpr) { return tpr < 256 ? 256 : tpr; }

template <typename T, int TPR, int NV>
__global__ __launch_bounds__(norm_threads(TPR)) void norm_kernel(NormParams p) {
  constexpr int VE = 16 / (int)sizeof(T);
  constexpr int RPB = norm_threads(TPR) / TPR;
  __shared__ float part_sum[norm_threads(TPR) / WAVE];
  __shared__ unsigned part_max[norm_threads(TPR) / WAVE], part_peak[norm_threads(TPR) / WAVE];
  const int row = (int)block_index() * RPB + threadIdx.x / TPR, t = threadIdx.x % TPR;
  if (row >= p.rows) return;  // whole waves, and with TPR > 64 whole workgroups
  const int dim = p.dim;
  const T *const x = (const T *)p.x + row * p.x_stride;
  const T *const r = p.residual ? (const T *)p.residual + row * p.residual_stride : nullptr;
  const T *const w = (const T *)p.weight;
  float h[NV][VE], g[NV][VE];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = (j * TPR + t) * VE;
    if (at + VE <= dim) {
      load_f32<T, VE>(h[j], x + at);
      load_f32<T, VE>(g[j], w + at);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        h[j][i] = at + i < dim ? (float)x[at + i] : 0.0f;
        g[j][i] = at + i < dim ? (float)w[at + i] : 0.0f;
      }
    }
  }
  if (r) {
    T *const s = p.sum ? (T *)p.sum + row * p.sum_stride : nullptr;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = (j * TPR + t) * VE;
      if (at + VE <= dim) {
        float b[VE];
        load_f32<T, VE>(b, r + at);
#pragma unroll
        for (int i = 0; i < VE; ++i) h[j][i] += b[i];
        if (s) store_f32<T, VE>(s + at, h[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (at + i < dim) {
            h[j][i] += (float)r[at + i];
            if (s) s[at + i] = (T)h[j][i];
          }
      }
    }
  }
  float ss = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VE; ++i) ss += h[j][i] * h[j][i];
  const float mean = row_sum<TPR>(ss, part_sum) / (float)dim + p.eps;
  float rms = 1.0f / sqrtf(mean);
  if (!(mean > 0x1p-90f && mean < INFINITY)) {
    // Squares that left binary32 (or none: zeros, a NaN, an infinity): once more with the row scaled by a
    // power of two that brings its largest value to [1, 2).  All threads of the row are here.
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const unsigned a = __float_as_uint(h[j][i]) & 0x7fffffffu;
        m = a > m ? a : m;
      }
    m = row_max<TPR>(m, part_peak);
    if (m > 0 && m < 0x7f800000u) {
      const int e = -ilogbf(__uint_as_float(m));
      ss = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          h[j][i] = ldexpf(h[j][i], e);
          ss += h[j][i] * h[j][i];
        }
      // (eps scaled alike may be no binary32 number)
      rms = (float)(1.0 / sqrt((double)row_sum<TPR>(ss, part_sum) / dim + ldexp((double)p.eps, 2 * e)));
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VE; ++i) h[j][i] = h[j][i] * rms * g[j][i];

  if (p.out) {
    T *const o = (T *)p.out + row * p.out_stride;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = (j * TPR + t) * VE;
      if (at + VE <= dim) {
        store_f32<T, VE>(o + at, h[j]);
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (at + i < dim) o[at + i] = (T)h[j][i];
      }
    }
  }
  if (p.q) {
    // the largest |y| by its bit pattern, which orders like the value and puts NaN above all else
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const unsigned a = __float_as_uint(h[j][i]) & 0x7fffffffu;
        m = a > m ? a : m;
      }
    const unsigned top = row_max<TPR>(m, part_max);
    const bool finite = top < 0x7f800000u;
    // 0 for a row of zeros and where binary32 holds no such number; a subnormal scale is rounded so coarsely
    // that a row's largest values may pass 127 times it
    const float scale = __uint_as_float(top) / 127.0f;
    if (t == 0) p.scale[row] = finite ? scale : __uint_as_float(0x7fc00000u);
    int8_t *const q = p.q + row * p.q_stride;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = (j * TPR + t) * VE;
      typename Raw<int8_t, VE>::type c;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float v = fminf(fmaxf(rintf(h[j][i] / scale), -127.0f), 127.0f);
        c[i] = finite && scale > 0.0f ? (int8_t)(int)v : (int8_t)0;
      }
      if (at + VE <= dim) {
        *(typename Raw<int8_t, VE>::type *)(q + at) = c;
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (at + i < dim) q[at + i] = c[i];
      }
    }
  }
}

template <typename T, int TPR, int NV>
int norm_launch(const NormParams &p, hipStream_t stream) {
  constexpr int RPB = norm_threads(TPR) / TPR;
  return launch(norm_kernel<T, TPR, NV>, (p.rows + RPB - 1) / RPB, norm_threads(TPR), stream, p);
}

template <typename T>
int norm_dispatch(const NormParams &p, hipStream_t stream) {
  constexpr int VE = 16 / (int)sizeof(T);
  const int v = (p.dim + VE - 1) / VE;  // vectors a row
  // A wave a row saves the exchange through LDS, but keeps only as many loads under way as one wave has
  // registers for: 4096 rows of 1024 (bf16, with a residual, in 8 bits; calls in a graph) take 11.1 us so and
  // 14.2 with four waves a row, 8191 rows of 4096 take 60 so and 46 with four waves, 256 rows of 4096 10.4 and 6.6.
  if (v <= 64) return norm_launch<T, 64, 1>(p, stream);
  if (v <= 128 && p.rows >= 1024) return norm_launch<T, 64, 2>(p, stream);
  if (v <= 256) return norm_launch<T, 256, 1>(p, stream);
  if (v <= 512) return norm_launch<T, 256, 2>(p, stream);
  if (v <= 1024) return norm_launch<T, 256, 4>(p, stream);
  if (v <= 2048) return norm_launch<T, 1024, 2>(p, stream);
  return norm_launch<T, 1024, 4>(p, stream);
}

int norm_check(const jdob_edge_norm_args *a) {
  if (!a || a->rows < 0 || a->dim < 1 || !(a->eps >= 0.0f) || !isfinite(a->eps))
    return JDOB_ERR_INVALID_ARG;
  if (a->dtype != JDOB_EDGE_BF16 && a->dtype != JDOB_EDGE_F16 && a->dtype != JDOB_EDGE_F32)
    return JDOB_ERR_UNSUPPORTED;
  if (a->dim > JDOB_EDGE_MAX_NORM_DIM || a->rows > JDOB_EDGE_MAX_ROWS) return JDOB_ERR_UNSUPPORTED;
  if (a->rows == 0) return JDOB_OK;
  if (!a->x || !a->weight || (!a->out && !a->q) || (a->q && !a->scale) || (a->sum && !a->residual))
    return JDOB_ERR_INVALID_ARG;
  if (a->x_stride < a->dim || (a->residual && a->residual_stride < a->dim) ||
      (a->sum && a->sum_stride < a->dim) || (a->out && a->out_stride < a->dim) ||
      (a->q && a->q_stride < a->dim))
    return JDOB_ERR_INVALID_ARG;
  return JDOB_OK;
}

}  // namespace
}  // namespace edge

extern "C" int jdob_edge_norm(const jdob_edge_norm_args *a, void *hip_stream) {
  using namespace edge;
  const int code = norm_check(a);
  if (code != JDOB_OK || a->rows == 0) return code;
  const NormParams p = {a->rows,       a->dim,     a->eps,        a->x,
                        a->residual,   a->weight,  a->sum,        a->out,
                        a->q,          a->scale,   a->x_stride,   a->residual_stride,
                        a->sum_stride, a->out_stride, a->q_stride};
  hipStream_t stream = (hipStream_t)hip_stream;
  if (a->dtype == JDOB_EDGE_BF16) return norm_dispatch<__bf16>(p, stream);
  if (a->dtype == JDOB_EDGE_F16) return norm_dispatch<_Float16>(p, stream);
  return norm_dispatch<float>(p, stream);
}
