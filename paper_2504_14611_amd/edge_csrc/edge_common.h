// Shared by the edge operators' kernels: element types, vector access, wave reductions, launches.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "jdob.h"
#include "jdob_edge.h"

namespace edge {

constexpr int WAVE = 64;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// N elements of T as they stand in memory: aligned to the element only (the hardware reads and
// writes 16 bytes at any address; whole lines are moved either way).
template <typename T, int N>
struct Raw {
  typedef T type __attribute__((ext_vector_type(N), aligned(alignof(T))));
};

template <typename T, int N>
__device__ inline void load_f32(float *dst, const T *src) {
  const typename Raw<T, N>::type v = *(const typename Raw<T, N>::type *)src;
#pragma unroll
  for (int i = 0; i < N; ++i) dst[i] = (float)v[i];
}

template <typename T, int N>
__device__ inline void store_f32(T *dst, const float *src) {
  typename Raw<T, N>::type v;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (T)src[i];
  *(typename Raw<T, N>::type *)dst = v;
}

__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

__device__ inline unsigned wave_max(unsigned x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const unsigned y = __shfl_xor(x, d);
    x = y > x ? y : x;
  }
  return x;
}

// Launches a kernel of one parameter struct and returns the status of this launch alone.
template <typename P>
inline int launch(void (*kernel)(P), dim3 grid, int threads, hipStream_t stream, P params) {
  void *args[] = {&params};
  return hipLaunchKernel((const void *)kernel, grid, dim3(threads), args, 0, stream) == hipSuccess
             ? JDOB_OK
             : JDOB_ERR_HIP;
}

}  // namespace edge
