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
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
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

// The thread's wave, as a value that the compiler knows to be the same for all lanes.
__device__ inline int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE); }

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

// Loads 16 bytes a lane from memory to LDS without registers between: lane l's to to + 16 l, where `to`
// is the same for all lanes of the wave.  The compiler does not count these loads (it would wait for
// all of them before the next read of any LDS array that it cannot tell from the target): whoever
// reads the target waits for them with wait_loads and passes a barrier first.  The source is the sum
// of the wave's own base and a lane's offset of 32 bits, or a lane's own address.  (M0, which holds the
// target, is not the compiler's to allocate: it writes M0 itself before each instruction that reads it.)
__device__ inline unsigned lds_address(const void *p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}
__device__ inline void load_to_lds(const void *base, unsigned offset, unsigned to) {
  const uint64_t b = (uint64_t)base;
  const uint64_t same = (uint64_t)__builtin_amdgcn_readfirstlane((unsigned)(b >> 32)) << 32 |
                        (unsigned)__builtin_amdgcn_readfirstlane((unsigned)b);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(same)
               : "memory");
}
__device__ inline void load_to_lds(const void *from, unsigned to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
               : "memory");
}

// Waits until at most N of the wave's loads are under way, and none of its LDS accesses.
template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "i"(N) : "memory");
}

// Between a wave's stores to LDS and other lanes' reads of them, and between those reads and the next
// stores: the hardware takes a wave's LDS accesses in order, and so must the compiler, which knows a lane's only.
__device__ inline void lanes_meet() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A barrier that waits for nothing but the waves.
__device__ inline void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A dimension of a grid takes fewer than 2^32 threads: more than FOLD workgroups stand in rows of FOLD, and
// those behind the last one, in the last row, have nothing to do.
constexpr int FOLD = 1 << 21, MAX_BLOCKS = 0x7fffffff - FOLD;

__device__ inline unsigned block_index() { return blockIdx.y * FOLD + blockIdx.x; }

// Launches a kernel of one parameter struct with `blocks` workgroups, to MAX_BLOCKS, in each of `layers`, and
// returns the status of this launch alone.
template <typename P>
inline int launch(void (*kernel)(P), int64_t blocks, int threads, hipStream_t stream, P params, int layers = 1) {
  void *args[] = {&params};
  const int64_t rows = (blocks + FOLD - 1) / FOLD;
  const dim3 grid((unsigned)(rows > 1 ? FOLD : blocks), (unsigned)rows, (unsigned)layers);
  return hipLaunchKernel((const void *)kernel, grid, dim3(threads), args, 0, stream) == hipSuccess
             ? JDOB_OK
             : JDOB_ERR_HIP;
}

}  // namespace edge
