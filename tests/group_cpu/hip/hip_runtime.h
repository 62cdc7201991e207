// Workgroups of several 64-lane waves on the CPU: what the edge operators' sources use of the HIP runtime and of
// the gfx950 builtins, so that they compile as C++ and run one workgroup at a time, for tests that check what a
// kernel reads and writes, and when, without a GPU.
//
// The lanes are coroutines.  A lane runs until it meets an operation that involves others: one of its wave (a
// matrix product, a lane move, a fence between lanes) waits for the wave's other lanes, a barrier for the
// workgroup's.  Lanes, and waves between two barriers, run one after the other, lowest first or highest first:
// what one of them must not do before another has read or written shows in the result.  Loads from memory to
// LDS are done when they are issued, or only when a wait asks for them.
#ifndef GROUP_CPU_H
#define GROUP_CPU_H

#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <deque>
#include <math.h>
#include <stdint.h>

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
typedef struct ihipStream_t *hipStream_t;

namespace group_cpu {

constexpr int MOST = 1024, WAVE = 64;
constexpr size_t STACK = 192 * 1024;

enum State { READY, AT_WAVE, AT_GROUP, DONE };
struct Load { const char *from; char *to; };

struct Wave {
  unsigned epoch;
  struct { const char *kind[WAVE]; uint64_t v[WAVE]; uint64_t present; } slot[2];
};

struct Group {
  void *main_sp, *sp[MOST];
  char *stack[MOST];
  State state[MOST];
  std::deque<Load> loads[MOST];
  Wave wave[MOST / WAVE];
  int threads = 0, lane = 0;
  dim3 block, grid;
  bool any[2];          // of the lanes at a barrier
  unsigned barriers;
  bool descending = false, late = false;
  void (*body)(void *);
  void *arg;
  int tile = 0;         // which tiles many rows are given (tests choose them)
};

inline Group &g() {
  static Group x;
  return x;
}

extern "C" void group_cpu_switch(void **from, void *to);
asm(".text\n.weak group_cpu_switch\n.type group_cpu_switch,@function\ngroup_cpu_switch:\n"
    "  push %rbp\n  push %rbx\n  push %r12\n  push %r13\n  push %r14\n  push %r15\n"
    "  mov %rsp, (%rdi)\n  mov %rsi, %rsp\n"
    "  pop %r15\n  pop %r14\n  pop %r13\n  pop %r12\n  pop %rbx\n  pop %rbp\n  ret\n"
    ".size group_cpu_switch, .-group_cpu_switch\n");

[[noreturn]] inline void die(const char *what) {
  fprintf(stderr, "group_cpu: %s (block %u %u %u, thread %d)\n", what, g().block.x, g().block.y, g().block.z, g().lane);
  fflush(stderr);
  abort();
}

inline void suspend(State s) {
  Group &x = g();
  x.state[x.lane] = s;
  group_cpu_switch(&x.sp[x.lane], x.main_sp);
}

inline void lane_main() {
  Group &x = g();
  x.body(x.arg);
  if (!x.loads[x.lane].empty()) die("loads to LDS are under way when the lane ends");
  suspend(DONE);
  abort();
}

// Waits for the wave's other lanes (those that wait for the workgroup aside) and returns what they brought.
struct Met { const uint64_t *v; uint64_t present; };
inline Met meet(const char *kind, uint64_t v) {
  Group &x = g();
  Wave &w = x.wave[x.lane / WAVE];
  const int l = x.lane % WAVE;
  auto &s = w.slot[(w.epoch + 1) & 1];
  s.kind[l] = kind;
  s.v[l] = v;
  suspend(AT_WAVE);
  auto &met = w.slot[w.epoch & 1];
  return {met.v, met.present};
}

inline bool barrier(bool b) {
  Group &x = g();
  const unsigned n = x.barriers;
  x.any[n & 1] |= b;
  suspend(AT_GROUP);
  return x.any[n & 1];
}

inline void release(int wave) {
  Group &x = g();
  Wave &w = x.wave[wave];
  auto &s = w.slot[++w.epoch & 1];
  s.present = 0;
  const char *kind = nullptr;
  for (int l = 0; l < WAVE; ++l) {
    const int t = wave * WAVE + l;
    if (x.state[t] != AT_WAVE) continue;
    if (kind && strcmp(kind, s.kind[l])) {
      fprintf(stderr, "group_cpu: %s and %s\n", kind, s.kind[l]);
      die("lanes of a wave meet different operations");
    }
    kind = s.kind[l];
    s.present |= uint64_t(1) << l;
    x.state[t] = READY;
  }
}

inline void run_block(int threads) {
  Group &x = g();
  const int waves = (threads + WAVE - 1) / WAVE;
  x.threads = threads;
  x.barriers = 0;
  x.any[0] = x.any[1] = false;
  for (int t = 0; t < threads; ++t) {
    if (!x.stack[t]) x.stack[t] = (char *)malloc(STACK);
    void **sp = (void **)(((uintptr_t)x.stack[t] + STACK) & ~uintptr_t(63));
    *--sp = nullptr;
    *--sp = (void *)&lane_main;
    for (int r = 0; r < 6; ++r) *--sp = nullptr;
    x.sp[t] = sp;
    x.state[t] = READY;
    x.loads[t].clear();
  }
  for (int w = 0; w < waves; ++w) x.wave[w].epoch = 0;
  for (;;) {
    bool waits = false;
    for (int i = 0; i < waves; ++i) {
      const int w = x.descending ? waves - 1 - i : i;
      for (;;) {
        bool met = false;
        for (int j = 0; j < WAVE; ++j) {
          const int t = w * WAVE + (x.descending ? WAVE - 1 - j : j);
          if (t < threads && x.state[t] == READY) {
            x.lane = t;
            group_cpu_switch(&x.main_sp, x.sp[t]);
          }
        }
        for (int t = w * WAVE; t < (w + 1) * WAVE && t < threads; ++t) {
          met |= x.state[t] == AT_WAVE;
          waits |= x.state[t] == AT_GROUP;
        }
        if (!met) break;
        release(w);
      }
    }
    if (!waits) return;
    x.any[++x.barriers & 1] = false;
    for (int t = 0; t < threads; ++t)
      if (x.state[t] == AT_GROUP) x.state[t] = READY;
  }
}

template <typename F>
bool run(F &&f, dim3 grid, int threads) {
  Group &x = g();
  if (threads > MOST) die("too many threads");
  x.body = [](void *p) { (*(typename std::remove_reference<F>::type *)p)(); };
  x.arg = &f;
  x.grid = grid;
  for (unsigned z = 0; z < grid.z; ++z)
    for (unsigned y = 0; y < grid.y; ++y)
      for (unsigned b = 0; b < grid.x; ++b) {
        x.block = dim3(b, y, z);
        run_block(threads);
      }
  return true;
}

// ---- memory to LDS: an LDS address is a distance from here
inline char here;
inline unsigned lds_offset(const void *p) { return (unsigned)((uintptr_t)p - (uintptr_t)&here); }
inline void load(const void *from, unsigned to) {
  Group &x = g();
  const Load l = {(const char *)from, (char *)((uintptr_t)&here + (intptr_t)(int)to) + x.lane % WAVE * 16};
  if (x.late) {
    x.loads[x.lane].push_back(l);
  } else {
    memcpy(l.to, l.from, 16);
  }
}
inline void wait(size_t most) {
  auto &q = g().loads[g().lane];
  for (; q.size() > most; q.pop_front()) memcpy(q.front().to, q.front().from, 16);
  meet("wait", 0);
}

template <typename V>
inline uint64_t bits(V v) {
  uint64_t u = 0;
  memcpy(&u, &v, sizeof v);
  return u;
}
template <typename V>
inline V value(uint64_t u) {
  V v;
  memcpy(&v, &u, sizeof v);
  return v;
}
template <typename V>
inline V of_lane(const char *kind, V v, int from) {
  const Met m = meet(kind, bits(v));
  if (from < 0 || from >= WAVE || !(m.present >> from & 1)) die("a value of a lane that is not there");
  return value<V>(m.v[from]);
}

// What f makes of the operands that the wave's lanes brought; none goes on before all have it.
template <typename R, typename A, typename F>
inline R together(const char *kind, const A &mine, F f) {
  const Met m = meet(kind, (uint64_t)&mine);
  if (m.present != ~uint64_t(0)) die("a wave's operation without all of its lanes");
  const A *all[WAVE];
  for (int l = 0; l < WAVE; ++l) all[l] = (const A *)m.v[l];
  const R r = f(all, g().lane % WAVE);
  meet("done", 0);
  return r;
}

// D = A B + C: SIDE rows and columns, lane l brings K elements of A's row and B's column l % SIDE from element
// l / SIDE * K on, and holds of column l % SIDE the rows 4 (l / SIDE) .. + 3, with 32 rows those of every eight.
template <int SIDE, int K, typename E, typename S, typename C>
inline C product(const void *a, const void *b, C c) {
  struct Operands { E a[K], b[K]; } mine;
  memcpy(mine.a, a, sizeof mine.a);
  memcpy(mine.b, b, sizeof mine.b);
  return together<C>("product", mine, [&](const Operands *const *all, int lane) {
    constexpr int PARTS = WAVE / SIDE;
    for (int e = 0; e < SIDE * SIDE / WAVE; ++e) {
      const int row = SIDE == 16 ? lane / 16 * 4 + e : 8 * (e / 4) + 4 * (lane / 32) + e % 4, col = lane % SIDE;
      S s = c[e];
      for (int p = 0; p < PARTS; ++p)
        for (int k = 0; k < K; ++k)
          s = (S)(s + (S)all[p * SIDE + row]->a[k] * (S)all[p * SIDE + col]->b[k]);
      c[e] = s;
    }
    return c;
  });
}

struct Dim { unsigned x; };

}  // namespace group_cpu

extern "C" inline void __attribute__((used)) group_cpu_mode(int descending, int late, int tile) {
  group_cpu::g().descending = descending;
  group_cpu::g().late = late;
  group_cpu::g().tile = tile;
}

#define __global__
#define __device__
#define __shared__ static
#define __align__(n) __attribute__((aligned(n)))
#define __launch_bounds__(...)
#define threadIdx (group_cpu::Dim{(unsigned)group_cpu::g().lane})
#define blockIdx (group_cpu::g().block)
#define gridDim (group_cpu::g().grid)
#define __syncthreads() ((void)group_cpu::barrier(false))
#define __syncthreads_or(b) group_cpu::barrier(b)

inline unsigned __float_as_uint(float v) { return group_cpu::value<unsigned>(group_cpu::bits(v)); }
inline float __uint_as_float(unsigned v) { return group_cpu::value<float>(v); }

inline unsigned long long __ballot(bool b) {
  const group_cpu::Met m = group_cpu::meet("ballot", b);
  unsigned long long r = 0;
  for (int l = 0; l < group_cpu::WAVE; ++l)
    if (m.present >> l & 1) r |= (unsigned long long)m.v[l] << l;
  return r;
}
inline bool __any(bool b) { return __ballot(b) != 0; }
template <typename V>
inline V __shfl_xor(V v, int m) {
  return group_cpu::of_lane("shfl_xor", v, group_cpu::g().lane % 64 ^ m);
}
template <typename V>
inline V __shfl_up(V v, int d) {
  const int l = group_cpu::g().lane % 64;
  return group_cpu::of_lane("shfl_up", v, l < d ? l : l - d);
}

#define __builtin_amdgcn_fence(...) ((void)group_cpu::meet("fence", 0))
#define __builtin_amdgcn_sched_barrier(n) ((void)0)
#define __builtin_amdgcn_s_barrier() ((void)group_cpu::barrier(false))
#define __builtin_amdgcn_readlane(v, l) group_cpu::of_lane<int>("readlane", (int)(v), (l))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_frexp_expf(x) group_cpu_exponent(x)
#define __builtin_amdgcn_permlane32_swap(a, b, fi, bc) group_cpu_swap32(a, b)
#define __builtin_amdgcn_permlane16_swap(a, b, fi, bc) group_cpu_swap16(a, b)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) group_cpu_transposed(p)
#define __builtin_amdgcn_readfirstlane(v) group_cpu_first(v)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) group_cpu_mfma<16, 8, __bf16, float>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) group_cpu_mfma<16, 8, _Float16, float>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) group_cpu_mfma<16, 1, float, float>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) group_cpu_mfma<32, 8, __bf16, float>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) group_cpu_mfma<32, 8, _Float16, float>(a, b, c)
#define __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, x, y, z) group_cpu_mfma<16, 16, signed char, unsigned>(a, b, c)
#define __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, x, y, z) group_cpu_mfma<32, 16, signed char, unsigned>(a, b, c)

// A window of memory: what is read from behind its end is zero, and nothing stands half behind it.
struct group_cpu_window {
  const char *at;
  unsigned bytes;
};
#define __amdgpu_buffer_rsrc_t group_cpu_window
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, n, flags) (group_cpu_window{(const char *)(p), (unsigned)(n)})
template <typename V>
inline V group_cpu_window_load(group_cpu_window w, unsigned offset) {
  V v;
  memset(&v, 0, sizeof v);
  if (offset >= w.bytes) return v;
  if (w.bytes - offset < sizeof v) group_cpu::die("a load stands half behind a window's end");
  memcpy(&v, w.at + offset, sizeof v);
  return v;
}
typedef unsigned group_cpu_u2 __attribute__((ext_vector_type(2)));
typedef unsigned group_cpu_u4 __attribute__((ext_vector_type(4)));
#define __builtin_amdgcn_raw_buffer_load_b16(w, v, s, a) group_cpu_window_load<unsigned short>(w, (v) + (s))
#define __builtin_amdgcn_raw_buffer_load_b32(w, v, s, a) group_cpu_window_load<unsigned>(w, (v) + (s))
#define __builtin_amdgcn_raw_buffer_load_b64(w, v, s, a) group_cpu_window_load<group_cpu_u2>(w, (v) + (s))
#define __builtin_amdgcn_raw_buffer_load_b128(w, v, s, a) group_cpu_window_load<group_cpu_u4>(w, (v) + (s))

inline int group_cpu_exponent(float x) {
  int e = 0;
  if (std::isfinite(x)) frexpf(x, &e);
  return e;
}
template <typename V>
inline V group_cpu_first(V v) {
  const group_cpu::Met m = group_cpu::meet("readfirstlane", group_cpu::bits(v));
  return group_cpu::value<V>(m.v[__builtin_ctzll(m.present)]);
}
struct group_cpu_two {
  unsigned v[2];
  unsigned operator[](int i) const { return v[i]; }
};
inline group_cpu_two group_cpu_swap32(unsigned a, unsigned b) {
  const int l = group_cpu::g().lane % 64;
  const unsigned lo = group_cpu::of_lane("permlane32", b, l & 31), hi = group_cpu::of_lane("permlane32", a, l | 32);
  return {{l < 32 ? a : lo, l < 32 ? hi : b}};
}
inline group_cpu_two group_cpu_swap16(unsigned a, unsigned b) {  // odd rows of 16 of a and even rows of b change places
  const int l = group_cpu::g().lane % 64;
  const unsigned lo = group_cpu::of_lane("permlane16", b, l & ~16), hi = group_cpu::of_lane("permlane16", a, l | 16);
  return {{l & 16 ? lo : a, l & 16 ? b : hi}};
}
// Sixteen lanes' eight bytes are four rows of sixteen elements; a lane gets its column.
template <typename V>
inline V group_cpu_transposed(V *p) {
  return group_cpu::together<V>("transpose", p, [](V *const *const *all, int lane) {
    V r;
    for (int i = 0; i < 4; ++i) r[i] = (**all[lane / 16 * 16 + i * 4 + lane % 16 / 4])[lane % 4];
    return r;
  });
}
template <int SIDE, int K, typename E, typename S, typename F, typename C>
inline C group_cpu_mfma(const F &a, const F &b, C c) {
  return group_cpu::product<SIDE, K, E, S>(&a, &b, c);
}

#endif  // GROUP_CPU_H
