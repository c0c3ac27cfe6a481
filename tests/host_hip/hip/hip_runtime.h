// Enough of HIP's names to compile the kernels' sources for the CPU and to run a workgroup of them there: every thread of the
// workgroup is a fiber, barriers and the operations of a wave switch between them. Launches do nothing, matrix and memory
// builtins are names only.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <ucontext.h>

#include <cmath>
#include <functional>
#include <initializer_list>
#include <memory>
#include <string>
#include <vector>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __shared__ thread_local  // of the one OS thread that all fibers run on
#define __align__(n) __attribute__((aligned(n)))
#define __launch_bounds__(...)
#define hipLaunchKernelGGL(...) ((void)0)
#define hipExtLaunchKernelGGL(...) ((void)0)

struct uint2 { unsigned x, y; };
struct uint4 { unsigned x, y, z, w; };
struct int4 { int x, y, z, w; };
struct float2 { float x, y; };
struct float4 { float x, y, z, w; };
inline uint2 make_uint2(unsigned x, unsigned y) { return {x, y}; }
inline uint4 make_uint4(unsigned x, unsigned y, unsigned z, unsigned w) { return {x, y, z, w}; }
inline int4 make_int4(int x, int y, int z, int w) { return {x, y, z, w}; }
inline float2 make_float2(float x, float y) { return {x, y}; }
inline float4 make_float4(float x, float y, float z, float w) { return {x, y, z, w}; }
struct dim3 {
  unsigned x, y, z;
  dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
typedef void* hipStream_t;
typedef void* hipEvent_t;
typedef int hipError_t;
enum { hipSuccess = 0 };
inline hipError_t hipGetLastError() { return hipSuccess; }
inline const char* hipGetErrorString(hipError_t) { return ""; }

// ------------------------------------------------------------------------------------------------ a workgroup of fibers
struct HostGroup {
  struct Fiber {
    ucontext_t at;
    std::unique_ptr<char[]> stack;
    bool done = false;
    int waits = 0;  // 0: runs; 1: at a barrier; 2: at an operation of its wave
    unsigned long long value = 0;
  };
  std::vector<Fiber> fibers;
  ucontext_t back;
  int current = 0;
  dim3 block, index, dim, grid;
  std::function<void()> body;
  static HostGroup*& get() {
    static HostGroup* g = nullptr;
    return g;
  }
  static void enter() {
    HostGroup* g = get();
    g->body();
    g->fibers[g->current].done = true;
    swapcontext(&g->fibers[g->current].at, &g->back);
  }
  void wait(int kind) {
    Fiber& f = fibers[current];
    f.waits = kind;
    swapcontext(&f.at, &back);
  }
  bool arrived(int a, int b, int kind) const {
    for (int i = a; i < b; i++)
      if (fibers[i].done || fibers[i].waits != kind) return false;
    return true;
  }
  // false: some threads wait for others that never come
  bool run(int threads, std::function<void()> f) {
    get() = this;
    body = f;
    dim = dim3(threads);
    fibers = std::vector<Fiber>(threads);
    for (Fiber& x : fibers) {
      x.stack.reset(new char[1 << 16]);
      getcontext(&x.at);
      x.at.uc_stack.ss_sp = x.stack.get();
      x.at.uc_stack.ss_size = 1 << 16;
      x.at.uc_link = nullptr;
      makecontext(&x.at, enter, 0);
    }
    for (;;) {
      bool all = true, moved = false;
      for (current = 0; current < threads; current++) {
        if (fibers[current].done || fibers[current].waits) continue;
        index = dim3(current, 0, 0);
        swapcontext(&back, &fibers[current].at);
        moved = true;
      }
      for (const Fiber& x : fibers) all = all && x.done;
      if (all) return true;
      if (arrived(0, threads, 1)) {
        for (Fiber& x : fibers) x.waits = 0;
        moved = true;
      }
      for (int w = 0; w < threads; w += 64)
        if (arrived(w, w + 64, 2)) {
          for (int i = w; i < w + 64; i++) fibers[i].waits = 0;
          moved = true;
        }
      if (!moved) return false;
    }
  }
};
#define threadIdx (HostGroup::get()->index)
#define blockDim (HostGroup::get()->dim)
#define blockIdx (HostGroup::get()->block)
#define gridDim (HostGroup::get()->grid)
inline void __syncthreads() { HostGroup::get()->wait(1); }

// Every lane of the wave gives a value and reads those of the others.
template <typename F>
inline unsigned long long host_wave(unsigned long long v, F pick) {
  HostGroup* g = HostGroup::get();
  const int me = g->current, lane = me & 63;
  g->fibers[me].value = v;
  g->wait(2);
  const unsigned long long r = pick([&](int l) { return g->fibers[(me & ~63) + l].value; }, lane);
  g->wait(2);
  return r;
}
inline unsigned long long __ballot(int p) {
  return host_wave(p != 0, [](auto at, int) {
    unsigned long long m = 0;
    for (int l = 0; l < 64; l++) m |= at(l) << l;
    return m;
  });
}
inline int __any(int p) { return __ballot(p) != 0; }
inline int __all(int p) { return __ballot(p) == ~0ull; }
template <typename T>
inline T __shfl(T v, int from, int width = 64) {
  unsigned long long u = 0;
  __builtin_memcpy(&u, &v, sizeof(T));
  u = host_wave(u, [=](auto at, int l) { return at((l & ~(width - 1)) | (from & (width - 1))); });
  __builtin_memcpy(&v, &u, sizeof(T));
  return v;
}
template <typename T>
inline T __shfl_xor(T v, int d, int width = 64) {
  unsigned long long u = 0;
  __builtin_memcpy(&u, &v, sizeof(T));
  u = host_wave(u, [=](auto at, int l) { return at(l ^ d); });
  __builtin_memcpy(&v, &u, sizeof(T));
  return v;
}
inline int host_readlane(int v, int from) {
  return (int)host_wave((unsigned)v, [=](auto at, int) { return at(from); });
}
// The moves between lanes that a scan uses: `old` where a row is masked out, 0 (no bound) where no lane is the source.
inline int host_dpp(int old, int src, int ctrl, int rows, int, bool) {
  return (int)host_wave((unsigned)src, [=](auto at, int l) -> unsigned long long {
    const int row = l >> 4;
    if (!(rows >> row & 1)) return (unsigned)old;
    if (ctrl >= 0x111 && ctrl <= 0x11f) return (l & 15) >= (ctrl & 15) ? at(l - (ctrl & 15)) : (unsigned)old;
    if (ctrl == 0x142) return row > 0 ? at(row * 16 - 1) : (unsigned)old;
    if (ctrl == 0x143) return l >= 32 ? at(31) : (unsigned)old;
    __builtin_trap();
  });
}
#define __builtin_amdgcn_update_dpp host_dpp
#define __builtin_amdgcn_readlane host_readlane
#define __builtin_amdgcn_readfirstlane(v) host_readlane(v, 0)

template <typename T, typename U>
inline T atomicAdd(T* p, U v) { const T o = *p; *p = o + (T)v; return o; }
template <typename T, typename U>
inline T atomicSub(T* p, U v) { const T o = *p; *p = o - (T)v; return o; }
template <typename T, typename U>
inline T atomicMax(T* p, U v) { const T o = *p; if ((T)v > o) *p = (T)v; return o; }
template <typename T, typename U>
inline T atomicOr(T* p, U v) { const T o = *p; *p = o | (T)v; return o; }

template <typename A, typename B>
inline auto min(A a, B b) -> decltype(a + b) { return a < b ? a : b; }
template <typename A, typename B>
inline auto max(A a, B b) -> decltype(a + b) { return a > b ? a : b; }
inline int __popcll(unsigned long long m) { return __builtin_popcountll(m); }
inline int __clz(int v) { return v ? __builtin_clz((unsigned)v) : 32; }
inline float __uint_as_float(uint32_t u) { float f; __builtin_memcpy(&f, &u, 4); return f; }
inline uint32_t __float_as_uint(float f) { uint32_t u; __builtin_memcpy(&u, &f, 4); return u; }
unsigned long long wall_clock64();

#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_load(p, ...) (*(p))
#define __hip_atomic_store(p, v, ...) ((void)(*(p) = (v)))
#define __hip_atomic_fetch_max(p, v, ...) atomicMax(p, v)

// Names that no test on the CPU runs.
template <typename T>
struct HostName {
  template <typename... A>
  T operator()(A...) const { __builtin_trap(); }
};
typedef __bf16 host_bf16x4 __attribute__((ext_vector_type(4)));
#define __builtin_amdgcn_s_waitcnt HostName<void>()
#define __builtin_amdgcn_perm HostName<unsigned>()
#define __builtin_amdgcn_exp2f HostName<float>()
#define __builtin_amdgcn_fdot2_f32_bf16 HostName<float>()
#define __builtin_amdgcn_global_load_lds HostName<void>()
#define __builtin_amdgcn_ds_read_tr16_b64_v4bf16 HostName<host_bf16x4>()
#define __builtin_amdgcn_sched_group_barrier HostName<void>()
