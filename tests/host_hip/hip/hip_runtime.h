// Stands in for HIP's header of the same name where a kernel file is compiled
// as host code, so that the kernel's own indexing runs on a CPU, on arrays that
// end at a page without access. A launch runs its workgroups one after the
// other and a workgroup's threads as fibers; a fiber runs until it meets
// others (a barrier, an exchange between lanes) or sleeps. Waves have 64 lanes.
// Exchanges expect all lanes of a wave that have not returned.
#pragma once

#include <ucontext.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <vector>

#include "hip_runtime_api.h"

#define __device__
#define __host__
#define __global__
#define __launch_bounds__(...)
#define __shared__ static
#ifndef __HIP_MEMORY_SCOPE_AGENT
#define __HIP_MEMORY_SCOPE_AGENT 4
#endif

using std::max;
using std::min;

struct uint4 {
  unsigned x, y, z, w;
};
inline uint4 make_uint4(unsigned x, unsigned y, unsigned z, unsigned w) { return {x, y, z, w}; }
struct dim3 {
  unsigned x, y, z;
  dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};

namespace host_hip {

struct Meeting {  // of the lanes of a wave, or the threads of a workgroup
  int here = 0;
  uint64_t round = 0;
  uint64_t values[2][64];
};
struct Fiber {
  ucontext_t context;
  std::vector<char> stack;
  dim3 thread;
  int index = 0;
  bool done = false;
};
struct Group {
  std::vector<Fiber> fibers;
  std::vector<Meeting> waves;
  std::vector<int> alive;  // lanes of each wave that have not returned
  Meeting all;
  int left = 0;
  dim3 block, grid, size;
  ucontext_t scheduler;
  Fiber* now = nullptr;
  std::function<void()> body;
};
inline Group& group() {
  static Group g;
  return g;
}

inline void pause() {
  Group& g = group();
  swapcontext(&g.now->context, &g.scheduler);
}

inline void threads_meet() {
  Group& g = group();
  const uint64_t round = g.all.round;
  ++g.all.here;
  while (g.all.round == round) {
    if (g.all.here >= g.left) {
      g.all.here = 0;
      ++g.all.round;
    } else {
      pause();
    }
  }
}

// Every lane's value, in each lane of the wave.
inline const uint64_t* lanes_meet(uint64_t value) {
  Group& g = group();
  const int wave = g.now->index / 64;
  Meeting& m = g.waves[wave];
  const uint64_t round = m.round;
  if (m.here == 0) std::memset(m.values[round & 1], 0, sizeof(m.values[0]));
  m.values[round & 1][g.now->index % 64] = value;
  ++m.here;
  while (m.round == round) {
    if (m.here >= g.alive[wave]) {
      m.here = 0;
      ++m.round;
    } else {
      pause();
    }
  }
  return m.values[round & 1];
}

inline void enter_fiber() {
  Group& g = group();
  g.body();
  g.now->done = true;
  --g.left;
  --g.alive[g.now->index / 64];
  swapcontext(&g.now->context, &g.scheduler);
}

inline void launch(dim3 grid, dim3 size, std::function<void()> body) {
  Group& g = group();
  const int n = (int)(size.x * size.y * size.z);
  g.body = std::move(body);
  g.grid = grid;
  g.size = size;
  g.fibers.resize(n);
  for (unsigned z = 0; z < grid.z; ++z)
    for (unsigned y = 0; y < grid.y; ++y)
      for (unsigned x = 0; x < grid.x; ++x) {
        g.block = dim3(x, y, z);
        g.waves.assign((n + 63) / 64, Meeting());
        g.alive.assign((n + 63) / 64, 0);
        g.all = Meeting();
        g.left = n;
        for (int i = 0; i < n; ++i) {
          Fiber& f = g.fibers[i];
          ++g.alive[i / 64];
          f.index = i;
          f.done = false;
          f.thread = dim3(i % size.x, i / size.x % size.y, i / (size.x * size.y));
          f.stack.resize(64 << 10);
          getcontext(&f.context);
          f.context.uc_stack.ss_sp = f.stack.data();
          f.context.uc_stack.ss_size = f.stack.size();
          f.context.uc_link = nullptr;
          makecontext(&f.context, enter_fiber, 0);
        }
        while (g.left > 0)
          for (int i = 0; i < n; ++i)
            if (!g.fibers[i].done) {
              g.now = &g.fibers[i];
              swapcontext(&g.scheduler, &g.now->context);
            }
      }
}

struct Pair {
  uint32_t v[2];
  uint32_t operator[](int i) const { return v[i]; }
};
// (a, a): the even (lower) row's values in the first result, the odd one's in the second.
inline Pair row_swap(uint32_t a, int row) {
  const int lane = group().now->index % 64;
  const uint64_t* v = lanes_meet(a);
  return {{(uint32_t)v[lane & ~row], (uint32_t)v[lane | row]}};
}

template <class T>
T shuffle_xor(T x, int by) {
  uint64_t w = 0;
  std::memcpy(&w, &x, sizeof(T));
  const int lane = group().now->index % 64;
  w = lanes_meet(w)[lane ^ by];
  std::memcpy(&x, &w, sizeof(T));
  return x;
}

inline uint64_t ballot(bool b) {
  const uint64_t* v = lanes_meet(b);
  uint64_t r = 0;
  for (int i = 0; i < 64; ++i) r |= (v[i] & 1) << i;
  return r;
}

// The vector instructions' lane permutations in rows of 16 that the kernels use.
inline int permuted(int x, int control) {
  const int lane = group().now->index % 64;
  int from = lane;
  if (control == 0xb1) from = lane ^ 1;
  else if (control == 0x4e) from = lane ^ 2;
  else if (control == 0x141) from = (lane & ~7) | (7 - (lane & 7));
  else if (control == 0x140) from = (lane & ~15) | (15 - (lane & 15));
  else std::abort();
  return (int)lanes_meet((uint32_t)x)[from];
}

}  // namespace host_hip

#define threadIdx (host_hip::group().now->thread)
#define blockIdx (host_hip::group().block)
#define gridDim (host_hip::group().grid)
#define blockDim (host_hip::group().size)

inline void __syncthreads() { host_hip::threads_meet(); }
inline uint64_t __ballot(bool b) { return host_hip::ballot(b); }
inline int __ffs(int x) { return __builtin_ffs(x); }
template <class T>
T __shfl_xor(T x, int by, int) {
  return host_hip::shuffle_xor(x, by);
}
inline int atomicAdd(int* p, int v) {
  const int old = *p;
  *p += v;
  return old;
}
#define __hip_atomic_load(p, order, scope) (*(p))
#define __hip_atomic_store(p, v, order, scope) (*(p) = (v))
#define __builtin_amdgcn_permlane16_swap(a, b, x, y) host_hip::row_swap(a, 16)
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) host_hip::row_swap(a, 32)
#define __builtin_amdgcn_mov_dpp(v, control, x, y, z) host_hip::permuted(v, control)
#define __builtin_amdgcn_sched_barrier(n)
#define __builtin_amdgcn_s_waitcnt(n) std::abort()
#define __builtin_amdgcn_global_load_lds(...) std::abort()
#define __builtin_amdgcn_s_sleep(n) host_hip::pause()
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_exp2f(x) std::exp2(x)
#define __builtin_amdgcn_readfirstlane(x) ((int)host_hip::lanes_meet((uint32_t)(x))[0])
