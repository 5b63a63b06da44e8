// Just enough of HIP to run one workgroup of a kernel on the host: a fiber per thread, lanes of 64.  Threads are switched
// at barriers, wave operations and atomics, the next one drawn at random, so that what depends on the order of
// atomics shows.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <ucontext.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <memory>
#include <random>
#include <vector>

#define __host__
#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(n)
typedef int hipError_t;
typedef void* hipStream_t;
struct int2 {
  int x, y;
};
struct Dim {
  unsigned x;
};
inline Dim threadIdx;

using std::max;
using std::min;

namespace emu {

struct Fiber {
  ucontext_t at;
  std::unique_ptr<char[]> stack;
  bool done = false;
  int wave_op = 0, barrier = 0;   // how many it has reached
};
struct Group {
  std::vector<Fiber> f;
  ucontext_t main;
  std::vector<unsigned> ready;
  std::vector<unsigned long long> value;   // what each lane gave to the current wave operation
  std::mt19937 rng;
  const std::function<void()>* body = nullptr;
};
inline Group g;

inline void die(const char* what) {
  std::fprintf(stderr, "FAIL %s\n", what);
  std::exit(1);
}
inline void leave() {   // to the scheduler, and back when drawn again
  const unsigned me = threadIdx.x;
  swapcontext(&g.f[me].at, &g.main);
  threadIdx.x = me;
}
inline void start() {
  (*g.body)();
  g.f[threadIdx.x].done = true;
  leave();
}
template <class F>
void wait_for(F there) {
  while (!there()) leave();
}
// All lanes of the wave (or threads of the group) that have not ended reach the same operation.
inline void meet(int Fiber::*count, unsigned first, unsigned n) {
  const int mine = ++(g.f[threadIdx.x].*count);
  wait_for([&] {
    for (unsigned t = first; t < first + n; ++t)
      if (!g.f[t].done && g.f[t].*count < mine) return false;
    return true;
  });
}
inline unsigned wave0() { return threadIdx.x & ~63u; }
template <class T>
T exchange(T v, unsigned from) {
  static_assert(sizeof(T) <= 8);
  std::memcpy(&g.value[threadIdx.x], &v, sizeof(T));
  meet(&Fiber::wave_op, wave0(), 64);
  T r;
  std::memcpy(&r, &g.value[wave0() + from], sizeof(T));
  meet(&Fiber::wave_op, wave0(), 64);
  return r;
}

inline void run(unsigned threads, unsigned seed, const std::function<void()>& body) {
  g.rng.seed(seed);
  g.body = &body;
  g.value.assign(threads, 0);
  if (g.f.size() != threads) g.f = std::vector<Fiber>(threads);
  g.ready.resize(threads);
  constexpr size_t kStack = 64 << 10;
  for (unsigned t = 0; t < threads; ++t) {
    Fiber& f = g.f[t];
    if (!f.stack) f.stack = std::make_unique<char[]>(kStack);
    getcontext(&f.at);
    f.at.uc_stack.ss_sp = f.stack.get();
    f.at.uc_stack.ss_size = kStack;
    f.at.uc_link = nullptr;
    f.done = false;
    f.wave_op = f.barrier = 0;
    makecontext(&f.at, start, 0);
    g.ready[t] = t;
  }
  for (size_t left = threads; left;) {   // rounds, each in an order of its own
    std::shuffle(g.ready.begin(), g.ready.begin() + left, g.rng);
    for (size_t i = 0; i < left; ++i) {
      threadIdx.x = g.ready[i];
      swapcontext(&g.main, &g.f[g.ready[i]].at);
    }
    left = std::partition(g.ready.begin(), g.ready.begin() + left, [](unsigned t) { return !g.f[t].done; }) - g.ready.begin();
  }
}

}  // namespace emu

inline void __syncthreads() { emu::meet(&emu::Fiber::barrier, 0, (unsigned)emu::g.f.size()); }
template <class T>
T __shfl(T v, int from) {
  return emu::exchange(v, from & 63);
}
template <class T>
T __shfl_up(T v, int by) {
  const int lane = threadIdx.x & 63;
  return emu::exchange(v, lane >= by ? lane - by : lane);
}
template <class T>
T __shfl_xor(T v, int by) {
  return emu::exchange(v, (threadIdx.x & 63) ^ by);
}
inline unsigned long long __ballot(bool p) {
  unsigned long long r = 0;
  emu::g.value[threadIdx.x] = p;
  emu::meet(&emu::Fiber::wave_op, emu::wave0(), 64);
  for (int l = 0; l < 64; ++l) r |= emu::g.value[emu::wave0() + l] << l;
  emu::meet(&emu::Fiber::wave_op, emu::wave0(), 64);
  return r;
}
inline int __popcll(unsigned long long v) { return __builtin_popcountll(v); }
template <class T, class V, class F>
T emu_atomic(T* p, V v, F f) {
  emu::leave();
  const T old = *p;
  *p = f(old, (T)v);
  return old;
}
template <class T, class V>
T atomicAdd(T* p, V v) {
  return emu_atomic(p, v, [](T a, T b) { return a + b; });
}
template <class T, class V>
T atomicOr(T* p, V v) {
  return emu_atomic(p, v, [](T a, T b) { return a | b; });
}
template <class T, class V>
T atomicMax(T* p, V v) {
  return emu_atomic(p, v, [](T a, T b) { return std::max(a, b); });
}
