// Runs the kernels of a HIP source on the CPU, as the source stands, for tests: each thread of a
// workgroup is a fiber, the lanes of a wavefront meet in every operation between lanes, and the
// threads of a workgroup in __syncthreads.  What the kernels of vpce_seq.hip use, and no more.
// Lanes that meet in different operations, or read a lane that is not there, end the program.
#pragma once
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <functional>
#include <memory>
#include <vector>

#define __global__
#define __device__
#define __forceinline__ inline
#define __shared__ static
#define __launch_bounds__(...)

using std::max;
using std::min;

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
typedef struct ihipStream_t* hipStream_t;
enum hipError_t { hipSuccess = 0, hipErrorInvalidConfiguration = 9 };

inline dim3 threadIdx, blockIdx, gridDim;

namespace cpu {

[[noreturn]] inline void die(const char* what) {
  printf("FAILED in a kernel: %s (block %u of %u, thread %u)\n", what, blockIdx.x, gridDim.x, threadIdx.x);
  fflush(stdout);
  _Exit(1);
}

// Saves the registers that a call keeps on the stack, and goes on at another stack (x86-64; the
// library's own switch makes two system calls).
extern "C" void cpu_switch(void** from, void* to);
asm(R"(
  .text
cpu_switch:
  push %rbp
  push %rbx
  push %r12
  push %r13
  push %r14
  push %r15
  mov %rsp, (%rdi)
  mov %rsi, %rsp
  pop %r15
  pop %r14
  pop %r13
  pop %r12
  pop %rbx
  pop %rbp
  ret
)");

enum Op { NONE, BALLOT, READLANE, FIRSTLANE, SHUFFLE, DPP, BARRIER, DONE };
struct Fiber {
  void* at;  // its stack pointer while it waits
  std::unique_ptr<char[]> stack;
  Op wait = NONE;
  uint64_t value = 0;
};
struct Wave {
  uint64_t value[64];
  uint64_t active = 0;  // lanes that took part in the last operation
};
constexpr size_t kStack = 128 << 10;
inline std::vector<Fiber> fibers(1024);
inline Wave waves[16];
inline void* scheduler;
inline const std::function<void()>* body;
inline hipError_t last_error = hipSuccess;
inline long launches = 0;

inline void entry() {
  (*body)();
  Fiber& f = fibers[threadIdx.x];
  f.wait = DONE;
  cpu_switch(&f.at, scheduler);
}
inline Wave& meet(Op op, uint64_t v = 0) {
  const unsigned me = threadIdx.x;
  fibers[me].wait = op;
  fibers[me].value = v;
  cpu_switch(&fibers[me].at, scheduler);
  return waves[me / 64];
}
inline int lane() { return threadIdx.x & 63; }

inline void run_block(unsigned threads) {
  for (unsigned i = 0; i < threads; ++i) {
    Fiber& f = fibers[i];
    if (!f.stack) f.stack.reset(new char[kStack]);
    f.wait = NONE;
    // six registers, then where the switch returns to, at an address that a call would leave
    uintptr_t top = ((uintptr_t)f.stack.get() + kStack) & ~(uintptr_t)15;
    void** sp = (void**)(top - 64);
    std::fill(sp, sp + 6, nullptr);
    sp[6] = (void*)entry;
    f.at = sp;
  }
  for (;;) {
    unsigned done = 0;
    // a wavefront at a time, up to its end or to a barrier
    for (unsigned first = 0; first < threads; first += 64) {
      const unsigned last = min(threads, first + 64);
      Wave& wave = waves[first / 64];
      for (;;) {
        for (unsigned i = first; i < last; ++i)
          if (fibers[i].wait == NONE) {
            threadIdx.x = i;
            cpu_switch(&scheduler, fibers[i].at);
          }
        Op op = DONE;
        wave.active = 0;
        for (unsigned i = first; i < last; ++i) {
          const Fiber& f = fibers[i];
          if (f.wait == DONE) continue;
          threadIdx.x = i;
          if (op != DONE && f.wait != op) die("the lanes of a wavefront are in different operations");
          op = f.wait;
          wave.active |= 1ull << (i & 63);
          wave.value[i & 63] = f.value;
        }
        if (op == DONE || op == BARRIER) break;
        for (unsigned i = first; i < last; ++i)
          if (fibers[i].wait != DONE) fibers[i].wait = NONE;
      }
      done += wave.active == 0;
    }
    if (done == (threads + 63) / 64) return;
    for (unsigned i = 0; i < threads; ++i)
      if (fibers[i].wait == BARRIER) fibers[i].wait = NONE;
  }
}
inline void launch(dim3 grid, dim3 block, const std::function<void()>& f) {
  ++launches;
  if (grid.x == 0 || block.x == 0 || block.x > 1024 || grid.y != 1 || grid.z != 1 ||
      (uint64_t)grid.x * block.x >= 1ull << 32) {
    last_error = hipErrorInvalidConfiguration;
    return;
  }
  body = &f;
  gridDim = grid;
  for (unsigned b = 0; b < grid.x; ++b) {
    blockIdx.x = b;
    run_block(block.x);
  }
}

template <class T>
uint64_t bits(T v) {
  uint64_t u = 0;
  memcpy(&u, &v, sizeof v);
  return u;
}
template <class T>
T value(uint64_t u) {
  T v;
  memcpy(&v, &u, sizeof v);
  return v;
}
template <class T>
T from(Op op, T v, int source) {  // the value of another lane
  const Wave& w = meet(op, bits(v));
  if (source < 0 || source > 63 || !(w.active >> source & 1)) die("a lane that is not there is read");
  return value<T>(w.value[source]);
}
inline uint64_t ballot(bool p) {
  const Wave& w = meet(BALLOT, p);
  uint64_t m = 0;
  for (int i = 0; i < 64; ++i)
    if (w.active >> i & 1) m |= w.value[i] << i;
  return m;
}
inline int first_lane(int v) {
  const Wave& w = meet(FIRSTLANE, bits(v));
  return value<int>(w.value[__builtin_ctzll(w.active)]);
}
template <class T>
T shuffle(T v, int source) {
  return from(SHUFFLE, v, source < 0 || source > 63 ? lane() : source);
}
// quad_perm, row_shr, row_mirror, row_half_mirror, row_bcast15 and row_bcast31
inline int dpp(int old, int v, int ctrl, int rows, int banks, bool bound) {
  if (banks != 0xf || bound) die("a lane selection that is not written here");
  const int l = lane(), row = l / 16, in = l % 16;
  int s = -1;
  if (ctrl < 0x100)
    s = (l & ~3) + (ctrl >> 2 * (l & 3) & 3);
  else if (ctrl > 0x110 && ctrl < 0x120)
    s = in >= ctrl - 0x110 ? l - (ctrl - 0x110) : -1;
  else if (ctrl == 0x140)
    s = row * 16 + 15 - in;
  else if (ctrl == 0x141)
    s = (l & ~7) + 7 - (l & 7);
  else if (ctrl == 0x142)
    s = row > 0 ? row * 16 - 1 : -1;
  else if (ctrl == 0x143)
    s = l >= 32 ? 31 : -1;
  else
    die("a lane selection that is not written here");
  const Wave& w = meet(DPP, bits(v));
  if (s < 0 || !(rows >> row & 1) || !(w.active >> s & 1)) return old;
  return value<int>(w.value[s]);
}

}  // namespace cpu

inline hipError_t hipGetLastError() {
  const hipError_t e = cpu::last_error;
  cpu::last_error = hipSuccess;
  return e;
}
#define hipLaunchKernelGGL(kernel, grid, block, shared, stream, ...) \
  cpu::launch(grid, block, [&] { (kernel)(__VA_ARGS__); })

inline void __syncthreads() { cpu::meet(cpu::BARRIER); }
inline uint64_t __ballot(int p) { return cpu::ballot(p != 0); }
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
template <class T>
T __shfl_xor(T v, int m) {
  return cpu::shuffle(v, cpu::lane() ^ m);
}
template <class T>
T __shfl_up(T v, int n) {
  return cpu::shuffle(v, cpu::lane() - n);
}
template <class T>
T __shfl_down(T v, int n) {
  return cpu::shuffle(v, cpu::lane() + n);
}
inline int __float_as_int(float v) { return cpu::value<int>(cpu::bits(v)); }
inline float __int_as_float(int v) { return cpu::value<float>(cpu::bits(v)); }
#define __builtin_amdgcn_readlane(v, l) cpu::from(cpu::READLANE, (int)(v), l)
#define __builtin_amdgcn_readfirstlane(v) cpu::first_lane(v)
#define __builtin_amdgcn_update_dpp(old, v, ctrl, rows, banks, bound) cpu::dpp(old, v, ctrl, rows, banks, bound)
