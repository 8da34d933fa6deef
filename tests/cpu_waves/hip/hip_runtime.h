// Kernels on the CPU, for tests of which memory they touch: stands in for the HIP
// runtime's header where a kernel's source is compiled for the host.  A workgroup's
// threads are threads, and the lanes of a wave meet at every operation across lanes
// (so those have to be reached by all lanes, as in the kernels tested here).
// Conversions to and from FP4 give zeros.
#pragma once

#include <algorithm>
#include <barrier>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <thread>
#include <type_traits>
#include <vector>

#define __global__
#define __device__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
inline thread_local dim3 threadIdx, blockIdx;
inline dim3 gridDim;
struct uint2 { uint32_t x, y; };
struct uint4 { uint32_t x, y, z, w; };
struct float2 { float x, y; };
struct float4 { float x, y, z, w; };
struct double2 { double x, y; };
typedef int hipError_t;
typedef void *hipStream_t;
typedef void *hipEvent_t;
constexpr int hipSuccess = 0;
inline int hipGetLastError() { return hipSuccess; }
using std::max;
using std::min;

namespace cpu {

struct Wave {
  std::barrier<> meet{64};
  int64_t lane[64];
};
inline Wave *waves;
inline std::barrier<> *group;
inline int lane() { return threadIdx.x & 63; }

// fn(what every lane gave)
template <typename F>
auto across(int64_t x, F &&fn) {
  Wave &w = waves[threadIdx.x >> 6];
  w.lane[lane()] = x;
  w.meet.arrive_and_wait();
  const auto r = fn(w.lane);
  w.meet.arrive_and_wait();
  return r;
}
inline int readlane(int x, int l) { return across(x, [&](int64_t *v) { return (int)v[l & 63]; }); }
inline int readfirstlane(int x) { return x; }   // (of values that all lanes agree on)
inline int dpp(int old, int x, int ctrl, int rows, int, bool) {
  return across(x, [&](int64_t *v) {
    const int l = lane(), row = l / 16;
    if ((rows >> row & 1) == 0) return old;
    if (ctrl > 0x110 && ctrl < 0x120) return l % 16 >= (ctrl & 15) ? (int)v[l - (ctrl & 15)] : old;   // shift in the row
    if (ctrl == 0x142) return row > 0 ? (int)v[16 * row - 1] : old;   // the last lane of the row before
    if (ctrl == 0x143) return row > 1 ? (int)v[31] : old;
    std::abort();
  });
}
template <typename... T> uint32_t zero(T...) { return 0; }

template <typename F>
void launch(dim3 grid, dim3 block, F &&fn) {
  gridDim = grid;
  for (unsigned y = 0; y < grid.y; ++y) {
    for (unsigned x = 0; x < grid.x; ++x) {
      std::unique_ptr<Wave[]> w(new Wave[block.x / 64]);
      std::barrier<> g(block.x);
      waves = w.get();
      group = &g;
      std::vector<std::thread> threads;
      for (unsigned t = 0; t < block.x; ++t)
        threads.emplace_back([&, t] {
          threadIdx = dim3(t);
          blockIdx = dim3(x, y);
          fn();
          w[t >> 6].meet.arrive_and_drop();
          g.arrive_and_drop();
        });
      for (auto &t : threads) t.join();
    }
  }
}

}  // namespace cpu

inline unsigned long long __ballot(bool on) {
  return cpu::across(on, [](int64_t *v) {
    unsigned long long m = 0;
    for (int l = 0; l < 64; ++l) m |= (unsigned long long)v[l] << l;
    return m;
  });
}
inline int __any(bool on) { return __ballot(on) != 0; }
inline int __shfl_xor(int x, int m) { return cpu::across(x, [&](int64_t *v) { return (int)v[cpu::lane() ^ m]; }); }
inline int __shfl_up(int x, int d) {
  return cpu::across(x, [&](int64_t *v) { return (int)v[cpu::lane() >= d ? cpu::lane() - d : cpu::lane()]; });
}
inline void __syncthreads() { cpu::group->arrive_and_wait(); }
inline int atomicOr(int32_t *p, int bits) { return __atomic_fetch_or(p, bits, __ATOMIC_SEQ_CST); }
inline double __dmul_rn(double a, double b) { return a * b; }
inline double __dadd_rn(double a, double b) { return a + b; }
inline double __dsub_rn(double a, double b) { return a - b; }

#define __builtin_amdgcn_readlane(x, l) cpu::readlane(x, l)
#define __builtin_amdgcn_readfirstlane(x) cpu::readfirstlane(x)
#define __builtin_amdgcn_update_dpp(...) cpu::dpp(__VA_ARGS__)
#define __builtin_amdgcn_fence(...) cpu::waves[threadIdx.x >> 6].meet.arrive_and_wait()
#define __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(...) cpu::zero(__VA_ARGS__)
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(...) cpu::zero(__VA_ARGS__)
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) cpu::launch(grid, block, [&] { kernel(__VA_ARGS__); })
