// What the kernels around a generated token use beyond hip_runtime.h, on the CPU.  MFMAs
// leave their sums as they are.
#pragma once

#include <hip/hip_runtime.h>

template <typename T>
T any_lane(T x, int l) {
  static_assert(sizeof(T) <= 8);
  int64_t bits = 0;
  std::memcpy(&bits, &x, sizeof(T));
  bits = cpu::across(bits, [&](int64_t *v) { return v[l & 63]; });
  T y;
  std::memcpy(&y, &bits, sizeof(T));
  return y;
}
inline float __shfl_xor(float x, int m) { return any_lane(x, cpu::lane() ^ m); }
inline double __shfl_xor(double x, int m) { return any_lane(x, cpu::lane() ^ m); }
inline int __shfl(int x, int l) { return any_lane(x, l); }
inline double __shfl(double x, int l) { return any_lane(x, l); }
inline uint32_t atomicOr(uint32_t *p, uint32_t bits) { return __atomic_fetch_or(p, bits, __ATOMIC_SEQ_CST); }
inline int atomicAdd(int32_t *p, int n) { return __atomic_fetch_add(p, n, __ATOMIC_SEQ_CST); }
inline unsigned long long atomicAdd(unsigned long long *p, unsigned long long n) {
  return __atomic_fetch_add(p, n, __ATOMIC_SEQ_CST);
}
template <typename A, typename B, typename C>
C same(A, B, C c, int, int, int) { return c; }

struct int2 { int x, y; };
// The moves within 16 lanes that hip_runtime.h has not.
inline int more_dpp(int old, int x, int ctrl, int rows, int banks, bool bound) {
  const int l = cpu::lane();
  switch (ctrl) {
    case 0xB1: return any_lane(x, l ^ 1);
    case 0x4E: return any_lane(x, l ^ 2);
    case 0x124: return any_lane(x, (l & ~15) | ((l - 4) & 15));
    case 0x128: return any_lane(x, (l & ~15) | ((l - 8) & 15));
    case 0x141: return any_lane(x, l ^ 7);
    case 0x140: return any_lane(x, l ^ 15);
  }
  return cpu::dpp(old, x, ctrl, rows, banks, bound);
}
#undef __builtin_amdgcn_update_dpp
#define __builtin_amdgcn_update_dpp(...) more_dpp(__VA_ARGS__)

// 16 bytes a lane to LDS, zeros from outside the buffer
struct Buffer {
  const char *base;
  uint32_t bytes;
};
inline void buffer_to_lds(Buffer b, void *to, int size, uint32_t lane_offset, uint32_t offset, int, int) {
  char *mine = static_cast<char *>(to) + size * cpu::lane();
  if ((uint64_t)lane_offset + offset + size <= b.bytes) std::memcpy(mine, b.base + lane_offset + offset, size);
  else std::memset(mine, 0, size);
}

#define __builtin_amdgcn_make_buffer_rsrc(p, stride, n, flags) (Buffer{static_cast<const char *>(p), n})
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(...) buffer_to_lds(__VA_ARGS__)
#define __builtin_amdgcn_s_waitcnt(n) cpu::waves[threadIdx.x >> 6].meet.arrive_and_wait()
#define address_space(n) aligned(1)
#define __builtin_amdgcn_exp2f(x) std::exp2(x)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(...) same(__VA_ARGS__)

#include <sys/mman.h>

#include <cstdio>

// `bytes` of memory that end where the next page begins, which cannot be touched, and begin
// behind one that cannot (to the page).
inline void *guarded(size_t bytes, size_t align) {
  const size_t size = (bytes + 4095) / 4096 * 4096;
  char *m = static_cast<char *>(mmap(nullptr, size + 8192, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0)) + 4096;
  if (size > 0 && mprotect(m, size, PROT_READ | PROT_WRITE) != 0) std::abort();
  return m + (size - bytes) / align * align;
}

// An array of `n` from standard input.
template <typename T>
T *input(size_t n, size_t align = sizeof(T)) {
  T *p = static_cast<T *>(guarded(n * sizeof(T), align));
  if (std::fread(p, sizeof(T), n, stdin) != n) std::abort();
  return p;
}
template <typename T>
void output(const T *p, size_t n) {
  if (std::fwrite(p, sizeof(T), n, stdout) != n) std::abort();
}
