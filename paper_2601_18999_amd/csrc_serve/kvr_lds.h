// kvr_lds.h - loads from memory straight to LDS, and the waits for them; LDS
// beyond a kernel's default limit.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

namespace kvr {
namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef const __attribute__((address_space(1))) int32_t* global_ints;
typedef const __attribute__((address_space(1))) char* global_bytes;

// Loads from memory straight to LDS: lane i's 16 (4) bytes to `to` + 16 i
// (4 i), `to` the same in all lanes.  The compiler does not see these loads:
// wait_loads<n> waits until at most n of them are in flight.  (M0 may not be
// read in the cycle after it is written.  The compiler keeps values of its own
// there, so it is named as written.)
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_char*)p);
}
__device__ __forceinline__ void load16_to_lds(global_bytes from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from),
               "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory", "m0");
}
__device__ __forceinline__ void load4_to_lds(global_ints from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from),
               "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory", "m0");
}
// The same with one base for the wave and 32-bit offsets.
__device__ __forceinline__ void load16_to_lds(uint64_t base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// every read of LDS by this wave has been answered
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// a barrier that does not wait for loads in flight
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Once a device: LDS beyond the default limit.
template <auto Kernel>
hipError_t allow_lds(int bytes) {
  static std::atomic<uint64_t> allowed{0};
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (!(allowed.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void*)Kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    allowed.fetch_or(bit, std::memory_order_relaxed);
  }
  return hipSuccess;
}

}  // namespace
}  // namespace kvr
