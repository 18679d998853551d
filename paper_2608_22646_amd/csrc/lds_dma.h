// Loads from memory to LDS (LDS-DMA) and what orders them.
#pragma once
#include "common.h"

namespace dllm {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint32_t lo = uniform((int)(uint64_t)p), hi = uniform((int)((uint64_t)p >> 32));
  return (const char*)((uint64_t)hi << 32 | lo);
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
__device__ __forceinline__ void barrier_nofence() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Of a wave's LDS accesses, which run in order: the compiler moves none past this.
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }
// Buffer descriptor of `bytes` bytes from p on (both the same in every lane):
// reads past its end give zeros.
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ rsrc_t rsrc_of(const char* p, uint32_t bytes) {
  return rsrc_t{(uint32_t)uniform((int)(uint64_t)p), (uint32_t)uniform((int)((uint64_t)p >> 32)) & 0xffffu, (uint32_t)uniform((int)bytes), 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// 16 bytes per lane from the buffer to LDS at `to` + 16 lane.  Written out, since
// the compiler lets no transposing LDS read pass while an LDS-DMA load that it
// knows of is in flight; the waits for these loads are wait_vmcnt's alone.  m0, which
// the compiler cannot be told of, is left as it was.  (The idle cycles are what a
// descriptor fresh from readfirstlane needs before its use.)
__device__ __forceinline__ void dma16(rsrc_t rs, uint32_t off, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(uniform((int)to)), "v"(off), "s"(rs)
               : "memory");
}

}  // namespace dllm
