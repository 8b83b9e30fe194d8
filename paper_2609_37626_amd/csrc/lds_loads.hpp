// Loads straight to LDS, and the waits around them (gfx950 device code).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace splash {

// s_waitcnt with only vmcnt constrained.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
// Workgroup barrier that leaves loads to LDS in flight.
__device__ __forceinline__ void lds_barrier() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt((0x3F & 15) | (7 << 4) | (0 << 8) | ((0x3F >> 4) << 14));  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}
// 16 bytes a lane from base + offset + ADD straight to LDS at `lds` + 16 * lane.  Through
// asm, so that the compiler does not wait for it at every LDS read; the kernel does.  (The
// instruction's own offset moves the LDS address as well: M0 is set that much lower.  M0 is a
// reserved register: the compiler allocates nothing to it, writes it only for an
// instruction that takes it, and refuses it as a clobber.  It is not restored: nothing else
// in the kernels that include this takes it, which their listings show as no mention of m0
// but these.)
template <int ADD>
__device__ __forceinline__ void load_lds(const void* from, uint32_t offset, uint32_t to) {
  const uint64_t at = (uint64_t)from;
  const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int32_t)(at >> 32)) << 32 |
                        (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)at);
  const uint32_t lds = __builtin_amdgcn_readfirstlane((int32_t)to);
  asm volatile("s_sub_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" ::"s"(lds), "v"(offset), "s"(base), "n"(ADD) : "memory", "scc");
}
// The same from an address of the lane's own.
__device__ __forceinline__ void load_lds_from(const void* from, uint32_t to) {
  const uint32_t lds = __builtin_amdgcn_readfirstlane((int32_t)to);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}

}  // namespace splash
