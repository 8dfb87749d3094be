// Loads from memory straight into LDS, in assembly (private). The compiler does not know them: it would wait for every load into LDS that it
// knows of in front of the next barrier, while these stay in flight until wait_vm() asks for them. Included with <>, so that the tests' build for the
// host CPU can put its own in their place.
#ifndef CKV_DMA_H_
#define CKV_DMA_H_

#include <hip/hip_runtime.h>

namespace ckv {

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)p);
}

// 16 bytes a lane from `from` to lds + 16 * lane; lds is the same for the wave. STREAM: data that is used once.
template <bool STREAM>
__device__ __forceinline__ void dma_16(const char *from, char *lds) {
  if constexpr (STREAM)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" : : "s"(lds_address(lds)), "v"(from) : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_address(lds)), "v"(from) : "memory");
}
// Four bytes a lane, to lds + 4 * lane.
__device__ __forceinline__ void dma_4(const void *from, void *lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_address(lds)), "v"(from) : "memory");
}

// At most N of this wave's vector memory operations are still in flight (they complete in issue order), and no access to LDS moves
// across.
template <int N>
__device__ __forceinline__ void wait_vm_at_most() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
// This wave's reads of LDS are done: what they read may be overwritten.
__device__ __forceinline__ void wait_lds_reads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}

}  // namespace ckv
#endif
