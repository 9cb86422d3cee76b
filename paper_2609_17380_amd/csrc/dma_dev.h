// dma_dev.h - loads from global memory straight into LDS, and the wait for them.
//
// Written as assembly so that the compiler does not track them: it would otherwise wait for all of them before every LDS read,
// which defeats loading ahead; the kernels wait for them themselves (vm_left) and issue no other instruction that uses m0.
#pragma once
#include <hip/hip_runtime.h>

namespace canon {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 (or 4) bytes a lane: lane l's to lds + 16 l (4 l), lds wavefront-uniform
__device__ __forceinline__ void dma16(const void* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop
// waits until at most N vector-memory operations of this wavefront are outstanding (they complete in order)
template <int N>
__device__ __forceinline__ void vm_left() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x70 | 0xF00);  // expcnt, lgkmcnt left at max
}

}  // namespace canon
