// Loads from memory straight to LDS, written out (gfx950).
#pragma once

#include "device.h"

namespace dckv {

// The LDS address of a pointer to shared memory.
__device__ __forceinline__ uint32_t lds_address(unsigned char* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)(p)));
}

// 16 bytes a lane from global memory (base, uniform, + lane_at) to LDS, in lane order from
// `lds` on.  Written out, as is the wait for them (loads_done): the compiler cannot tell
// which buffer such a load fills and lets every LDS read wait for it.  It writes no
// register.
__device__ __forceinline__ void load_lds16(const uint8_t* base, uint32_t lane_at, uint32_t lds) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(lane_at), "s"(base) : "memory", "m0");
#endif
}

__device__ __forceinline__ void load_lds4(const uint8_t* base, uint32_t lane_at, uint32_t lds) {
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :: "s"(lds), "v"(lane_at), "s"(base) : "memory", "m0");
#endif
}

// Every load of the wave has landed: those written out, and those that the compiler knows of
// (in a loop it would otherwise wait again for what was loaded before the loop).
__device__ __forceinline__ void loads_done() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0)
}

}  // namespace dckv
