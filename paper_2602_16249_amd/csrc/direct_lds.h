// Loads from memory straight into LDS through a buffer whose end the hardware checks.
#pragma once

#include "device_util.h"

namespace affmae {

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr uint32_t kNowhere = 0x80000000u;  // beyond every buffer: such loads bring 0

// A buffer of at most 2^31 - 1 bytes from `base` on: what lies beyond reads as 0.
__device__ __forceinline__ i32x4 buffer_of(const char* base, long long bytes) {
  const uint64_t p = (uint64_t)base;
  const int n = (int)(bytes < 0 ? 0 : bytes < 0x7fffffffll ? bytes : 0x7fffffffll);
  return i32x4{(int)(uint32_t)p, (int)((uint32_t)(p >> 32) & 0xffffu), n, 0x00020000};
}
__device__ __forceinline__ i32x4 uniform(i32x4 v) {
  return i32x4{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), __builtin_amdgcn_readfirstlane(v.w)};
}

// From a buffer straight into LDS (lane l's bytes land at dst + W l).  By hand: for the compiler every LDS read might read what
// such a load still writes, and it would wait for what is on its way before it reads what is there.  (The waits: m0 for the load, and five
// states between a vector instruction that writes a scalar of `rsrc` and the load, which the compiler does not see in here.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is reserved: written only for the next instruction, never held)
template <int W>
__device__ __forceinline__ void lds_load(uint32_t dst, i32x4 rsrc, uint32_t off) {
  if constexpr (W == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(off), "s"(rsrc) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(dst), "v"(off), "s"(rsrc) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(size_t)(__attribute__((address_space(3))) const char*)p; }

}  // namespace affmae
