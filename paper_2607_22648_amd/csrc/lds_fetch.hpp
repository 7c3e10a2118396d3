// Loads from memory to LDS that pass no registers, and the waits for them (latent_attend.hip,
// latent_prompt.hip, weigh.hip).
#pragma once

#include <hip/hip_runtime.h>

namespace ptsd {

// Memory to LDS, 16 bytes (4) a lane: lane i's go to `lds` + 16 i (4 i). The compiler does not
// count these loads, so that it waits for none of them by itself: `arrive` does. It does know the register that
// they take `lds` from, m0, as an operand; the s_nop is the cycle that the load needs after its last write.
__device__ inline void fetch16(const uint8_t* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "{m0}"(lds)
                 : "memory");
}
__device__ inline void fetch16_at(const uint8_t* at, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(at), "{m0}"(lds) : "memory");
}
// The same for what is read once: past the caches' usual order.
__device__ inline void fetch16_once(const uint8_t* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(base), "{m0}"(lds)
                 : "memory");
}
__device__ inline void fetch16_once_at(const uint8_t* at, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(at), "{m0}"(lds) : "memory");
}
__device__ inline void fetch4_at(const void* at, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(at), "{m0}"(lds) : "memory");
}
// Waits until at most kLeft of the wave's loads are under way; its LDS reads are done, too.
template <int kLeft>
__device__ inline void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft) : "memory");
}
__device__ inline void barrier() { asm volatile("s_barrier" ::: "memory"); }

// The LDS address of a shared array, as those loads take it.
__device__ inline uint32_t lds_of(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p;
}

}  // namespace ptsd
