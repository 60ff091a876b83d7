// LDS DMA (global_load_lds_dwordx4): 16 bytes a lane from global memory to LDS address lds + 16 lane, lds the same for
// the whole wave.  Written in asm, because the compiler would wait for all of it before every read of LDS; so the wait states
// that the instruction needs are in the asm too, which the compiler does not look into: one after a write of M0 by
// the scalar unit, and five after a write by the vector unit (v_readfirstlane is one) of a scalar register that holds the base.
// The base therefore passes through a scalar move, which takes what the vector unit has written without
// wait states and is the one that M0 needs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rift {

// From a 64-bit wave-uniform base and a lane's byte offset (below 2^31), which the hardware adds.  NT: nontemporal.
template <bool NT = false>
__device__ __forceinline__ void lds_dma16(const void* base, uint32_t offset, uint32_t lds) {
    const uint64_t b = (uint64_t)(uintptr_t)base;
    // (through uint32_t: readfirstlane gives a signed int, and the low word is to be zero-extended)
    const uint64_t ub = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b) |
                        ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32);
    uint64_t from;
    if constexpr (NT)
        asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0 nt"
                     : "=&s"(from) : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(ub) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0"
                     : "=&s"(from) : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(ub) : "memory", "m0");
}

// From an address of each lane's own.
__device__ __forceinline__ void lds_dma16_lanes(const void* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(from) : "memory", "m0");
}

}  // namespace rift
