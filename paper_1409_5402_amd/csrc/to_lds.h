// Loads from memory straight to LDS, and the wait for them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace same {

// 16 or 4 bytes per lane from base + offset straight to consecutive places of LDS from `to` on.  Written as assembly because the
// compiler takes the builtin for a store that any later read from LDS may depend on, and waits for it there: here the only
// readers are behind arrived().  No vector register is written.  The copy of the base is for two waits that the compiler does not
// look for inside: a base that the vector unit has just written, and the state between writing m0 and using it.
__device__ __forceinline__ void to_lds_16(const uint8_t* base, uint32_t offset, const void* to)
{
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)to;
    uint64_t copy;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(copy) : "s"(at), "v"(offset), "s"(base) : "m0");
}
__device__ __forceinline__ void to_lds_4(const uint8_t* base, uint32_t offset, const void* to)
{
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)to;
    uint64_t copy;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0" : "=&s"(copy) : "s"(at), "v"(offset), "s"(base) : "m0");
}

// An address that is the same for the whole wave, in scalar registers wherever it was computed.
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p)
{
    const uint64_t at = (uint64_t)(uintptr_t)p;
    return (const uint8_t*)(uintptr_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at));
}

// All of this wave's loads but the last N have come (they end in their order), then all waves'.
template <int N>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    __syncthreads();
}

}  // namespace same
