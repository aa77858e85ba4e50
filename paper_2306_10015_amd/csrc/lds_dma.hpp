// lds_dma.hpp — loads from global memory straight into LDS, and the waits they
// need.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mezo {

// The LDS byte offset of a __shared__ object.
__device__ __forceinline__ uint32_t lds_offset(const void* p)
{
    return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)(p)));
}

// Start a load of 16 bytes a lane: lane l's go from base + its offset to LDS byte
// lds + 16 l (base and lds are the wave's, uniform). The instruction is written out
// because after the builtin the compiler waits for every such load before the next
// LDS read of the kernel, also of another buffer, which undoes the overlap of loads
// with the work on the stage before. It has no result register, so nothing but
// the LDS bytes is in flight: dma_wait() before they are read. m0 is a reserved
// register: the compiler sets it right before each use of its own and keeps
// nothing in it. The copy of base gives m0 its wait state, and it is what makes the load
// safe wherever base comes from: a memory instruction may read a scalar register that a
// vector instruction wrote (v_readfirstlane_b32) only five wait states later, which the
// compiler does not see to in here; a scalar instruction waits by itself.
__device__ __forceinline__ void dma_to_lds(uint64_t base, uint32_t offset, uint32_t lds)
{
    uint64_t at;
    asm volatile("s_mov_b32 m0, %3\n\t"
                 "s_mov_b64 %0, %2\n\t"
                 "global_load_lds_dwordx4 %1, %0"
                 : "=&s"(at)
                 : "v"(offset), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory");
}

// 4 bytes a lane: lane l's go to LDS byte lds + 4 l.
__device__ __forceinline__ void dma_word_to_lds(uint64_t base, uint32_t offset, uint32_t lds)
{
    uint64_t at;
    asm volatile("s_mov_b32 m0, %3\n\t"
                 "s_mov_b64 %0, %2\n\t"
                 "global_load_lds_dword %1, %0"
                 : "=&s"(at)
                 : "v"(offset), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory");
}

// Wait until at most kLeft of the wave's loads (the latest) are still in flight.
template <int kLeft = 0>
__device__ __forceinline__ void dma_wait()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLeft) : "memory");
}

// Wait for the wave's LDS accesses.
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// A barrier of the workgroup that waits for the wave's LDS accesses but not for
// its loads in flight.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

}  // namespace mezo
