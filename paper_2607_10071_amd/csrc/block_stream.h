// Loads from memory to LDS that pass no registers.
#pragma once

#include "block_common.h"

namespace {

__device__ const __attribute__((aligned(16))) uint32_t kZeros[4] = {0, 0, 0, 0};

// 16 bytes of each lane to LDS at `lds` + 16 lane.  Written in assembly, without
// registers to be written: the compiler would wait for every load in flight before
// the next LDS read, whichever stage it reads.  m0, which holds the place in LDS, is an
// operand, so that the compiler knows it (s_nop: the wait between its write and the load).
__device__ __forceinline__ void to_lds(const void *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "{m0}"(lds), "v"(off), "s"(base) : "memory");
}

__device__ __forceinline__ void to_lds(const void *p, uint32_t lds)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "{m0}"(lds), "v"(p) : "memory");
}

// 4 bytes of each lane to LDS at `lds` + 4 lane.
__device__ __forceinline__ void word_to_lds(const void *p, uint32_t lds)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" :: "{m0}"(lds), "v"(p) : "memory");
}

// Until at most N vector memory operations are in flight: s_waitcnt with vmcnt N
// (bits 3..0 and 15..14) and no other limit.  Not in assembly: the compiler has to
// know that its own loads are back, or it waits for them inside the loop.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
    asm volatile("" ::: "memory");
}

}  // namespace
