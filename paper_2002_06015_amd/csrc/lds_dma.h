// Loads from global memory straight into LDS, and the waits that go with them (gfx950).
#pragma once

#include <hip/hip_runtime.h>

namespace kfac {

// An address in LDS, in bytes.
typedef unsigned lds_address;
__device__ __forceinline__ lds_address address_in_lds(void *p)
{
    return (unsigned)(unsigned long long)(__attribute__((address_space(3))) void *)p;
}

// 16 bytes a lane: lane l's, at base + offset (both in bytes), go to lds + 16 l.  base and lds are the same in all lanes of the wave.
// Written as one block, so that the compiler, which takes every LDS read for a possible reader of every such load in flight and
// waits for all of them, leaves the waits to the kernel (wait_loads).
__device__ __forceinline__ void load_to_lds(const void *base, unsigned offset, lds_address lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}

// Waits until at most `newest` loads of this wave are in flight and its LDS accesses are done, then for the other waves.
template <int newest>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(newest) : "memory");
}

// The same without a wait for loads.
__device__ __forceinline__ void wait_lds()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

}  // namespace kfac
