// Loads from global memory straight into LDS (gfx950).
#pragma once

#include <hip/hip_runtime.h>

namespace {

// global_load_lds_dwordx4 moves 16 bytes per lane, 1 KiB per wave instruction, into
// LDS at M0 + 16 * lane.  The instruction is written out because the compiler, which
// cannot tell a ring's slots apart, would otherwise wait for every such load before
// each LDS access; the kernels wait themselves.  The LDS address is an operand bound to
// M0, so the compiler writes M0 itself and knows it is read here; the s_nop is the one
// wait state the hardware needs between that write and the load.
__device__ __forceinline__ void lds_dma16(const void *gsrc, unsigned lds_addr) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :
                 : "v"(gsrc), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr))
                 : "memory");
}
// The same from a scalar base and an offset for each lane.
__device__ __forceinline__ void lds_dma16(const char *base, unsigned off, unsigned lds_addr) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(off), "s"(base), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr))
                 : "memory");
}

}  // namespace
