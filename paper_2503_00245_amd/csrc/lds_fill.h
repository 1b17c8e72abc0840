// Operands from memory straight into LDS, and the end of a phase of a kernel that is fed that way (internal).
#pragma once

#include "common.h"

namespace moe {

typedef __attribute__((address_space(3))) char lds_char;

// 64 lanes x 16 bytes from memory straight to 1 KB of LDS at byte address lds (wave-uniform).  The compiler
// does not see these loads: they are waited for by hand (wait_vm), and what it inserts for loads of
// its own can only wait longer.  NT: the data is used once, here; it need not stay in the caches.  (m0 is
// reserved to the compiler, which sets it right before an instruction of its own that reads it and accepts no
// clobber of it; these kernels have no such instruction: every m0 in their assembly is one of these moves.)
template <bool NT>
__device__ __forceinline__ void dma16(unsigned lds, const char* base, unsigned off) {
#if defined(__HIP_DEVICE_COMPILE__)
    if (NT)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base)
                     : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
                     : "memory");
#endif
}
// at most N of the wave's memory loads are still in flight afterwards (they complete in order)
template <int N>
__device__ __forceinline__ void wait_vm() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
#endif
}
// The wave's LDS reads have landed, and all waves have come here.  (The wait is the compiler's own instruction: one that it does not see it
// makes again, fragment by fragment between a phase's MFMAs, eight for 64: 16384 tokens of 2048 / 5632 1809 us with these, 1786 without, 2048 tokens
// 305.8 and 302.7, of rank 1024 263.0 and 261.6.)
__device__ __forceinline__ void phase_end() {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0) alone
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#endif
}

}  // namespace moe
