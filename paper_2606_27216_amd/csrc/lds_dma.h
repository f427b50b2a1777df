// Copies from memory to LDS that pass no register (global_load_lds), for kernels that
// feed a ring of LDS buffers.
#pragma once

#include "ns_device.h"

namespace himuon {
namespace dev {

HM_DEV uint32_t lds_offset(const void* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)(p);
}

// The address in scalar registers (it is the same in all lanes).
HM_DEV uint64_t uniform_address(const void* q)
{
    const uint64_t v = (uint64_t)(uintptr_t)q;
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32)) << 32;
}

// 64 lanes x 16 bytes from base + voff to LDS bytes dst .. dst + 1023, lane order.
// (An asm statement without outputs: the compiler would otherwise order every
// LDS read behind all DMA in flight. The waits are dma_wait_barrier's.)
HM_DEV void dma16(uint32_t dst, uint32_t voff, uint64_t base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(voff), "s"(base)
                 : "m0", "memory");
}

// N of them, to LDS bytes dst, dst + 1024, ..: the instruction's offset counts for both sides, so
// voff[i] is 1024 i less than where lane i's bytes lie, and m0 is set once.
template <int N> HM_DEV void dma16_run(uint32_t dst, const uint32_t (&voff)[N], uint64_t base)
{
    static_assert(N == 1 || N == 2 || N == 4, "");
    if constexpr (N == 1) {
        dma16(dst, voff[0], base);
    } else if constexpr (N == 2) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(dst),
                     "v"(voff[0]), "v"(voff[1]), "s"(base)
                     : "m0", "memory");
    } else {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:%6\n\t"
                     "global_load_lds_dwordx4 %3, %5 offset:%7\n\tglobal_load_lds_dwordx4 %4, %5 offset:%8" ::"s"(dst),
                     "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(base), "n"(1024), "n"(2 * 1024), "n"(3 * 1024)
                     : "m0", "memory");
    }
}

// The same with 4 bytes a lane: LDS bytes dst .. dst + 255.
HM_DEV void dma4(uint32_t dst, uint32_t voff, uint64_t base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(dst), "v"(voff), "s"(base)
                 : "m0", "memory");
}

// Waits until at most N of this wave's DMA are in flight and its LDS reads
// have returned, then for the other waves. (Builtins, so that the compiler
// knows that earlier LDS reads need no further wait.)
template <int N> HM_DEV void dma_wait_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace dev
}  // namespace himuon
