// Helpers of the kernels that stream operand tiles through LDS (gemm.hip, i8.hip).
#pragma once

#include "common.h"

namespace ebrl {

typedef __attribute__((address_space(3))) void* lds_ptr_t;

// s_waitcnt on the vector-memory counter only (gfx9 encoding: expcnt and
// lgkmcnt fields at their maxima), and on the LDS counter only.
template <int N> EBRL_DEV void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | 0x70 | 0xF00 | ((N >> 4) << 14));
}
EBRL_DEV void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// Waits until at most min(later, MAX) groups of PER loads each are in flight.
template <int MAX, int PER> EBRL_DEV void wait_tiles(int later) {
    if constexpr (MAX > 0) {
        if (later < MAX) { wait_tiles<MAX - 1, PER>(later); return; }
    }
    wait_vmcnt<MAX * PER>();
}

// Workgroup barrier without the waits of __syncthreads: the kernels below
// count their own loads.  Neither memory accesses nor MFMAs move across it.
EBRL_DEV void wg_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// global_load_lds_dwordx4 issued as inline assembly: the compiler neither
// counts these loads nor guards LDS reads against them, so its own waits
// stay partial; kernels that use it wait on vmcnt and synchronise
// themselves before reading what the DMA filled.
EBRL_DEV void dma16_to_lds(const void* g, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :: "v"(g), "s"(lds_addr) : "memory", "m0");
}
// The same with the non-temporal hint, for weights that no other workgroup of
// the launch reads again (streaming them keeps the activations cached).
EBRL_DEV void dma16_to_lds_nt(const void* g, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
                 :: "v"(g), "s"(lds_addr) : "memory", "m0");
}
// The same DMA in its scalar-base form: a wave-uniform 64-bit base in SGPRs
// plus a 32-bit per-lane byte offset, so a wave's row offsets stay fixed
// across K tiles (only the scalar base advances) and take one VGPR each.
EBRL_DEV void dma16_to_lds_s(const void* sbase, uint32_t voff, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(voff), "s"(sbase), "s"(lds_addr) : "memory", "m0");
}
EBRL_DEV void dma16_to_lds_s_nt(const void* sbase, uint32_t voff, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                 :: "v"(voff), "s"(sbase), "s"(lds_addr) : "memory", "m0");
}
// Four bytes a lane, lane i's at lds_addr + 4 i.
EBRL_DEV void dma4_to_lds(const void* g, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
                 :: "v"(g), "s"(lds_addr) : "memory", "m0");
}
// A wave-uniform address pinned to SGPRs (readfirstlane returns int: each half
// goes through uint32_t, so the low half is zero-extended).
EBRL_DEV const char* uniform_ptr(const void* p) {
    const uint64_t b = (uint64_t)(uintptr_t)p;
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32));
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b);
    return (const char*)(uintptr_t)(((uint64_t)hi << 32) | (uint64_t)lo);
}

// Row-tile-major groups of four row tiles: consecutive tiles share weights
// (four at a time) and activations.
EBRL_DEV void tile_origin(int v, int tiles_m, int tiles_n, int bm, int bn, int& m0, int& n0) {
    constexpr int G = 4;
    const int group = G * tiles_n, gi = v / group, first_m = gi * G;
    const int gsz = min(tiles_m - first_m, G), within = v - gi * group;
    m0 = (first_m + within % gsz) * bm;
    n0 = (within / gsz) * bn;
}

}  // namespace ebrl
