// Buffer loads that write LDS directly, waits for them, and the order of output
// tiles over the XCDs: shared by the tiled matrix kernels.
#pragma once

#include "mq_device.h"

#include <type_traits>

namespace mq {

constexpr uint32_t kPastEnd = 0x80000000u;   // buffer offset past every operand (< 2 GB): reads zero

// Tile order: blocks are dealt to the 8 XCDs round-robin, so give each XCD a
// contiguous range of a grouped tile order (the CUs of one XCD then share
// operand strips in their L2).
constexpr int kGroupM = 8;
__device__ __forceinline__ void tile_coords(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int nt = tiles_m * tiles_n;
    const int xcd = b % 8, k = b / 8;
    const int per = nt / 8, rem = nt % 8;
    const int t = xcd < rem ? xcd * (per + 1) + k : rem * (per + 1) + (xcd - rem) * per + k;
    // grouped order inside the range: bands of kGroupM tile rows, M fastest
    // within a band, so the tiles an XCD holds at once form a near-square
    // patch and share its L2 for both operands
    const int band = t / (kGroupM * tiles_n);
    const int first = band * kGroupM;
    const int h = min(tiles_m - first, kGroupM);
    const int r = t - band * kGroupM * tiles_n;
    tm = first + r % h;
    tn = r / h;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}

// the same as the four dwords that the LDS DMA takes
__device__ __forceinline__ i32x4 make_desc(const void* base, uint32_t bytes) {
    const uint64_t at = (uint64_t)(uintptr_t)base;
    return i32x4{(int)(uint32_t)at, (int)((uint32_t)(at >> 32) & 0xFFFFu), (int)bytes, 0x00020000};
}

__device__ __forceinline__ uint4 bload16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff) {
    const i32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0);
    return make_uint4((uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]);
}

typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(4))) int32_t cint32_t;   // read-only (scalar-loadable) int32

// LDS DMA (buffer loads that write LDS, lane l's bytes at dst + size * l),
// issued from inline assembly so that the compiler does not track them: its
// wait-count pass would otherwise make every later LDS read wait for all of
// them, including the prefetches of later groups.  The kernel waits for them
// itself (wait_loads_and_sync), before the barrier that publishes a stage.
// The compiler's own vector-memory waits stay correct: loads return in order,
// so loads it does not know of can only make its waits longer.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
    return (uint32_t)(uintptr_t)(lds_ptr_t)p;
}
// reads at LDS byte address addr (aligned to the size read)
__device__ __forceinline__ uint4 lds_read16(uint32_t addr) {
    const i32x4 v = *(__attribute__((address_space(3))) const i32x4*)(uintptr_t)addr;
    return make_uint4((uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]);
}
__device__ __forceinline__ uint2 lds_read8(uint32_t addr) {
    const i32x2 v = *(__attribute__((address_space(3))) const i32x2*)(uintptr_t)addr;
    return make_uint2((uint32_t)v[0], (uint32_t)v[1]);
}
__device__ __forceinline__ uint16_t lds_read2(uint32_t addr) {
    return *(__attribute__((address_space(3))) const uint16_t*)(uintptr_t)addr;
}
// An LDS DMA reads M0; after an SALU write of M0 it needs one wait state
// (the compiler adds none inside inline assembly, hence the s_nop).  The
// destination and the resource are wave-uniform; readfirstlane makes that
// explicit, so they are always in scalar registers (a no-op when they are).
__device__ __forceinline__ i32x4 uniform4(const i32x4 d) {
    return i32x4{__builtin_amdgcn_readfirstlane(d[0]), __builtin_amdgcn_readfirstlane(d[1]),
                 __builtin_amdgcn_readfirstlane(d[2]), __builtin_amdgcn_readfirstlane(d[3])};
}
// Four 1 KB blocks at dst + 1024 k from voff + soff + 1024 k (k = 0 .. 3): the
// instruction's immediate offset moves both the memory and the LDS address.
__device__ __forceinline__ void dma16x4(const i32x4 desc, uint32_t dst, uint32_t voff, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %1, %2, %3 offen lds\n\t"
                 "buffer_load_dwordx4 %1, %2, %3 offen offset:1024 lds\n\t"
                 "buffer_load_dwordx4 %1, %2, %3 offen offset:2048 lds\n\t"
                 "buffer_load_dwordx4 %1, %2, %3 offen offset:3072 lds"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(voff), "s"(uniform4(desc)),
                    "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory", "m0");
}
// two 1 KB blocks
__device__ __forceinline__ void dma16x2(const i32x4 desc, uint32_t dst, uint32_t voff, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %1, %2, %3 offen lds\n\t"
                 "buffer_load_dwordx4 %1, %2, %3 offen offset:1024 lds"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(voff), "s"(uniform4(desc)),
                    "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory", "m0");
}
// one 1 KB block
__device__ __forceinline__ void dma16s(const i32x4 desc, uint32_t dst, uint32_t voff, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(voff), "s"(uniform4(desc)),
                    "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory", "m0");
}
// 256 bytes, one dword a lane
__device__ __forceinline__ void dma4(const i32x4 desc, uint32_t dst, uint32_t voff, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(voff), "s"(uniform4(desc)),
                    "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory", "m0");
}

// f(std::integral_constant<int, I>{}) for I = 0 .. N-1, in order
template <int I, int N, typename F>
__device__ __forceinline__ void static_for_from(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for_from<I + 1, N>(f);
    }
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_from<0, N>(f);
}

// Waits until all of this wave's vector-memory loads have landed (the LDS DMA
// does not raise the compiler's own waits), then meets the other waves of
// the workgroup.
__device__ __forceinline__ void wait_loads_and_sync() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace mq
