// e4m3 codes, and the layout of the 8-bit cache (documented in mq.h).
#pragma once

#include "mq_float.h"

namespace mq {

constexpr float kE4m3Max = 448.0f;
constexpr int kBlockTokens = 32;        // tokens that share a scale for each head

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two numbers to e4m3, ties to even, in the lower (or upper, HIGH) half of `into`: |a|, |b| <= 448, or NaN.
template <bool HIGH>
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, uint32_t into) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)into, HIGH);
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
    return to_e4m3<true>(c, d, to_e4m3<false>(a, b, 0u));
}
// Bytes 0, 1 (or 2, 3) of w, as fp32.
template <bool HIGH>
__device__ __forceinline__ f32x2 from_e4m3(uint32_t w) {
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HIGH));
}

// Eight codes as fp16, exactly.
__device__ __forceinline__ f16x8 operand8(uint32_t a, uint32_t b) {
    struct {
        f16x2 v[4];
    } r = {{__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true),
            __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true)}};
    return __builtin_bit_cast(f16x8, r);
}

// What other lanes of the wave have written to LDS is there.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// One cache as the kernels take it.
struct Cache8 {
    uint8_t *k, *v;
    uint8_t *ke, *ve;       // exponents of the blocks' scales, + 127
    int pages, heads;
    int page_bits;          // log2 of the page size
};

// First token row of block `block` of a sequence for a head (its codes are at D times that, its exponents at that / 32), or
// -1 where no page of the cache holds it.  A block lies in one page.
__device__ __forceinline__ int64_t block_row8(const Cache8& c, const int32_t* table, int table_pages, int64_t block, int head) {
    const int64_t at = block * kBlockTokens, column = at >> c.page_bits;
    if (column >= table_pages) return -1;
    const int page = table[column];
    if (page < 0 || page >= c.pages) return -1;
    return (((int64_t)page * c.heads + head) << c.page_bits) + (at & ((1 << c.page_bits) - 1));
}

// Byte of channel c of a block's token t.  Both are the operands of the 16 x 16 x 32 matrix instruction, 8 bytes a lane,
// two of them side by side in a lane's 16 bytes, so a wave loads 1 KB in a row.  Keys: row t % 16 of tile t / 16,
// lane quarter and half by the channel.
template <int D>
__device__ __forceinline__ int key_offset8(int t, int c) {
    return t / 16 * (16 * D) + c / 64 * 1024 + (c % 64 / 16 * 16 + t % 16) * 16 + c % 16;
}
// Values, transposed: row c % 16 of tile c / 16; a quarter's eight tokens are 4 q .. + 3 and 16 + 4 q .. + 3, as a lane
// has the scores of two tiles of 16 tokens.
__device__ __forceinline__ int value_offset8(int t, int c) {
    return c / 32 * 1024 + (t % 16 / 4 * 16 + c % 16) * 16 + c % 32 / 16 * 8 + t / 16 * 4 + t % 4;
}

}  // namespace mq
