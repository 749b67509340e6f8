// Layout of the 4-bit cache (documented in mq.h) and the pieces that its
// writers and readers share.
#pragma once

#include "mq_float.h"

namespace mq {

// One cache as the kernels take it.
struct Cache4 {
    uint8_t *k, *v;
    uint32_t *kp, *vp;      // parameters: scale in the low half, minimum in the high half, both fp16
    int pages, heads;
    int page_bits;          // log2 of the page size
};

// Codes lie in a 16-bit word in fours: the words of a fp16 pair (two of them)
// masked with 0x000F000F, or 0x00F000F0, are two subnormal fp16 numbers, n 2^-24
// and 16 n 2^-24, exactly: one operation turns four bits into an operand of the
// matrix instruction, which takes subnormals as they are.
//
// Keys, a row of D codes of one token: dword c holds channels 8c .. 8c + 7,
// channel 8c + 2j at bit 4j, channel 8c + 2j + 1 at bit 16 + 4j.
// Values, blocks of four tokens: the unit of channels (D / 16) r .. of them, r =
// 0 .. 15, is D / 64 words of 64 bits, each a 16-bit word for each token in turn
// with four channels, the first in the lowest bits.
__device__ __forceinline__ int64_t row_index(const Cache4& c, int64_t slot, int head) {
    const int64_t page = slot >> c.page_bits;
    return ((page * c.heads + head) << c.page_bits) + (slot & ((1 << c.page_bits) - 1));
}
// code of channel j of the eight in a key's dword
__device__ __forceinline__ uint32_t key_code(uint32_t w, int j) { return (w >> (4 * (j / 2) + 16 * (j % 2))) & 15u; }
// byte offset, in a page and head's values, of the 16-bit word of four channels 4 f .. 4 f + 3 of a token
template <int D>
__device__ __forceinline__ int value_offset(int token, int f) {
    return (token >> 2) * (2 * D) + f * 8 + (token & 3) * 2;
}

}  // namespace mq
