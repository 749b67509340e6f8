// Keys and values of new tokens into the paged 8-bit cache, and back.
//
// A block of 32 tokens of a sequence and head has one scale 2^e for its keys and
// one for its values, e the least with |x| <= 448 2^e; codes are e4m3(x 2^-e).
// Later tokens of the block may raise e: the codes that are there are then
// divided by the power of two, exactly but where they pass below 2^-6.  Where the
// tokens that raised it have been taken back (the sequence's length went down), it
// goes down again, and codes are multiplied, exactly.
//
// One wave takes one block and head: what the block holds comes to LDS, new codes
// go there, and it goes back in whole lines.  Nobody else writes the block, so
// nothing depends on order.  Memory and the vector unit bound it together: 16381 bf16
// tokens of 8 heads of 128, 101 MB, 28 us; one token each of 32 sequences 8.2 us,
// latency (the block comes, then goes).  Heads of 128 spill 74 scalar registers to lanes.
#include "kv8.h"

#include <type_traits>

namespace mq {

struct Append8Args {
    Cache8 c;
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;   // strides, in elements
    const int32_t *table, *lens, *starts;       // starts may be null: one token a sequence
    int sequences, tokens, table_pages;
};

// Blocks that the tokens of sequences before b can reach, and two for each: a bound that ascends and needs no pass over
// the sequences (n tokens reach at most n / 32 + 2 blocks).
__device__ __forceinline__ int64_t first_unit(const int32_t* starts, int b) { return starts[b] / kBlockTokens + 2 * (int64_t)b; }

// The last sequence with first_unit <= unit (the wave looks at 64 of them at a time), -1 for none.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int sequences, int64_t unit) {
    const int lane = threadIdx.x & 63;
    int first = 0, n = sequences;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lane * step;
        const int count = __popcll(__ballot(i < n && first_unit(starts, first + i) <= unit));
        if (count == 0) return -1;
        first += (count - 1) * step;
        n = min(step, n - (count - 1) * step);
    }
    return first;
}

// Least e with 2^by amax <= 448 2^e = 1.75 2^(e + 8), for the exponent's byte: e + 127 in 0 .. 254.
__device__ __forceinline__ int exponent_byte(uint32_t amax_bits, int by = 0) {
    const int x = (int)(amax_bits >> 23) + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return amax_bits ? max(x - 8 + by, 0) : 0;
}

// The bytes of four codes that are NaN, as 0xFF.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t d) { return ((d & 0x7F7F7F7Fu) + 0x01010101u & 0x80808080u) / 0x80u * 0xFFu; }

template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(Append8Args a) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, TURNS = kBlockTokens / ROWS, BYTES = kBlockTokens * D, PIECES = BYTES / 1024;
    __shared__ __attribute__((aligned(16))) uint8_t image[4][2][BYTES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
    const int head = (int)(unit % a.c.heads), ch = 8 * (lane % LANES), sub = lane / LANES;
    const int64_t which = unit / a.c.heads;
    const int b = a.starts ? sequence_of(a.starts, a.sequences, which) : (int)min(which, (int64_t)a.sequences);
    if (b < 0 || b >= a.sequences) return;                  // (waves do not meet)
    const int first_new = a.starts ? a.starts[b] : b, count = a.starts ? a.starts[b + 1] - first_new : 1;
    const int64_t len = a.lens[b], had = len - count;       // had < 0: the first -had tokens have no place
    const int64_t block = (had > 0 ? had : 0) / kBlockTokens + (a.starts ? which - first_unit(a.starts, b) : 0);
    const int64_t at = block * kBlockTokens;
    if (count <= 0 || at < 0 || at >= len) return;          // (below 0: starts that do not ascend)
    const int64_t row = block_row8(a.c, a.table + (int64_t)b * a.table_pages, a.table_pages, block, head);
    if (row < 0) return;
    const int64_t base = row * D, blk = row / kBlockTokens;

    // The block's new tokens, and which of them are finite in key and value (bits, the same in every lane).  Of keys a lane has
    // eight channels of TURNS tokens; of values two channels of every token (of a half of them where rows have 64), so that
    // four tokens of a channel, which lie side by side in the cache, are one word (byte by byte, 16381 tokens of 8 heads
    // 31 us, so 27.5).
    typedef T t2 __attribute__((ext_vector_type(2)));
    constexpr int PAIRS = D / 2, QUADS = kBlockTokens / 4 * PAIRS / 64;
    const int pair = lane % PAIRS, half = lane / PAIRS;     // lanes of half h have the quads h, h + 64 / PAIRS, ..
    typename Vec8<T>::type k8[TURNS];
    t2 v2[QUADS][4];
    // tokens t of the block that are new, and have their row among those given: from <= t < to
    const int64_t row0 = first_new + at - had, from = max(max(had - at, -row0), (int64_t)0);
    const int64_t to = min(min(len - at, a.tokens - row0), (int64_t)kBlockTokens);
    const uint32_t fresh = to <= from ? 0u : (uint32_t)((1ull << to) - (1ull << from));
    auto row_of = [&](int t) { return row0 + t; };
    uint32_t bad = 0, amax[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int t = i * ROWS + sub;
        k8[i] = (typename Vec8<T>::type)(T)0.0f;
        if (fresh >> t & 1) k8[i] = *reinterpret_cast<const typename Vec8<T>::type*>(static_cast<const T*>(a.k) + row_of(t) * a.k_token + head * a.k_head + ch);
    }
#pragma unroll
    for (int i = 0; i < QUADS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = 4 * (i * (64 / PAIRS) + half) + j;
            v2[i][j] = (t2)(T)0.0f;
            if (fresh >> t & 1) v2[i][j] = *reinterpret_cast<const t2*>(static_cast<const T*>(a.v) + row_of(t) * a.v_token + head * a.v_head + 2 * pair);
        }
    auto bits_of = [](T x) { return __float_as_uint((float)x) & 0x7FFFFFFFu; };
    uint32_t most_k[TURNS], most_v[QUADS][4];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        most_k[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most_k[i] = max(most_k[i], bits_of(k8[i][j]));
        const uint64_t lanes = __ballot(most_k[i] >= kFloatInf);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) bad |= (uint32_t)((lanes >> (r * LANES) & ((1ull << LANES) - 1)) != 0) << (i * ROWS + r);
    }
#pragma unroll
    for (int i = 0; i < QUADS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            most_v[i][j] = max(bits_of(v2[i][j][0]), bits_of(v2[i][j][1]));
            const uint64_t lanes = __ballot(most_v[i][j] >= kFloatInf);
#pragma unroll
            for (int h = 0; h < 64 / PAIRS; ++h)
                bad |= (uint32_t)((PAIRS == 64 ? lanes : lanes >> (h * PAIRS) & ((1ull << (PAIRS % 64)) - 1)) != 0) << (4 * (i * (64 / PAIRS) + h) + j);
        }
#pragma unroll
    for (int i = 0; i < TURNS; ++i)
        if (!(bad >> (i * ROWS + sub) & 1)) amax[0] = max(amax[0], most_k[i]);
#pragma unroll
    for (int i = 0; i < QUADS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!(bad >> (4 * (i * (64 / PAIRS) + half) + j) & 1)) amax[1] = max(amax[1], most_v[i][j]);
    const bool whole = fresh == 0xFFFFFFFFu;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint8_t *codes = (w ? a.c.v : a.c.k) + base, *held = (w ? a.c.ve : a.c.ke) + blk;
        uint8_t* im = image[wave][w];
        int e = exponent_byte(wave_max_dpp(amax[w]));
        if (!whole) {
            const int e_old = *held, kept = (int)min(had - at, (int64_t)kBlockTokens);      // tokens from before
            uint4 p[PIECES];
#pragma unroll
            for (int i = 0; i < PIECES; ++i) p[i] = ldg16(codes + i * 1024 + lane * 16);
            if (kept > 0) {
                // The kept tokens' bytes: of keys a lane has one token for each tile of 16, of values four for each.
                uint32_t keep[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int n = w ? kept - 16 * h - lane / 16 * 4 : 4 * (kept - 16 * h - lane % 16);
                    keep[h] = n >= 4 ? ~0u : n > 0 ? (1u << (8 * n)) - 1u : 0u;
                }
                auto each = [&](auto&& f) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        const uint32_t d[4] = {p[i].x, p[i].y, p[i].z, p[i].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) f(d[j] & 0x7F7F7F7Fu & keep[w ? j % 2 : i / (PIECES / 2)]);
                    }
                };
                // A scale that one of them needed shows as a code of 224 (0x76) and more, not NaN.
                uint32_t needed = 0;
                each([&](uint32_t d) { needed |= (d + 0x0A0A0A0Au) & ~(d + 0x01010101u); });
                int e_kept = e_old;
                if (__ballot((needed & 0x80808080u) != 0) == 0) {
                    uint32_t most = 0;
                    each([&](uint32_t d) {
                        d &= ~nan_bytes(d);
                        const f32x2 lo = from_e4m3<false>(d), hi = from_e4m3<true>(d);
                        most = max(most, __float_as_uint(fmaxf(fmaxf(lo[0], lo[1]), fmaxf(hi[0], hi[1]))));
                    });
                    e_kept = exponent_byte(wave_max_dpp(most), e_old - 127);
                }
                e = max(e, e_kept);
                if (e != e_old) {
                    auto moved = [&](uint32_t d) {
                        const f32x2 lo = from_e4m3<false>(d), hi = from_e4m3<true>(d);
                        // (codes behind the kept ones may pass the largest where the scale goes down)
                        auto by = [&](float x) { return __builtin_amdgcn_fmed3f(ldexpf(x, e_old - e), -kE4m3Max, kE4m3Max); };
                        const uint32_t to = to_e4m3x4(by(lo[0]), by(lo[1]), by(hi[0]), by(hi[1])), nan = nan_bytes(d);
                        return (to & ~nan) | (d & nan);     // a NaN stays the one it was
                    };
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) p[i] = make_uint4(moved(p[i].x), moved(p[i].y), moved(p[i].z), moved(p[i].w));
                }
            }
#pragma unroll
            for (int i = 0; i < PIECES; ++i) *reinterpret_cast<uint4*>(im + i * 1024 + lane * 16) = p[i];
            wave_sync();
        }
        auto scaled = [&](T x) { return ldexpf((float)x, 127 - e); };
        // a token that is not finite: NaN throughout its key, and a value of zeros
        if (w == 0) {
#pragma unroll
            for (int i = 0; i < TURNS; ++i) {
                const int t = i * ROWS + sub;
                if (!(fresh >> t & 1)) continue;
                uint32_t q[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    q[h] = bad >> t & 1 ? 0x7F7F7F7Fu : to_e4m3x4(scaled(k8[i][4 * h]), scaled(k8[i][4 * h + 1]), scaled(k8[i][4 * h + 2]), scaled(k8[i][4 * h + 3]));
                *reinterpret_cast<uint2*>(im + key_offset8<D>(t, ch)) = make_uint2(q[0], q[1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < QUADS; ++i) {
                const int t0 = 4 * (i * (64 / PAIRS) + half);
                const uint32_t news = fresh >> t0 & 15u, bads = bad >> t0 & 15u;
                if (news == 0) continue;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float f[4];
                    uint32_t mask = 0;                      // bytes of the new tokens
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        f[j] = bads >> j & 1 ? 0.0f : scaled(v2[i][j][c]);
                        mask |= news >> j & 1 ? 0xFFu << (8 * j) : 0u;
                    }
                    uint32_t* to = reinterpret_cast<uint32_t*>(im + value_offset8(t0, 2 * pair + c));
                    const uint32_t q = to_e4m3x4(f[0], f[1], f[2], f[3]);
                    *to = mask == 0xFFFFFFFFu ? q : (*to & ~mask) | (q & mask);
                }
            }
        }
        wave_sync();
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            *reinterpret_cast<uint4*>(codes + i * 1024 + lane * 16) = *reinterpret_cast<const uint4*>(im + i * 1024 + lane * 16);
        if (lane == 0) *held = (uint8_t)e;
    }
}

struct Read8Args {
    Cache8 c;
    void *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    const int64_t* slots;
    int tokens;
};

// A wave takes 512 / D tokens of a head.  Where they are neighbours in a block, four tokens of a channel of values are one word
// (byte by byte, 16381 tokens of 8 heads 38 us, so 30.5).
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_read_kernel(Read8Args a) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, PAIRS = D / 2;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(unit % a.c.heads), ch = 8 * (lane % LANES), sub = lane / LANES;
    const int64_t first = unit / a.c.heads * ROWS, token = first + sub;
    const int64_t slot = token < a.tokens ? a.slots[token] : -1;
    const bool inside = slot >= 0 && slot < (int64_t)a.c.pages << a.c.page_bits;
    auto base_of = [&](int64_t s) {                         // row of its block
        const int64_t page = s >> a.c.page_bits, in = s & ((1 << a.c.page_bits) - 1);
        return ((page * a.c.heads + head) << a.c.page_bits) + in / kBlockTokens * kBlockTokens;
    };
    const int64_t slot0 = __shfl((long long)slot, 0);
    const bool together = __ballot(inside && slot == slot0 + sub) == ~0ull && slot0 % ROWS == 0;
    if (token >= a.tokens) return;
    f32x8 kx{}, vx{};
    if (inside) {
        const int64_t row = base_of(slot);
        const int t = (int)(slot % kBlockTokens), ke = a.c.ke[row / kBlockTokens] - 127;
        const uint2 kw = *reinterpret_cast<const uint2*>(a.c.k + row * D + key_offset8<D>(t, ch));
        auto values = [](uint32_t a, uint32_t b, int e) {
            const f32x2 p[4] = {from_e4m3<false>(a), from_e4m3<true>(a), from_e4m3<false>(b), from_e4m3<true>(b)};
            f32x8 y;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = ldexpf(p[j / 2][j % 2], e);
            return y;
        };
        kx = values(kw.x, kw.y, ke);
        const int ve = a.c.ve[row / kBlockTokens] - 127;
        if (together) {
            typedef T t2 __attribute__((ext_vector_type(2)));
            const int pair = lane % PAIRS, t0 = (int)(slot0 % kBlockTokens) + 4 * (lane / PAIRS);
            f32x2 y[2][2];                                  // of a channel, by token
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(a.c.v + row * D + value_offset8(t0, 2 * pair + c));
                y[c][0] = from_e4m3<false>(w);
                y[c][1] = from_e4m3<true>(w);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                t2 v;
#pragma unroll
                for (int c = 0; c < 2; ++c) v[c] = (T)ldexpf(y[c][j / 2][j % 2], ve);
                *reinterpret_cast<t2*>(static_cast<T*>(a.v) + (first + 4 * (lane / PAIRS) + j) * a.v_token + head * a.v_head + 2 * pair) = v;
            }
        } else {
            uint32_t vw[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) vw[j / 4] |= (uint32_t)a.c.v[row * D + value_offset8(t, ch + j)] << (8 * (j % 4));
            vx = values(vw[0], vw[1], ve);
        }
    }
    store8(static_cast<T*>(a.k) + token * a.k_token + head * a.k_head + ch, kx);
    if (!together) store8(static_cast<T*>(a.v) + token * a.v_token + head * a.v_head + ch, vx);
}

// What a cache has to be, for every call that takes one.
mq_status check_cache8(const mq_kv8_cache* c) {
    if (!c || c->pages < 0 || c->heads < 0 || c->page_size < 0 || c->head_dim < 0) return MQ_ERR_INVALID_ARG;
    if ((c->head_dim != 64 && c->head_dim != 128) || c->page_size < kBlockTokens || c->page_size > 65536 ||
        (c->page_size & (c->page_size - 1)) != 0 || c->heads < 1 || c->heads > 65535 || c->pages < 1)
        return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!c->k || !c->v || !c->k_scales || !c->v_scales) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(c->k, 16) || !mq_host::aligned(c->v, 16)) return MQ_ERR_MISALIGNED;
    return MQ_OK;
}
Cache8 device_cache8(const mq_kv8_cache* c) {
    return Cache8{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), static_cast<uint8_t*>(c->k_scales),
                  static_cast<uint8_t*>(c->v_scales), c->pages, c->heads, __builtin_ctz((unsigned)c->page_size)};
}

static bool strides_ok(int64_t kt, int64_t kh, int64_t vt, int64_t vh) {
    for (int64_t s : {kt, kh, vt, vh})
        if (s < 0 || s % 8 != 0) return false;
    return true;
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_kv8_code_bytes(int pages, int page_size, int heads, int head_dim) {
    if (pages < 1 || page_size < 1 || heads < 1 || head_dim < 1) return 0;
    return (size_t)pages * page_size * heads * head_dim;
}

extern "C" mq_status mq_kv8_append(const mq_kv8_cache* cache, int sequences, int T, mq_dtype type, const void* K,
                                   int64_t k_token, int64_t k_head, const void* V, int64_t v_token, int64_t v_head,
                                   const int32_t* page_table, int table_pages, const int32_t* kv_lens, const int32_t* cu_new,
                                   hipStream_t stream) {
    if (T < 0 || sequences < 0 || table_pages < 0 || !mq_host::is_half_type(type) || (!cu_new && T != sequences))
        return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_cache8(cache); st != MQ_OK) return st;
    if (!strides_ok(k_token, k_head, v_token, v_head)) return MQ_ERR_UNSUPPORTED_SHAPE;
    const int64_t units = cu_new ? (int64_t)T / kBlockTokens + 2 * (int64_t)sequences : sequences;
    const int64_t groups = (units * cache->heads + 3) / 4;
    if (!mq_host::launch_holds(groups, 256)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (T == 0 || sequences == 0) return MQ_OK;
    if (!K || !V || !page_table || !kv_lens) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(K, 16) || !mq_host::aligned(V, 16) || !mq_host::aligned(page_table, 4) ||
        !mq_host::aligned(kv_lens, 4) || !mq_host::aligned(cu_new, 4))
        return MQ_ERR_MISALIGNED;
    const Append8Args a{device_cache8(cache), K, V, k_token, k_head, v_token, v_head, page_table, kv_lens, cu_new,
                        sequences, T, table_pages};
    return mq_host::with_half_type(type, [&](auto z) {
        using E = decltype(z);
        if (cache->head_dim == 64) hipLaunchKernelGGL((kv8_append_kernel<E, 64>), dim3((unsigned)groups), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((kv8_append_kernel<E, 128>), dim3((unsigned)groups), dim3(256), 0, stream, a);
        return mq_host::launch_status();
    });
}

extern "C" mq_status mq_kv8_read(const mq_kv8_cache* cache, int T, mq_dtype type, const int64_t* slots, void* K,
                                 int64_t k_token, int64_t k_head, void* V, int64_t v_token, int64_t v_head, hipStream_t stream) {
    if (T < 0 || !mq_host::is_half_type(type)) return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_cache8(cache); st != MQ_OK) return st;
    const int rows = 512 / cache->head_dim;
    const int64_t groups = (((int64_t)T + rows - 1) / rows * cache->heads + 3) / 4;
    if (!strides_ok(k_token, k_head, v_token, v_head) || !mq_host::launch_holds(groups, 256)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return MQ_OK;
    if (!K || !V || !slots) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(K, 16) || !mq_host::aligned(V, 16) || !mq_host::aligned(slots, 8)) return MQ_ERR_MISALIGNED;
    const Read8Args a{device_cache8(cache), K, V, k_token, k_head, v_token, v_head, slots, T};
    return mq_host::with_half_type(type, [&](auto z) {
        using E = decltype(z);
        if (cache->head_dim == 64) hipLaunchKernelGGL((kv8_read_kernel<E, 64>), dim3((unsigned)groups), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((kv8_read_kernel<E, 128>), dim3((unsigned)groups), dim3(256), 0, stream, a);
        return mq_host::launch_status();
    });
}
