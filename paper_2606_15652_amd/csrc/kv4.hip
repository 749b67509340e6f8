// Keys and values of new tokens into the paged 4-bit cache, and back.
//
//   z = fp16(min x),  s = fp16(max(max x - z, 0) / 15),  n = clamp(round_half_even((x - z) / s), 0, 15)
//
// for each row of a token and head; the value that a code stands for is z + s n.
#include "kv4.h"

#include <type_traits>

namespace mq {

struct Rows4 {
    const void *k, *v;
    void *ko, *vo;
    int64_t k_token, k_head, v_token, v_head;   // strides, in elements
    const int64_t* slots;
    int tokens;
};

// Combines v over a row's lanes (8 or 16 neighbours) by DPP: within pairs, quads, eights, sixteens.
template <int LANES, typename F>
__device__ __forceinline__ float row_reduce(float v, F f) {
    auto step = [&](auto ctrl) {
        v = f(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)));
    };
    step(std::integral_constant<int, 0xB1>{});                                  // quad_perm 1, 0, 3, 2
    step(std::integral_constant<int, 0x4E>{});                                  // quad_perm 2, 3, 0, 1
    step(std::integral_constant<int, 0x141>{});                                 // row_half_mirror
    if constexpr (LANES == 16) step(std::integral_constant<int, 0x140>{});      // row_mirror
    return v;
}

// The codes (whole numbers) and parameters of a row, eight values of which this lane holds.  The quotients are
// products with the reciprocal, less than 2^-17 off (of at most 32), and divided after all where one of the lane's is
// that near a tie (bf16 rows of 128: 16381 tokens of 8 heads in scattered slots 32.7 us with divisions only, which the
// vector unit bounded, 26; in slots that follow one another 24.5).
template <int LANES>
__device__ __forceinline__ uint32_t quantise4(const f32x8 x, float (&n)[8]) {
    float lo = x[0], hi = x[0], nan = 0.0f;                 // NaN if a value is infinity or NaN
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
        nan = __builtin_fmaf(x[j], 0.0f, nan);
    }
    lo = row_reduce<LANES>(lo, [](float a, float b) { return fminf(a, b); });
    hi = row_reduce<LANES>(hi, [](float a, float b) { return fmaxf(a, b); });
    const uint64_t bad = __ballot(!(nan == 0.0f));
    const int lane = threadIdx.x & 63;
    const bool row_finite = ((bad >> (lane & ~(LANES - 1))) & ((1u << LANES) - 1)) == 0;
    const uint16_t zb = float_to_half_bits(lo);
    const float z = half_bits_to_float(zb);
    // z may be rounded past every value of a bf16 row: no spread is left then, and the scale is +0
    const uint16_t sb = float_to_half_bits(fmaxf(hi - z, 0.0f) / 15.0f) & 0x7FFFu;
    const float s = half_bits_to_float(sb);
    const bool ok = row_finite && (zb & 0x7FFFu) < kHalfInf && sb < kHalfInf;
    const float inv = __builtin_amdgcn_rcpf(s);
    float far = 0.0f;                                       // the largest distance from a whole number
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float q = (x[j] - z) * inv, whole = rintf(q);
        far = fmaxf(far, fabsf(q - whole));
        n[j] = __builtin_amdgcn_fmed3f(whole, 0.0f, 15.0f);
    }
    if (!ok || s == 0.0f || far > 0.5f - 0x1p-16f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = ok && s > 0.0f ? __builtin_amdgcn_fmed3f(rintf((x[j] - z) / s), 0.0f, 15.0f) : 0.0f;
    }
    return ok ? (uint32_t)sb | (uint32_t)zb << 16 : 0x7E007E00u;
}

// four codes to 16 bits, the first lowest
__device__ __forceinline__ uint32_t word4(float a, float b, float c, float d) {
    return (uint32_t)__builtin_fmaf(d, 4096.0f, __builtin_fmaf(c, 256.0f, __builtin_fmaf(b, 16.0f, a)));
}

// A row of a token and head takes D / 8 lanes; a wave takes 512 / D neighbouring tokens of one head.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(Rows4 r, Cache4 c) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(unit % c.heads), ch = lane % LANES;
    const int64_t token = unit / c.heads * ROWS + lane / LANES;
    const int64_t slot = token < r.tokens ? r.slots[token] : -1;
    const bool there = slot >= 0 && slot < (int64_t)c.pages << c.page_bits;
    f32x8 kx{}, vx{};
    if (there) {
        kx = load8(static_cast<const T*>(r.k) + token * r.k_token + head * r.k_head + 8 * ch);
        vx = load8(static_cast<const T*>(r.v) + token * r.v_token + head * r.v_head + 8 * ch);
    }
    float kn[8], vn[8];
    const uint32_t kp = quantise4<LANES>(kx, kn), vp = quantise4<LANES>(vx, vn);
    if (!there) return;
    const int64_t row = row_index(c, slot, head), first = row & ~(int64_t)((1 << c.page_bits) - 1);
    const int in_page = (int)(row - first);
    if (ch == 0) {
        c.kp[row] = kp;
        c.vp[row] = vp;
    }
    *reinterpret_cast<uint32_t*>(c.k + row * (D / 2) + 4 * ch) =
        word4(kn[0], kn[2], kn[4], kn[6]) | word4(kn[1], kn[3], kn[5], kn[7]) << 16;
    uint8_t* values = c.v + first * (D / 2);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        *reinterpret_cast<uint16_t*>(values + value_offset<D>(in_page, 2 * ch + h)) =
            (uint16_t)word4(vn[4 * h], vn[4 * h + 1], vn[4 * h + 2], vn[4 * h + 3]);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(Rows4 r, Cache4 c) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(unit % c.heads), ch = lane % LANES;
    const int64_t token = unit / c.heads * ROWS + lane / LANES;
    if (token >= r.tokens) return;
    const int64_t slot = r.slots[token];
    f32x8 kx{}, vx{};
    if (slot >= 0 && slot < (int64_t)c.pages << c.page_bits) {
        const int64_t row = row_index(c, slot, head), first = row & ~(int64_t)((1 << c.page_bits) - 1);
        const uint32_t kp = c.kp[row], vp = c.vp[row];
        const uint32_t kw = *reinterpret_cast<const uint32_t*>(c.k + row * (D / 2) + 4 * ch);
        const uint8_t* values = c.v + first * (D / 2);
        uint32_t vw = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            vw |= (uint32_t)*reinterpret_cast<const uint16_t*>(values + value_offset<D>((int)(row - first), 2 * ch + h)) << (16 * h);
        const float ks = half_bits_to_float((uint16_t)kp), kz = half_bits_to_float((uint16_t)(kp >> 16));
        const float vs = half_bits_to_float((uint16_t)vp), vz = half_bits_to_float((uint16_t)(vp >> 16));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            kx[j] = __builtin_fmaf(ks, (float)key_code(kw, j), kz);
            vx[j] = __builtin_fmaf(vs, (float)((vw >> (4 * j)) & 15u), vz);
        }
    }
    store8(static_cast<T*>(r.ko) + token * r.k_token + head * r.k_head + 8 * ch, kx);
    store8(static_cast<T*>(r.vo) + token * r.v_token + head * r.v_head + 8 * ch, vx);
}

// What a cache has to be, for every call that takes one.
mq_status check_cache4(const mq_kv4_cache* c) {
    if (!c || c->pages < 0 || c->heads < 0 || c->page_size < 0 || c->head_dim < 0) return MQ_ERR_INVALID_ARG;
    if ((c->head_dim != 64 && c->head_dim != 128) || c->page_size < 16 || c->page_size > 65536 ||
        (c->page_size & (c->page_size - 1)) != 0 || c->heads < 1 || c->heads > 65535 || c->pages < 1)
        return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!c->k || !c->v || !c->k_params || !c->v_params) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(c->k, 16) || !mq_host::aligned(c->v, 16) || !mq_host::aligned(c->k_params, 16) ||
        !mq_host::aligned(c->v_params, 16))
        return MQ_ERR_MISALIGNED;
    return MQ_OK;
}
Cache4 device_cache4(const mq_kv4_cache* c) {
    return Cache4{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), static_cast<uint32_t*>(c->k_params),
                  static_cast<uint32_t*>(c->v_params), c->pages, c->heads, __builtin_ctz((unsigned)c->page_size)};
}

// workgroups of four waves, of 512 / head_dim rows each
static int64_t row_blocks(const mq_kv4_cache* c, int T) {
    const int rows = 512 / c->head_dim;
    return (((int64_t)T + rows - 1) / rows * c->heads + 3) / 4;
}

static mq_status check_rows(const mq_kv4_cache* c, int T, const void* K, int64_t kt, int64_t kh, const void* V, int64_t vt,
                            int64_t vh, const int64_t* slots, mq_dtype type) {
    if (T < 0 || !mq_host::is_half_type(type)) return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_cache4(c); st != MQ_OK) return st;
    for (int64_t s : {kt, kh, vt, vh})
        if (s < 0 || s % 8 != 0) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!mq_host::launch_holds(row_blocks(c, T), 256)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return MQ_OK;
    if (!K || !V || !slots) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(K, 16) || !mq_host::aligned(V, 16) || !mq_host::aligned(slots, 8)) return MQ_ERR_MISALIGNED;
    return MQ_OK;
}

template <typename F>
static mq_status launch_rows(const mq_kv4_cache* c, int T, mq_dtype type, F&& run) {
    if (T == 0) return MQ_OK;
    const int64_t blocks = row_blocks(c, T);
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        if (c->head_dim == 64) run(T{}, std::integral_constant<int, 64>{}, dim3((unsigned)blocks));
        else run(T{}, std::integral_constant<int, 128>{}, dim3((unsigned)blocks));
        return mq_host::launch_status();
    });
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_kv4_code_bytes(int pages, int page_size, int heads, int head_dim) {
    if (pages < 1 || page_size < 1 || heads < 1 || head_dim < 1) return 0;
    return (size_t)pages * page_size * heads * head_dim / 2;
}

extern "C" mq_status mq_kv4_append(const mq_kv4_cache* cache, int T, mq_dtype type, const void* K, int64_t k_token,
                                   int64_t k_head, const void* V, int64_t v_token, int64_t v_head, const int64_t* slots,
                                   hipStream_t stream) {
    if (mq_status st = check_rows(cache, T, K, k_token, k_head, V, v_token, v_head, slots, type); st != MQ_OK) return st;
    const Rows4 r{K, V, nullptr, nullptr, k_token, k_head, v_token, v_head, slots, T};
    return launch_rows(cache, T, type, [&](auto z, auto d, dim3 grid) {
        hipLaunchKernelGGL((kv4_append_kernel<decltype(z), decltype(d)::value>), grid, dim3(256), 0, stream, r, device_cache4(cache));
    });
}

extern "C" mq_status mq_kv4_read(const mq_kv4_cache* cache, int T, mq_dtype type, const int64_t* slots, void* K, int64_t k_token,
                                 int64_t k_head, void* V, int64_t v_token, int64_t v_head, hipStream_t stream) {
    if (mq_status st = check_rows(cache, T, K, k_token, k_head, V, v_token, v_head, slots, type); st != MQ_OK) return st;
    const Rows4 r{nullptr, nullptr, K, V, k_token, k_head, v_token, v_head, slots, T};
    return launch_rows(cache, T, type, [&](auto z, auto d, dim3 grid) {
        hipLaunchKernelGGL((kv4_read_kernel<decltype(z), decltype(d)::value>), grid, dim3(256), 0, stream, r, device_cache4(cache));
    });
}
