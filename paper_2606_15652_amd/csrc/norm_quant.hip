// Residual addition, RMS norm and per-token INT8 quantisation in one pass over
// the row, and the values that INT8 codes stand for.
//
//   h = rn(x + r),  t = h gamma,  rho = 1 / sqrt(mean(h^2) + eps),  y = rho t,
//   s = rho max|t| / 127,  q = clamp(round_half_even(y / s), -127, 127)
//
// h and gamma have at most 11 significant bits, so t is exact in fp32, and in
// rows (fp32 scales) y / s = 127 t / max|t| does not depend on rho at all.  The
// row stays in registers from its one read to its codes; sum of squares and
// maximum are reduced together.  The sum, and what is made of it for the row, are
// fp64 (the scale is rounded to fp32, and in the A8 layout from there to fp16, as
// the other quantisers' are), and a code is rounded from one fp32 rounding of its
// quotient, multiplied as two parts: memory bounds the kernel, which leaves room
// for both.  8192 rows of 8192 with residual: in rows 93 us, in the A8 layout 106, 4.8-5.0 TB/s of the 4.9 that a
// copy reaches; without the norm 44 us, 4.6; their values read back from rows 37 us, 5.4 TB/s, from the A8 layout 66,
// 3.6 (two threads read a chunk's low bytes).  Four pieces a thread (K > 32768) spill 23-25 registers: 1024 rows of
// 65536 with residual 149 us, 3.2 TB/s.
#include "mq_float.h"

#include <math.h>

#include <algorithm>

namespace mq {

constexpr int kNormMaxThreads = 1024;

// Sum of v over the wave, in a fixed order; every lane has the result.
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// 16 values at p, of which the first n (16, 8 or 0) are there; the others are 0.
template <typename T>
__device__ __forceinline__ void load_piece(const T* p, int n, f32x8 (&v)[2]) {
    v[0] = v[1] = f32x8{};
    if (n > 0) v[0] = load8(p);
    if (n > 8) v[1] = load8(p + 8);
}

// P: pieces of 16 values that a thread keeps.
template <typename T, bool NORM, bool A8, int P>
__global__ __launch_bounds__(kNormMaxThreads) void norm_quant_kernel(
    const T* X, const T* R, const T* __restrict__ gamma, T* H, int M, int K,
    int64_t ldx, int64_t ldr, int64_t ldh, float eps, uint8_t* __restrict__ Xq, int64_t ldq, void* __restrict__ s_x) {
    __shared__ double sums[kNormMaxThreads / 64];
    __shared__ uint32_t maxima[kNormMaxThreads / 64];
    const int m = blockIdx.x, t = threadIdx.x, threads = blockDim.x;

    f32x8 v[P][2];
    double sum = 0.0;
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int k = 16 * (t + i * threads), n = min(16, K - k);
        load_piece(X + m * ldx + k, n, v[i]);
        if (NORM && R) {
            f32x8 r[2];
            load_piece(R + m * ldr + k, n, r);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // the stream that the next reader sees: rounded to its type, and normalised as rounded
                const auto h = __builtin_convertvector(v[i][e] + r[e], typename Vec8<T>::type);
                if (n > 8 * e) *reinterpret_cast<typename Vec8<T>::type*>(H + m * ldh + k + 8 * e) = h;
                v[i][e] = __builtin_convertvector(h, f32x8);
            }
        }
        if constexpr (NORM) {
            f32x8 g[2];
            load_piece(gamma + k, n, g);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const double h = (double)v[i][e][j];
                    sum = __builtin_fma(h, h, sum);
                }
                v[i][e] *= g[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = max(amax, __float_as_uint(v[i][e][j]) & 0x7FFFFFFFu);
    }
    amax = wave_max_dpp(amax);
    if constexpr (NORM) sum = wave_sum(sum);
    if (threads > 64) {
        if ((t & 63) == 0) {
            maxima[t >> 6] = amax;
            sums[t >> 6] = sum;
        }
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < threads / 64; ++w) {
            amax = max(amax, maxima[w]);
            sum += sums[w];
        }
    }
    const double rho = NORM ? 1.0 / sqrt(sum / (double)K + (double)eps) : 1.0;
    const float top = __uint_as_float(amax);
    const double exact = (double)top * rho / (double)kQmax8;
    bool finite = amax < kFloatInf && (!NORM || (float)sum < INFINITY) && exact == exact;   // (0 / 0: zeros, and no eps)
    double inv;                                             // codes are t inv, rounded
    if constexpr (A8) {
        float single = (float)exact;
        asm("" : "+v"(single));                             // two roundings: contracted, they would be one
        const uint16_t sb = float_to_half_bits(single);
        const float s = half_bits_to_float(sb);
        finite = finite && sb < kHalfInf;
        inv = s == 0.0f ? 0.0 : rho / (double)s;
        if (t == 0) static_cast<uint16_t*>(s_x)[m] = finite ? sb : (uint16_t)0x7E00;
    } else {
        const float s = (float)exact;
        // a subnormal scale has too few bits for 127 / max to be the same
        inv = s == 0.0f ? 0.0 : s < 0x1p-126f ? rho / (double)s : (double)kQmax8 / (double)top;
        if (t == 0) static_cast<float*>(s_x)[m] = finite ? s : __uint_as_float(0x7FC00000u);
    }
    if (inv > 0x1p64) {                                     // rows so small that fp32 may not hold it, 2^165 at most
        inv *= 0x1p-64;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) v[i][e] *= 0x1p64f;
    }
    const float inv_hi = (float)inv, inv_lo = (float)(inv - (double)inv_hi);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int k = 16 * (t + i * threads);
        if (k >= K) break;
        float q[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = v[i][e / 8][e % 8];
            const float c = __builtin_amdgcn_fmed3f(rintf(__builtin_fmaf(x, inv_hi, x * inv_lo)) + 0.0f, -127.0f, 127.0f);   // no -0
            q[e] = finite ? c : 0.0f;
        }
        if constexpr (A8) {
            const int g = k / kGroup, j = (k % kGroup) / 16;    // chunk j of group g
            float hi[16], lo[16];
            uint32_t hb[4];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                hi[e] = floorf(q[e] * 0.125f);
                lo[e] = __builtin_fmaf(-8.0f, hi[e], q[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int b = __builtin_amdgcn_cvt_pk_fp8_f32(hi[4 * e], hi[4 * e + 1], 0, false);
                hb[e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[4 * e + 2], hi[4 * e + 3], b, true);
            }
            const u32x6 d = operand_dwords(lo);
            *reinterpret_cast<uint4*>(Xq + ((int64_t)g * M + m) * 128 + hi_chunk_offset(j)) = make_uint4(hb[0], hb[1], hb[2], hb[3]);
            *reinterpret_cast<uint2*>(Xq + (int64_t)M * K + piece_offset(M, m, g) + 8 * j) =
                make_uint2(d[0] | (d[2] & kFoldA), d[1] | (d[2] & kFoldB));
        } else {
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                b[e] = ((uint32_t)(int)q[4 * e] & 0xFFu) | ((uint32_t)(int)q[4 * e + 1] & 0xFFu) << 8 |
                       ((uint32_t)(int)q[4 * e + 2] & 0xFFu) << 16 | (uint32_t)(int)q[4 * e + 3] << 24;
            // rows are 16 bytes aligned and padded: past K the codes are 0
            *reinterpret_cast<uint4*>(Xq + m * ldq + k) = make_uint4(b[0], b[1], b[2], b[3]);
        }
    }
}

// y = rn(s q): eight values a thread, `chunks` workgroups a row
template <typename T, bool A8>
__global__ __launch_bounds__(256) void dequant_act8_kernel(const uint8_t* __restrict__ Xq, int64_t ldq,
                                                           const void* __restrict__ s_x, int M, int K, int chunks,
                                                           T* __restrict__ Y, int64_t ldy) {
    const int m = blockIdx.x / chunks, k = 8 * (blockIdx.x % chunks * blockDim.x + threadIdx.x);
    if (k >= K) return;
    f32x8 v;
    float s;
    if constexpr (A8) {
        s = half_bits_to_float(static_cast<const uint16_t*>(s_x)[m]);
        const int g = k / kGroup, j = (k % kGroup) / 16;
        const uint2 hb = *reinterpret_cast<const uint2*>(Xq + ((int64_t)g * M + m) * 128 + hi_chunk_offset(j) + k % 16);
        const uint2 lb = *reinterpret_cast<const uint2*>(Xq + (int64_t)M * K + piece_offset(M, m, g) + 8 * j);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = ((e < 4 ? hb.x : hb.y) >> (8 * (e % 4))) & 0xFFu;
            v[e] = (float)(8 * int_of_e4m3(b) + chunk_code(lb.x, lb.y, k % 16 + e));
        }
    } else {
        s = static_cast<const float*>(s_x)[m];
        const uint2 b = *reinterpret_cast<const uint2*>(Xq + m * ldq + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? b.x : b.y) >> (8 * (e % 4)));
    }
    store8(Y + m * ldy + k, v * s);
}

struct NormArgs {
    int M, K;
    const void *X, *R, *gamma;
    void* H;
    int ldx, ldr, ldh;
    float eps;
    void* Xq;
    int ldq;
    void* s_x;
};

// threads of a row: one for 16 values, a wave at least
static int norm_threads(int K) { return std::min(((K + 15) / 16 + 63) / 64 * 64, kNormMaxThreads); }

template <typename T, bool NORM, bool A8>
static mq_status launch_norm(const NormArgs& a, hipStream_t stream) {
    auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(a.M), dim3(norm_threads(a.K)), 0, stream, static_cast<const T*>(a.X),
                           static_cast<const T*>(a.R), static_cast<const T*>(a.gamma), static_cast<T*>(a.H), a.M, a.K,
                           a.ldx, a.ldr, a.ldh, a.eps, static_cast<uint8_t*>(a.Xq), a.ldq, a.s_x);
        return mq_host::launch_status();
    };
    const int pieces = (a.K + 15) / 16;
    if (pieces <= kNormMaxThreads) return run(norm_quant_kernel<T, NORM, A8, 1>);
    if (pieces <= 2 * kNormMaxThreads) return run(norm_quant_kernel<T, NORM, A8, 2>);
    return run(norm_quant_kernel<T, NORM, A8, 4>);
}

// K and leading dimensions that the row kernels take.
static bool rows_ok(int K, int ld) { return ld >= K && ld % 8 == 0; }
static mq_status check_codes(int M, int K, mq_act8_layout layout, const void* Xq, int ldq, const void* s_x) {
    if (M < 0 || K < 0 || (layout != MQ_ACT8_ROWS && layout != MQ_ACT8_A8)) return MQ_ERR_INVALID_ARG;
    if (M > (1 << 24) || K < 8 || K % 8 != 0 || K > MQ_NORM_MAX_K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (layout == MQ_ACT8_A8 ? K % kGroup != 0 : ldq < (K + 15) / 16 * 16 || ldq % 16 != 0) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    if (!Xq || !s_x) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Xq, 16) || !mq_host::aligned(s_x, layout == MQ_ACT8_A8 ? 2 : 4)) return MQ_ERR_MISALIGNED;
    return MQ_OK;
}

}  // namespace mq

using namespace mq;

extern "C" mq_status mq_rms_norm_quantize8(int M, int K, mq_dtype type, const void* X, int ldx, const void* R, int ldr,
                                           const void* gamma, float eps, void* H, int ldh, mq_act8_layout layout,
                                           void* Xq8, int ldq, void* s_x, hipStream_t stream) {
    if (!mq_host::is_half_type(type) || !(eps >= 0.0f)) return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_codes(M, K, layout, Xq8, ldq, s_x); st != MQ_OK) return st;
    if (!rows_ok(K, ldx) || (R && (!rows_ok(K, ldr) || !rows_ok(K, ldh))) || !mq_host::launch_holds(M, norm_threads(K)))
        return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    if (!X || !gamma || (R != nullptr) != (H != nullptr)) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(X, 16) || !mq_host::aligned(R, 16) || !mq_host::aligned(gamma, 16) || !mq_host::aligned(H, 16))
        return MQ_ERR_MISALIGNED;
    const NormArgs a{M, K, X, R, gamma, H, ldx, ldr, ldh, eps, Xq8, ldq, s_x};
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        return layout == MQ_ACT8_A8 ? launch_norm<T, true, true>(a, stream) : launch_norm<T, true, false>(a, stream);
    });
}

extern "C" mq_status mq_quantize_rows8(int M, int K, mq_dtype type, const void* X, int ldx, void* Xq8, int ldq,
                                       void* s_x, hipStream_t stream) {
    if (!mq_host::is_half_type(type)) return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_codes(M, K, MQ_ACT8_ROWS, Xq8, ldq, s_x); st != MQ_OK) return st;
    if (!rows_ok(K, ldx) || !mq_host::launch_holds(M, norm_threads(K))) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    if (!X) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(X, 16)) return MQ_ERR_MISALIGNED;
    const NormArgs a{M, K, X, nullptr, nullptr, nullptr, ldx, 0, 0, 0.0f, Xq8, ldq, s_x};
    return mq_host::with_half_type(type, [&](auto z) { return launch_norm<decltype(z), false, false>(a, stream); });
}

extern "C" mq_status mq_dequantize_act8(int M, int K, mq_act8_layout layout, const void* Xq8, int ldq, const void* s_x,
                                        mq_dtype type, void* Y, int ldy, hipStream_t stream) {
    if (!mq_host::is_half_type(type)) return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_codes(M, K, layout, Xq8, ldq, s_x); st != MQ_OK) return st;
    const int threads = std::min((K / 8 + 63) / 64 * 64, 256), chunks = (K / 8 + threads - 1) / threads;
    if (!rows_ok(K, ldy) || !mq_host::launch_holds((int64_t)M * chunks, threads)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    if (!Y) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Y, 16)) return MQ_ERR_MISALIGNED;
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        auto run = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(M * chunks)), dim3(threads), 0, stream, static_cast<const uint8_t*>(Xq8),
                               ldq, s_x, M, K, chunks, static_cast<T*>(Y), ldy);
            return mq_host::launch_status();
        };
        return layout == MQ_ACT8_A8 ? run(dequant_act8_kernel<T, true>) : run(dequant_act8_kernel<T, false>);
    });
}
