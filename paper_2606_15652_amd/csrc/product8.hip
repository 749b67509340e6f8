// Product of 8-bit activations and 8-bit weights with scales for each token and
// channel:  Y[m,n] = rn(s_x[m] s_w[n] sum_k Xq[m,k] Wq[n,k] + bias[n]).
//
// The sums run on v_mfma_i32_16x16x64_i8 in exact int32.  Weights are laid out
// once in the instruction's operand order: the piece of 16 rows (channels) and
// 64 codes is 1 KB, lane l's 16 bytes (row l % 16, codes 16 (l / 16) ..) at 16 l.
// Rows past N and codes past K are zero, so whatever X holds past K adds nothing.
#include "mq_float.h"

namespace mq {

constexpr int kPieceRows = 16, kPieceK = 64, kPieceBytes = 1024;

struct Product8Args {
    int M, N, K;
    const uint8_t* X;
    int64_t ldx;
    const float* s_x;
    const uint8_t* W;
    const float* s_w;
    const void* bias;
    void* Y;
    int64_t ldy;
};

template <typename T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }

// 32 x 32 outputs a wave, four waves a workgroup side by side along N.
template <typename T>
__global__ __launch_bounds__(256) void product8_kernel(Product8Args a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, quad = lane >> 4;
    const int tiles_n = (a.N + 127) / 128;
    const int n0 = (blockIdx.x % tiles_n * 4 + wave) * 32, m0 = blockIdx.x / tiles_n * 32;
    const int pieces_k = (a.K + kPieceK - 1) / kPieceK, pieces_n = (a.N + kPieceRows - 1) / kPieceRows;
    if (n0 >= a.N) return;
    const uint8_t* w[2];
    const uint8_t* x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[i] = a.W + (int64_t)min(n0 / kPieceRows + i, pieces_n - 1) * pieces_k * kPieceBytes + 16 * lane;
        x[i] = a.X + min(m0 + 16 * i + row, a.M - 1) * a.ldx;
    }
    i32x4 acc[2][2] = {};
    const int last = (a.K - 1) / 16 * 16;                   // first code of a row's last 16
    for (int p = 0; p < pieces_k; ++p) {
        i32x4 wv[2], xv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            wv[i] = *reinterpret_cast<const i32x4*>(w[i] + (int64_t)p * kPieceBytes);
            xv[i] = *reinterpret_cast<const i32x4*>(x[i] + min(p * kPieceK + 16 * quad, last));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[i], xv[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int m = m0 + 16 * j + row;
        if (m >= a.M) continue;
        const float sx = a.s_x[m];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = n0 + 16 * i + 4 * quad + r;
                if (n >= a.N) continue;
                float y = (float)acc[i][j][r] * (sx * a.s_w[n]);
                if (a.bias) y += to_float(static_cast<const T*>(a.bias)[n]);
                static_cast<T*>(a.Y)[m * a.ldy + n] = (T)y;
            }
    }
}

// Per-channel INT8 weights: s = max|w| / 127 (fp32), q = clamp(round_half_even(w / s), -127, 127),
// and canonical codes into pieces: one workgroup per 16 rows.
struct FromFloat {
    const float* W;
    int64_t ldw;
    float* s_w;
};
struct FromCodes {
    const int8_t* W;
    int64_t ldw;
};

template <typename From>
__global__ __launch_bounds__(1024) void pack_weight8_kernel(From from, int N, int K, uint8_t* __restrict__ Wq) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int pieces_k = (K + kPieceK - 1) / kPieceK;
    const int row0 = blockIdx.x * kPieceRows;
    __shared__ float scale[kPieceRows];
    if constexpr (__is_same(From, FromFloat)) {
        for (int r = wave; r < kPieceRows; r += waves) {
            uint32_t amax = 0;
            if (row0 + r < N)
                for (int k = lane; k < K; k += 64)
                    amax = max(amax, __float_as_uint(from.W[(row0 + r) * from.ldw + k]) & 0x7FFFFFFFu);
            amax = wave_max_dpp(amax);
            const float s = __uint_as_float(amax) / (float)kQmax8;
            if (lane == 0) {
                scale[r] = s;
                if (row0 + r < N) from.s_w[row0 + r] = s;
            }
        }
        __syncthreads();
    }
    const int row = row0 + (lane & 15);
    for (int p = wave; p < pieces_k; p += waves) {
        const int k0 = p * kPieceK + 16 * (lane >> 4);
        uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            int q = 0;
            if (row < N && k0 + e < K) {
                if constexpr (__is_same(From, FromFloat)) {
                    const float s = scale[lane & 15];
                    const float c = rintf(from.W[row * from.ldw + k0 + e] / s);
                    // a row that is not finite: codes 0 (its scale is not finite either)
                    q = s > 0.0f && __float_as_uint(s) < kFloatInf ? (int)__builtin_amdgcn_fmed3f(c, -127.0f, 127.0f) : 0;
                } else {
                    q = from.W[row * from.ldw + k0 + e];
                }
            }
            b[e / 4] |= ((uint32_t)q & 0xFFu) << (8 * (e % 4));
        }
        *reinterpret_cast<uint4*>(Wq + ((int64_t)blockIdx.x * pieces_k + p) * kPieceBytes + 16 * lane) = make_uint4(b[0], b[1], b[2], b[3]);
    }
}

__global__ __launch_bounds__(256) void unpack_weight8_kernel(const uint8_t* __restrict__ Wq, int N, int K,
                                                             int8_t* __restrict__ Wc, int64_t ldw) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)N * K) return;
    const int n = (int)(i / K), k = (int)(i % K), pieces_k = (K + kPieceK - 1) / kPieceK;
    const int lane = n % 16 + 16 * (k % kPieceK / 16);
    Wc[n * ldw + k] = (int8_t)Wq[((int64_t)(n / 16) * pieces_k + k / kPieceK) * kPieceBytes + 16 * lane + k % 16];
}

static bool shape8_ok(int N, int K) { return N >= 1 && N <= (1 << 24) && K >= 1 && K <= MQ_W8A8_MAX_K; }

}  // namespace mq

using namespace mq;

extern "C" size_t mq_weight8_bytes(int N, int K) {
    if (!shape8_ok(N, K)) return 0;
    return (size_t)((N + kPieceRows - 1) / kPieceRows) * ((K + kPieceK - 1) / kPieceK) * kPieceBytes;
}

extern "C" mq_status mq_quantize_weight8(const float* W, int N, int K, int ldw, uint8_t* Wq8, float* s_w, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!W || !Wq8 || !s_w) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(W, 4) || !mq_host::aligned(Wq8, 16) || !mq_host::aligned(s_w, 4)) return MQ_ERR_MISALIGNED;
    hipLaunchKernelGGL(pack_weight8_kernel<FromFloat>, dim3((N + 15) / 16), dim3(1024), 0, stream, FromFloat{W, ldw, s_w}, N, K, Wq8);
    return mq_host::launch_status();
}

extern "C" mq_status mq_repack_weight8(int N, int K, const int8_t* Wc, int ldw, uint8_t* Wq8, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Wc || !Wq8) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Wq8, 16)) return MQ_ERR_MISALIGNED;
    hipLaunchKernelGGL(pack_weight8_kernel<FromCodes>, dim3((N + 15) / 16), dim3(1024), 0, stream, FromCodes{Wc, ldw}, N, K, Wq8);
    return mq_host::launch_status();
}

extern "C" mq_status mq_unpack_weight8(int N, int K, const uint8_t* Wq8, int8_t* Wc, int ldw, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Wc || !Wq8) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Wq8, 16)) return MQ_ERR_MISALIGNED;
    const int64_t blocks = ((int64_t)N * K + 255) / 256;
    if (blocks > INT32_MAX) return MQ_ERR_UNSUPPORTED_SHAPE;
    hipLaunchKernelGGL(unpack_weight8_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, Wq8, N, K, Wc, ldw);
    return mq_host::launch_status();
}

extern "C" size_t mq_gemm_w8a8_workspace_size(int M, int N, int K) {
    (void)M, (void)N, (void)K;
    return 0;
}

extern "C" mq_status mq_gemm_w8a8(int M, int N, int K, const int8_t* Xq8, int ldx, const float* s_x, const uint8_t* Wq8,
                                  const float* s_w, mq_dtype type, const void* bias, void* Y, int ldy, void* workspace,
                                  size_t ws_bytes, hipStream_t stream) {
    if (M < 0 || N < 0 || K < 0 || (!mq_host::is_half_type(type) && type != MQ_FP32)) return MQ_ERR_INVALID_ARG;
    if (M > (1 << 24) || !shape8_ok(N, K) || ldx < (K + 15) / 16 * 16 || ldx % 16 != 0 || ldy < N) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    if (!Xq8 || !s_x || !Wq8 || !s_w || !Y) return MQ_ERR_INVALID_ARG;
    const size_t size = type == MQ_FP32 ? 4 : 2;
    if (!mq_host::aligned(Xq8, 16) || !mq_host::aligned(Wq8, 16) || !mq_host::aligned(s_x, 4) || !mq_host::aligned(s_w, 4) ||
        !mq_host::aligned(bias, size) || !mq_host::aligned(Y, size))
        return MQ_ERR_MISALIGNED;
    const size_t need = mq_gemm_w8a8_workspace_size(M, N, K);
    if (need > 0 && (!workspace || ws_bytes < need)) return MQ_ERR_WORKSPACE;
    const Product8Args a{M, N, K, reinterpret_cast<const uint8_t*>(Xq8), ldx, s_x, Wq8, s_w, bias, Y, ldy};
    auto run = [&](auto z) {
        using T = decltype(z);
        const int64_t tiles = (int64_t)((N + 127) / 128) * ((M + 31) / 32);
        if (tiles > INT32_MAX) return MQ_ERR_UNSUPPORTED_SHAPE;
        hipLaunchKernelGGL(product8_kernel<T>, dim3((unsigned)tiles), dim3(256), 0, stream, a);
        return mq_host::launch_status();
    };
    return type == MQ_FP32 ? run(float{}) : mq_host::with_half_type(type, run);
}
