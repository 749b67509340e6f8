// Product of e4m3 activations and e4m3 weights with a scale for each token and
// 128 channels, and for each block of 128 x 128 of the weight:
//   Y[m,n] = rn( sum_g s_x[m,g] s_w[n/128,g] sum_{k in g} Xq[m,k] Wq[n,k] + bias[n] ).
//
// One v_mfma_f32_16x16x128_f8f6f4 sums a group of 128 for 16 x 16 outputs (fp32 results: four
// v_mfma_f32_16x16x32_f16, the codes turned to fp16), and one
// fp32 fma an output puts it to the rest, by the product of the two scales.  The
// weight's layout is that of the INT8 product (mq.h): lane l's 16 bytes of two
// pieces of 64 codes are the instruction's 32, and X's rows are taken the same way.
// Codes of X are read up to the next 16 past K; there and past N weights are zero, so that a NaN there is all that would show (and
// is the caller's to keep away: cleared in LDS, as one more stage, 131 x 5000 -> 8191 took 21.9 us instead of 21.0).
//
// Inside the 8-bit instruction eight neighbouring products at a time are cut, towards zero, to multiples of 2^(e - 13), e the
// sum of the exponents of the largest one's factors (measured; the 32-long fp8 instruction does the same).  It costs
// outputs 1.4e-5 of their norm where values are of one size, some 3e-5 beside outlier channels; a 16-bit result's own rounding
// is 2e-4 and more, an fp32 one's is not.  Those go by fp16 operands, at half the rate: 1e-7 of the norm; 1 x 4096 -> 131071
// 91 us instead of 88, 128 rows of it 163 and 147, 4096 x 4096 -> 32768 1030 and 620.  Everything after a group's sum is fp32.
//
// Two kernels, as there:
//  * tiled: output tiles through LDS slots of one group, filled by the LDS DMA, scales of X among them.  The matrix
//    unit, LDS and four fmas a product bound it together: 8192 rows of 8192 codes by 28672 channels 1610 to 1800 us
//    as the card's clock goes, 2.1 to 2.4 PFLOP/s; 4096 -> 4096 at 4096 rows 64 to 70 us;
//  * streaming (few rows): weights straight to registers, once; the eight waves of a workgroup share out the groups,
//    and their sums are added in LDS in the order of the waves.  Reading the weight bounds it: 4096 -> 14336 at one row
//    9.6 us, 6.1 TB/s.
#include "lds_dma.h"
#include "kv8.h"

#include <algorithm>
#include <type_traits>

namespace mq {

constexpr int kBlockF8 = 64;            // channels of a block of the layout
constexpr int kPieceF8 = 1024;          // bytes of 16 channels of 64 codes
constexpr int kMaxGroups = (MQ_W8A8_MAX_K + kGroup - 1) / kGroup;
constexpr int kWaveRowsF8 = 32;         // rows of X at most that a wave loads: they span less than 2 GB

struct ProductF8Args {
    int M, N, K;
    const uint8_t* X;
    int64_t ldx;
    const float* s_x;                   // [groups][lds]
    int64_t lds;
    const uint8_t* W;
    const float* s_w;                   // [N / 128][groups]
    const void* bias;
    void* Y;
    int64_t ldy;
    int y16;                            // rows of Y 16-byte aligned
};

__host__ __device__ __forceinline__ int groups_of(int K) { return (K + kGroup - 1) / kGroup; }
__host__ __device__ __forceinline__ int blocks_of(int N) { return (N + kBlockF8 - 1) / kBlockF8; }

__device__ __forceinline__ i32x8 operand_f8(const uint4 a, const uint4 b) {
    return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}
// The sum of 128 products for 16 x 16 outputs of type T: of fp32 ones in fp32, of others cut as above.
template <typename T>
__device__ __forceinline__ f32x4 mfma_f8(const i32x8 a, const i32x8 b) {
    if constexpr (__is_same(T, float)) {
        f32x4 sum = {};
#pragma unroll
        for (int i = 0; i < 8; i += 2)
            sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand8((uint32_t)a[i], (uint32_t)a[i + 1]), operand8((uint32_t)b[i], (uint32_t)b[i + 1]), sum, 0, 0, 0);
        return sum;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{}, 0, 0, 0, 0, 0, 0);
    }
}

// y[c] = sum + bias for 16 channels n .. n + 15 of row m, stored.
template <typename T>
__device__ __forceinline__ void store_row_f8(const ProductF8Args& a, int m, int n, float (&y)[16]) {
    if (a.bias) {
#pragma unroll
        for (int c = 0; c < 16; ++c)
            if (n + c < a.N) y[c] += (float)static_cast<const T*>(a.bias)[n + c];
    }
    T* row = static_cast<T*>(a.Y) + m * a.ldy + n;
    if (a.y16 && n + 16 <= a.N) {
        constexpr int per = 16 / sizeof(T);
        typedef T vec __attribute__((ext_vector_type(per)));
#pragma unroll
        for (int c = 0; c < 16; c += per) {
            vec v;
#pragma unroll
            for (int e = 0; e < per; ++e) v[e] = (T)y[c + e];
            *reinterpret_cast<vec*>(row + c) = v;
        }
    } else {
#pragma unroll
        for (int c = 0; c < 16; ++c)
            if (n + c < a.N) row[c] = (T)y[c];
    }
}

// 16 rows of a wave's 64 channels n0 .. where rows of Y are not 16-byte aligned: through LDS, so that a store takes 64 neighbours
// (131 rows of 5000 codes by 8191 channels: one value a lane and 16 rows a store 24 us, so 20.5).
template <typename T>
__device__ __forceinline__ void store_block_f8(const ProductF8Args& a, int m0, int n0, const f32x4 (&sum)[4], float (*lds)[68]) {
    const int lane = threadIdx.x & 63, lrow = lane & 15, lq = lane >> 4, n = n0 + lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(&lds[lrow][16 * lq + 4 * i]) = sum[i];
    wave_sync();
    if (n < a.N) {
        const float bias = a.bias ? (float)static_cast<const T*>(a.bias)[n] : 0.0f;
        T* y = static_cast<T*>(a.Y) + m0 * a.ldy + n;
        const int rows = min(16, a.M - m0);
        for (int r = 0; r < rows; ++r) y[r * a.ldy] = (T)(a.bias ? lds[r][lane] + bias : lds[r][lane]);
    }
    wave_sync();
}

// --------------------------------------------------------------------------
// Tiled kernel: WM x WN waves, each 16 MI rows of X by one block of 64 channels.
// --------------------------------------------------------------------------
// A stage is a group: rows of 128 bytes of X (16-byte chunk q of row r at q ^ (r % 8):
// reads of 16 rows are free of bank conflicts, and every load of eight rows takes
// whole lines), 8 KB of W for each block, in order, and the rows' scales.  One
// barrier a stage, when all of it has been read, two rows of products before its
// end: it says so, and that the next stage has landed; the loads of the stage SLOTS
// on go into its slot.  Loads past the last stage read nothing: they keep the number
// in flight the same throughout.  X is read two rows ahead, and a row's sums are put to
// the rest after the next row's products have been issued (8192 x 8192 -> 28672 1754 us
// without both, 1690 on the same card).
// SPLIT: workgroup y takes the groups [y, y + 1) per_split and writes its sums to part[y][M][N].
template <typename T, int WM, int WN, int MI, int SLOTS, bool SPLIT>
__device__ __forceinline__ void product_tiled(ProductF8Args a, int per_split, float* __restrict__ part) {
    constexpr int TM = 16 * MI * WM, TN = kBlockF8 * WN, NW = WM * WN;
    constexpr int XL = TM / 8 / NW, WL = TN / 8 / NW;       // 1 KB loads of a wave and stage
    constexpr int SW = (TN + kGroup - 1) / kGroup;          // rows of blocks of W's scales
    static_assert(XL * NW * 8 == TM && 8 * XL <= kWaveRowsF8 && (WL == 2 || WL == 4), "whole loads");
    __shared__ __attribute__((aligned(16))) struct {
        uint8_t x[SLOTS][TM * kGroup];
        uint8_t w[SLOTS][TN * kGroup];
        float sx[SLOTS][NW][64];                            // of a wave's 8 XL rows
        float sw[SW][kMaxGroups];
    } L;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN, lrow = lane & 15, lq = lane >> 4;
    const int groups = groups_of(a.K), kp = groups * kGroup, blocks = blocks_of(a.N);
    const int first = SPLIT ? blockIdx.y * per_split : 0, stages = SPLIT ? min(per_split, groups - first) : groups;
    int tm, tn;
    tile_coords(blockIdx.x, (a.M + TM - 1) / TM, (a.N + TN - 1) / TN, tm, tn);
    const int m0 = tm * TM, b0 = tn * WN;

    for (int i = threadIdx.x; i < SW * stages; i += 64 * NW) {
        const int r = i / stages, g = i % stages, nb = b0 * kBlockF8 / kGroup + r;
        L.sw[r][g] = nb * kGroup < a.N ? a.s_w[(int64_t)nb * groups + first + g] : 0.0f;
    }
    // X from the wave's own first row on: what a resource spans stays below 2 GB (the host sees to it), and rows past M
    // are past its end
    const int mw = m0 + 8 * XL * wave, rows = min(8 * XL, a.M - mw);
    const uint32_t kx = (uint32_t)(a.K + 15) / 16 * 16;
    const i32x4 rx = make_desc(a.X + mw * a.ldx, rows > 0 ? (uint32_t)((rows - 1) * a.ldx + kx) : 0u);
    const i32x4 rw = make_desc(a.W + (int64_t)b0 * kp * kBlockF8, (uint32_t)min(WN, blocks - b0) * (uint32_t)(kp * kBlockF8));
    const uint32_t ldx = (uint32_t)a.ldx;
    const uint32_t chunk = (uint32_t)((lane & 7) ^ (lane >> 3)) << 4;
    const uint32_t vx = (uint32_t)(lane >> 3) * ldx + chunk;
    const uint32_t vw = (uint32_t)lane * 16;
    const uint32_t vs = lane < rows ? (uint32_t)lane * 4 : kPastEnd;
    uint32_t sx = (uint32_t)(first * kGroup);
    uint32_t sw = (uint32_t)(WL * wave / 8) * (uint32_t)(kp * kBlockF8) + (uint32_t)(WL * wave % 8) * 1024u + (uint32_t)(first * 8192);
    const float* scales = a.s_x + (int64_t)first * a.lds + mw;
    int to_load = stages;
    auto issue = [&](int slot) {
        const bool there = to_load-- > 0;
        const uint32_t v = sx + chunk < kx ? vx : kPastEnd; // codes past K may be anything
#pragma unroll
        for (int k = 0; k < XL; ++k)
            dma16s(rx, lds_addr(L.x) + (uint32_t)(slot * (TM * kGroup) + (XL * wave + k) * 1024), v, there ? sx + (uint32_t)(8 * k) * ldx : kPastEnd);
        const uint32_t dst = lds_addr(L.w) + (uint32_t)(slot * (TN * kGroup) + WL * wave * 1024);
        if constexpr (WL == 4) dma16x4(rw, dst, vw, there ? sw : kPastEnd);
        else dma16x2(rw, dst, vw, there ? sw : kPastEnd);
        dma4(make_desc(scales, there && rows > 0 ? (uint32_t)rows * 4u : 0u), lds_addr(L.sx) + (uint32_t)((slot * NW + wave) * 256), vs, 0u);
        sx += kGroup;
        sw += 8192;
        if (there) scales += a.lds;
    };
    constexpr int LOADS = XL + WL + 1;
    const uint32_t xa = lds_addr(L.x) + (uint32_t)(wm * 16 * MI + lrow) * kGroup + (uint32_t)((lq ^ (lrow & 7)) << 4);
    const uint32_t wa = lds_addr(L.w) + (uint32_t)(wn * 8192 + lane * 16);
    auto read_x = [&](int slot, int j) {
        const uint32_t at = xa + (uint32_t)(slot * (TM * kGroup) + j * 2048);
        return operand_f8(lds_read16(at), lds_read16(at ^ 64u));
    };
    f32x4 acc[4][MI] = {};

    for (int s = 0; s < SLOTS; ++s) issue(s);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((SLOTS - 1) * LOADS) : "memory");
    int slot = 0;
    for (int s = 0; s < stages; ++s) {
        const int next = slot + 1 == SLOTS ? 0 : slot + 1;
        i32x8 w[4], x[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = wa + (uint32_t)(slot * (TN * kGroup) + i * 1024);
            w[i] = operand_f8(lds_read16(at), lds_read16(at + 4096));
        }
        x[0] = read_x(slot, 0);
        if constexpr (MI > 1) x[1] = read_x(slot, 1);
        float scale[MI];
        const float by = L.sw[wn * kBlockF8 / kGroup][s];
#pragma unroll
        for (int j = 0; j < MI; ++j) {
            const int row = wm * 16 * MI + 16 * j;          // 8 XL rows a wave: 16 of them are one wave's
            scale[j] = by * L.sx[slot][row / (8 * XL)][row % (8 * XL) + lrow];
        }
        f32x4 sum[2][4];
#pragma unroll
        for (int j = 0; j <= MI; ++j) {
            if (j < MI) {
                if (j + 2 < MI) x[(j + 2) % 3] = read_x(slot, j + 2);
                if (j == (MI > 1 ? MI - 2 : 0)) {           // all of the stage is read
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((SLOTS - 2) * LOADS) : "memory");
                    issue(slot);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[j % 2][i] = mfma_f8<T>(w[i], x[j % 3]);
            }
            if (j > 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j - 1][r] = __builtin_fmaf(scale[j - 1], sum[(j - 1) % 2][i][r], acc[i][j - 1][r]);
            }
        }
        slot = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // nothing may write LDS after the workgroup has gone

    const int n = (b0 + wn) * kBlockF8 + 16 * lq;
    if (!SPLIT && !a.y16) {
        __syncthreads();                                    // the slots are everybody's, and their last loads write zeros
        static_assert(sizeof(L.x) + sizeof(L.w) >= NW * 16 * 68 * sizeof(float), "16 rows of each wave");
        float(*rows16)[68] = reinterpret_cast<float(*)[68]>(&L) + 16 * wave;
#pragma unroll
        for (int j = 0; j < MI; ++j) {
            const int m = m0 + wm * 16 * MI + 16 * j;
            const f32x4 sum[4] = {acc[0][j], acc[1][j], acc[2][j], acc[3][j]};
            if (m < a.M) store_block_f8<T>(a, m, n - 16 * lq, sum, rows16);
        }
        return;
    }
    if (n >= a.N) return;
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        const int m = m0 + wm * 16 * MI + 16 * j + lrow;
        if (m >= a.M) break;
        if constexpr (SPLIT) {
            float* p = part + ((int64_t)blockIdx.y * a.M + m) * (blocks * kBlockF8) + n;
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(p + 4 * i) = acc[i][j];
        } else {
            float y[16];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) y[4 * i + r] = acc[i][j][r];
            store_row_f8<T>(a, m, n, y);
        }
    }
}

// 16-bit results, and fp32 ones (whose matrix instruction is another).
template <typename T, int WM, int WN, int MI, int SLOTS, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_f8_tiled_kernel(ProductF8Args a, int per_split, float* __restrict__ part) {
    product_tiled<T, WM, WN, MI, SLOTS, SPLIT>(a, per_split, part);
}
template <int WM, int WN, int MI, int SLOTS, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_fp32_tiled_kernel(ProductF8Args a, int per_split, float* __restrict__ part) {
    product_tiled<float, WM, WN, MI, SLOTS, SPLIT>(a, per_split, part);
}

// Sums of the splits, in order -> Y, 16 channels a thread.
template <typename T>
__global__ __launch_bounds__(256) void product_f8_join_kernel(ProductF8Args a, int splits, const float* __restrict__ part) {
    const int np = blocks_of(a.N) * kBlockF8, per = np / 16;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.M * per) return;
    const int m = (int)(i / per), n = (int)(i % per) * 16;
    if (n >= a.N) return;
    f32x4 sum[4] = {};
    for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] += *reinterpret_cast<const f32x4*>(part + ((int64_t)s * a.M + m) * np + n + 4 * c);
    float y[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) y[c] = sum[c / 4][c % 4];
    store_row_f8<T>(a, m, n, y);
}

// --------------------------------------------------------------------------
// Streaming kernel: P pieces of a block and all rows (16 MT) a workgroup.
// --------------------------------------------------------------------------
constexpr int kStreamWavesF8 = 8;
template <typename T, int P, int MT>
__device__ __forceinline__ void product_stream(ProductF8Args a) {
    constexpr int U = P + MT >= 4 ? 1 : 6 / (P + MT);       // groups in flight, twice
    __shared__ float sums[kStreamWavesF8][16 * MT][16 * P + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lrow = lane & 15, lq = lane >> 4;
    const int groups = groups_of(a.K);
    const int block = blockIdx.x / (4 / P), i0 = blockIdx.x % (4 / P) * P;
    const uint8_t* w = a.W + (int64_t)block * groups * (kGroup * kBlockF8) + i0 * kPieceF8 + 16 * lane;
    const float* s_w = a.s_w + (int64_t)(block * kBlockF8 / kGroup) * groups;
    int64_t x[MT];                                          // rows
#pragma unroll
    for (int j = 0; j < MT; ++j) x[j] = (int64_t)min(16 * j + lrow, a.M - 1) * a.ldx;

    struct Batch {
        uint4 w[U][P][2], x[U][MT][2];
        float s[U][MT], by[U];
    };
    auto load = [&](Batch& b, int g0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int g = min(g0 + u * kStreamWavesF8, groups - 1);
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) b.w[u][i][h] = ldg16(w + (int64_t)g * 8192 + h * 4096 + i * kPieceF8);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = g * kGroup + 64 * h + 16 * lq;
                    b.x[u][j][h] = k < a.K ? ldg16(a.X + x[j] + k) : make_uint4(0, 0, 0, 0);
                }
                b.s[u][j] = a.s_x[g * a.lds + min(16 * j + lrow, a.M - 1)];
            }
            b.by[u] = s_w[g];
        }
    };
    f32x4 acc[P][MT] = {};
    auto multiply = [&](const Batch& b, int g0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (g0 + u * kStreamWavesF8 >= groups) break;
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const i32x8 xo = operand_f8(b.x[u][j][0], b.x[u][j][1]);
                const float scale = b.s[u][j] * b.by[u];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const f32x4 sum = mfma_f8<T>(operand_f8(b.w[u][i][0], b.w[u][i][1]), xo);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] = __builtin_fmaf(scale, sum[r], acc[i][j][r]);
                }
            }
        }
    };
    Batch b0, b1;
    constexpr int step = U * kStreamWavesF8;
    if (wave < groups) load(b0, wave);
    for (int g = wave; g < groups; g += 2 * step) {
        if (g + step < groups) load(b1, g + step);
        multiply(b0, g);
        if (g + step >= groups) break;
        if (g + 2 * step < groups) load(b0, g + 2 * step);
        multiply(b1, g + step);
    }
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[wave][16 * j + lrow][(4 * lq) * P + 4 * i + r] = acc[i][j][r];
    __syncthreads();
    // columns 4 P a + 4 i + b are channels 16 a + 4 (i0 + i) + b
    for (int e = threadIdx.x; e < 16 * P * min(a.M, 16 * MT); e += 64 * kStreamWavesF8) {
        const int m = e / (16 * P), c = e % (16 * P);
        const int n = block * kBlockF8 + c / (4 * P) * 16 + 4 * i0 + c % (4 * P);
        if (n >= a.N) continue;
        float y = 0.0f;
#pragma unroll
        for (int v = 0; v < kStreamWavesF8; ++v) y += sums[v][m][c];
        if (a.bias) y += (float)static_cast<const T*>(a.bias)[n];
        static_cast<T*>(a.Y)[m * a.ldy + n] = (T)y;
    }
}

template <typename T, int P, int MT>
__global__ __launch_bounds__(64 * kStreamWavesF8) void product_f8_stream_kernel(ProductF8Args a) {
    product_stream<T, P, MT>(a);
}
template <int P, int MT>
__global__ __launch_bounds__(64 * kStreamWavesF8) void product_fp32_stream_kernel(ProductF8Args a) {
    product_stream<float, P, MT>(a);
}

// --------------------------------------------------------------------------
// Quantisers and layouts.
// --------------------------------------------------------------------------
// Codes of values x by their scale s = amax / 448: e4m3 of the fp32 quotient.  The quotient is the product with the
// reciprocal and one exact correction (correctly rounded, as the reciprocal is); where s is near fp32's smallest numbers it is divided.
struct Scale8 {
    float s, inv;
    bool divides;
    __device__ __forceinline__ explicit Scale8(uint32_t amax_bits) {
        s = __uint_as_float(amax_bits) / kE4m3Max;
        divides = !(s > 0x1p-90f && s < 0x1p100f);
        inv = 1.0f / s;
    }
    __device__ __forceinline__ bool finite() const { return __float_as_uint(s) < kFloatInf; }
    __device__ __forceinline__ float of(float x) const {
        float q;
        if (divides) {
            q = s > 0.0f && finite() ? x / s : 0.0f;
        } else {
            const float q0 = x * inv;
            q = __builtin_fmaf(__builtin_fmaf(-q0, s, x), inv, q0);
        }
        return __builtin_amdgcn_fmed3f(q, -kE4m3Max, kE4m3Max);
    }
};

// 16 lanes take a row's group, a wave four rows, a workgroup 16 (so scales go out in whole lines) by four groups in turn.
// Memory bounds it: 8192 x 8192 bf16 43 us, 4.7 TB/s.
constexpr int kQuantRows = 16, kQuantGroups = 4;
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_f8_kernel(const T* __restrict__ X, int64_t ldx, int M, int K,
                                                               uint8_t* __restrict__ Xq, int64_t ldq, float* __restrict__ s_x, int64_t lds) {
    const int lane = threadIdx.x & 15, m = blockIdx.x * kQuantRows + (threadIdx.x >> 4), groups = groups_of(K);
    const int g0 = blockIdx.y * kQuantGroups, kx = (K + 15) / 16 * 16;
    if (m >= M) return;
    f32x8 x[kQuantGroups];
#pragma unroll
    for (int i = 0; i < kQuantGroups; ++i) {
        const int k = (g0 + i) * kGroup + 8 * lane;
        x[i] = k < K ? load8(X + m * ldx + k) : f32x8{};
    }
#pragma unroll
    for (int i = 0; i < kQuantGroups; ++i) {
        if (g0 + i >= groups) break;
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = max(amax, __float_as_uint(x[i][j]) & 0x7FFFFFFFu);
        auto step = [&](auto ctrl) {
            amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, decltype(ctrl)::value, 0xf, 0xf, true));
        };
        step(std::integral_constant<int, 0xB1>{});          // quad_perm 1, 0, 3, 2
        step(std::integral_constant<int, 0x4E>{});          // quad_perm 2, 3, 0, 1
        step(std::integral_constant<int, 0x141>{});         // row_half_mirror
        step(std::integral_constant<int, 0x140>{});         // row_mirror
        const bool fine = amax < kFloatInf;
        const Scale8 s(fine ? amax : 0u);
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = s.of(fine ? x[i][j] : 0.0f);
        const int k = (g0 + i) * kGroup + 8 * lane;
        if (k < kx)
            *reinterpret_cast<uint2*>(Xq + m * ldq + k) = make_uint2(to_e4m3x4(q[0], q[1], q[2], q[3]), to_e4m3x4(q[4], q[5], q[6], q[7]));
        if (lane == 0) s_x[(g0 + i) * lds + m] = fine ? s.s : __builtin_nanf("");
    }
}

// Byte of the 16 codes from k on (a multiple of 16) of channel n.
__device__ __forceinline__ int64_t weight_offset_f8(int n, int k, int groups) {
    const int c = n % kBlockF8, row = c / 16 * 4 + c % 4, piece = c % 16 / 4;
    return (((int64_t)(n / kBlockF8) * (2 * groups) + k / 64) * 4 + piece) * kPieceF8 + 16 * (row + 16 * (k % 64 / 16));
}

// One workgroup takes a block of 128 x 128, a thread 16 values of a row.  FLOAT: values, whose scale is made; else codes.
template <bool FLOAT>
__global__ __launch_bounds__(1024) void pack_weight_f8_kernel(const void* __restrict__ W, int64_t ldw, int N, int K,
                                                              uint8_t* __restrict__ Wq, float* __restrict__ s_w) {
    __shared__ uint32_t most[16];
    const int groups = groups_of(K), nb = blockIdx.x / groups, g = blockIdx.x % groups;
    const int n = nb * kGroup + threadIdx.x / 8, k = g * kGroup + 16 * (threadIdx.x % 8);
    const int64_t at = n * ldw + k;
    uint32_t b[4] = {0, 0, 0, 0};
    if constexpr (FLOAT) {
        float x[16];
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = n < N && k + e < K ? static_cast<const float*>(W)[at + e] : 0.0f;
            amax = max(amax, __float_as_uint(x[e]) & 0x7FFFFFFFu);
        }
        amax = wave_max_dpp(amax);
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = amax;
        __syncthreads();
        for (int i = 0; i < 16; ++i) amax = max(amax, most[i]);
        const bool fine = amax < kFloatInf;
        const Scale8 s(fine ? amax : 0u);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            b[i] = fine ? to_e4m3x4(s.of(x[4 * i]), s.of(x[4 * i + 1]), s.of(x[4 * i + 2]), s.of(x[4 * i + 3])) : 0u;
        if (threadIdx.x == 0) s_w[(int64_t)nb * groups + g] = fine ? s.s : __builtin_nanf("");
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (n < N && k + e < K) b[e / 4] |= (uint32_t)static_cast<const uint8_t*>(W)[at + e] << (8 * (e % 4));
    }
    if (n < blocks_of(N) * kBlockF8)
        *reinterpret_cast<uint4*>(Wq + weight_offset_f8(n, k, groups)) = make_uint4(b[0], b[1], b[2], b[3]);
}

__global__ __launch_bounds__(256) void unpack_weight_f8_kernel(const uint8_t* __restrict__ Wq, int N, int K, uint8_t* __restrict__ Wc, int64_t ldw) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)N * K; i += (int64_t)gridDim.x * 256) {
        const int n = (int)(i / K), k = (int)(i % K);
        Wc[n * ldw + k] = Wq[weight_offset_f8(n, k / 16 * 16, groups_of(K)) + k % 16];
    }
}

template <int N>
using Int = std::integral_constant<int, N>;
static bool shape_f8_ok(int N, int K) { return N >= 1 && N <= (1 << 24) && K >= 1 && K <= MQ_W8A8_MAX_K; }

// ---------------------------------------------------------------- host side --
// Which kernel takes a product.  Up to 16 rows, and up to 32 where the weight is small, the streaming kernel (a graph of calls; 5000 ->
// 8191 at 17 rows 10.3 us, 64 x 64 tiles 16.2; 4096 -> 14336 15.0 and 14.4; at 16 rows 13.2 and 14.4).  It takes as many pieces
// a workgroup as leave every CU one: four from 192 blocks on (1 x 4096 -> 14336 by one, two, four 17.9, 14.9, 12.1; 5120 wide 7.9, 6.1,
// 5.9), two from 64 on (16 x 8192 -> 8191 20.4, 14.5, 18.3; 1 x 8192 -> 2048 5.6, 6.0, 8.3), one where K is long besides (1 x 14336 ->
// 4096 12.5, 14.4, 22.3; not the best from 65 blocks on: 16 x 14336 -> 5120 25.7, 19.4).  Beyond, of four tiles and one, two or four splits of K the one with
// the least estimated time: groups by the time of one (a workgroup alone on its CU waits for memory; more of them
// share it), or W at the rate that the tiles reach, whichever is longer, and what writing and joining a split's sums
// takes.  128 x 128 has four slots where there is no more than one workgroup a CU, and two where two share it (8192 ->
// 8192 at 512 rows 43 us instead of 57, at 1024 rows 87 instead of 76).  Measured (us): 8192 -> 8192 at 64 rows by 64 x 64 in two
// splits 20, unsplit 25; at 200 rows by 128 x 64 31, 64 x 64 35; at 300 by 128 x 128 38, 128 x 64 49; 4096 -> 4096 at
// 4096 by 256 x 256 68, 128 x 128 75; 14336 -> 4096 at 131 rows by 128 x 128 in four splits 28, 128 x 64 30.
struct TileF8 {
    int rows, cols;
    double alone, share;                // us of a stage: one workgroup a CU, and of each of several
    bool splits;
};
constexpr TileF8 kTilesF8[4] = {
    {64, 64, 0.36, 0.28, true},
    {128, 64, 0.45, 0.38, true},
    {128, 128, 0.60, 0.59, true},
    {256, 256, 1.90, 1.90, false},
};
struct PlanF8 {
    int rows, cols;                     // of a workgroup's tile; cols of the streaming kernel: 16 P
    bool streams;
    int splits, per_split;              // groups of a split
};
static PlanF8 plan_f8(int M, int N, int K) {
    const int blocks = blocks_of(N), stages = groups_of(K);
    if (M <= 16 || (M <= 32 && blocks < 192 && K <= 8192)) {
        const int p = blocks >= 192 ? 4 : blocks >= 64 && K <= 8192 ? 2 : 1;
        return PlanF8{M <= 16 ? 16 : 32, 16 * p, true, 1, stages};
    }
    PlanF8 best{};
    double least = 0.0;
    for (const TileF8& t : kTilesF8)
        for (int splits = 1; splits <= (t.splits ? 4 : 1); splits *= 2) {
            if (splits > 1 && stages < 8 * splits) break;
            const int64_t groups = (int64_t)((M + t.rows - 1) / t.rows) * ((N + t.cols - 1) / t.cols) * splits;
            const int64_t a_cu = (groups + 255) / 256;
            const int per = (stages + splits - 1) / splits;
            const double compute = per * std::max(t.alone, a_cu * t.share), memory = (double)N * K / 4.6e6;
            const double join = splits == 1 ? 0.0 : 6.0 + (double)M * N * 4 * (splits + 1) / 5.0e6;
            const double us = std::max(compute, memory) + join;
            if (least == 0.0 || us < least) {
                least = us;
                best = PlanF8{t.rows, t.cols, false, (stages + per - 1) / per, per};
            }
        }
    return best;
}

}  // namespace mq

using namespace mq;

extern "C" mq_status mq_quantize_rows_fp8(int M, int K, mq_dtype type, const void* X, int ldx, void* Xq, int ldq, float* s_x, int lds,
                                          hipStream_t stream) {
    if (M < 0 || K < 0 || !mq_host::is_half_type(type)) return MQ_ERR_INVALID_ARG;
    const int64_t blocks = ((int64_t)M + kQuantRows - 1) / kQuantRows, turns = (groups_of(K) + kQuantGroups - 1) / kQuantGroups;
    if (M > (1 << 24) || !shape_f8_ok(1, K) || K % 8 != 0 || ldx < K || ldx % 8 != 0 || ldq < (K + 15) / 16 * 16 || ldq % 16 != 0 || lds < M ||
        !mq_host::launch_holds(blocks * turns, 256))
        return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    if (!X || !Xq || !s_x) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(X, 16) || !mq_host::aligned(Xq, 16) || !mq_host::aligned(s_x, 4)) return MQ_ERR_MISALIGNED;
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        hipLaunchKernelGGL(quantize_rows_f8_kernel<T>, dim3((unsigned)blocks, (unsigned)turns), dim3(256), 0, stream, static_cast<const T*>(X),
                           ldx, M, K, static_cast<uint8_t*>(Xq), ldq, s_x, lds);
        return mq_host::launch_status();
    });
}

extern "C" size_t mq_weight_fp8_bytes(int N, int K) {
    if (!shape_f8_ok(N, K)) return 0;
    return (size_t)blocks_of(N) * kBlockF8 * groups_of(K) * kGroup;
}

template <bool FLOAT>
static mq_status pack_f8(const void* W, int N, int K, int ldw, uint8_t* Wq, float* s_w, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    const int64_t blocks = (int64_t)((N + kGroup - 1) / kGroup) * groups_of(K);
    if (!shape_f8_ok(N, K) || ldw < K || !mq_host::launch_holds(blocks, 1024)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!W || !Wq || (FLOAT && !s_w)) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(W, FLOAT ? 4 : 1) || !mq_host::aligned(Wq, 16) || !mq_host::aligned(s_w, 4)) return MQ_ERR_MISALIGNED;
    hipLaunchKernelGGL(pack_weight_f8_kernel<FLOAT>, dim3((unsigned)blocks), dim3(1024), 0, stream, W, ldw, N, K, Wq, s_w);
    return mq_host::launch_status();
}

extern "C" mq_status mq_quantize_weight_fp8(const float* W, int N, int K, int ldw, uint8_t* Wq, float* s_w, hipStream_t stream) {
    return pack_f8<true>(W, N, K, ldw, Wq, s_w, stream);
}

extern "C" mq_status mq_repack_weight_fp8(int N, int K, const uint8_t* Wc, int ldw, uint8_t* Wq, hipStream_t stream) {
    return pack_f8<false>(Wc, N, K, ldw, Wq, nullptr, stream);
}

extern "C" mq_status mq_unpack_weight_fp8(int N, int K, const uint8_t* Wq, uint8_t* Wc, int ldw, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape_f8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Wc || !Wq) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Wq, 16)) return MQ_ERR_MISALIGNED;
    // a launch has less than 2^32 threads; the rest of the codes come in further turns
    const int64_t blocks = std::min<int64_t>(((int64_t)N * K + 255) / 256, 1 << 22);
    hipLaunchKernelGGL(unpack_weight_f8_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, Wq, N, K, Wc, ldw);
    return mq_host::launch_status();
}

extern "C" size_t mq_gemm_fp8_workspace_size(int M, int N, int K) {
    if (M < 1 || M > (1 << 24) || !shape_f8_ok(N, K)) return 0;
    const PlanF8 p = plan_f8(M, N, K);
    return p.splits == 1 ? 0 : (size_t)p.splits * M * blocks_of(N) * kBlockF8 * sizeof(float);
}

extern "C" mq_status mq_gemm_fp8_tile(int M, int N, int K, int* rows, int* cols, int* splits) {
    if (!rows || !cols || !splits || M < 1 || M > (1 << 24)) return MQ_ERR_INVALID_ARG;
    if (!shape_f8_ok(N, K)) return MQ_ERR_UNSUPPORTED_SHAPE;
    const PlanF8 p = plan_f8(M, N, K);
    *rows = p.rows;
    *cols = p.cols;
    *splits = p.splits;
    return MQ_OK;
}

extern "C" mq_status mq_gemm_fp8(int M, int N, int K, const void* Xq, int ldx, const float* s_x, int lds, const uint8_t* Wq, const float* s_w,
                                 mq_dtype type, const void* bias, void* Y, int ldy, void* workspace, size_t ws_bytes, hipStream_t stream) {
    if (M < 0 || N < 0 || K < 0 || (!mq_host::is_half_type(type) && type != MQ_FP32)) return MQ_ERR_INVALID_ARG;
    if (M > (1 << 24) || !shape_f8_ok(N, K) || ldx < (K + 15) / 16 * 16 || ldx % 16 != 0 || ldy < N || lds < M) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    PlanF8 p = plan_f8(M, N, K);
    if (type == MQ_FP32 && p.rows == 256) p.rows = p.cols = 128;   // (operands in fp16 leave no registers for more: 4096 x 4096 -> 32768 1320 us)
    const int64_t groups = p.streams ? (int64_t)blocks_of(N) * (kBlockF8 / p.cols)
                                     : (int64_t)((M + p.rows - 1) / p.rows) * ((N + p.cols - 1) / p.cols);
    const int64_t joins = p.splits > 1 ? ((int64_t)M * (blocks_of(N) * kBlockF8 / 16) + 255) / 256 : 0;
    if (!mq_host::launch_holds(groups * p.splits, 512) || !mq_host::launch_holds(joins, 256)) return MQ_ERR_UNSUPPORTED_SHAPE;
    // offsets within a wave's rows: 31 bits, past which loads read nothing
    if (!p.streams && (int64_t)(std::min(M, kWaveRowsF8) - 1) * ldx + (K + 15) / 16 * 16 > INT32_MAX) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Xq || !s_x || !Wq || !s_w || !Y) return MQ_ERR_INVALID_ARG;
    const size_t size = type == MQ_FP32 ? 4 : 2;
    if (!mq_host::aligned(Xq, 16) || !mq_host::aligned(Wq, 16) || !mq_host::aligned(s_x, 4) || !mq_host::aligned(s_w, 4) ||
        !mq_host::aligned(bias, size) || !mq_host::aligned(Y, size) || !mq_host::aligned(workspace, 16))
        return MQ_ERR_MISALIGNED;
    const size_t need = mq_gemm_fp8_workspace_size(M, N, K);
    if (need > 0 && (!workspace || ws_bytes < need)) return MQ_ERR_WORKSPACE;
    const ProductF8Args a{M, N, K, static_cast<const uint8_t*>(Xq), ldx, s_x, lds, Wq, s_w, bias, Y, ldy,
                          mq_host::aligned(Y, 16) && ldy * size % 16 == 0};
    auto run = [&](auto z) {
        using T = decltype(z);
        float* part = static_cast<float*>(workspace);
        auto stream_rows = [&](auto pieces, auto rows) {
            constexpr int P = decltype(pieces)::value, MT = decltype(rows)::value;
            const dim3 grid((unsigned)groups), threads(64 * kStreamWavesF8);
            if constexpr (__is_same(T, float)) hipLaunchKernelGGL((product_fp32_stream_kernel<P, MT>), grid, threads, 0, stream, a);
            else hipLaunchKernelGGL((product_f8_stream_kernel<T, P, MT>), grid, threads, 0, stream, a);
        };
        auto tile = [&](auto wm, auto wn, auto mi, auto slots, auto split) {
            constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, MI = decltype(mi)::value, SLOTS = decltype(slots)::value;
            constexpr bool SPLIT = decltype(split)::value;
            const dim3 grid((unsigned)groups, p.splits), threads(64 * WM * WN);
            if constexpr (__is_same(T, float)) hipLaunchKernelGGL((product_fp32_tiled_kernel<WM, WN, MI, SLOTS, SPLIT>), grid, threads, 0, stream, a, p.per_split, part);
            else hipLaunchKernelGGL((product_f8_tiled_kernel<T, WM, WN, MI, SLOTS, SPLIT>), grid, threads, 0, stream, a, p.per_split, part);
        };
        constexpr Int<1> _1{};
        constexpr Int<2> _2{};
        constexpr Int<3> _3{};
        constexpr Int<4> _4{};
        constexpr std::true_type split{};
        constexpr std::false_type whole{};
        if (p.streams && p.rows == 16) {
            if (p.cols == 64) stream_rows(_4, _1);
            else if (p.cols == 32) stream_rows(_2, _1);
            else stream_rows(_1, _1);
        } else if (p.streams) {
            if (p.cols == 32) stream_rows(_2, _2);
            else stream_rows(_1, _2);
        } else if (p.rows == 256) {
            if constexpr (!__is_same(T, float)) tile(_2, _4, Int<8>{}, _2, whole);
        } else if (p.cols == 128) {
            if (p.splits > 1) tile(_4, _2, _2, _4, split);
            else if (groups <= 256) tile(_4, _2, _2, _4, whole);
            else tile(_4, _2, _2, _2, whole);
        } else if (p.rows == 128) {
            if (p.splits > 1) tile(_4, _1, _2, _3, split);
            else tile(_4, _1, _2, _3, whole);
        } else {
            if (p.splits > 1) tile(_4, _1, _1, _4, split);
            else tile(_4, _1, _1, _4, whole);
        }
        if (p.splits > 1)
            hipLaunchKernelGGL(product_f8_join_kernel<T>, dim3((unsigned)joins), dim3(256), 0, stream, a, p.splits, part);
        return mq_host::launch_status();
    };
    return type == MQ_FP32 ? run(float{}) : mq_host::with_half_type(type, run);
}
