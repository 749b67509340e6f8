// Product of 8-bit activations and 8-bit weights with scales for each token and
// channel:  Y[m,n] = rn(s_x[m] s_w[n] sum_k Xq[m,k] Wq[n,k] + bias[n]).
//
// The sums run on v_mfma_i32_16x16x64_i8 in exact int32.  Weights are laid out
// once in the instruction's operand order: a block of 64 channels holds, for
// every 64 codes, four pieces of 16 channels x 64 codes, 1 KB each, lane l's 16
// bytes (row l % 16, codes 16 (l / 16) ..) at 16 l.  Row 4 a + b of piece i is
// channel 16 a + 4 i + b of the block: a lane's results of the four pieces are
// 16 neighbouring channels.  Channels past N and codes past K are zero, so
// whatever X holds past K adds nothing.
//
// Two kernels:
//  * tiled: output tiles of 64 x 64 to 256 x 256, both operands through two to
//    four LDS slots of 128 codes, filled by the LDS DMA.  The matrix unit and LDS
//    bound it: 8192 rows of 8192 codes by 28672 channels 1480-1540 us, 2.5-2.6
//    POP/s (65 % of the cycles have a product running);
//  * streaming (few rows): weights go straight to registers, once; the eight
//    waves of a workgroup share out K and add their sums in LDS (integers: in
//    any order).  Reading the weight bounds it: 4096 -> 14336 at one row 10.2 us,
//    5.7 TB/s.
#include "lds_dma.h"
#include "mq_float.h"

#include <algorithm>

namespace mq {

constexpr int kBlock8 = 64;             // channels of a block
constexpr int kPieceK = 64, kPieceBytes = 1024;
constexpr int kStageK = 128;            // codes of a slot; K is padded to a multiple
constexpr int kWaveRows = 32;           // rows of X at most that a wave loads: they span less than 2 GB (streaming kernel: 4)

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
    int y16;                            // rows of Y 16-byte aligned
};

__host__ __device__ __forceinline__ int padded_k8(int K) { return (K + kStageK - 1) / kStageK * kStageK; }

__host__ __device__ __forceinline__ int padded_n8(int N) { return (N + kBlock8 - 1) / kBlock8 * kBlock8; }

// y[c] = s_x s_w sum + bias for 16 channels n .. n + 15 of row m, stored.
template <typename T>
struct Scales16 {
    float w[16], b[16];
    __device__ __forceinline__ Scales16() {}
    __device__ __forceinline__ Scales16(const Product8Args& a, int n) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            w[c] = n + c < a.N ? a.s_w[n + c] : 0.0f;
            b[c] = a.bias && n + c < a.N ? (float)static_cast<const T*>(a.bias)[n + c] : 0.0f;
        }
    }
};
template <typename T>
__device__ __forceinline__ void store_row16(const Product8Args& a, int m, int n, const int (&sum)[16], const Scales16<T>& s) {
    const float sx = a.s_x[m];
    float y[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        y[c] = (float)sum[c] * (sx * s.w[c]);
        if (a.bias) y[c] += s.b[c];
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

// --------------------------------------------------------------------------
// Tiled kernel: WM x WN waves, each 16 MI rows of X by one block of 64 channels.
// --------------------------------------------------------------------------
// A stage is 128 codes: rows of 128 bytes of X (16-byte chunk q of row r at q ^
// (r % 8): reads of 16 rows are free of bank conflicts, and every load of eight
// rows takes whole lines) and 8 KB of W for each block, in order.  One barrier a
// stage, in its middle: it says that the next stage has landed and that this one
// has been read (its second half is in registers by then), and the loads of the
// stage SLOTS on go into its slot.  Loads past the last stage read nothing: they
// keep the number in flight the same throughout.
// SPLIT: workgroup y takes the stages [y, y + 1) per_split and writes its sums,
// int32, to part[y][M][N].
template <typename T, int WM, int WN, int MI, int SLOTS, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN, 2) void product8_tiled_kernel(Product8Args a, int per_split, int* __restrict__ part) {
    constexpr int TM = 16 * MI * WM, TN = kBlock8 * WN, NW = WM * WN;
    constexpr int XL = TM / 8 / NW, WL = TN / 8 / NW;       // 1 KB loads of a wave and stage
    static_assert(XL * NW * 8 == TM && 8 * XL <= kWaveRows && (WL == 2 || WL == 4), "whole loads");
    __shared__ __attribute__((aligned(16))) struct {
        uint8_t x[SLOTS][TM * kStageK];
        uint8_t w[SLOTS][TN * kStageK];
    } L;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN, lrow = lane & 15, lq = lane >> 4;
    const int kp = padded_k8(a.K), blocks = (a.N + kBlock8 - 1) / kBlock8;
    const int first = SPLIT ? blockIdx.y * per_split : 0, stages = SPLIT ? min(per_split, kp / kStageK - first) : kp / kStageK;
    int tm, tn;
    tile_coords(blockIdx.x, (a.M + TM - 1) / TM, (a.N + TN - 1) / TN, tm, tn);
    const int m0 = tm * TM, b0 = tn * WN;

    // X from the wave's own first row on: what a resource spans stays below 2 GB (the host sees to it), and rows past M
    // are past its end
    const int mw = m0 + 8 * XL * wave, rows = min(8 * XL, a.M - mw);
    const i32x4 rx = make_desc(a.X + mw * a.ldx, rows > 0 ? (uint32_t)((rows - 1) * a.ldx + (a.K + 15) / 16 * 16) : 0u);
    const i32x4 rw = make_desc(a.W + (int64_t)b0 * kp * kBlock8, (uint32_t)min(WN, blocks - b0) * (uint32_t)(kp * kBlock8));
    const uint32_t ldx = (uint32_t)a.ldx;
    const uint32_t vx = (uint32_t)(lane >> 3) * ldx + (uint32_t)(((lane & 7) ^ (lane >> 3)) << 4);
    const uint32_t vw = (uint32_t)lane * 16;
    uint32_t sx = (uint32_t)(first * kStageK);
    uint32_t sw = (uint32_t)(WL * wave / 8) * (uint32_t)(kp * kBlock8) + (uint32_t)(WL * wave % 8) * 1024u + (uint32_t)(first * 8192);
    int to_load = stages;
    auto issue = [&](int slot) {
        const bool there = to_load-- > 0;
#pragma unroll
        for (int k = 0; k < XL; ++k)
            dma16s(rx, lds_addr(L.x) + (uint32_t)(slot * (TM * kStageK) + (XL * wave + k) * 1024), vx, there ? sx + (uint32_t)(8 * k) * ldx : kPastEnd);
        const uint32_t dst = lds_addr(L.w) + (uint32_t)(slot * (TN * kStageK) + WL * wave * 1024);
        if constexpr (WL == 4) dma16x4(rw, dst, vw, there ? sw : kPastEnd);
        else dma16x2(rw, dst, vw, there ? sw : kPastEnd);
        sx += kStageK;
        sw += 8192;
    };
    // the stage after the one being read has landed: those of SLOTS - 2 more are in flight
    auto wait_and_sync = [] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((SLOTS - 2) * (XL + WL)) : "memory"); };
    const uint32_t xa = lds_addr(L.x) + (uint32_t)(wm * 16 * MI + lrow) * kStageK + (uint32_t)((lq ^ (lrow & 7)) << 4);
    const uint32_t wa = lds_addr(L.w) + (uint32_t)(wn * 8192 + lane * 16);
    struct Half {
        i32x4 w[4], x[MI];
    };
    auto read = [&](Half& h, int slot, int kk) {
        const uint32_t xs = (kk ? xa ^ 64u : xa) + (uint32_t)(slot * (TM * kStageK)), ws = wa + (uint32_t)(slot * (TN * kStageK));
#pragma unroll
        for (int i = 0; i < 4; ++i) h.w[i] = __builtin_bit_cast(i32x4, lds_read16(ws + kk * 4096 + i * 1024));
#pragma unroll
        for (int j = 0; j < MI; ++j) h.x[j] = __builtin_bit_cast(i32x4, lds_read16(xs + j * 2048));
    };
    i32x4 acc[4][MI] = {};
    auto multiply = [&](const Half& h) {
#pragma unroll
        for (int j = 0; j < MI; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(h.w[i], h.x[j], acc[i][j], 0, 0, 0);
    };

    for (int s = 0; s < SLOTS; ++s) issue(s);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((SLOTS - 1) * (XL + WL)) : "memory");
    Half h0, h1;
    read(h0, 0, 0);
    int slot = 0;
    for (int s = 0; s < stages; ++s) {
        const int next = slot + 1 == SLOTS ? 0 : slot + 1;
        read(h1, slot, 1);
        multiply(h0);
        wait_and_sync();
        issue(slot);
        read(h0, next, 0);                                  // past the last stage: zeros, unused
        multiply(h1);
        slot = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // nothing may write LDS after the workgroup has gone

    const int n = (b0 + wn) * kBlock8 + 16 * lq;
    if (n >= a.N) return;
    const Scales16<T> scales = SPLIT ? Scales16<T>{} : Scales16<T>(a, n);
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        const int m = m0 + wm * 16 * MI + 16 * j + lrow;
        if (m >= a.M) break;
        if constexpr (SPLIT) {
            int* p = part + ((int64_t)blockIdx.y * a.M + m) * padded_n8(a.N) + n;
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<i32x4*>(p + 4 * i) = acc[i][j];
        } else {
            int sum[16];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[4 * i + r] = acc[i][j][r];
            store_row16(a, m, n, sum, scales);
        }
    }
}

// Sums of the splits -> Y, 16 channels a thread.
template <typename T>
__global__ __launch_bounds__(256) void product8_join_kernel(Product8Args a, int splits, const int* __restrict__ part) {
    const int np = padded_n8(a.N), per = np / 16;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.M * per) return;
    const int m = (int)(i / per), n = (int)(i % per) * 16;
    if (n >= a.N) return;
    i32x4 sum[4] = {};
    for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] += *reinterpret_cast<const i32x4*>(part + ((int64_t)s * a.M + m) * np + n + 4 * c);
    int flat[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) flat[c] = sum[c / 4][c % 4];
    store_row16(a, m, n, flat, Scales16<T>(a, n));
}

// --------------------------------------------------------------------------
// Streaming kernel: P pieces of a block and all rows (16 MT) a workgroup.
// --------------------------------------------------------------------------
constexpr int kStreamWaves = 8;
template <typename T, int P, int MT>
__global__ __launch_bounds__(64 * kStreamWaves) void product8_stream_kernel(Product8Args a) {
    static_assert(16 * MT <= kWaveRows, "rows span less than 4 GB");
    constexpr int U = P + MT >= 8 ? 1 : 12 / (P + MT);       // pieces of K in flight, twice
    __shared__ int sums[16 * MT][16 * P + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lrow = lane & 15, lq = lane >> 4;
    const int kp = padded_k8(a.K), pieces = kp / kPieceK;
    const int block = blockIdx.x / (4 / P), i0 = blockIdx.x % (4 / P) * P;
    const uint8_t* w = a.W + (int64_t)block * kp * kBlock8 + i0 * kPieceBytes + 16 * lane;
    uint32_t x[MT];                                         // rows, from X: less than 4 GB (the host sees to it)
#pragma unroll
    for (int j = 0; j < MT; ++j) x[j] = (uint32_t)min(16 * j + lrow, a.M - 1) * (uint32_t)a.ldx;
    const int last = (a.K - 1) / 16 * 16;                   // first code of a row's last 16
    for (int i = threadIdx.x; i < 16 * MT * (16 * P + 1); i += 64 * kStreamWaves) (&sums[0][0])[i] = 0;

    struct Batch {
        i32x4 w[U][P], x[U][MT];
    };
    auto load = [&](Batch& b, int p0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = min(p0 + u * kStreamWaves, pieces - 1);
#pragma unroll
            for (int i = 0; i < P; ++i) b.w[u][i] = *reinterpret_cast<const i32x4*>(w + (int64_t)p * 4096 + i * kPieceBytes);
#pragma unroll
            for (int j = 0; j < MT; ++j) b.x[u][j] = *reinterpret_cast<const i32x4*>(a.X + (x[j] + (uint32_t)min(p * kPieceK + 16 * lq, last)));
        }
    };
    i32x4 acc[P][MT] = {};
    auto multiply = [&](const Batch& b, int p0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u * kStreamWaves >= pieces) break;
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i < P; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b.w[u][i], b.x[u][j], acc[i][j], 0, 0, 0);
        }
    };
    Batch b0, b1;
    constexpr int step = U * kStreamWaves;
    load(b0, wave);
    for (int p = wave; p < pieces; p += 2 * step) {
        if (p + step < pieces) load(b1, p + step);
        multiply(b0, p);
        if (p + step >= pieces) break;
        if (p + 2 * step < pieces) load(b0, p + 2 * step);
        multiply(b1, p + step);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) atomicAdd(&sums[16 * j + lrow][(4 * lq) * P + 4 * i + r], acc[i][j][r]);
    __syncthreads();
    // columns 4 P a + 4 i + b are channels 16 a + 4 (i0 + i) + b
    for (int e = threadIdx.x; e < 16 * P * min(a.M, 16 * MT); e += 64 * kStreamWaves) {
        const int m = e / (16 * P), c = e % (16 * P);
        const int n = block * kBlock8 + c / (4 * P) * 16 + 4 * i0 + c % (4 * P);
        if (n >= a.N) continue;
        float y = (float)sums[m][c] * (a.s_x[m] * a.s_w[n]);
        if (a.bias) y += (float)static_cast<const T*>(a.bias)[n];
        static_cast<T*>(a.Y)[m * a.ldy + n] = (T)y;
    }
}

// Per-channel INT8 weights, once for a weight (4096 channels of 14336 codes: quantised in 733 us, laid out in 396, read
// back in 174; few and narrow loads bound them): s = max|w| / 127 (fp32), q = clamp(round_half_even(w / s), -127, 127),
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

// channel of row r of piece i of its block
__device__ __forceinline__ int channel8(int i, int r) { return 16 * (r / 4) + 4 * i + r % 4; }

template <typename From>
__global__ __launch_bounds__(1024) void pack_weight8_kernel(From from, int N, int K, uint8_t* __restrict__ Wq) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int pieces = padded_k8(K) / kPieceK * 4;
    const int row0 = blockIdx.x * kBlock8;
    __shared__ float scale[kBlock8];
    if constexpr (__is_same(From, FromFloat)) {
        for (int r = wave; r < kBlock8; r += waves) {
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
    for (int p = wave; p < pieces; p += waves) {
        const int k0 = p / 4 * kPieceK + 16 * (lane >> 4), c = channel8(p % 4, lane & 15), row = row0 + c;
        uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            int q = 0;
            if (row < N && k0 + e < K) {
                if constexpr (__is_same(From, FromFloat)) {
                    const float s = scale[c];
                    const float f = rintf(from.W[row * from.ldw + k0 + e] / s);
                    // a row that is not finite: codes 0 (its scale is not finite either)
                    q = s > 0.0f && __float_as_uint(s) < kFloatInf ? (int)__builtin_amdgcn_fmed3f(f, -127.0f, 127.0f) : 0;
                } else {
                    q = from.W[row * from.ldw + k0 + e];
                }
            }
            b[e / 4] |= ((uint32_t)q & 0xFFu) << (8 * (e % 4));
        }
        *reinterpret_cast<uint4*>(Wq + ((int64_t)blockIdx.x * pieces + p) * kPieceBytes + 16 * lane) = make_uint4(b[0], b[1], b[2], b[3]);
    }
}

__global__ __launch_bounds__(256) void unpack_weight8_kernel(const uint8_t* __restrict__ Wq, int N, int K,
                                                             int8_t* __restrict__ Wc, int64_t ldw) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)N * K; i += (int64_t)gridDim.x * 256) {
        const int n = (int)(i / K), k = (int)(i % K), c = n % kBlock8;
        const int row = c / 16 * 4 + c % 4, piece = c % 16 / 4;     // channel8's inverse
        const int64_t at = ((int64_t)(n / kBlock8) * (padded_k8(K) / kPieceK) + k / kPieceK) * 4 + piece;
        Wc[n * ldw + k] = (int8_t)Wq[at * kPieceBytes + 16 * (row + 16 * (k % kPieceK / 16)) + k % 16];
    }
}

static bool shape8_ok(int N, int K) { return N >= 1 && N <= (1 << 24) && K >= 1 && K <= MQ_W8A8_MAX_K; }

// ---------------------------------------------------------------- host side --
// Which kernel takes a product.  Up to 16 rows, and up to 32 where the weight is
// small, the streaming kernel (K = N = 4096: M = 16 5.9 us, M = 32 7.9; the 64 x
// 64 tiles 9.7 and 9.8; 4096 -> 14336 at M = 32 14.4 and 13.4).  Beyond, of four
// tiles and one, two or four splits of K the one with the least estimated time:
// stages of 128 codes by the time of one (a workgroup alone on its CU waits for
// memory; more of them share the CU), or W at the rate that the tiles reach,
// whichever is longer; and what writing, reading and joining a split's sums
// takes.  The estimates are within a fifth of what was measured (K = 14336, N =
// 4096: M = 64 in four splits 19.9 us, unsplit 34.5; M = 512 by 128 x 64 51.2,
// 64 x 64 56.5, 128 x 128 91; K = N = 8192 at M = 1157 by 256 x 256 97, 128 x 128
// 114; 5120 -> 25599 at M = 77 by 64 x 64 44.5, 128 x 128 42.8), but for few rows of
// 128 x 64, whose loads of W reach less than the rate assumed (the last by 128 x 64
// 38.1 us, estimated at 28.5).
struct Tile8 {
    int rows, cols;
    double alone, share;                // us of a stage: one workgroup a CU, and of each of several
    bool splits;
};
constexpr Tile8 kTiles8[4] = {
    {64, 64, 0.26, 0.25, true},
    {128, 64, 0.45, 0.345, true},
    {128, 128, 0.95, 0.60, false},
    {256, 256, 1.60, 1.60, false},
};
struct Plan8 {
    int rows, cols;                     // of a workgroup's tile; cols of the streaming kernel: 16 P
    bool streams;
    int splits, per_split;              // stages of a split
};
static Plan8 plan8(int M, int N, int K) {
    const int blocks = (N + kBlock8 - 1) / kBlock8, stages = padded_k8(K) / kStageK;
    if (M <= 16 || (M <= 32 && blocks < 192 && K <= 8192)) {
        // pieces of 16 channels a workgroup: four where that still makes three workgroups for four CUs (4096 -> 14336
        // 11.6 us, two 13.1), two where K is short and they fill half the CUs (K = N = 4096 5.7, one 6.6; 14336 ->
        // 4096 13.1 and 11.8), else one
        const int p = blocks >= 192 ? 4 : blocks >= 64 && K <= 8192 ? 2 : 1;
        return Plan8{M <= 16 ? 16 : 32, 16 * p, true, 1, stages};
    }
    Plan8 best{};
    double least = 0.0;
    for (const Tile8& t : kTiles8)
        for (int splits = 1; splits <= (t.splits ? 4 : 1); splits *= 2) {
            if (splits > 1 && stages < 8 * splits) break;
            const int64_t groups = (int64_t)((M + t.rows - 1) / t.rows) * ((N + t.cols - 1) / t.cols) * splits;
            const int64_t a_cu = (groups + 255) / 256;
            const int per = (stages + splits - 1) / splits;
            const double compute = per * std::max(t.alone, a_cu * t.share), memory = (double)N * K / 4.6e6;
            const double join = splits == 1 ? 0.0 : 7.0 + (double)M * N * 4 * (splits + 1) / 5.0e6;
            const double us = std::max(compute, memory) + join;
            if (least == 0.0 || us < least) {
                least = us;
                best = Plan8{t.rows, t.cols, false, (stages + per - 1) / per, per};
            }
        }
    return best;
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_weight8_bytes(int N, int K) {
    if (!shape8_ok(N, K)) return 0;
    return (size_t)((N + kBlock8 - 1) / kBlock8) * kBlock8 * padded_k8(K);
}

extern "C" mq_status mq_quantize_weight8(const float* W, int N, int K, int ldw, uint8_t* Wq8, float* s_w, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!W || !Wq8 || !s_w) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(W, 4) || !mq_host::aligned(Wq8, 16) || !mq_host::aligned(s_w, 4)) return MQ_ERR_MISALIGNED;
    hipLaunchKernelGGL(pack_weight8_kernel<FromFloat>, dim3((N + kBlock8 - 1) / kBlock8), dim3(1024), 0, stream, FromFloat{W, ldw, s_w}, N, K, Wq8);
    return mq_host::launch_status();
}

extern "C" mq_status mq_repack_weight8(int N, int K, const int8_t* Wc, int ldw, uint8_t* Wq8, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Wc || !Wq8) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Wq8, 16)) return MQ_ERR_MISALIGNED;
    hipLaunchKernelGGL(pack_weight8_kernel<FromCodes>, dim3((N + kBlock8 - 1) / kBlock8), dim3(1024), 0, stream, FromCodes{Wc, ldw}, N, K, Wq8);
    return mq_host::launch_status();
}

extern "C" mq_status mq_unpack_weight8(int N, int K, const uint8_t* Wq8, int8_t* Wc, int ldw, hipStream_t stream) {
    if (N < 0 || K < 0) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K) || ldw < K) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Wc || !Wq8) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Wq8, 16)) return MQ_ERR_MISALIGNED;
    // a launch has less than 2^32 threads; the rest of the codes come in further turns
    const int64_t blocks = std::min<int64_t>(((int64_t)N * K + 255) / 256, 1 << 22);
    hipLaunchKernelGGL(unpack_weight8_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, Wq8, N, K, Wc, ldw);
    return mq_host::launch_status();
}

extern "C" size_t mq_gemm_w8a8_workspace_size(int M, int N, int K) {
    if (M < 1 || M > (1 << 24) || !shape8_ok(N, K)) return 0;
    const Plan8 p = plan8(M, N, K);
    return p.splits == 1 ? 0 : (size_t)p.splits * M * padded_n8(N) * sizeof(int);
}

extern "C" mq_status mq_gemm_w8a8_tile(int M, int N, int K, int* rows, int* cols, int* splits) {
    if (!rows || !cols || !splits || M < 1 || M > (1 << 24)) return MQ_ERR_INVALID_ARG;
    if (!shape8_ok(N, K)) return MQ_ERR_UNSUPPORTED_SHAPE;
    const Plan8 p = plan8(M, N, K);
    *rows = p.rows;
    *cols = p.cols;
    *splits = p.splits;
    return MQ_OK;
}

extern "C" mq_status mq_gemm_w8a8(int M, int N, int K, const int8_t* Xq8, int ldx, const float* s_x, const uint8_t* Wq8,
                                  const float* s_w, mq_dtype type, const void* bias, void* Y, int ldy, void* workspace,
                                  size_t ws_bytes, hipStream_t stream) {
    if (M < 0 || N < 0 || K < 0 || (!mq_host::is_half_type(type) && type != MQ_FP32)) return MQ_ERR_INVALID_ARG;
    if (M > (1 << 24) || !shape8_ok(N, K) || ldx < (K + 15) / 16 * 16 || ldx % 16 != 0 || ldy < N) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (M == 0) return MQ_OK;
    const Plan8 p = plan8(M, N, K);
    const int64_t groups = p.streams ? (int64_t)((N + kBlock8 - 1) / kBlock8) * (kBlock8 / p.cols)
                                     : (int64_t)((M + p.rows - 1) / p.rows) * ((N + p.cols - 1) / p.cols);
    const int64_t joins = p.splits > 1 ? ((int64_t)M * (padded_n8(N) / 16) + 255) / 256 : 0;
    if (!mq_host::launch_holds(groups, 512) || !mq_host::launch_holds(joins, 256)) return MQ_ERR_UNSUPPORTED_SHAPE;
    // offsets within a wave's rows: 32 bits, of which the tiled kernels' loads past the end take the upper half
    if ((int64_t)(std::min(M, kWaveRows) - 1) * ldx + (K + 15) / 16 * 16 > (p.streams ? (int64_t)UINT32_MAX : INT32_MAX))
        return MQ_ERR_UNSUPPORTED_SHAPE;
    if (!Xq8 || !s_x || !Wq8 || !s_w || !Y) return MQ_ERR_INVALID_ARG;
    const size_t size = type == MQ_FP32 ? 4 : 2;
    if (!mq_host::aligned(Xq8, 16) || !mq_host::aligned(Wq8, 16) || !mq_host::aligned(s_x, 4) || !mq_host::aligned(s_w, 4) ||
        !mq_host::aligned(bias, size) || !mq_host::aligned(Y, size) || !mq_host::aligned(workspace, 16))
        return MQ_ERR_MISALIGNED;
    const size_t need = mq_gemm_w8a8_workspace_size(M, N, K);
    if (need > 0 && (!workspace || ws_bytes < need)) return MQ_ERR_WORKSPACE;
    const Product8Args a{M, N, K, reinterpret_cast<const uint8_t*>(Xq8), ldx, s_x, Wq8, s_w, bias, Y, ldy,
                         mq_host::aligned(Y, 16) && ldy * size % 16 == 0};
    auto run = [&](auto z) {
        using T = decltype(z);
        int* part = static_cast<int*>(workspace);
        auto stream_rows = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * kStreamWaves), 0, stream, a); };
        auto tile = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups, p.splits), dim3(threads), 0, stream, a, p.per_split, part);
        };
        if (p.streams && p.rows == 16) {
            if (p.cols == 64) stream_rows(product8_stream_kernel<T, 4, 1>);
            else if (p.cols == 32) stream_rows(product8_stream_kernel<T, 2, 1>);
            else stream_rows(product8_stream_kernel<T, 1, 1>);
        } else if (p.streams) {
            if (p.cols == 32) stream_rows(product8_stream_kernel<T, 2, 2>);
            else stream_rows(product8_stream_kernel<T, 1, 2>);
        } else if (p.rows == 256) {
            tile(product8_tiled_kernel<T, 2, 4, 8, 2, false>, 512);
        } else if (p.cols == 128) {
            tile(product8_tiled_kernel<T, 4, 2, 2, 2, false>, 512);
        } else if (p.rows == 128) {
            if (p.splits > 1) tile(product8_tiled_kernel<T, 4, 1, 2, 3, true>, 256);
            else tile(product8_tiled_kernel<T, 4, 1, 2, 3, false>, 256);
        } else {
            if (p.splits > 1) tile(product8_tiled_kernel<T, 4, 1, 1, 4, true>, 256);
            else tile(product8_tiled_kernel<T, 4, 1, 1, 4, false>, 256);
        }
        if (p.splits > 1) {
            hipLaunchKernelGGL(product8_join_kernel<T>, dim3((unsigned)joins), dim3(256), 0, stream, a, p.splits, part);
        }
        return mq_host::launch_status();
    };
    return type == MQ_FP32 ? run(float{}) : mq_host::with_half_type(type, run);
}
