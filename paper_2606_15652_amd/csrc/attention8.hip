// Attention over the paged 8-bit cache.
//
//   o = sum_t p_t v_t / sum_t p_t,   p_t = exp(scale q.k_t),
//   k_t = 2^ek nk_t,  v_t = 2^ev nv_t   (n: e4m3 codes; ek, ev: of the token's block of 32 and head)
//
// Columns are the queries of one sequence and key head: position qi and head hg
// of the group at column qi group + hg.  A wave takes blocks of 32 tokens for 16
// NT columns: codes go from memory to registers in operand order, become fp16
// there (exactly), and the matrix instruction's two products of a block are
//   scores  S = K Q^T  (tokens x columns),   O += V^T W  (channels x columns),
// the lanes' scores being, in place, the operand W of the second.  Scales act on
// scores and weights, D times fewer than codes.
//
// With s = log2(e) scale q.k and, for each column, whole numbers m (running
// maximum of s, by up to 2^kSlack too low) and J (the same of s - m + ev):
//   p = 2^(s - m),  l = sum p,   w = p 2^(ev - J + kLift) in fp16,  O = sum w nv,
//   o = 2^(J - kLift) O / l.
// Only differences of s enter, so scores may be of any size, and a block of large
// values that a column gives no weight takes nothing from the others.  Moving m or
// J multiplies by powers of two.
//
// Two kernels: for few columns, whose waves share out the tokens and load codes straight
// to registers, memory bounds it (two contexts of up to 131072 tokens 86 us, 5.5 TB/s; 64 of up
// to 8191 107 us, 5.2; with the join 90 and 115); for many, whose waves share the tokens' codes in
// LDS, the vector unit (8192 queries over 8192 tokens 575 to 590 us as the card's clock goes, 930 to
// 955 TFLOP/s; four ragged prompts of up to 2047 queries 210 to 222 us with the order of their work).
#include "kv8.h"

#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

namespace mq {

mq_status check_cache8(const mq_kv8_cache* c);
Cache8 device_cache8(const mq_kv8_cache* c);

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;          // weights up to 2^kSlack before a maximum moves
constexpr float kLift = 7.0f;           // and as operands up to 2^(kSlack + kLift) < 65504, down to 2^-24
constexpr float kLowest = -FLT_MAX;     // m of a column that has seen nothing
constexpr float kNone = -1e30f;         // and its J: below any that a token gives

struct Attn8Args {
    Cache8 c;
    const void* q;
    void* o;
    int64_t q_token, q_head, o_token, o_head;
    const int32_t *table, *lens, *starts;
    int table_pages, tokens, group, max_q, causal;
    float scale;                        // times log2(e)
    int64_t max_kv;
    int chunk, chunks;                  // tokens that a workgroup takes, and chunks of the longest sequence
    const int2* order;                  // sequence and block of columns of each workgroup, or null
    float* part;                        // sums (sums_at): O[D], then m, J, l in `stats`
    float* stats;
};

// Where the sums of a column are: entries are the order's blocks or else the sequences, of `cols` columns each (a block's, or
// max_q queries'), by key head, chunk and column.
__device__ __forceinline__ int64_t sums_at(const Attn8Args& a, int entry_head, int chunk, int cols, int col) {
    return ((int64_t)entry_head * a.chunks + chunk) * cols + col;
}

// One sequence's lengths, as the arguments bound them.
struct Sequence8 {
    int64_t len;                        // tokens
    int first, queries;                 // rows of Q; queries that are computed
    int64_t shift;                      // query i is at token i + shift
    __device__ __forceinline__ Sequence8(const Attn8Args& a, int b) {
        const int64_t n = a.lens[b];
        len = n < 0 ? 0 : n < a.max_kv ? n : a.max_kv;
        first = a.starts ? a.starts[b] : b;
        const int count = a.starts ? a.starts[b + 1] - first : 1;
        shift = n - count;
        queries = min(count, a.max_q);
    }
    // tokens that query i sees: those before this
    __device__ __forceinline__ int64_t seen(const Attn8Args& a, int i) const {
        if (!a.causal) return len;
        const int64_t n = shift + i + 1;
        return n < 0 ? 0 : n < len ? n : len;
    }
};

// A product that is rounded before anything is taken from it.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// The largest of v over the lanes l, l ^ 16, l ^ 32, l ^ 48 (a column's).
__device__ __forceinline__ float column_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// The columns of one wave: their queries as operands, and what has been summed up for them.
template <typename T, int D, int NT>
struct Columns8 {
    static constexpr int STEPS = D / 32, TILES = D / 16;    // of 32 channels of keys, of 16 channels of values
    // fp16 results show one rounding of the weights to fp16 (2.9e-4 of their norm off, 2.1e-4 of it their own rounding): the rest
    // of a weight is a second operand (single tokens take as long, four ragged prompts 289 us instead of 226); in bf16 it does not
    // show.
    static constexpr int WEIGHTS = __is_same(T, _Float16) ? 2 : 1;
    f16x8 q[NT][STEPS];
    int by[NT];                                             // queries as operands are 2^by of what they are
    int sees[NT];                                           // tokens that the column sees
    int least, most;                                        // over the columns that are there
    f32x4 o[TILES][NT];
    float m[NT], jj[NT], l[NT];

    __device__ __forceinline__ Columns8(const Attn8Args& a, const Sequence8& seq, int head, int col0) {
        const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4, columns = seq.queries * a.group;
        least = (int)seq.len;
        most = 0;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int c = col0 + 16 * n + col;
            const bool there = c < columns;
            const int qi = there ? c / a.group : 0, hg = there ? c % a.group : 0;
            const int64_t row = (int64_t)seq.first + qi;
            const bool has = there && row >= 0 && row < a.tokens;
            sees[n] = has ? (int)seq.seen(a, qi) : 0;
            const T* p = static_cast<const T*>(a.q) + (has ? row * a.q_token + (int64_t)(head * a.group + hg) * a.q_head : 0) + 16 * quarter;
            f32x8 x[STEPS];
            uint32_t big = 0;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                x[s] = has ? load8(p + s / 2 * 64 + s % 2 * 8) : f32x8{};
#pragma unroll
                for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint(x[s][j]) & 0x7FFFFFFFu);
            }
            big = max(big, (uint32_t)__shfl_xor((int)big, 16));
            big = max(big, (uint32_t)__shfl_xor((int)big, 32));
            // bf16: by a power of two so that the largest is in [2^14, 2^15).  A query that is not finite is NaN throughout.
            by[n] = __is_same(T, __bf16) && big ? 141 - (int)(big >> 23) : 0;
            const bool bad = big >= kFloatInf;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) q[n][s][j] = bad ? (_Float16)__builtin_nanf("") : (_Float16)ldexpf(x[s][j], by[n]);
            least = has && sees[n] < least ? sees[n] : least;
            most = max(most, sees[n]);
            m[n] = kLowest;
            jj[n] = kNone;
            l[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < TILES; ++i) o[i][n] = f32x4{};
        }
#pragma unroll
        for (int k = 32; k >= 1; k >>= 1) {
            least = min(least, __shfl_xor(least, k));
            most = max(most, __shfl_xor(most, k));
        }
        least = __builtin_amdgcn_readfirstlane(least);
        most = __builtin_amdgcn_readfirstlane(most);
    }

    // One block of 32 tokens: key(t, s) and value(i) give the operands of its two tiles of tokens, and of its channels.  A block
    // that no page holds (ve < 0) is seen by none; it is not left out, as a branch around the products makes the compiler
    // copy the accumulators.
    template <typename K, typename V>
    __device__ __forceinline__ void take(float scale, int block, int ke, int ve, K&& key, V&& value) {
        const int quarter = (threadIdx.x & 63) >> 4;
        f32x4 s[NT][2] = {};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const f16x8 k = key(t, i);
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[n][i], s[n][t], 0, 0, 0);
            }
        // the two products and what is between them each load their own operands: loaded ahead of that they cost registers, and with
        // them a wave (8 contexts of 4096 tokens by 2048 queries 1110 us, 880)
        __builtin_amdgcn_sched_barrier(0);
        const float ev = (float)(ve - 127);
        float c[NT], e[NT];
        bool moves = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // (by both powers at once: by one of them it may be below fp32's normal numbers); not 0: hidden scores stay -infinity
            c[n] = fminf(fmaxf(ldexpf(scale, ke - 127 - by[n]), FLT_MIN), FLT_MAX);
            if ((block + 1) * kBlockTokens > least || ve < 0) {
                const int left = ve < 0 ? 0 : sees[n] - block * kBlockTokens - 4 * quarter;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * t + r >= left) s[n][t][r] = -INFINITY;
            }
            e[n] = ev - jj[n] + kLift;
            float high = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) high = fmaxf(high, s[n][j / 4][j % 4]);
            // p <= 2^kSlack, w <= 2^(kSlack + kLift)
            moves |= rounded_product(high, c[n]) - m[n] > kSlack + fminf(kLift - e[n], 0.0f);
        }
        if (__ballot(moves)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float high = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) high = fmaxf(high, s[n][j / 4][j % 4]);
                const float top = rounded_product(column_max(high), c[n]), was = m[n];
                const bool up = top > was + kSlack || ceilf(top - was) + ev > jj[n] + kSlack;
                m[n] = up ? fmaxf(was, ceilf(top)) : was;
                const float old = jj[n] + (was - m[n]);     // J of what O holds, by the new m
                jj[n] = up ? fmaxf(fmaxf(old, ceilf(top - m[n]) + ev), kNone) : old;
                l[n] *= __builtin_amdgcn_exp2f(was - m[n]);
                const float by = __builtin_amdgcn_exp2f(old - jj[n]);
#pragma unroll
                for (int i = 0; i < TILES; ++i) o[i][n] *= by;
                e[n] = ev - jj[n] + kLift;
            }
        }
        // Scores as they are usual: the product less m and the weights' exponent in one operation, and p from w.  Not so in a
        // column where m passes 2^20 (m is a rounded product: an exact one may differ from it by more than any weight
        // allows), or where w may lose what p still has.
        f16x8 w[NT][WEIGHTS];
        auto put = [&](int n, int j, float p) {
            w[n][0][j] = (_Float16)p;
            if constexpr (WEIGHTS == 2) w[n][1][j] = (_Float16)(p - (float)w[n][0][j]);
        };
        auto usual = [&](int n) {
            const float from = e[n] - m[n];
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][j / 4][j % 4], c[n], from));
                sum += p;
                put(n, j, p);
            }
            l[n] = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(-e[n]), l[n]);
        };
        auto is_far = [&](int n) { return !(fabsf(m[n]) < 0x1p20f) || e[n] < -60.0f; };
        bool far = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) far |= is_far(n);
        if (__ballot(far)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (is_far(n)) {
                    const int by = (int)fminf(e[n], 1000.0f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float p = __builtin_amdgcn_exp2f(rounded_product(s[n][j / 4][j % 4], c[n]) - m[n]);
                        l[n] += p;
                        put(n, j, ldexpf(p, by));
                    }
                } else {
                    usual(n);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) usual(n);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const f16x8 v = value(i);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < WEIGHTS; ++k) o[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[n][k], o[i][n], 0, 0, 0);
        }
    }

    __device__ __forceinline__ void sum_up() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
        }
    }
};

// Where a column's result goes: as values, or where chunks share the column as sums.
template <typename T, int D>
struct Target8 {
    T* out;
    float *sum, *stat;
    __device__ __forceinline__ Target8(const Attn8Args& a, const Sequence8& seq, int head, int c, int entry_cols, int entry_col, bool direct) {
        out = nullptr;
        sum = stat = nullptr;
        const int64_t row = (int64_t)seq.first + c / a.group;
        if (row < 0 || row >= a.tokens) return;
        if (direct) {
            out = static_cast<T*>(a.o) + row * a.o_token + (int64_t)(head * a.group + c % a.group) * a.o_head;
        } else {
            const int64_t at = sums_at(a, blockIdx.x, blockIdx.z, entry_cols, entry_col);
            sum = a.part + at * D;
            stat = a.stats + 3 * at;
        }
    }
    // four channels ch ..
    __device__ __forceinline__ void store(int ch, f32x4 o, float m, float j, float l) const {
        if (out) {
            typedef T t4 __attribute__((ext_vector_type(4)));
            f32x4 y;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = l == 0.0f ? 0.0f : ldexpf(o[r] / l, (int)fmaxf(j - kLift, -1000.0f));
            *reinterpret_cast<t4*>(out + ch) = __builtin_convertvector(y, t4);
        } else if (sum) {
            *reinterpret_cast<f32x4*>(sum + ch) = o;
            if (ch == 0) {
                stat[0] = m;
                stat[1] = j;
                stat[2] = l;
            }
        }
    }
};

// What a workgroup takes: `cols` columns of a sequence and key head, and a chunk of the tokens that they see.
struct Part8 {
    int b, head, first_col, columns, chunks, from, until;
    bool empty;
    __device__ __forceinline__ Part8(const Attn8Args& a, int cols) {
        const int unit = blockIdx.x / a.c.heads;
        head = blockIdx.x % a.c.heads;
        const int2 item = a.order ? a.order[unit] : make_int2(unit, (int)(gridDim.y - 1 - blockIdx.y));     // the longest first
        b = item.x;
        empty = b < 0;
        if (empty) return;
        const Sequence8 seq(a, b);
        columns = seq.queries * a.group;
        first_col = item.y * cols;
        empty = first_col >= columns;
        if (empty) return;
        const int seen = (int)seq.seen(a, (min(first_col + cols, columns) - 1) / a.group);
        chunks = max(1, (int)(((int64_t)seen + a.chunk - 1) / a.chunk));
        empty = (int)blockIdx.z >= chunks;
        from = (int)blockIdx.z * a.chunk;                   // (below `seen` where it is not empty)
        until = (int)min((int64_t)from + a.chunk, (int64_t)seen);
    }
};

// Blocks of `cols` columns of all sequences, those that see the most tokens first (of the same 1024th in any order): the last
// ones to begin are then the shortest.  `most` entries; those behind the last block are -1.
__global__ __launch_bounds__(1024) void attention8_order_kernel(Attn8Args a, int sequences, int cols, int most, int2* __restrict__ order) {
    __shared__ uint32_t first[1024], sums[16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    first[t] = 0;
    __syncthreads();
    auto for_blocks = [&](auto&& f) {
        for (int b = wave; b < sequences; b += 16) {
            const Sequence8 seq(a, b);
            const int columns = seq.queries * a.group;
            for (int k = lane; k * cols < columns; k += 64) {
                const int64_t seen = seq.seen(a, (min((k + 1) * cols, columns) - 1) / a.group);
                f(b, k, 1023 - (int)(seen * 1024 / (a.max_kv + 1)));
            }
        }
    };
    for_blocks([&](int, int, int bin) { atomicAdd(&first[bin], 1u); });
    __syncthreads();
    const uint32_t mine = first[t];
    uint32_t v = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t o = __shfl_up(v, m);
        if (lane >= m) v += o;
    }
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) v += sums[w];
        all += sums[w];
    }
    first[t] = v - mine;
    __syncthreads();
    for_blocks([&](int b, int k, int bin) {
        const uint32_t at = atomicAdd(&first[bin], 1u);
        if (at < (uint32_t)most) order[at] = make_int2(b, k);
    });
    for (int i = (int)all + t; i < most; i += 1024) order[i] = make_int2(-1, 0);
}

// Few columns: the waves share out the tokens (WT of them; blocks in turn), 4 / WT take 16 NT columns of their own.  Codes go
// from memory to registers, a block ahead.
template <typename T, int D, int NT, int WT>
__global__ __launch_bounds__(256, 2) void attention8_kernel(Attn8Args a) {
    constexpr int COLS = 16 * NT, WC = 4 / WT, PIECES = D / 32, TILES = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wt = wave % WT, wc = wave / WT, col = lane & 15, quarter = lane >> 4;
    const Part8 part(a, WC * COLS);
    if (part.empty) return;
    const Sequence8 seq(a, part.b);
    Columns8<T, D, NT> cols(a, seq, part.head, part.first_col + wc * COLS);

    const int32_t* table = a.table + (int64_t)part.b * a.table_pages;
    struct Block {
        uint4 k[PIECES], v[PIECES];
        int ke, ve;                                         // ve < 0: no page holds it
    };
    auto load = [&](Block& x, int block) {
        const int64_t row = block_row8(a.c, table, a.table_pages, block, part.head);
        const int64_t at = row < 0 ? 0 : row;
        const uint8_t *k = a.c.k + at * D + lane * 16, *v = a.c.v + at * D + lane * 16;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) x.k[i] = ldg16(k + i * 1024);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) x.v[i] = ldg16(v + i * 1024);
        x.ke = a.c.ke[at / kBlockTokens];
        x.ve = row < 0 ? -1 : a.c.ve[at / kBlockTokens];
    };
    auto take = [&](const Block& x, int block) {
        auto half = [](const uint4 p, int h) { return h ? operand8(p.z, p.w) : operand8(p.x, p.y); };
        cols.take(a.scale, block, x.ke, __builtin_amdgcn_readfirstlane(x.ve), [&](int t, int s) { return half(x.k[t * (PIECES / 2) + s / 2], s % 2); },
                  [&](int i) { return half(x.v[i / 2], i % 2); });
    };
    const int first_block = part.from / kBlockTokens + wt;
    const int end_block = (min(part.until, cols.most) + kBlockTokens - 1) / kBlockTokens;
    Block x0, x1;
    if (first_block < end_block) load(x0, first_block);
    for (int block = first_block; block < end_block; block += 2 * WT) {
        if (block + WT < end_block) load(x1, block + WT);
        take(x0, block);
        if (block + WT >= end_block) break;
        if (block + 2 * WT < end_block) load(x0, block + 2 * WT);
        take(x1, block + WT);
    }
    cols.sum_up();

    // the waves' sums of a column, in LDS
    __shared__ float sums[4][COLS][D + 4], stat[4][COLS][3];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < TILES; ++i)
            *reinterpret_cast<f32x4*>(&sums[wave][16 * n + col][16 * i + 4 * quarter]) = cols.o[i][n];
        if (quarter == 0) {
            stat[wave][16 * n + col][0] = cols.m[n];
            stat[wave][16 * n + col][1] = cols.jj[n];
            stat[wave][16 * n + col][2] = cols.l[n];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < WC * COLS * (D / 4); e += 256) {
        const int c = e / (D / 4), ch = e % (D / 4) * 4, w0 = c / COLS * WT, cc = c % COLS;
        if (part.first_col + c >= part.columns) continue;
        float mm = kLowest, j = kNone, ll = 0.0f;
#pragma unroll
        for (int w = 0; w < WT; ++w) mm = fmaxf(mm, stat[w0 + w][cc][0]);
#pragma unroll
        for (int w = 0; w < WT; ++w) j = fmaxf(j, stat[w0 + w][cc][1] + (stat[w0 + w][cc][0] - mm));
        f32x4 sum = {};
#pragma unroll
        for (int w = 0; w < WT; ++w) {
            const float by = stat[w0 + w][cc][0] - mm;
            ll += stat[w0 + w][cc][2] * __builtin_amdgcn_exp2f(by);
            sum += *reinterpret_cast<const f32x4*>(&sums[w0 + w][cc][ch]) * __builtin_amdgcn_exp2f(stat[w0 + w][cc][1] + by - j);
        }
        Target8<T, D>(a, seq, part.head, part.first_col + c, a.max_q * a.group, part.first_col + c, part.chunks == 1).store(ch, sum, mm, j, ll);
    }
}

// Many columns: each wave takes 16 NT of them and all tokens.  A stage of 4096 / D tokens is turned to fp16 once, a share by each
// wave, and lies in LDS in operand order, in two slots: while one is used the next is on its way from memory, to be written
// after it.  One barrier a stage.
template <typename T, int D, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 3) void attention8_wide_kernel(Attn8Args a) {
    constexpr int COLS = 16 * NT, PIECES = D / 32, TILES = D / 16, STEPS = D / 32;
    constexpr int BLOCKS = 128 / D, LOADS = 8 / WAVES;      // of a stage; pieces of 1 KB of codes of a wave and stage
    __shared__ __attribute__((aligned(16))) f16x8 staged[2][BLOCKS][4 * PIECES][64];    // keys' steps by tile, values' tiles
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const Part8 part(a, WAVES * COLS);
    if (part.empty) return;
    const Sequence8 seq(a, part.b);
    Columns8<T, D, NT> cols(a, seq, part.head, part.first_col + wave * COLS);

    const int32_t* table = a.table + (int64_t)part.b * a.table_pages;
    const int first = part.from / kBlockTokens, end = (part.until + kBlockTokens - 1) / kBlockTokens;
    const int mine = min(end, (cols.most + kBlockTokens - 1) / kBlockTokens);
    struct Stage {
        uint4 p[LOADS];
        int ke[BLOCKS], ve[BLOCKS];                         // ve < 0: no page holds the block
    };
    auto load = [&](Stage& x, int block) {
        int64_t at[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const int64_t row = block + b < end ? block_row8(a.c, table, a.table_pages, block + b, part.head) : -1;
            at[b] = row < 0 ? 0 : row;
            x.ke[b] = a.c.ke[at[b] / kBlockTokens];
            x.ve[b] = row < 0 ? -1 : a.c.ve[at[b] / kBlockTokens];
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = wave * LOADS + i, b = piece / (2 * PIECES), r = piece % (2 * PIECES);
            const int64_t row = BLOCKS == 1 || b == 0 ? at[0] : at[BLOCKS - 1];
            x.p[i] = ldg16((r < PIECES ? a.c.k : a.c.v) + row * D + r % PIECES * 1024 + lane * 16);
        }
    };
    auto write = [&](const Stage& x, int slot) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int piece = wave * LOADS + i, b = piece / (2 * PIECES), r = piece % (2 * PIECES);
            staged[slot][b][2 * r][lane] = operand8(x.p[i].x, x.p[i].y);
            staged[slot][b][2 * r + 1][lane] = operand8(x.p[i].z, x.p[i].w);
        }
    };
    static_assert(2 * STEPS == 2 * PIECES && TILES == 2 * PIECES, "as many operands of keys as of values");
    Stage x;
    if (first < end) {
        load(x, first);
        write(x, 0);
    }
    int slot = 0, block = first;
    for (; block < mine; block += BLOCKS) {
        int ke[BLOCKS], ve[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            ke[b] = x.ke[b];
            ve[b] = __builtin_amdgcn_readfirstlane(x.ve[b]);
        }
        __syncthreads();                                    // this stage is written, and the one before is read
        load(x, block + BLOCKS);                            // (past the end: some page's, unused)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
            cols.take(a.scale, block + b, ke[b], ve[b], [&](int t, int s) { return staged[slot][b][t * STEPS + s][lane]; },
                      [&](int i) { return staged[slot][b][2 * PIECES + i][lane]; });
        slot ^= 1;
        write(x, slot);
    }
    for (; block < end; block += BLOCKS) {                  // what only other waves' columns see
        __syncthreads();
        load(x, block + BLOCKS);
        slot ^= 1;
        write(x, slot);
    }
    cols.sum_up();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = part.first_col + wave * COLS + 16 * n + col;
        if (c >= part.columns) continue;
        const Target8<T, D> to(a, seq, part.head, c, a.order ? WAVES * COLS : a.max_q * a.group, a.order ? c - part.first_col : c, part.chunks == 1);
#pragma unroll
        for (int i = 0; i < TILES; ++i) to.store(16 * i + 4 * quarter, cols.o[i][n], cols.m[n], cols.jj[n], cols.l[n]);
    }
}

// The chunks of one column to its result: one workgroup, D / 4 threads for four channels each, the rest share the chunks.
template <typename T, int D, bool ORDERED>
__global__ __launch_bounds__(256) void attention8_join_kernel(Attn8Args a, int block_cols) {
    constexpr int LANES = D / 4, PARTS = 256 / LANES;
    __shared__ float sums[PARTS][D + 4], ls[PARTS];
    const int cols = ORDERED ? block_cols : a.max_q * a.group;
    const int entry = blockIdx.x / cols, col = blockIdx.x % cols, head = entry % a.c.heads;
    const int2 item = ORDERED ? a.order[entry / a.c.heads] : make_int2(entry / a.c.heads, 0);
    if (item.x < 0) return;
    const Sequence8 seq(a, item.x);
    const int c = ORDERED ? item.y * block_cols + col : col;
    const int columns = seq.queries * a.group;
    if (c >= columns) return;
    const int64_t seen = seq.seen(a, (min(c / block_cols * block_cols + block_cols, columns) - 1) / a.group);
    const int chunks = max(1, (int)((seen + a.chunk - 1) / a.chunk));
    const int64_t row = (int64_t)seq.first + c / a.group;
    if (chunks == 1 || row < 0 || row >= a.tokens) return;
    const int64_t stride = cols, first = sums_at(a, entry, 0, cols, col);
    const int part = threadIdx.x / LANES, ch = threadIdx.x % LANES * 4;
    // every wave finds the maxima, 64 chunks at a time
    float m = kLowest, j = kNone;
    for (int i = threadIdx.x & 63; i < chunks; i += 64) m = fmaxf(m, a.stats[3 * (first + i * stride)]);
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    for (int i = threadIdx.x & 63; i < chunks; i += 64) {
        const float* s = a.stats + 3 * (first + i * stride);
        j = fmaxf(j, s[1] + (s[0] - m));
    }
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) j = fmaxf(j, __shfl_xor(j, k));
    f32x4 sum = {};
    float l = 0.0f;
#pragma unroll 4
    for (int i = part; i < chunks; i += PARTS) {
        const int64_t at = first + i * stride;
        const float by = a.stats[3 * at] - m;
        l += a.stats[3 * at + 2] * __builtin_amdgcn_exp2f(by);
        sum += *reinterpret_cast<const f32x4*>(a.part + at * D + ch) * __builtin_amdgcn_exp2f(a.stats[3 * at + 1] + by - j);
    }
    *reinterpret_cast<f32x4*>(&sums[part][ch]) = sum;
    if (ch == 0) ls[part] = l;
    __syncthreads();
    if (part != 0) return;
    sum = f32x4{};
    l = 0.0f;
    for (int p = 0; p < PARTS; ++p) {
        sum += *reinterpret_cast<const f32x4*>(&sums[p][ch]);
        l += ls[p];
    }
    typedef T t4 __attribute__((ext_vector_type(4)));
    f32x4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = l == 0.0f ? 0.0f : ldexpf(sum[r] / l, (int)fmaxf(j - kLift, -1000.0f));
    *reinterpret_cast<t4*>(static_cast<T*>(a.o) + row * a.o_token + (int64_t)(head * a.group + c % a.group) * a.o_head + ch) =
        __builtin_convertvector(y, t4);
}

// ---------------------------------------------------------------- host side --
struct Plan8a {
    int nt, wt;                         // few columns: 16 nt a wave, wt waves share out the tokens; wt = 0: many columns
    int cols;                           // of a workgroup
    int blocks;                         // of columns
    int chunk, chunks;                  // tokens of a workgroup, and the most of them of a sequence
    int items;                          // entries of the order, 0 for none
    int64_t sums;                       // columns whose chunks' sums are kept, 0 for one chunk
};
constexpr int kWideTiles = 2, kWideWaves = 4;
static bool plan_attention8(int sequences, int tokens, int heads, int group, int head_dim, int max_q, int64_t max_kv, Plan8a& p) {
    if (sequences < 0 || heads < 1 || heads > 65535 || group < 1 || group > 1024 || max_q < 0 || max_kv < 0 || max_kv > INT32_MAX - 65536 ||
        (head_dim != 64 && head_dim != 128))
        return false;
    const int64_t columns = (int64_t)max_q * group;
    if (columns > INT32_MAX / 2) return false;
    p.nt = columns <= 16 ? 1 : 2;
    p.wt = columns <= 32 ? 4 : columns <= 64 ? 2 : 0;
    p.cols = p.wt ? 16 * p.nt * (4 / p.wt) : 16 * kWideTiles * kWideWaves;
    const int cols = p.cols;
    const int64_t blocks = std::max<int64_t>(1, (columns + cols - 1) / cols);
    // many columns of several sequences: workgroups in order of their work, and none for blocks that are not there (prompts of
    // 1025 to 1877 queries over 1025 to 4095 tokens 365 us, in order 211).  Chunks' sums go by it, too: laid out for max_q
    // queries of every sequence, 64 of one token and one of 2048 over 8192 tokens took 1.6 GB and a million workgroups to join.
    const int64_t items = p.wt == 0 && sequences > 1 ? std::min((int64_t)tokens * group / cols + sequences, sequences * blocks) : 0;
    const int64_t units = (items ? items : sequences * blocks) * heads;
    // Chunks: as many as there are CUs for one query and little more, two or three a CU for more columns (8 contexts of 8192
    // tokens by 4 columns: 256 workgroups 32.7 us, 512 31.6, 1024 33.9; 32 of 2048 with heads of 64: 15.3, then 19.6, as 4 of it are
    // the join's; 8 of 8192 by 64 columns 57, 50 and 62; by 256 columns 172, 134, 137, and 768 of them 124), of 256 tokens at
    // least for each wave, or 128; where there are enough without, single tokens take 2048 at a time, as contexts may be
    // ragged (64 of 257 to 8191 tokens: in chunks of 2048 114 us, of 4096 118; 128 of 1000 tokens whole 51, in halves 64).
    const int64_t least = p.wt ? 256 * p.wt / p.nt : 128, want = (p.wt ? 256 * p.nt : 768) / std::max<int64_t>(1, units);
    // Sums take 1 GB at most: as many chunks as that holds, where a launch's bound is far above the contexts that are there (1024
    // sequences of 500 tokens, 8 queries each by 8 x 8 heads, bounded by 131072: in chunks of 2048 17.6 GB and 1680 us, so 0.8 and
    // 1010; with one of 131072 among them 1870 and 1860).
    const int64_t sums = p.wt ? (int64_t)sequences * heads * columns * (head_dim + 3) * (int64_t)sizeof(float) : 0;
    const int64_t holds = std::max<int64_t>(1, (1 << 30) / std::max<int64_t>(1, sums));
    const int64_t share = want > 1 ? (max_kv + want - 1) / want : p.wt ? std::max(std::min<int64_t>(max_kv, 2048), (max_kv + holds - 1) / holds) : max_kv;
    const int64_t chunk = std::max<int64_t>(least, (share + 31) / 32 * 32);
    const int64_t chunks = std::max<int64_t>(1, (max_kv + chunk - 1) / chunk);
    if ((!items && blocks > 65535) || chunks > 65535 || (int64_t)sequences * heads > INT32_MAX || !mq_host::launch_holds(units * chunks, 256))
        return false;
    p.sums = chunks == 1 ? 0 : (items ? items * cols : sequences * columns) * heads;
    if (!mq_host::launch_holds(p.sums, 256)) return false;
    p.chunk = (int)chunk;
    p.blocks = (int)blocks;
    p.chunks = (int)chunks;
    p.items = (int)items;
    return true;
}

}  // namespace mq

using namespace mq;

// The order, then the chunks' sums and what belongs to them.
static size_t order_bytes(const Plan8a& p) { return ((size_t)p.items * sizeof(int2) + 15) / 16 * 16; }
static size_t workspace_of(const Plan8a& p, int head_dim) { return order_bytes(p) + (size_t)p.sums * p.chunks * (head_dim + 3) * sizeof(float); }

extern "C" size_t mq_attention_kv8_workspace_size(int sequences, int tokens, int heads, int group, int head_dim, int max_q,
                                                  int64_t max_kv) {
    Plan8a p;
    if (tokens < 0 || !plan_attention8(sequences, tokens, heads, group, head_dim, max_q, max_kv, p)) return 0;
    return workspace_of(p, head_dim);
}

extern "C" mq_status mq_attention_kv8(const mq_kv8_cache* cache, int sequences, int tokens, int group, int max_q, int64_t max_kv,
                                      mq_dtype type, const void* Q, int64_t q_token, int64_t q_head, const int32_t* page_table,
                                      int table_pages, const int32_t* kv_lens, const int32_t* cu_q, float scale, int causal, void* O,
                                      int64_t o_token, int64_t o_head, void* workspace, size_t ws_bytes, hipStream_t stream) {
    if (sequences < 0 || tokens < 0 || group < 1 || max_q < 0 || max_kv < 0 || table_pages < 0 || !mq_host::is_half_type(type) ||
        !(scale > 0.0f) || !(scale <= FLT_MAX) || (!cu_q && tokens != sequences))
        return MQ_ERR_INVALID_ARG;
    if (mq_status st = check_cache8(cache); st != MQ_OK) return st;
    for (int64_t s : {q_token, q_head, o_token, o_head})
        if (s < 0 || s % 8 != 0) return MQ_ERR_UNSUPPORTED_SHAPE;
    Plan8a p;
    if (max_kv > (int64_t)table_pages * cache->page_size ||
        !plan_attention8(sequences, tokens, cache->heads, group, cache->head_dim, cu_q ? max_q : std::min(max_q, 1), max_kv, p))
        return MQ_ERR_UNSUPPORTED_SHAPE;
    if (tokens == 0 || sequences == 0 || max_q == 0) return MQ_OK;
    if (!Q || !O || !kv_lens || (!page_table && max_kv > 0)) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Q, 16) || !mq_host::aligned(O, 16) || !mq_host::aligned(page_table, 4) || !mq_host::aligned(kv_lens, 4) ||
        !mq_host::aligned(cu_q, 4) || !mq_host::aligned(workspace, 16))
        return MQ_ERR_MISALIGNED;
    if (!cu_q) max_q = 1;
    const size_t need = workspace_of(p, cache->head_dim);
    if (need > 0 && (!workspace || ws_bytes < need)) return MQ_ERR_WORKSPACE;
    Attn8Args a{device_cache8(cache), Q, O, q_token, q_head, o_token, o_head, page_table, kv_lens, cu_q, table_pages, tokens, group, max_q,
                causal != 0, std::min(scale * kLog2e, FLT_MAX), max_kv, p.chunk, p.chunks, nullptr, nullptr, nullptr};
    int2* order = static_cast<int2*>(workspace);
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + order_bytes(p));
    a.stats = a.part + (size_t)p.sums * p.chunks * cache->head_dim;
    const dim3 grid(p.items ? p.items * cache->heads : sequences * cache->heads, p.items ? 1 : p.blocks, p.chunks);
    if (p.items) {
        hipLaunchKernelGGL(attention8_order_kernel, dim3(1), dim3(1024), 0, stream, a, sequences, p.cols, p.items, order);
        a.order = order;
    }
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        auto run = [&](auto d) {
            constexpr int D = decltype(d)::value;
            auto few = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
            if (p.wt == 4 && p.nt == 1) few(attention8_kernel<T, D, 1, 4>);
            else if (p.wt == 4) few(attention8_kernel<T, D, 2, 4>);
            else if (p.wt == 2) few(attention8_kernel<T, D, 2, 2>);
            else hipLaunchKernelGGL((attention8_wide_kernel<T, D, kWideTiles, kWideWaves>), grid, dim3(64 * kWideWaves), 0, stream, a);
            auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)p.sums), dim3(256), 0, stream, a, p.cols); };
            if (p.chunks > 1) p.items ? join(attention8_join_kernel<T, D, true>) : join(attention8_join_kernel<T, D, false>);
        };
        if (cache->head_dim == 64) run(std::integral_constant<int, 64>{});
        else run(std::integral_constant<int, 128>{});
        return mq_host::launch_status();
    });
}
