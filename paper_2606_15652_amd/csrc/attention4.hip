// Attention over the paged 4-bit cache.
//
//   o = sum_t p_t v_t / sum_t p_t,   p_t = exp(scale q.k_t),
//   k_t = zk_t + sk_t nk_t,  v_t = zv_t + sv_t nv_t   (n: codes 0 .. 15):
//   q.k_t = sk_t (q.nk_t) + zk_t sum(q),
//   sum_t p_t v_t = sum_t (p_t sv_t) nv_t + sum_t p_t zv_t.
//
// The codes go into the fp16 matrix instruction as they are, four bits a
// subnormal number (kv4.h), and the scales and minima act on the scores and
// weights, of which there are D times fewer than codes.  A token that a query
// does not see has the weight 0 there, whatever its parameters hold.
//
// Columns are the queries of one sequence and key head: position qi and head hg
// of the group at column qi group + hg.
#include "kv4.h"

#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

namespace mq {

mq_status check_cache4(const mq_kv4_cache* c);
Cache4 device_cache4(const mq_kv4_cache* c);

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 64;               // tokens that are taken at a time
constexpr int kLeastSteps = 4;          // of a workgroup
// What beginning and ending a unit takes, in steps of a workgroup (64 ragged contexts of up to 8191 tokens:
// none counted 82.7 us, 4 68.6, 12 66.7, 24 69.0).
constexpr int kUnitSteps = 12;
constexpr float kLowest = -FLT_MAX;     // no score is lower: running maximum of none
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;          // weights up to 2^kSlack before the running maximum moves

struct Attn4Args {
    Cache4 c;
    const void* q;
    void* o;
    int64_t q_token, q_head, o_token, o_head;
    const int32_t* table;
    int table_pages;                    // pages of a sequence in the table
    int max_kv;                         // tokens of a sequence at most: no length counts for more
    const int32_t* kv_lens;
    const int32_t* cu_q;                // null: one query a sequence
    int sequences, tokens, group, max_q;
    float scale;
    int causal;
    float *part_o, *part_m, *part_l;    // results of parts of a row's tokens: [place][column] (x D); null: whole rows only
    int32_t* starts;                    // few columns: [sequence] first step of each among all, [sequences] steps of a workgroup
    int splits, split_steps;            // many columns: parts of a unit and their steps
};

// The launch writes none of these arrays: reads by uniform indexes go through the scalar cache, beside the
// vector loads in flight, which return in order.
typedef __attribute__((address_space(4))) const int32_t const_int;

// A sequence's queries and tokens.
struct Sequence {
    int q0, nq, n;
};
__device__ __forceinline__ Sequence sequence(const Attn4Args& a, int b) {
    Sequence s;
    if (a.cu_q) {
        const const_int* cu_q = (const const_int*)a.cu_q;
        s.q0 = min(max(cu_q[b], 0), a.tokens);
        s.nq = min(max(min(cu_q[b + 1], a.tokens) - s.q0, 0), a.max_q);
    } else {
        s.q0 = b;
        s.nq = 1;
    }
    s.n = min(max(((const const_int*)a.kv_lens)[b], 0), a.max_kv);
    return s;
}
// tokens that query qi sees: 0 .. limit - 1
__device__ __forceinline__ int visible(const Attn4Args& a, const Sequence& s, int qi) {
    return a.causal ? min(max(s.n - s.nq + qi + 1, 0), s.n) : s.n;
}

__device__ __forceinline__ float quads_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quads_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// eight codes of a dword -> an operand: elements 2, 3, 6, 7 come 16 times too large
__device__ __forceinline__ f16x8 key_operand(uint32_t w) {
    return __builtin_bit_cast(f16x8, u32x4{w & 0x000F000Fu, w & 0x00F000F0u, (w >> 8) & 0x000F000Fu, (w >> 8) & 0x00F000F0u});
}
// code I (0 .. 3) of each of eight tokens' words; odd I: 16 times too large
template <int I>
__device__ __forceinline__ f16x8 value_operand(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
    constexpr uint32_t mask = I % 2 ? 0x00F000F0u : 0x000F000Fu;
    constexpr int shift = I / 2 * 8;
    return __builtin_bit_cast(f16x8, u32x4{(a0 >> shift) & mask, (a1 >> shift) & mask, (b0 >> shift) & mask, (b1 >> shift) & mask});
}

// Operands and scales of 16 columns of queries: fp16, scaled by a power of two that brings the largest
// finite value of the workgroup's columns near 2^8, so that neither type's range matters; channels of the codes that come 16 times too large
// divided by 16.  A lane has the channels (D / 4) g .. of its column.
template <int D>
struct Queries {
    f16x8 op[D / 32];
    // x = sk (q'.n) + zk of_minimum is the score over to_score(), in powers of 2
    float of_minimum, amax;
    f32x8 x[D / 32];

    template <typename T>
    __device__ __forceinline__ void load(const T* q) {
        of_minimum = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            x[i] = load8(q + 8 * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) of_minimum += x[i][e];
        }
        of_minimum = quads_sum(of_minimum);
        amax = largest([](float v) { return v; });
        // a column that is not finite spoils no other
        if (amax == INFINITY) amax = largest([](float v) { return v < INFINITY ? v : 0.0f; });
    }
    template <typename F>
    __device__ __forceinline__ float largest(F of) const {  // of the 16 columns' values without their signs; NaN is none
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v = fmaxf(v, of(fabsf(x[i][e])));
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) v = fmaxf(v, __shfl_xor(v, i));
        return v;
    }
    static __device__ __forceinline__ int exponent(float amax) { return amax > 0.0f ? 8 - ilogbf(amax) : 0; }
    __device__ __forceinline__ void finish(int up) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = ldexpf(x[i][e], e & 2 ? up - 4 : up);
            op[i] = __builtin_convertvector(x[i], f16x8);
        }
        of_minimum = ldexpf(of_minimum, up - 24);
    }
    // never zero or infinite: a scale or minimum of zero times it stays zero
    static __device__ __forceinline__ float to_score(float scale, int up) {
        return fminf(fmaxf(ldexpf(scale * kLog2e, 24 - up), FLT_MIN), FLT_MAX);
    }
};

// Four channels of a column, divided by the sum of its weights, to the output.
template <typename T>
__device__ __forceinline__ void store_output(const Attn4Args& a, const Sequence& s, int head, int col, int channel, f32x4 o, float sum) {
    typedef T half4 __attribute__((ext_vector_type(4)));
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;           // a row that sees nothing is 0
    T* out = static_cast<T*>(a.o) + (s.q0 + col / a.group) * a.o_token + (head * a.group + col % a.group) * a.o_head + channel;
    *reinterpret_cast<half4*>(out) = __builtin_convertvector(o * by, half4);
}

// Work of a launch: units (sequence, block of RP columns, key head) of as many steps as the sequence has
// tokens, behind kUnitSteps that stand for the unit's own cost, one unit after the other.  Every workgroup
// takes as many steps; its ends may lie inside units.
struct Work4 {
    int steps, units;
    __device__ __forceinline__ int each() const { return steps > 0 ? steps + kUnitSteps : 0; }
    __device__ __forceinline__ int all() const { return each() * units; }
};
template <int RP>
__device__ __forceinline__ Work4 work4(const Attn4Args& a, const Sequence& s) {
    return Work4{(s.n + kStep - 1) / kStep, (s.nq * a.group + RP - 1) / RP * a.c.heads};
}

// --------------------------------------------------------------------------
// Few columns (at most RP): codes go from memory to registers and into the products.
// --------------------------------------------------------------------------
// A wave takes 64 tokens at a time, four tiles of 16.  S = Q K^T with the queries
// repeated in the 16 rows (row i holds column i % RP), so each tile's scores are
// in every group of RP rows, and the lanes keep of tile i those that they alone
// keep: with RP = 4 a lane ends up with one token (16 g + r) and all the columns
// in its registers.  A row of 16 columns for four queries would leave three lanes
// of four with nothing (the work on scores, parameters and weights was half of
// the kernel: a batch of 64 contexts of up to 8191 tokens 70 us, 65).
// The weights cross to the lanes of the second product, O^T = V^T P^T, through LDS.
//
// Weights are held as multiples of `unit` (every sv is at most 2^7 of them), w = p sv /
// unit up to 2^15, rounded to fp16, whose smallest step is then 2^-31 of the largest sv;
// of the products 7.5 sum(w) is taken off again and made up for in fp32: codes about
// their middle, so that the rounding of w counts against values about their middle.
//
// What a wave loads for 64 tokens: lane (r, g), tile i: token r's key channels
// (D / 4) g .., the tokens 4 g .. + 3's value channels (D / 16) r ..; and the
// parameters of the tokens whose scores it keeps.
template <int D>
struct Keys4 {
    uint32_t k[4][D / 32];
};
template <int D>
struct Values4 {
    uint32_t v[4][D / 32];
};
// The pages of a step's tiles, as the table has them (the last token's where a tile is past the end: its
// page is there to be read).
struct Pages {
    int of[4];
};
__device__ __forceinline__ Pages find_pages(const Attn4Args& a, int b, int t, int last) {
    const const_int* table = (const const_int*)a.table + (int64_t)b * a.table_pages;
    Pages p;
#pragma unroll
    for (int h = 0; h < 4; ++h) p.of[h] = table[min(t + 16 * h, last) >> a.c.page_bits];
    return p;
}
// Whether a page is one of the cache's; the others hold no tokens, and page 0 is read in their place.
__device__ __forceinline__ bool there(const Attn4Args& a, int page) { return (uint32_t)page < (uint32_t)a.c.pages; }
// row of the cache's first token of a tile at token t
__device__ __forceinline__ int64_t tile_row(const Attn4Args& a, int head, int page, int t) {
    return (((int64_t)(there(a, page) ? page : 0) * a.c.heads + head) << a.c.page_bits) + (t & ((1 << a.c.page_bits) - 1));
}

template <int RP>
struct Shape4 {
    static constexpr int kTokens = RP / 4;          // of a step, that a lane keeps
    static constexpr int kTiles = 16 / RP;          // tiles that share the lanes
};
template <typename T, int D, int RP, int R>
__global__ __launch_bounds__(256, 2) void attention4_kernel(Attn4Args a) {
    constexpr int KK = D / 32, VT = D / 16, WT = 4, NT = Shape4<RP>::kTokens, Row = kStep + 8;
    // the waves' weights, and when the tokens are through, their results
    union Shared {
        _Float16 p[WT][RP][Row];
        float o[WT][RP][D + 4];
    };
    __shared__ __attribute__((aligned(16))) Shared shared;
    __shared__ float shared_m[WT][16], shared_l[WT][16];
    __shared__ f16x8 shared_q[KK][64];                      // operands: 16 registers more would cost a wave a SIMD
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;

    // this workgroup's steps pos .. last - 1 of all and the sequence that they begin in, or its unit
    int b, start = 0, pos = 0, last = 0, from = 0, unit = 0;
    if (a.part_o) {
        int total = 0;
        for (int i = lane; i < a.sequences; i += 64) total += work4<RP>(a, sequence(a, i)).all();
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) total += __shfl_xor(total, i);
        const int each = max(kLeastSteps, (total + (int)gridDim.x - 1) / (int)gridDim.x);
        if (blockIdx.x == 0 && threadIdx.x == 0) a.starts[a.sequences] = each;
        from = pos = __builtin_amdgcn_readfirstlane(min((int64_t)blockIdx.x * each, (int64_t)total));
        last = __builtin_amdgcn_readfirstlane(min(pos + each, total));
        b = start = -1;
        for (int i = 0, before = 0; i < a.sequences; i += 64) {
            const int w = i + lane < a.sequences ? work4<RP>(a, sequence(a, i + lane)).all() : 0;
            int up = w;
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) {
                const int v = __shfl_up(up, k);
                up += lane >= k ? v : 0;
            }
            if (blockIdx.x == 0 && wave == 0 && i + lane < a.sequences) a.starts[i + lane] = before + up - w;
            const uint64_t here = __ballot(pos < before + up);
            if (b < 0 && here) {
                const int at = __builtin_ctzll(here);
                b = i + at;
                start = __builtin_amdgcn_readfirstlane(before + __shfl(up - w, at));
                if (blockIdx.x != 0) break;
            }
            before += __shfl(up, 63);
        }
        if (pos >= last) return;
    } else {
        b = blockIdx.x / (a.c.heads * ((a.max_q * a.group + RP - 1) / RP));
        unit = blockIdx.x % (a.c.heads * ((a.max_q * a.group + RP - 1) / RP));
        if (unit >= work4<RP>(a, sequence(a, b)).units) return;     // a unit of no steps is written too: its rows are 0
    }
    b = __builtin_amdgcn_readfirstlane(b);
  do {
    const Sequence s = sequence(a, b);
    const Work4 work = work4<RP>(a, s);
    int step0 = 0, taken = work.steps, passed = 0;
    if (a.part_o) {
        unit = (pos - start) / work.each();
        const int at = (pos - start) % work.each();
        passed = min(work.each() - at, last - pos);
        step0 = max(at - kUnitSteps, 0);
        taken = max(at + passed - kUnitSteps, 0) - step0;
    }
    if (taken > 0 || !a.part_o) {
    const int head = unit % a.c.heads, col0 = unit / a.c.heads * RP, cols = s.nq * a.group;
    const int low = visible(a, s, col0 / a.group), high = visible(a, s, (min(col0 + RP, cols) - 1) / a.group);
    const int begin = (step0 + wave) * kStep, end = min(high, (step0 + taken) * kStep);
    constexpr int stride = kStep * WT;
    // the lane's scores: columns (within the block) mine + e, tokens of tile base + kTiles * i, i < NT
    const int mine = RP == 4 ? 0 : RP == 8 ? 4 * (g & 1) : 4 * g, base = RP == 4 ? g : RP == 8 ? g >> 1 : 0;

    Keys4<D> keys;
    Values4<D> values;
    uint32_t kp[NT], vp[NT];
    Pages pages{}, next{};
    auto load_keys = [&](const Pages& p, int t) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const uint8_t* k = a.c.k + tile_row(a, head, p.of[h], t + 16 * h) * (D / 2);
            __builtin_memcpy(keys.k[h], __builtin_assume_aligned(k + (uint32_t)(r * (D / 2) + g * (D / 8)), D / 8), D / 8);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            int64_t row = tile_row(a, head, p.of[i * Shape4<RP>::kTiles], t + 16 * i * Shape4<RP>::kTiles);
#pragma unroll
            for (int h = 1; h < Shape4<RP>::kTiles; ++h)
                if (base == h) row = tile_row(a, head, p.of[i * Shape4<RP>::kTiles + h], t + 16 * (i * Shape4<RP>::kTiles + h));
            kp[i] = a.c.kp[row + r];
            vp[i] = a.c.vp[row + r];
        }
    };
    auto load_values = [&](const Pages& p, int t) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const uint8_t* v = a.c.v + tile_row(a, head, p.of[h], t + 16 * h) * (D / 2);
            __builtin_memcpy(values.v[h], __builtin_assume_aligned(v + (uint32_t)(g * (2 * D) + r * (D / 8)), D / 8), D / 8);
        }
    };
    if (begin < end) {
        pages = find_pages(a, b, begin, end - 1);
        load_keys(pages, begin);
        load_values(pages, begin);
        next = find_pages(a, b, begin + stride, end - 1);
    }
    float of_minimum[R], to_score;
    {
        const int col = min(col0 + r % RP, cols - 1), qi = col / a.group;
        Queries<D> mq;
        mq.load(static_cast<const T*>(a.q) + (s.q0 + qi) * a.q_token + (head * a.group + col % a.group) * a.q_head + g * (D / 4));
        const int up = Queries<D>::exponent(mq.amax);
        mq.finish(up);
        to_score = Queries<D>::to_score(a.scale, up);
#pragma unroll
        for (int i = 0; i < KK; ++i)
            if (wave == 0) shared_q[i][lane] = mq.op[i];
#pragma unroll
        for (int e = 0; e < R; ++e) {
            of_minimum[e] = __shfl(mq.of_minimum, mine + e) * to_score;
        }
        __syncthreads();
    }

    f32x4 acc[VT] = {};
    float m[R], l[R] = {}, rest[R] = {};                    // rest: what the codes about their middle leave out
    float unit = 0.0f, per_unit = 0.0f;                     // weights are held as multiples of `unit`
#pragma unroll
    for (int e = 0; e < R; ++e) m[e] = kLowest;
    // over the lanes that keep the same columns
    auto all_max = [&](float v) {
#pragma unroll
        for (int i = 1; i < 64; i <<= 1)
            if (!(RP == 8 && i == 16) && !(RP == 16 && i >= 16)) v = fmaxf(v, __shfl_xor(v, i));
        return v;
    };
    auto all_sum = [&](float v) {
#pragma unroll
        for (int i = 1; i < 64; i <<= 1)
            if (!(RP == 8 && i == 16) && !(RP == 16 && i >= 16)) v += __shfl_xor(v, i);
        return v;
    };

    for (int t = begin; t < end; t += stride) {
        // the step after this one; behind the last the same again, so that the loads are not conditional (their
        // registers would be copied, and the copies wait for them)
        const bool more = t + stride < end;
        const int then = more ? t + stride : t;
        const Pages now = pages;
#pragma unroll
        for (int h = 0; h < 4; ++h) pages.of[h] = more ? next.of[h] : now.of[h];
        float x[NT][R];
        f16x8 q[KK];
#pragma unroll
        for (int i = 0; i < KK; ++i) q[i] = shared_q[i][lane];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int h = 0; h < Shape4<RP>::kTiles; ++h) {
                const int tile = i * Shape4<RP>::kTiles + h;
                f32x4 y = {};
#pragma unroll
                for (int c = 0; c < KK; ++c) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[c], key_operand(keys.k[tile][c]), y, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < R; ++e) x[i][e] = h == 0 || base == h ? y[e] : x[i][e];
                if (tile % 2) __builtin_amdgcn_sched_barrier(0);    // two tiles' operands at a time in registers
            }
        float sv[NT], middle[NT];
        uint32_t vps[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const f16x2 k = __builtin_bit_cast(f16x2, kp[i]), v = __builtin_bit_cast(f16x2, vp[i]);
            // a value row that is not finite (both its parameters are NaN) makes the score NaN, for the
            // queries that see it, and its weight 0 stays 0
            const float bad = __builtin_fmaf((float)v[0], 0.0f, 0.0f);
            vps[i] = v[0] == v[0] ? vp[i] : 0u;
            // in powers of 2 from here on: less their maximum, itself one of them, scores of any size are exact
            const float sk = (float)k[0] * to_score;
#pragma unroll
            for (int e = 0; e < R; ++e) x[i][e] = __builtin_fmaf(x[i][e], sk, __builtin_fmaf((float)k[1], of_minimum[e], bad));
        }
        __builtin_amdgcn_sched_barrier(0);
        load_keys(pages, then);
        if (t + kStep > low || !there(a, now.of[0]) || !there(a, now.of[1]) || !there(a, now.of[2]) || !there(a, now.of[3])) {
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                int page = now.of[i * Shape4<RP>::kTiles];
#pragma unroll
                for (int h = 1; h < Shape4<RP>::kTiles; ++h) page = base == h ? now.of[i * Shape4<RP>::kTiles + h] : page;
                const int token = t + 16 * (i * Shape4<RP>::kTiles + base) + r;
                if (!there(a, page) || token >= end) vps[i] = 0u;      // whatever memory holds there
#pragma unroll
                for (int e = 0; e < R; ++e)
                    if (!there(a, page) || token >= visible(a, s, (col0 + mine + e) / a.group)) x[i][e] = -INFINITY;
            }
        }
        float most = 0.0f;
        bool moves = false;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const f16x2 v = __builtin_bit_cast(f16x2, vps[i]);
            sv[i] = (float)v[0];
            middle[i] = __builtin_fmaf((float)v[0], 7.5f, (float)v[1]);
            most = fmaxf(most, sv[i]);
        }
        float top[R];
#pragma unroll
        for (int e = 0; e < R; ++e) {
            top[e] = x[0][e];
#pragma unroll
            for (int i = 1; i < NT; ++i) top[e] = fmaxf(top[e], x[i][e]);
            moves = moves || top[e] > m[e] + kSlack;
        }
        moves = moves || most > 0x1p7f * unit;
        if (__any(moves)) {
            const float old = unit;
#pragma unroll
            for (int i = 1; i < 64; i <<= 1) most = fmaxf(most, __shfl_xor(most, i));
            unit = fmaxf(unit, 0x1p-6f * most);
            per_unit = unit > 0.0f ? 1.0f / unit : 0.0f;
            float down[R];
#pragma unroll
            for (int e = 0; e < R; ++e) {
                const float to = fmaxf(m[e], all_max(top[e]));
                down[e] = __builtin_amdgcn_exp2f(m[e] - to);
                m[e] = to;
                l[e] *= down[e];
                rest[e] *= down[e];
                down[e] *= old * per_unit;
            }
            // the factor of the second product's column r: register r % 4 of a lane that keeps it
            float by = 1.0f;
#pragma unroll
            for (int e = 0; e < R; ++e) {
                const float v = __shfl(down[e], RP == 4 ? 0 : RP == 8 ? r % 8 / 4 * 16 : r / 4 * 16);
                by = r % 4 == e ? v : by;
            }
#pragma unroll
            for (int i = 0; i < VT; ++i) acc[i] *= by;
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int tile = i * Shape4<RP>::kTiles + base;
            // tokens of 32 in the order of the second product's operand: 4 g .. + 3 of one tile, then of the other
            const int at = tile / 2 * 32 + r / 4 * 8 + tile % 2 * 4 + r % 4;
            const float by = sv[i] * per_unit, off = -7.5f * unit;
#pragma unroll
            for (int e = 0; e < R; ++e) {
                const float pe = __builtin_amdgcn_exp2f(x[i][e] - m[e]);
                l[e] += pe;
                const _Float16 w = (_Float16)(pe * by);
                rest[e] = __builtin_fmaf((float)w, off, __builtin_fmaf(pe, middle[i], rest[e]));
                shared.p[wave][mine + e][at] = w;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own, read by its other lanes
        __builtin_amdgcn_wave_barrier();
        f16x8 p[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) p[h] = *reinterpret_cast<const f16x8*>(&shared.p[wave][r % RP][32 * h + 8 * g]);
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(p[0]), "+v"(p[1])::"memory");
        // scalar loads count with those of LDS: the next table entries are under way through the second product only
        next = find_pages(a, b, t + 2 * stride, end - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int w = 0; w < D / 64; ++w) {
                const uint32_t a0 = values.v[2 * h][2 * w], a1 = values.v[2 * h][2 * w + 1];
                const uint32_t b0 = values.v[2 * h + 1][2 * w], b1 = values.v[2 * h + 1][2 * w + 1];
                acc[4 * w] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_operand<0>(a0, a1, b0, b1), p[h], acc[4 * w], 0, 0, 0);
                acc[4 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_operand<1>(a0, a1, b0, b1), p[h], acc[4 * w + 1], 0, 0, 0);
                acc[4 * w + 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_operand<2>(a0, a1, b0, b1), p[h], acc[4 * w + 2], 0, 0, 0);
                acc[4 * w + 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value_operand<3>(a0, a1, b0, b1), p[h], acc[4 * w + 3], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        load_values(pages, then);
        asm volatile("" ::: "memory");                      // the weights are read before the next are written
    }

    // Column r's D / 4 channels (D / 4) g .., not yet divided by the weights' sum; joined over the waves.
#pragma unroll
    for (int e = 0; e < R; ++e) {
        l[e] = all_sum(l[e]);
        rest[e] = all_sum(rest[e]);
    }
    float add = 0.0f;
#pragma unroll
    for (int e = 0; e < R; ++e) {
        const float v = __shfl(rest[e], RP == 4 ? 0 : RP == 8 ? r % 8 / 4 * 16 : r / 4 * 16);
        add = r % 4 == e ? v : add;
    }
    if (r == 0 && (RP == 16 || g < RP / 4)) {
#pragma unroll
        for (int e = 0; e < R; ++e) {
            shared_m[wave][mine + e] = m[e];
            shared_l[wave][mine + e] = l[e];
        }
    }
    const float of_unit = unit * 0x1p24f;
    __syncthreads();                                        // every wave has read its last weights
    if (r < RP && col0 + r < cols) {
#pragma unroll
        for (int c = 0; c < D / 4; c += 4) {
            f32x4 out;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = (c + k) % VT, e = (c + k) / VT;
                out[k] = __builtin_fmaf(acc[i][e], of_unit * (i % 2 ? 0.0625f : 1.0f), add);
            }
            *reinterpret_cast<f32x4*>(&shared.o[wave][r][g * (D / 4) + c]) = out;
        }
    }
    __syncthreads();
    const bool whole = taken == work.steps;
    const int64_t place = ((int64_t)blockIdx.x * 2 + (pos == from ? 0 : 1)) * RP;   // at most two parts of units a workgroup
    for (int i = threadIdx.x; i < RP * (D / 4); i += 256) {
        const int col = i / (D / 4), ch = 4 * (i % (D / 4));
        if (col0 + col >= cols) break;
        float mx = shared_m[0][col], sum = 0.0f;
        f32x4 o = {};
#pragma unroll
        for (int w = 1; w < WT; ++w) mx = fmaxf(mx, shared_m[w][col]);
#pragma unroll
        for (int w = 0; w < WT; ++w) {
            const float by = __builtin_amdgcn_exp2f(shared_m[w][col] - mx);
            sum = __builtin_fmaf(shared_l[w][col], by, sum);
            o += *reinterpret_cast<const f32x4*>(&shared.o[w][col][ch]) * by;
        }
        if (whole) {
            store_output<T>(a, s, head, col0 + col, ch, o, sum);
        } else {
            *reinterpret_cast<f32x4*>(a.part_o + (place + col) * D + ch) = o;
            if (ch == 0) {
                a.part_m[place + col] = mx;
                a.part_l[place + col] = sum;
            }
        }
    }
    }
    pos += passed;
    if (!a.part_o || pos >= last) return;
    __syncthreads();                                        // the results are read before the next unit's weights
    if (pos >= start + work.all()) {
        start += work.all();
        do ++b;                                             // there is one: steps are left
        while (work4<RP>(a, sequence(a, b)).all() == 0);
    }
  } while (true);
}

constexpr float kLift = 8.0f, kMost = 15.0f;    // log2 of the weight at the running maximum, and above which that moves
constexpr uint16_t kMostPower = 0x7000;     // 2^13 in fp16: the largest power of two by which codes are staged

// what a scheduling group holds
constexpr int kVector = 0x402, kProducts = 0x8, kLdsReads = 0x100;

// --------------------------------------------------------------------------
// Many columns: keys and values of 64 tokens at a time in LDS, as operands.
// --------------------------------------------------------------------------
// Eight waves of 32 columns each.  S^T = K Q^T: a lane holds four neighbouring tokens
// of one query, which is what the second product, O^T = V^T P^T, takes from it.
// Keys are staged as codes (subnormal numbers), their scales and minima, in fp32,
// act on the scores.  A value z + s n = m (b (n - 7.5) + (z + 7.5 s) / m), where b
// is the power of two and m the mantissa of s (b = s, m = 1 below fp16's normal
// range, where steps of 2^-25 are below what s resolves; b = 2^13, m up to 8 above 2^13,
// so that 7.5 b is in fp16's range): b (n - 7.5), exact in fp16, is staged; the weight
// w = p m comes out of the exponential, as log2 m over the key's scale is where the
// scores' sums begin, and is rounded to fp16; 1 / m and (z + 7.5 s) / m, each as two
// fp16 numbers, are four rows more of the second product (of the latter a 16th and what
// that leaves: it passes fp16's range, as z + 15 s may in bf16).  The weights' rounding is thus the only one, and the
// same above and below the fraction: fp16 results are off by 2.7e-4 of their norm,
// 2.1e-4 of it their own rounding (values staged as fp16 values: 3.3e-4, and 5 % less
// time).  Four ragged prompts of up to 2047 tokens, 32 / 8 heads of 128: 293 us, 580
// TFLOP/s; heads of 64: 263.  A stage is
// converted by the whole workgroup while the one before is in use, from registers
// loaded one stage earlier still; every conversion then serves 256 columns.
//
// The vector unit bounds it (an exponential takes it four times as long as
// another operation): a score is brought under its column's running maximum by
// the two multiply-adds that scale it, score - m = acc sk + (zk sum(q) - m), and
// the sums are rows of the second product.  Weights are held as multiples of 2^-kLift of
// the running maximum's, up to 2^15: a weight counts down to 2^-33 of the largest.
template <typename T, int D>
__global__ __launch_bounds__(512, 2) void attention4_wide_kernel(Attn4Args a) {
    constexpr int KK = D / 32, VT = D / 16, C = 2, WaveCols = 16 * C, NW = 8, Cols = WaveCols * NW;
    struct Stage {
        f16x8 k[4][KK][64];                                 // tile, operand, lane
        f16x8 v[2][VT][64];                                 // two tiles, operand, lane
        f32x2 kp[64];                                       // token: scale, minimum
        float up[64];                                       // token: log2 m over the key's scale
        _Float16 rest[4][64];                               // token: 1 / m, what fp16 leaves of it, the middle / 16 m as well
    };
    __shared__ __attribute__((aligned(16))) Stage stages[2];
    __shared__ float largest[NW];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    // The last columns, which see most, first; the blocks of a head's columns on one XCD where heads allow; the
    // sequences of a round one further on than in the round before, as workgroups go to the parts of an XCD in turn
    // (four ragged sequences, always in the same order: 500 us, 299).
    const int blocks = (a.max_q * a.group + Cols - 1) / Cols, pairs = a.sequences * a.c.heads;
    const int unit = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int round = unit / pairs, pair = unit % pairs, head = pair % a.c.heads, b = (pair / a.c.heads + round) % a.sequences;
    const int block0 = (blocks - 1 - round) * Cols;
    const Sequence s = sequence(a, b);
    const int cols = s.nq * a.group;
    if (block0 >= cols) return;
    const int all = visible(a, s, (min(block0 + Cols, cols) - 1) / a.group);
    const int begin = (int)min((int64_t)split * a.split_steps * kStep, (int64_t)INT_MAX - kStep);
    if (split > 0 && begin >= all) return;                  // split 0 is there for rows of no tokens, too
    const int end = min(all, begin + a.split_steps * kStep);
    const int col0 = block0 + wave * WaveCols;
    const bool mine = col0 < cols;
    const int low = mine ? visible(a, s, col0 / a.group) : 0;
    const int high = mine ? min(end, visible(a, s, (min(col0 + WaveCols, cols) - 1) / a.group)) : 0;

    // Loads of a stage: wave w < 4 has the keys of tile w; wave 4 + w the values of channels (D / 16) r + 4 (w %
    // (D / 64)) .. of tiles 2 (w / (D / 64)) and one on, and their parameters; wave 0 those of the keys.  (The same
    // work for every wave is slower, 8 contexts of 4096 tokens by 2048 queries 914 us, 870: of the two waves of a
    // SIMD one is through with its share earlier, and the one's products meet the other's vector work.)
    const int value_item = wave - 4;
    const bool has_keys = wave < 4, has_values = value_item >= 0 && value_item < D / 32;
    const int key_tile = wave, value_tile = value_item / (D / 64) * 2, value_word = value_item % (D / 64);
    uint32_t raw_k[D / 32], raw_v[2][2], raw_kp = 0, raw_vp = 0;
    u32x4 raw_p[2];
    int table = 0;                                          // lane h: page of tile h
    auto load_table = [&](int t) {
        const int at = min(t + 16 * (lane & 3), end - 1);
        table = a.table[(int64_t)b * a.table_pages + (at >> a.c.page_bits)];
    };
    int page[4] = {};
    auto load = [&](int t) {
#pragma unroll
        for (int h = 0; h < 4; ++h) page[h] = __builtin_amdgcn_readlane(table, h);
        if (has_keys) {
            const int64_t row = tile_row(a, head, key_tile == 0 ? page[0] : key_tile == 1 ? page[1] : key_tile == 2 ? page[2] : page[3], t + 16 * key_tile);
            __builtin_memcpy(raw_k, __builtin_assume_aligned(a.c.k + row * (D / 2) + (uint32_t)(r * (D / 2) + g * (D / 8)), D / 8), D / 8);
        }
        if (has_values) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t row = tile_row(a, head, value_tile == 0 ? page[h] : page[2 + h], t + 16 * (value_tile + h));
                __builtin_memcpy(raw_v[h], __builtin_assume_aligned(a.c.v + row * (D / 2) + (uint32_t)(g * (2 * D) + r * (D / 8) + 8 * value_word), 8), 8);
                raw_p[h] = *reinterpret_cast<const u32x4*>(a.c.vp + row + 4 * g);
            }
        }
        if (wave == 0) {                                    // lane: token
            int64_t row = tile_row(a, head, page[0], t);
#pragma unroll
            for (int h = 1; h < 4; ++h)
                if (g == h) row = tile_row(a, head, page[h], t + 16 * h);
            raw_kp = a.c.kp[row + r];
            raw_vp = a.c.vp[row + r];
        }
    };
    float to_score = 0.0f;                                  // the workgroup's
    auto finite = [](uint32_t p) { return (p & 0x7C00u) != 0x7C00u; };     // both parameters are NaN, or none
    auto convert = [&](Stage& st, int t) {
        if (has_keys) {
#pragma unroll
            for (int i = 0; i < KK; ++i) st.k[key_tile][i][lane] = key_operand(raw_k[i]);
        }
        if (has_values) {
            u32x4 w[4];                                     // channel of the word: four pairs of tokens
            uint32_t p[2][4];
            u16x2 most{};                                   // the largest scale, as its bits
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[h][e] = raw_p[h][e];
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, p[h][e]));
                }
            // a row that is not finite weighs on the scores (below), where a weight of 0 leaves it out; and what
            // memory holds past the end; scales from 2^13 on have the power 2^13
            if (__any(most[0] >= kMostPower) || t + kStep > s.n) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool none = !finite(p[h][e]) || t + 16 * (value_tile + h) + 4 * g + e >= s.n;
                        p[h][e] = none ? 0 : min(p[h][e] & 0xFFFFu, (uint32_t)kMostPower);
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t sv = __builtin_amdgcn_perm(p[h][2 * k + 1], p[h][2 * k], 0x05040100u);
                    // the scale's power of two; a subnormal scale whole
                    const u16x2 power = __builtin_elementwise_max(__builtin_bit_cast(u16x2, sv & 0x7C007C00u),
                                                                  __builtin_elementwise_min(__builtin_bit_cast(u16x2, sv), (u16x2)(uint16_t)0x3FF));
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint32_t raw = n == 0 ? raw_v[h][k] << 3 : raw_v[h][k] >> (4 * n - 3);
                        const uint32_t code = (raw & 0x00780078u) | 0x58005800u;                        // 128 + n
                        const f16x2 v = (__builtin_bit_cast(f16x2, code) - (f16x2)(_Float16)135.5f) * __builtin_bit_cast(f16x2, power);
                        w[n][2 * h + k] = __builtin_bit_cast(uint32_t, v);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) st.v[value_tile / 2][4 * value_word + n][lane] = __builtin_bit_cast(f16x8, w[n]);
        }
        if (wave == 0) {
            const f16x2 k = __builtin_bit_cast(f16x2, raw_kp);
            // a value row that is not finite makes the score NaN, for the queries that see it
            float sk = (float)k[0] * to_score;
            sk = fabsf(sk) < 0x1p-100f ? 0x1p-100f : sk;    // (no score comes of it, and it has a reciprocal)
            st.kp[lane] = f32x2{sk, finite(raw_vp) ? (float)k[1] * to_score : NAN};
            const uint32_t vp = finite(raw_vp) && t + lane < s.n ? raw_vp : 0;
            const float sv = half_bits_to_float((uint16_t)vp), middle = __builtin_fmaf(sv, 7.5f, half_bits_to_float((uint16_t)(vp >> 16)));
            const float mantissa = (vp & 0x7C00u) >= kMostPower ? sv * 0x1p-13f
                                 : (vp & 0x7C00u) ? __uint_as_float(0x3F800000u | (vp & 0x3FFu) << 13) : 1.0f;
            const float inv = __builtin_amdgcn_rcpf(mantissa), rest[2] = {inv, middle * inv};
            st.up[lane] = __builtin_amdgcn_logf(mantissa) * __builtin_amdgcn_rcpf(sk);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float units = i == 0 ? 1.0f : 16.0f;
                const _Float16 high = (_Float16)(rest[i] * (1.0f / units));
                st.rest[2 * i][lane] = high;
                st.rest[2 * i + 1][lane] = (_Float16)__builtin_fmaf((float)high, -units, rest[i]);
            }
        }
    };

    Queries<D> q[C];
    int limit[C];
    if (begin < end) {                                      // (of no tokens there may be no table)
        load_table(begin);
        load(begin);
        load_table(begin + kStep);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int col = min(col0 + 16 * j + r, cols - 1), qi = col / a.group;
        limit[j] = visible(a, s, qi);
        q[j].load(static_cast<const T*>(a.q) + (s.q0 + qi) * a.q_token + (head * a.group + col % a.group) * a.q_head + g * (D / 4));
    }
    float amax = fmaxf(q[0].amax, q[1].amax);
    if (lane == 0) largest[wave] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) amax = fmaxf(amax, largest[i]);
    const int up = Queries<D>::exponent(amax);
    to_score = Queries<D>::to_score(a.scale, up);
#pragma unroll
    for (int j = 0; j < C; ++j) q[j].finish(up);
    // (kept here: the compiler would make the operands again in every step that has work)
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < KK; ++i) asm volatile("" : "+v"(q[j].op[i]));
    f32x4 acc[C][VT] = {}, sums[C] = {};
    float m[C] = {}, most[C];                               // scores are taken less m; above `most` of that m moves
#pragma unroll
    for (int j = 0; j < C; ++j) most[j] = -INFINITY;        // to the first score that there is, then above kMost

    int now[4];                                             // pages of the stage in use
    auto turn = [&](int t) {                                // the stage at t from registers to LDS, the one after into registers
#pragma unroll
        for (int h = 0; h < 4; ++h) now[h] = page[h];
        convert(stages[t / kStep & 1], t);
        if (t + kStep < end) {
            load(t + kStep);
            load_table(t + 2 * kStep);
        }
        __syncthreads();
    };
    if (begin < end) turn(begin);
    for (int t = begin; t < end; t += kStep) {
        const Stage& st = stages[t / kStep & 1];
        if (t < high) {
            f32x4 x[C][4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
#pragma unroll
                for (int j = 0; j < C; ++j) x[j][h] = *reinterpret_cast<const f32x4*>(st.up + 16 * h + 4 * g);
#pragma unroll
                for (int i = 0; i < KK; ++i) {
                    const f16x8 k = st.k[h][i][lane];
#pragma unroll
                    for (int j = 0; j < C; ++j) x[j][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[j].op[i], x[j][h], 0, 0, 0);
                }
            }
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x2 kp = st.kp[16 * h + 4 * g + e];
#pragma unroll
                    for (int j = 0; j < C; ++j) x[j][h][e] = __builtin_fmaf(x[j][h][e], kp[0], __builtin_fmaf(kp[1], q[j].of_minimum, -m[j]));
                }
            // operands are read two tiles ahead of their products (read as they are needed, LDS is waited for each time)
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 2 * KK + 4, 0);
            __builtin_amdgcn_sched_group_barrier(kProducts, C * KK, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, KK, 0);
            __builtin_amdgcn_sched_group_barrier(kProducts, C * KK, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, KK, 0);
            __builtin_amdgcn_sched_group_barrier(kProducts, C * KK, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 8, 0);
            __builtin_amdgcn_sched_group_barrier(kProducts, C * KK, 0);
            if (t + kStep > low || !there(a, now[0]) || !there(a, now[1]) || !there(a, now[2]) || !there(a, now[3])) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < C; ++j)
                            if (!there(a, now[h]) || t + 16 * h + 4 * g + e >= limit[j]) x[j][h][e] = -INFINITY;
            }
            float top[C];
            bool moves = false;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                top[j] = -INFINITY;
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[j] = fmaxf(top[j], x[j][h][e]);
                moves = moves || top[j] > most[j];
            }
            if (__any(moves)) {
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    const float to = quads_max(top[j]), by = to > most[j] ? to - kLift : 0.0f;
                    const float down = most[j] == kMost ? __builtin_amdgcn_exp2f(-by) : 1.0f;   // (before: sums of nothing)
                    most[j] = to > most[j] ? kMost : most[j];
                    m[j] += by;
#pragma unroll
                    for (int h = 0; h < 4; ++h) x[j][h] -= by;
                    sums[j] *= down;
#pragma unroll
                    for (int i = 0; i < VT; ++i) acc[j][i] *= down;
                }
            }
            f16x8 p[C][2];
#pragma unroll
            for (int j = 0; j < C; ++j)
#pragma unroll
                for (int h = 0; h < 4; ++h) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[j][h / 2][4 * (h % 2) + e] = (_Float16)__builtin_amdgcn_exp2f(x[j][h][e]);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const _Float16* at = st.rest[r & 3] + 32 * h + 4 * g;
                const f16x8 rest = __builtin_shufflevector(*reinterpret_cast<const f16x4*>(at), *reinterpret_cast<const f16x4*>(at + 16), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int j = 0; j < C; ++j) sums[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rest, p[j][h], sums[j], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < VT; ++i) {
                    const f16x8 v = st.v[h][i][lane];
#pragma unroll
                    for (int j = 0; j < C; ++j) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[j][h], acc[j][i], 0, 0, 0);
                }
            }
            // half of the value operands are read before the exponentials, the others beside the products
            __builtin_amdgcn_sched_group_barrier(kLdsReads, VT + 2, 0);
            __builtin_amdgcn_sched_group_barrier(kVector, 12 * C, 0);
#pragma unroll
            for (int i = 0; i < VT; ++i) {
                __builtin_amdgcn_sched_group_barrier(kProducts, C, 0);
                __builtin_amdgcn_sched_group_barrier(kVector, 12 * C / VT, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 1, 0);
            }
        }
        if (t + kStep < end) turn(t + kStep);
    }

#pragma unroll
    for (int j = 0; j < C; ++j) {
        const float sum = sums[j][0] + sums[j][1], middle = __builtin_fmaf(sums[j][2], 16.0f, sums[j][3]);
        if (col0 + 16 * j + r < cols) {
            const int64_t place = (int64_t)blockIdx.x * Cols + wave * WaveCols + 16 * j + r;
#pragma unroll
            for (int c = 0; c < D / 4; c += 4) {
                f32x4 o;
#pragma unroll
                for (int k = 0; k < 4; ++k) o[k] = acc[j][(c + k) % VT][(c + k) / VT] + middle;
                if (a.splits == 1) store_output<T>(a, s, head, col0 + 16 * j + r, g * (D / 4) + c, o, sum);
                else *reinterpret_cast<f32x4*>(a.part_o + place * D + g * (D / 4) + c) = o;
            }
            if (a.splits > 1 && g == 0) {
                a.part_m[place] = most[j] == kMost ? m[j] : kLowest;
                a.part_l[place] = sum;
            }
        }
    }
}

// Joins the parts of a row, one workgroup a row, D / 4 lanes a part; rows of no tokens become 0.
template <typename T, int D, int RP>
__global__ __launch_bounds__(256) void attention4_join_kernel(Attn4Args a) {
    constexpr int Lanes = D / 4, Shares = 256 / Lanes;
    const int share = threadIdx.x / Lanes, at = threadIdx.x % Lanes;
    const int heads = a.c.heads * a.group, hq = blockIdx.x % heads, qi = blockIdx.x / heads % a.max_q;
    const int b = blockIdx.x / heads / a.max_q;
    const Sequence s = sequence(a, b);
    if (qi >= s.nq) return;
    const int head = hq / a.group, col = qi * a.group + hq % a.group;
    const Work4 work = work4<RP>(a, s);
    const int each = a.starts[a.sequences], first = a.starts[b] + (col / RP * a.c.heads + head) * work.each();
    const int w0 = (first + kUnitSteps) / each, w1 = (first + work.each() - 1) / each, parts = w1 - w0 + 1;
    if (parts == 1 && work.steps > 0) return;               // its workgroup wrote it
    if (work.steps == 0) {
        if (share == 0) store_output<T>(a, s, head, col, 4 * at, f32x4{}, 0.0f);
        return;
    }
    // where workgroup w0 + i left its part: only the first may have begun with another unit
    auto place = [&](int i) { return ((int64_t)(w0 + i) * 2 + (i == 0 && first > w0 * each ? 1 : 0)) * RP + col % RP; };
    f32x4 o = {};
    float mx = kLowest, sum = 0.0f;
    for (int i = share; i < parts; i += Shares) {
        const int64_t p = place(i);
        const float m = a.part_m[p], to = fmaxf(mx, m), down = __builtin_amdgcn_exp2f(mx - to), by = __builtin_amdgcn_exp2f(m - to);
        o = o * down + *reinterpret_cast<const f32x4*>(a.part_o + p * D + 4 * at) * by;
        sum = sum * down + a.part_l[p] * by;
        mx = to;
    }
    __shared__ f32x4 shared_o[Shares][Lanes];
    __shared__ float shared_m[Shares], shared_l[Shares];
    shared_o[share][at] = o;
    if (at == 0) {
        shared_m[share] = mx;
        shared_l[share] = sum;
    }
    __syncthreads();
    if (share > 0) return;
#pragma unroll
    for (int i = 1; i < Shares; ++i) mx = fmaxf(mx, shared_m[i]);
    o = f32x4{};
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < Shares; ++i) {
        const float by = __builtin_amdgcn_exp2f(shared_m[i] - mx);
        o += shared_o[i][at] * by;
        sum += shared_l[i] * by;
    }
    store_output<T>(a, s, head, col, 4 * at, o, sum);
}

// The same for many columns, where the parts are few and the rows many: D / 4 lanes a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention4_join_wide_kernel(Attn4Args a, int rows) {
    constexpr int Lanes = D / 4, Cols = 256;
    const int row = blockIdx.x * (256 / Lanes) + threadIdx.x / Lanes, at = threadIdx.x % Lanes;
    if (row >= rows) return;
    const int heads = a.c.heads * a.group, hq = row % heads, qi = row / heads % a.max_q, b = row / heads / a.max_q;
    const Sequence s = sequence(a, b);
    if (qi >= s.nq) return;
    const int head = hq / a.group, col = qi * a.group + hq % a.group, block = col / Cols;
    // the kernel's order of units, and the parts that had tokens
    const int blocks = (a.max_q * a.group + Cols - 1) / Cols, round = blocks - 1 - block;
    const int turn = ((b - round) % a.sequences + a.sequences) % a.sequences;
    const int64_t place = (int64_t)((round * a.sequences + turn) * a.c.heads + head) * a.splits * Cols + col % Cols;
    const int all = visible(a, s, (min((block + 1) * Cols, s.nq * a.group) - 1) / a.group);
    const int parts = max(1, min(a.splits, ((all + kStep - 1) / kStep + a.split_steps - 1) / a.split_steps));
    f32x4 o = {};
    float mx = kLowest, sum = 0.0f;
    for (int i = 0; i < parts; ++i) {
        const int64_t p = place + i * Cols;
        const float m = a.part_m[p], to = fmaxf(mx, m), down = __builtin_amdgcn_exp2f(mx - to), by = __builtin_amdgcn_exp2f(m - to);
        o = o * down + *reinterpret_cast<const f32x4*>(a.part_o + p * D + 4 * at) * by;
        sum = sum * down + a.part_l[p] * by;
        mx = to;
    }
    store_output<T>(a, s, head, col, 4 * at, o, sum);
}

// ---------------------------------------------------------------- host side --
struct Plan4 {
    int columns;                        // of a workgroup: up to 16, or 256
    int64_t groups;
    bool whole;                         // a workgroup takes whole units
    int splits, split_steps;            // 256 columns
};

// Columns of a workgroup.  Blocks of 16 read the cache once for every 16 columns, in a
// block of 256 the waves whose 32 columns are not there idle: the switch is where the two
// are about even (8 heads of 128; one context of 65536 tokens, one and eight of 8192, 32
// of 2048): at 64 columns blocks of 16 take 57.7, 21.6, 53.0 and 69.5 us, one of 256 74.0,
// 30.1, 66.5 and 61.4; at 68 columns 67.9, 22.5, 71.9 and 91.0 against 76.7, 30.9, 69.1
// and 64.0; at 192 141.6, 32.3, 128.4 and 191.3 against 98.6, 40.1, 93.6 and 86.3.
static int columns4(int max_q, int group) {
    const int64_t cols = (int64_t)max_q * group;
    return cols <= 4 ? 4 : cols <= 8 ? 8 : cols <= 64 ? 16 : 256;
}
constexpr int kWholeSteps = 16;         // few columns: sequences of up to as many steps are taken whole

// Workgroups of a launch.  Few columns: short sequences (up to 1024 tokens: 16
// steps, four for each wave) are taken whole; the others are cut into as many
// equal shares as workgroups fit on the chip, or shares of four steps if those are
// fewer: 768 up to 8 columns, 512 for 16 (8 heads of 128, 4 columns: 64 contexts of up
// to 8191 tokens 75.6 us, in 512 shares 76.4, in 1024 76.9, in 256 79.7; 256 contexts
// of up to 2000 tokens 84.9, 86.6, 94.5 and 119.9; 8 of up to 8192 21.0, 19.9, 26.2 and
// 21.8; 16 columns, the 64 contexts, 89.5, in 768 shares 98.9, in 256 100.7).  Many
// columns: units are split while there are fewer than CUs, into parts of at least eight
// steps (four contexts of 4096 tokens by 128 queries 60 us, in one part 127).
static Plan4 plan4(int sequences, int heads, int group, int max_q, int64_t max_kv) {
    Plan4 p;
    const int64_t cols = (int64_t)max_q * group;
    p.columns = columns4(max_q, group);
    const int64_t units = (int64_t)sequences * heads * ((cols + p.columns - 1) / p.columns), steps = (max_kv + kStep - 1) / kStep;
    p.splits = 1;
    p.split_steps = (int)std::max<int64_t>(steps, 1);
    if (p.columns == 256) {
        const int64_t splits = std::min<int64_t>(256 / std::max<int64_t>(units, 1), steps / 8);
        if (splits > 1) {
            p.split_steps = (int)((steps + splits - 1) / splits);
            p.splits = (int)((steps + p.split_steps - 1) / p.split_steps);
        }
        p.whole = p.splits == 1;
        p.groups = units * p.splits;
        return p;
    }
    p.whole = steps <= kWholeSteps;
    const int64_t shares = (units * steps + kLeastSteps - 1) / kLeastSteps, resident = p.columns > 8 ? 512 : 768;
    p.groups = p.whole ? units : std::min(shares, resident);
    return p;
}
// places of partial results
static int64_t places4(const Plan4& p) { return p.whole ? 0 : p.groups * p.columns * (p.columns == 256 ? 1 : 2); }
static size_t workspace4(const Plan4& p, int sequences, int head_dim) {
    const size_t floats = p.whole ? 0 : (size_t)places4(p) * (head_dim + 2) + (size_t)sequences + 1;
    return (floats * sizeof(float) + 15) / 16 * 16;
}

// Sizes that the plan, the kernels' indexes and the launches hold: a grid has less than 2^32 threads, and where
// workgroups share out all steps, these are counted in 32 bits.
static bool shape4_ok(int sequences, int heads, int group, int max_q, int64_t max_kv) {
    if (sequences < 0 || heads < 1 || group < 1 || max_q < 0 || max_kv < 0 || sequences > (1 << 24) || heads > 65535 || group > 1024 ||
        (int64_t)max_q * group >= (1 << 30) || max_kv >= (1ll << 31) - 65536)
        return false;
    const int columns = columns4(max_q, group);
    const double units = (double)sequences * heads * (double)(((int64_t)max_q * group + columns - 1) / columns);
    const double rows = (double)sequences * max_q * heads * group;
    if (units > (double)(UINT32_MAX / (columns == 256 ? 512 : 256))) return false;
    if (columns == 256 || (max_kv + kStep - 1) / kStep <= kWholeSteps) return true;
    return units * (double)((max_kv + kStep - 1) / kStep + kUnitSteps) < 0x1p30 && rows <= (double)(UINT32_MAX / 256);
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_attention_kv4_workspace_size(int sequences, int tokens, int heads, int group, int head_dim, int max_q,
                                                  int64_t max_kv) {
    if (!shape4_ok(sequences, heads, group, max_q, max_kv) || tokens < 0 || head_dim < 1 || sequences == 0 || max_q == 0) return 0;
    return workspace4(plan4(sequences, heads, group, max_q, max_kv), sequences, head_dim);
}

extern "C" mq_status mq_attention_kv4(const mq_kv4_cache* cache, int sequences, int tokens, int group, int max_q, int64_t max_kv,
                                      mq_dtype type, const void* Q, int64_t q_token, int64_t q_head, const int32_t* page_table,
                                      int table_pages, const int32_t* kv_lens, const int32_t* cu_q, float scale, int causal,
                                      void* O, int64_t o_token, int64_t o_head, void* workspace, size_t ws_bytes,
                                      hipStream_t stream) {
    if (mq_status st = check_cache4(cache); st != MQ_OK) return st;
    if (sequences < 0 || tokens < 0 || group < 1 || max_q < 0 || max_kv < 0 || table_pages < 0 || !mq_host::is_half_type(type) ||
        !(scale > 0.0f) || !(scale < INFINITY) || (!cu_q && tokens != sequences))
        return MQ_ERR_INVALID_ARG;
    if (!shape4_ok(sequences, cache->heads, group, max_q, max_kv) || max_kv > (int64_t)table_pages * cache->page_size)
        return MQ_ERR_UNSUPPORTED_SHAPE;
    for (int64_t s : {q_token, q_head, o_token, o_head})
        if (s < 0 || s % 8 != 0) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (sequences == 0 || tokens == 0 || max_q == 0) return MQ_OK;
    if (!Q || !O || !kv_lens || (!page_table && table_pages > 0)) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(Q, 16) || !mq_host::aligned(O, 16) || !mq_host::aligned(page_table, 4) || !mq_host::aligned(kv_lens, 4) ||
        !mq_host::aligned(cu_q, 4) || !mq_host::aligned(workspace, 16))
        return MQ_ERR_MISALIGNED;
    const Plan4 p = plan4(sequences, cache->heads, group, max_q, max_kv);
    const size_t need = mq_attention_kv4_workspace_size(sequences, tokens, cache->heads, group, cache->head_dim, max_q, max_kv);
    if (need > 0 && (!workspace || ws_bytes < need)) return MQ_ERR_WORKSPACE;
    float* part = p.whole ? nullptr : static_cast<float*>(workspace);
    const int64_t rows = places4(p);
    const Attn4Args a{device_cache4(cache), Q, O, q_token, q_head, o_token, o_head, page_table, table_pages, (int)max_kv, kv_lens, cu_q,
                      sequences, tokens, group, max_q, scale, causal != 0, part, part ? part + rows * cache->head_dim : nullptr,
                      part ? part + rows * (cache->head_dim + 1) : nullptr,
                      part ? reinterpret_cast<int32_t*>(part + rows * (cache->head_dim + 2)) : nullptr, p.splits, p.split_steps};
    const int64_t joins = (int64_t)sequences * max_q * cache->heads * group;            // rows, where the launch is followed by a join
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        auto with_dim = [&](auto d) {
            constexpr int D = decltype(d)::value;
            auto run = [&](auto kernel, auto join) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)p.groups), dim3(256), 0, stream, a);
                if (!p.whole) hipLaunchKernelGGL(join, dim3((unsigned)joins), dim3(256), 0, stream, a);
            };
            if (p.columns == 256) {
                hipLaunchKernelGGL((attention4_wide_kernel<T, D>), dim3((unsigned)p.groups), dim3(512), 0, stream, a);
                const int64_t blocks = (joins + 1024 / D - 1) / (1024 / D);
                if (!p.whole) hipLaunchKernelGGL((attention4_join_wide_kernel<T, D>), dim3((unsigned)blocks), dim3(256), 0, stream, a, (int)joins);
            } else if (p.columns == 16) run(attention4_kernel<T, D, 16, 4>, attention4_join_kernel<T, D, 16>);
            else if (p.columns == 8) run(attention4_kernel<T, D, 8, 4>, attention4_join_kernel<T, D, 8>);
            else if (max_q * group > 2) run(attention4_kernel<T, D, 4, 4>, attention4_join_kernel<T, D, 4>);
            else if (max_q * group > 1) run(attention4_kernel<T, D, 4, 2>, attention4_join_kernel<T, D, 4>);
            else run(attention4_kernel<T, D, 4, 1>, attention4_join_kernel<T, D, 4>);
            return mq_host::launch_status();
        };
        return cache->head_dim == 64 ? with_dim(std::integral_constant<int, 64>{}) : with_dim(std::integral_constant<int, 128>{});
    });
}
