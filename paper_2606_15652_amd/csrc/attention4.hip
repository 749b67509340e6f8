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
// The scores are computed transposed, S^T = K Q^T: a lane then holds four
// neighbouring tokens of one query, which is what the second product, O^T =
// V^T P^T, takes from it.  Nothing goes through LDS but the waves' results.
//
// Columns are the queries of one sequence and key head: position qi and head hg
// of the group at column qi group + hg.
#include "kv4.h"

#include <float.h>
#include <math.h>

namespace mq {

mq_status check_cache4(const mq_kv4_cache* c);
Cache4 device_cache4(const mq_kv4_cache* c);

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;               // tokens that a wave takes at a time
constexpr int kMostSplits = 64;         // of a sequence's tokens
constexpr float kLowest = -1e30f;       // below every score: running maximum of none
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
    int splits, chunk;                  // tokens of a split, a multiple of kStep
    float *part_o, *part_m, *part_l;    // [split][token][head] (x D)
};

// A sequence's queries and tokens.
struct Sequence {
    int q0, nq, n;
};
__device__ __forceinline__ Sequence sequence(const Attn4Args& a, int b) {
    Sequence s;
    if (a.cu_q) {
        s.q0 = min(max(a.cu_q[b], 0), a.tokens);
        s.nq = min(max(min(a.cu_q[b + 1], a.tokens) - s.q0, 0), a.max_q);
    } else {
        s.q0 = b;
        s.nq = 1;
    }
    s.n = min(max(a.kv_lens[b], 0), a.max_kv);
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

// Operands and scales of 16 columns of queries: fp16, each column scaled by a power of two (its largest
// value near 2^8, so that neither type's range matters), channels of the codes that come 16 times too
// large divided by 16.  A lane has the channels (D / 4) g .. of its column.
template <int D>
struct Queries {
    f16x8 op[D / 32];
    // x = sk (q'.n) + zk of_minimum is the score over to_score, in powers of 2
    float to_score, of_minimum;

    template <typename T>
    __device__ __forceinline__ void load(const T* q, float scale) {
        f32x8 x[D / 32];
        float sum = 0.0f, amax = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            x[i] = load8(q + 8 * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum += x[i][e];
                amax = fmaxf(amax, fabsf(x[i][e]));
            }
        }
        sum = quads_sum(sum);
        amax = quads_max(amax);
        const int up = amax > 0.0f && amax < INFINITY ? 8 - ilogbf(amax) : 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = ldexpf(x[i][e], e & 2 ? up - 4 : up);
            op[i] = __builtin_convertvector(x[i], f16x8);
        }
        // never zero or infinite, so that a hidden token's -infinity stays that
        to_score = fminf(fmaxf(ldexpf(scale * kLog2e, 24 - up), FLT_MIN), FLT_MAX);
        of_minimum = ldexpf(sum, up - 24);
    }
};

// A result row (or part of one) of column col, not yet divided by the weights' sum: to the output, or
// with splits to the partial results.
template <typename T, int D, int N>
__device__ __forceinline__ void store_result(const Attn4Args& a, const Sequence& s, int head, int split, int col, int channel,
                                             const float (&values)[N], float mx, float sum, bool first) {
    const int qi = col / a.group, h = head * a.group + col % a.group;
    if (a.splits > 1) {
        const int64_t row = ((int64_t)split * a.tokens + s.q0 + qi) * (a.c.heads * a.group) + h;
#pragma unroll
        for (int e = 0; e < N; e += 4)
            *reinterpret_cast<f32x4*>(a.part_o + row * D + channel + e) = f32x4{values[e], values[e + 1], values[e + 2], values[e + 3]};
        if (first) {
            a.part_m[row] = mx;
            a.part_l[row] = sum;
        }
    } else {
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;       // a row that sees nothing is 0
        T* o = static_cast<T*>(a.o) + (s.q0 + qi) * a.o_token + h * a.o_head + channel;
        typedef T half4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int e = 0; e < N; e += 4)
            *reinterpret_cast<half4*>(o + e) = __builtin_convertvector(
                (f32x4{values[e] * by, values[e + 1] * by, values[e + 2] * by, values[e + 3] * by}), half4);
    }
}

// --------------------------------------------------------------------------
// Few columns: codes go from memory to registers and into the products.
// --------------------------------------------------------------------------
// What a wave loads for 16 tokens: lane (r, g) has token r's key channels
// (D / 4) g .., the tokens 4 g .. + 3's value channels (D / 16) r .. and parameters.
template <int D>
struct Tile4 {
    uint32_t k[D / 32], v[D / 32];
    u32x4 kp, vp;
};
// The pages of a step's two tiles (the last token's where a tile is past the end: its page is there to be
// read); negative: outside the cache.
struct Pages {
    int of[2];
};
__device__ __forceinline__ Pages find_pages(const Attn4Args& a, int b, int t, int last) {
    Pages p;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int page = a.table[(int64_t)b * a.table_pages + (min(t + 16 * h, last) >> a.c.page_bits)];
        p.of[h] = __builtin_amdgcn_readfirstlane((uint32_t)page < (uint32_t)a.c.pages ? page : -1);
    }
    return p;
}
template <int D>
__device__ __forceinline__ void load_tile(Tile4<D>& x, const Attn4Args& a, int head, int page, int t, int lane) {
    const int r = lane & 15, g = lane >> 4;
    const int64_t row = (((int64_t)max(page, 0) * a.c.heads + head) << a.c.page_bits) + (t & ((1 << a.c.page_bits) - 1));
    const uint8_t* k = a.c.k + row * (D / 2);
    const uint8_t* v = a.c.v + row * (D / 2);
    __builtin_memcpy(x.k, __builtin_assume_aligned(k + (uint32_t)(r * (D / 2) + g * (D / 8)), D / 8), D / 8);
    __builtin_memcpy(x.v, __builtin_assume_aligned(v + (uint32_t)(g * (2 * D) + r * (D / 8)), D / 8), D / 8);
    x.kp = *reinterpret_cast<const u32x4*>(a.c.kp + row + (uint32_t)(4 * g));
    x.vp = *reinterpret_cast<const u32x4*>(a.c.vp + row + (uint32_t)(4 * g));
}

// Every wave takes all the columns (16 C) and a share of the tokens; the step after
// the one in hand is loaded meanwhile.  The parameters stay fp16 and are widened
// inside mixed multiply-adds.  Weights w = p sv (in units of `unit`, at least every
// sv) are rounded to fp16 for the second product, of which 7.5 sum(w) is taken off
// again: codes about their middle, so that the rounding of w counts against values
// about their middle.
template <typename T, int D, int C>
__global__ __launch_bounds__(256) void attention4_kernel(Attn4Args a) {
    constexpr int KK = D / 32, VT = D / 16, WT = 4, Cols = 16 * C;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int blocks = (a.max_q * a.group + Cols - 1) / Cols;
    int u = blockIdx.x;
    const int split = u % a.splits;
    u /= a.splits;
    const int col0 = u % blocks * Cols;
    u /= blocks;
    const int head = u % a.c.heads, b = u / a.c.heads;
    const Sequence s = sequence(a, b);
    const int cols = s.nq * a.group;
    if (col0 >= cols) return;
    const int low = visible(a, s, col0 / a.group), high = visible(a, s, (min(col0 + Cols, cols) - 1) / a.group);
    const int64_t first = (int64_t)split * a.chunk;
    if (a.splits > 1 && first >= high) return;
    const int begin = (int)first + wave * kStep, end = (int)min((int64_t)high, first + a.chunk);
    constexpr int stride = kStep * WT;

    Tile4<D> tile[2];
    Pages pages{}, next{};
    if (begin < end) {
        pages = find_pages(a, b, begin, end - 1);
        next = find_pages(a, b, begin + stride, end - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) load_tile<D>(tile[h], a, head, pages.of[h], begin + 16 * h, lane);
    }
    Queries<D> q[C];
    int limit[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int col = min(col0 + 16 * j + r, cols - 1), qi = col / a.group;
        limit[j] = visible(a, s, qi);
        q[j].load(static_cast<const T*>(a.q) + (s.q0 + qi) * a.q_token + (head * a.group + col % a.group) * a.q_head + g * (D / 4), a.scale);
    }

    f32x4 acc[C][VT] = {};
    float m[C], l[C] = {}, zs[C] = {}, ws[C] = {};
    float unit = 0.0f, per_unit = 0.0f;
#pragma unroll
    for (int j = 0; j < C; ++j) m[j] = kLowest;

    for (int t = begin; t < end; t += stride) {
        const Tile4<D> now[2] = {tile[0], tile[1]};
        const bool all = pages.of[0] >= 0 && pages.of[1] >= 0, there[2] = {pages.of[0] >= 0, pages.of[1] >= 0};
        pages = next;
        if (t + stride < end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) load_tile<D>(tile[h], a, head, pages.of[h], t + stride + 16 * h, lane);
            next = find_pages(a, b, t + 2 * stride, end - 1);
        }
        f32x4 x[C][2] = {};
        f16x2 vp[2][4];                                     // scale, minimum; finite
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < KK; ++i) {
                const f16x8 k = key_operand(now[h].k[i]);
#pragma unroll
                for (int j = 0; j < C; ++j) x[j][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[j].op[i], x[j][h], 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t kw = now[h].kp[e], vw = now[h].vp[e];
                const f16x2 kp = __builtin_bit_cast(f16x2, kw), v = __builtin_bit_cast(f16x2, vw);
                // a value row that is not finite makes the score NaN, for the queries that see it
                const float bad = __builtin_fmaf((float)v[0], 0.0f, __builtin_fmaf((float)v[1], 0.0f, 0.0f));
                vp[h][e] = __builtin_elementwise_max(v, (f16x2)(_Float16)-65504.0f);    // and its weight 0 stays 0
#pragma unroll
                for (int j = 0; j < C; ++j)
                    x[j][h][e] = __builtin_fmaf(x[j][h][e], (float)kp[0], __builtin_fmaf((float)kp[1], q[j].of_minimum, bad));
            }
        }
        if (t + kStep > low || !all) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int token = t + 16 * h + 4 * g + e;
                    if (!there[h] || token >= end) vp[h][e] = f16x2{};                  // whatever memory holds there
#pragma unroll
                    for (int j = 0; j < C; ++j)
                        if (!there[h] || token >= limit[j]) x[j][h][e] = -INFINITY;
                }
        }
        float top[C];
        bool moves = false;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            top[j] = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[j] = fmaxf(top[j], x[j][h][e]);
            top[j] *= q[j].to_score;
            moves = moves || top[j] > m[j] + kSlack;
        }
        // the largest scale, and minimum, of which only the scale is used
        f16x2 both = __builtin_elementwise_max(vp[0][0], vp[0][1]);
#pragma unroll
        for (int i = 2; i < 8; ++i) both = __builtin_elementwise_max(both, vp[i / 4][i % 4]);
        const float most = (float)both[0];
        moves = moves || most > unit;
        if (__any(moves)) {
            const float old = unit;
            unit = fmaxf(unit, 2.0f * quads_max(most));
            per_unit = unit > 0.0f ? 1.0f / unit : 0.0f;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const float to = fmaxf(m[j], quads_max(top[j])), down = __builtin_amdgcn_exp2f(m[j] - to);
                m[j] = to;
                l[j] *= down;
                zs[j] *= down;
                ws[j] *= down * (old * per_unit);
#pragma unroll
                for (int i = 0; i < VT; ++i) acc[j][i] *= down * (old * per_unit);
            }
        }
        f16x8 p[C];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float sv[4], middle[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sv[e] = (float)vp[h][e][0] * per_unit;
                middle[e] = __builtin_fmaf((float)vp[h][e][0], 7.5f, (float)vp[h][e][1]);
            }
#pragma unroll
            for (int j = 0; j < C; ++j) {
                f32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float pe = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j][h][e], q[j].to_score, -m[j]));
                    l[j] += pe;
                    zs[j] = __builtin_fmaf(pe, middle[e], zs[j]);
                    w[e] = pe * sv[e];
                }
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const f16x2 pair = __builtin_convertvector((f32x2{w[e], w[e + 1]}), f16x2);
                    ws[j] = __builtin_amdgcn_fdot2(pair, (f16x2)(_Float16)1.0f, ws[j], false);
                    p[j][4 * h + e] = pair[0];
                    p[j][4 * h + e + 1] = pair[1];
                }
            }
        }
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            const uint32_t a0 = now[0].v[2 * h], a1 = now[0].v[2 * h + 1], b0 = now[1].v[2 * h], b1 = now[1].v[2 * h + 1];
            const f16x8 v[4] = {value_operand<0>(a0, a1, b0, b1), value_operand<1>(a0, a1, b0, b1),
                                value_operand<2>(a0, a1, b0, b1), value_operand<3>(a0, a1, b0, b1)};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < C; ++j)
                    acc[j][4 * h + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[i], p[j], acc[j][4 * h + i], 0, 0, 0);
        }
    }

    // The lane's column and its D / 4 channels (D / 4) g .., not yet divided by the weights' sum; joined over the waves.
    __shared__ float shared_o[WT][Cols][D + 4];
    __shared__ float shared_m[WT][Cols], shared_l[WT][Cols];
    const float of_unit = unit * 0x1p24f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int col = 16 * j + r;
        const float rest = quads_sum(__builtin_fmaf(-7.5f * unit, ws[j], zs[j])), sum = quads_sum(l[j]);
        float out[D / 4];
#pragma unroll
        for (int i = 0; i < VT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e * VT + i] = __builtin_fmaf(acc[j][i][e], of_unit * (i % 2 ? 0.0625f : 1.0f), rest);
        if (col0 + col < cols) {
#pragma unroll
            for (int e = 0; e < D / 4; e += 4)
                *reinterpret_cast<f32x4*>(&shared_o[wave][col][g * (D / 4) + e]) = f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]};
        }
        if (g == 0) {
            shared_m[wave][col] = m[j];
            shared_l[wave][col] = sum;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < Cols * (D / 4); i += 256) {
        const int col = i / (D / 4), ch = 4 * (i % (D / 4));
        if (col0 + col >= cols) break;
        float mx = shared_m[0][col], sum = 0.0f, o[4] = {};
#pragma unroll
        for (int w = 1; w < WT; ++w) mx = fmaxf(mx, shared_m[w][col]);
#pragma unroll
        for (int w = 0; w < WT; ++w) {
            const float by = __builtin_amdgcn_exp2f(shared_m[w][col] - mx);
            sum = __builtin_fmaf(shared_l[w][col], by, sum);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(shared_o[w][col][ch + e], by, o[e]);
        }
        store_result<T, D, 4>(a, s, head, split, col0 + col, ch, o, mx, sum, ch == 0);
    }
}

// Joins the splits of a row, one wave a row: lane i weighs split i.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention4_join_kernel(Attn4Args a) {
    const int lane = threadIdx.x & 63;
    const int64_t u = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = a.c.heads * a.group, head = (int)(u % heads), qi = (int)(u / heads % a.max_q);
    const int64_t b = u / heads / a.max_q;
    if (b >= a.sequences) return;
    const Sequence s = sequence(a, (int)b);
    if (qi >= s.nq) return;
    const int seen = visible(a, s, qi), active = seen > 0 ? (seen - 1) / a.chunk + 1 : 0;   // at most a.splits: chunk splits >= n
    const int64_t row = (int64_t)(s.q0 + qi) * heads + head, step = (int64_t)a.tokens * heads;
    const bool mine = lane < min(active, a.splits);
    const float m = mine ? a.part_m[row + lane * step] : kLowest;
    float mx = m;
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
    const float by = mine ? exp2f(m - mx) : 0.0f;
    float sum = mine ? by * a.part_l[row + lane * step] : 0.0f;
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) sum += __shfl_xor(sum, i);
    constexpr int N = D / 64;
    float o[N] = {};
    for (int i = 0; i < min(active, a.splits); ++i) {
        const float w = __shfl(by, i);
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = __builtin_fmaf(a.part_o[(row + i * step) * D + lane * N + e], w, o[e]);
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* out = static_cast<T*>(a.o) + (s.q0 + qi) * a.o_token + head * a.o_head + lane * N;
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = (T)(o[e] * inv);
}

// ---------------------------------------------------------------- host side --
struct Plan4 {
    int columns;                        // of a workgroup
    int blocks, splits, chunk;
};

static Plan4 plan4(int sequences, int heads, int group, int max_q, int64_t max_kv) {
    Plan4 p;
    const int64_t cols = (int64_t)max_q * group;
    p.columns = cols <= 16 ? 16 : 32;
    p.blocks = (int)((cols + p.columns - 1) / p.columns);
    const int64_t units = (int64_t)sequences * heads * p.blocks, least = 4 * kStep;
    int64_t splits = (1024 + units - 1) / units;
    splits = splits > kMostSplits ? kMostSplits : splits;
    const int64_t room = (max_kv + least - 1) / least;
    splits = splits > room ? room : splits;
    if (splits < 1) splits = 1;
    const int64_t chunk = ((max_kv + splits - 1) / splits + least - 1) / least * least;
    p.chunk = (int)(chunk < least ? least : chunk > (INT32_MAX / least) * least ? (INT32_MAX / least) * least : chunk);
    p.splits = splits == 1 ? 1 : (int)((max_kv + p.chunk - 1) / p.chunk);
    return p;
}

static bool shape4_ok(int sequences, int heads, int group, int max_q, int64_t max_kv) {
    return sequences >= 0 && heads >= 1 && group >= 1 && max_q >= 0 && max_kv >= 0 && sequences <= (1 << 24) && heads <= 65535 &&
           group <= 1024 && (int64_t)max_q * group < (1 << 30) && max_kv < (1ll << 31) - 65536;
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_attention_kv4_workspace_size(int sequences, int tokens, int heads, int group, int head_dim, int max_q,
                                                  int64_t max_kv) {
    if (!shape4_ok(sequences, heads, group, max_q, max_kv) || tokens < 0 || head_dim < 1 || sequences == 0 || max_q == 0) return 0;
    const Plan4 p = plan4(sequences, heads, group, max_q, max_kv);
    return p.splits == 1 ? 0 : (size_t)p.splits * tokens * heads * group * (head_dim + 2) * sizeof(float);
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
    const int64_t rows = (int64_t)p.splits * tokens * cache->heads * group;
    float* part = static_cast<float*>(workspace);
    const Attn4Args a{device_cache4(cache), Q, O, q_token, q_head, o_token, o_head, page_table, table_pages, (int)max_kv, kv_lens, cu_q,
                      sequences, tokens, group, max_q, scale, causal != 0, p.splits, p.chunk, part,
                      part ? part + rows * cache->head_dim : nullptr, part ? part + rows * (cache->head_dim + 1) : nullptr};
    const int64_t grid = (int64_t)sequences * cache->heads * p.blocks * p.splits;
    const int64_t joins = ((int64_t)sequences * max_q * cache->heads * group + 3) / 4;
    if (grid > INT32_MAX || joins > INT32_MAX) return MQ_ERR_UNSUPPORTED_SHAPE;
    return mq_host::with_half_type(type, [&](auto z) {
        using T = decltype(z);
        auto run = [&](auto d) {
            constexpr int D = decltype(d)::value;
            if (p.columns == 16) hipLaunchKernelGGL((attention4_kernel<T, D, 1>), dim3((unsigned)grid), dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((attention4_kernel<T, D, 2>), dim3((unsigned)grid), dim3(256), 0, stream, a);
            if (p.splits > 1) hipLaunchKernelGGL((attention4_join_kernel<T, D>), dim3((unsigned)joins), dim3(256), 0, stream, a);
            return mq_host::launch_status();
        };
        return cache->head_dim == 64 ? run(std::integral_constant<int, 64>{}) : run(std::integral_constant<int, 128>{});
    });
}
