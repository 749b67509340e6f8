// A token drawn from the logits of each row.
//
//   w_i = exp((x_i - max x) / T);  order: x descending, the index ascending among equals;
//   kept: of the first top_k the shortest beginning whose sum is top_p of theirs, and of it those with w >= min_p;
//   the first kept token whose running sum passes u times the sum of all kept.
//
// Weights are whole numbers of 2^-43 (fp64 rounded): sums of up to 2^20 of them fit
// 64 bits, are exact and the same in every order, so that atomics may make them.
// One workgroup takes a row:
//  1. the row's maximum (and whether a value is NaN);
//  2. with top_k, a logit that k are not below: if few enough are not, those are listed in LDS, and the rest is done there;
//  3. otherwise counts and sums by bins of d = (max - x) log2(e) / T, kBinsPerUnit to a factor of two: a bin's tokens all
//     come before those of the next, and what has d >= kUnits has the weight 0 and no part in any of it;
//  4. in turn the k-th token, the end of top_p and the drawn token: the bin that it is in, whose tokens are listed, then
//     one of 1024 parts of the list, whose few tokens one wave compares.  A bin of more than kList tokens is split by
//     the logit's bits first (equal logits by the index's).
// A bin is a range of logits, found once, so passes that look for its tokens only compare.
//
// 1 x 32003 fp32 with top-k and top-p 22 us, which barriers and the first run through the code bound; 128 x 131071 with
// all filters 48 us, reading the rows twice by 128 CUs; 203 x 50000 bf16 with top-p alone 66 us, of which the
// exponentials in 64 bits and their additions in LDS are 22.  Temperature 0: 8.7, 23.6 and 11.2 us.  1024 threads leave a
// wave 128 registers: 30 vector ones are spilled for fp32 logits (11 for 16-bit ones), and 130 scalar ones to lanes of others.
#include "mq_float.h"

#include <float.h>

#include <type_traits>

namespace mq {

constexpr int kShift = 43;              // weights are multiples of 2^-kShift
static_assert(MQ_SAMPLE_MAX_VOCAB == 1 << (63 - kShift), "sums fit 64 bits");
constexpr int kThreads = 1024;
constexpr int kUnits = 45;              // weights below 2^-44 round to 0
constexpr int kBins = 2048;
constexpr double kBinsPerUnit = 45.5;   // kUnits of them fill the bins
constexpr int kList = 4096;             // tokens that are sorted in LDS

struct SampleArgs {
    const void* x;
    int64_t ldx;
    int rows, vocab;
    const float *u, *temperature, *top_p, *min_p;       // of each row, or null
    const int32_t* top_k;
    float temperature1, top_p1, min_p1;                 // for all rows, where there is no pointer
    int top_k1;
    int64_t* tokens;
    float* probs;
};

// Larger keys for larger values; -0 and +0 have one.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

// 2^-d in units of 2^-kShift for 0 <= d: of the fraction by its series (relative error below 2^-46), then rounded: a sum
// with 2^52 has the whole number in its low bits.
__device__ __forceinline__ uint64_t weight_of(double d) {
    if (!(d < kUnits)) return 0;                        // (infinite and NaN, too)
    const double n = rint(d), f = (n - d) * 0.69314718055994530942;     // |f| <= 0.3466
    double y = 1.0 / 39916800.0;                        // 1 / 11!
    y = __builtin_fma(y, f, 1.0 / 3628800.0);
    y = __builtin_fma(y, f, 1.0 / 362880.0);
    y = __builtin_fma(y, f, 1.0 / 40320.0);
    y = __builtin_fma(y, f, 1.0 / 5040.0);
    y = __builtin_fma(y, f, 1.0 / 720.0);
    y = __builtin_fma(y, f, 1.0 / 120.0);
    y = __builtin_fma(y, f, 1.0 / 24.0);
    y = __builtin_fma(y, f, 1.0 / 6.0);
    y = __builtin_fma(y, f, 0.5);
    y = __builtin_fma(y, f, 1.0);
    y = __builtin_fma(y, f, 1.0);
    const double up = 4503599627370496.0;               // 2^52
    return (uint64_t)__double_as_longlong(ldexp(y, kShift - (int)n) + up) - (uint64_t)__double_as_longlong(up);
}

// f s rounded down (or UP) for 0 <= f < 1: f = m 2^-k, exactly.
template <bool UP>
__device__ __forceinline__ uint64_t part_of(float f, uint64_t s) {
    const uint32_t b = __float_as_uint(f);
    const int e = (int)(b >> 23), k = 150 - (e ? e : 1);    // k >= 24
    const uint64_t m = e ? (b & 0x7FFFFFu) | 0x800000u : b;
    const unsigned __int128 p = (unsigned __int128)m * s;
    if (k >= 96) return UP && p ? 1 : 0;                    // p < 2^88
    return (uint64_t)((p + (UP ? ((unsigned __int128)1 << k) - 1 : 0)) >> k);
}

struct Row {
    double slope, max;                  // log2(e) / T, the largest logit
    // 0 for the largest, infinite or NaN for what has no weight
    __device__ __forceinline__ double distance(float x) const { return (double)x == max ? 0.0 : (max - (double)x) * slope; }
};
// Bins ascend with the distance (every operation keeps order), so a bin's tokens come before the next one's.
__device__ __forceinline__ int bin_of(double d) { return d < kBins / kBinsPerUnit ? (int)(d * kBinsPerUnit) : kBins; }

struct SampleLds {
    uint64_t sums[kBins];               // of the bins, then running, the bin's own among it
    uint32_t counts[kBins];
    uint64_t part_sums[kThreads];       // of parts of the list, running; of a long bin's parts
    uint32_t part_counts[kThreads];
    uint32_t few_keys[64];              // one part of the list
    int32_t few_at[64];
    uint32_t keys[kList];               // the list: larger first
    int32_t at[kList];
    uint64_t scan[kThreads / 64];
    uint32_t scan_counts[kThreads / 64];
    uint32_t listed, few, bounds[2];
    int found, token, nan;
    uint64_t found_before, found_count, found_tokens, found_sum, found_weight;
    float best[kThreads / 64];
};

// The least float x (as its key) with before(x), which holds for all from there to the key `top`: six bits of it at a time, by
// every wave.
template <typename F>
__device__ __forceinline__ uint32_t least_key(uint32_t top, F&& before) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t key = 0;
#pragma unroll 1
    for (int shift = 26; shift > -6; shift -= 6) {
        // the first of 64 ranges of keys whose last one says yes (the last round: of 4 keys)
        const int down = shift < 0 ? 0 : shift;
        const uint32_t k = key + (lane << down) + ((1u << down) - 1u);
        const uint64_t yes = __ballot((k >= top || k < key) || before(value_of_key(k)));
        key += (uint32_t)__builtin_ctzll(yes) << down;
    }
    return key;
}

// Inclusive running sums over the wave, by DPP: within rows of 16 lanes, then the rows' sums carried on.
__device__ __forceinline__ void scan_wave(uint64_t& v, uint32_t& c) {
    auto step = [&](auto ctrl, auto rows) {
        auto from = [&](uint32_t x) {
            return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, true);
        };
        const uint32_t lo = from((uint32_t)v), hi = from((uint32_t)(v >> 32)), n = from(c);
        v += (uint64_t)hi << 32 | lo;
        c += n;
    };
    constexpr std::integral_constant<int, 0xf> every{};
    step(std::integral_constant<int, 0x111>{}, every);                              // row_shr:1, 2, 4, 8
    step(std::integral_constant<int, 0x112>{}, every);
    step(std::integral_constant<int, 0x114>{}, every);
    step(std::integral_constant<int, 0x118>{}, every);
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}); // row_bcast:15, to rows 1 and 3
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}); // row_bcast:31, to rows 2 and 3
}

// Inclusive running sums (and numbers) over the workgroup's threads, and the sum (and number) of all.
__device__ __forceinline__ void scan_threads(SampleLds& L, uint64_t& v, uint32_t& c, uint64_t& all, uint32_t& all_count) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    scan_wave(v, c);
    __syncthreads();
    if (lane == 63) {
        L.scan[wave] = v;
        L.scan_counts[wave] = c;
    }
    __syncthreads();
    all = 0;
    all_count = 0;
    uint64_t before = 0;
    uint32_t before_count = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w == wave) {
            before = all;
            before_count = all_count;
        }
        all += L.scan[w];
        all_count += L.scan_counts[w];
    }
    v += before;
    c += before_count;
}

// f(v, i, E) for E logits v of the row at i(j), j < E, at a time: all of them, by all threads, AHEAD loads at once and the
// next ones on their way meanwhile.  Where fewer are left the rest of v is -infinity, which is nothing to any of the passes.
template <int AHEAD, typename T, typename F>
__device__ __forceinline__ void for_parts(const T* x, int n, F&& f) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int per = 16 / sizeof(T);
    // up to the first 16-byte border one by one
    const int head = min(n, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T)), body = (n - head) / per;
    const vec* v = reinterpret_cast<const vec*>(x + head);
    auto load = [&](vec (&y)[AHEAD], int c) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            y[a] = (vec)(T)-INFINITY;
            if (c + a * kThreads < body) y[a] = v[c + a * kThreads];
        }
    };
    vec y[AHEAD], next[AHEAD];
    load(y, threadIdx.x);
    for (int c = threadIdx.x; c < body; c += AHEAD * kThreads) {
        load(next, c + AHEAD * kThreads);
        float z[AHEAD * per];
#pragma unroll
        for (int j = 0; j < AHEAD * per; ++j) z[j] = (float)y[j / per][j % per];
        f(z, [&](int j) { return head + (c + j / per * kThreads) * per + j % per; }, std::integral_constant<int, AHEAD * per>{});
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) y[a] = next[a];
    }
    const int rest = n - body * per;                        // fewer than 2 per: one for each of the first threads
    if ((int)threadIdx.x < rest) {
        const int i = (int)threadIdx.x < head ? threadIdx.x : body * per + threadIdx.x;
        const float z[1] = {(float)x[i]};
        f(z, [&](int) { return i; }, std::integral_constant<int, 1>{});
    }
}
template <int AHEAD, typename T, typename F>
__device__ __forceinline__ void for_row(const T* x, int n, F&& f) {
    for_parts<AHEAD>(x, n, [&](const auto& v, auto&& at, auto each) {
#pragma unroll
        for (int j = 0; j < decltype(each)::value; ++j) f(v[j], at(j));
    });
}

// One step of a bitonic sort among a wave's lanes: element i and the one at i ^ j, in stage k.
__device__ __forceinline__ void sort_step(uint32_t& key, int& at, int i, int j, int k) {
    const uint32_t ok = (uint32_t)__shfl_xor((int)key, j);
    const int oa = __shfl_xor(at, j);
    const bool other_first = ok > key || (ok == key && oa < at);
    // the lower of the pair keeps the first where the stage ascends, the upper one the second
    if (other_first == (((i & j) == 0) == ((i & k) == 0))) {
        key = ok;
        at = oa;
    }
}

// Sorts the list (keys descending, index ascending among equals): bitonic, a wave's 64 neighbours by their lanes, further
// ones through LDS.
__device__ __forceinline__ void sort_list(SampleLds& L, int n) {
    const int t = threadIdx.x, lane = t & 63;
    int size = 64;
    while (size < n) size <<= 1;
    for (int i = n + t; i < size; i += kThreads) {
        L.keys[i] = 0;
        L.at[i] = INT32_MAX;
    }
    __syncthreads();
    // the steps j, j / 2, .. 1 of stage k for the elements that this wave holds, 64 at a time
    auto by_lanes = [&](int first_stage, int last_stage, int most) {
        for (int base = t - lane; base < size; base += kThreads) {
            const int i = base + lane;
            uint32_t key = L.keys[i];
            int at = L.at[i];
            for (int k = first_stage; k <= last_stage; k <<= 1)
                for (int j = min(k >> 1, most); j > 0; j >>= 1) sort_step(key, at, i, j, k);
            L.keys[i] = key;
            L.at[i] = at;
        }
        __syncthreads();
    };
    by_lanes(2, 64, 32);
    for (int k = 128; k <= size; k <<= 1) {
        for (int j = k >> 1; j >= 64; j >>= 1) {
            for (int p = t; p < size / 2; p += kThreads) {
                const int a = (p & ~(j - 1)) * 2 + (p & (j - 1)), b = a + j;
                const uint32_t ka = L.keys[a], kb = L.keys[b];
                const int ia = L.at[a], ib = L.at[b];
                const bool first = ka > kb || (ka == kb && ia < ib);    // a comes before b
                if (first != ((a & k) == 0)) {
                    L.keys[a] = kb;
                    L.keys[b] = ka;
                    L.at[a] = ib;
                    L.at[b] = ia;
                }
            }
            __syncthreads();
        }
        by_lanes(k, k, 32);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    __shared__ SampleLds L;
    const int r = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6, n = a.vocab;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const float temperature = a.temperature ? a.temperature[r] : a.temperature1;
    const float top_p = a.top_p ? a.top_p[r] : a.top_p1, min_p = a.min_p ? a.min_p[r] : a.min_p1;
    const int top_k = a.top_k ? a.top_k[r] : a.top_k1;
    const float u = a.u ? a.u[r] : 0.0f;

    // 1. the maximum, the two largest that this thread has seen, and whether there is a NaN
    float best = -INFINITY, second = -INFINITY;
    uint32_t bits = 0;
    for_row<4>(x, n, [&](float v, int) {
        second = fmaxf(second, fminf(best, v));
        best = fmaxf(best, v);
        bits = max(bits, __float_as_uint(v) & 0x7FFFFFFFu);
    });
    const float first = best;
    const bool nan = __ballot(bits > kFloatInf) != 0;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) best = fmaxf(best, __shfl_xor(best, m));
    if (t == 0) {
        L.nan = 0;
        L.token = INT32_MAX;
    }
    for (int i = t; i < kBins; i += kThreads) {
        L.sums[i] = 0;
        L.counts[i] = 0;
    }
    __syncthreads();
    if (lane == 0) {
        L.best[wave] = best;
        if (nan) L.nan = 1;
    }
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w) best = fmaxf(best, L.best[w]);
    auto answer = [&](int64_t token, float p) {
        a.tokens[r] = token;
        a.probs[r] = p;
    };
    if (L.nan || best == -INFINITY) {                   // nothing to draw from
        if (t == 0) answer(-1, L.nan ? __builtin_nanf("") : 0.0f);
        return;
    }
    if (!(temperature > 0.0f)) {                        // the first of its places
        int at = INT32_MAX;
        for_row<4>(x, n, [&](float v, int i) { at = v == best && i < at ? i : at; });
        if (at != INT32_MAX) atomicMin(&L.token, at);
        __syncthreads();
        if (t == 0) answer(L.token, 1.0f);
        return;
    }
    const Row row{1.4426950408889634074 / (double)temperature, (double)best};

    const uint32_t top = order_key(best);
    const uint64_t least = min_p > 0.0f ? (uint64_t)ceil((double)fminf(min_p, 1.0f) * (double)(1ull << kShift)) : 0;
    auto drawn = [&](uint64_t sum) { return u < 1.0f ? part_of<false>(fmaxf(u, 0.0f), sum) : sum - 1; };
    // the least beginning with a sum of top_p of it at least: it passes that less one
    auto cut = [&](uint64_t sum) { return max(part_of<true>(fmaxf(top_p, 0.0f), sum), (uint64_t)1) - 1; };
    auto add = [](uint64_t& to, uint64_t w) { atomicAdd(reinterpret_cast<unsigned long long*>(&to), (unsigned long long)w); };
    // a token's place in the order: 32 bits of its logit, the larger the lower, and 20 of its index
    constexpr int BITS = 52;
    auto place = [](float v, int i) { return (uint64_t)~order_key(v) << 20 | (uint64_t)i; };
    static_assert(kBins == 2 * kThreads, "two bins a thread");

    // The list: tokens in question, in any order, before which there are `before_count` with the sum `before`.  Thread t has
    // its tokens t, t + 1024, ..: their weights, and in which of 1024 equal ranges they are (by key, and by index among equals).
    constexpr int EACH = kList / kThreads;
    uint64_t w[EACH], before = 0, before_count = 0;
    uint32_t part[EACH];
    bool all_listed = false, sorted = false;            // whether it has every token in question; whether it is in order
    int in_list = -1;                                   // the bin that it holds
    uint64_t sum = 0, kept = 0, count = 0;              // of all tokens in question, of those that min_p keeps; their number

    // Turn -1: the list of few tokens down to the k-th, or the sums by bins.  Then in turn the k-th token, the end of top_p, the drawn
    // token.  (Every step has one place in the code: what a workgroup runs through once is bound by its loading.)
#pragma unroll 1
    for (int turn = -1; turn < 3; ++turn) {
        const bool by_count = turn == 0;
        if (by_count ? top_k <= 0 || (uint64_t)top_k >= count : turn == 1 && !(top_p < 1.0f)) continue;
        if (turn == 2 && least) sum = min(sum, kept);
        const uint64_t target = by_count ? (uint64_t)top_k - 1 : turn == 1 ? cut(sum) : turn == 2 ? drawn(sum) : 0;
        int bin = -1;
        __syncthreads();
        if (t == 0) L.found = -1;
        __syncthreads();
        if (turn < 0 && top_k > 0 && top_k <= 3 * kThreads / 2) {
            // The k-th largest of the threads' two largest logits is no more than the k-th of all, so its bin is the last in
            // question.  Of logits in no order, k = 1000 of the 2048 are found among some 1130 tokens, 1536 among 2070; where
            // they are more than the list holds, the sums by bins are taken.
            for (float v : {first, second})
                if (const int b = bin_of(row.distance(v)); b < kBins) atomicAdd(&L.counts[b], 1u);
            __syncthreads();
            const uint32_t c0 = L.counts[2 * t], c1 = L.counts[2 * t + 1], k = (uint32_t)top_k;
            uint64_t zero = 0, none;
            uint32_t down = c0 + c1, number;
            scan_threads(L, zero, down, none, number);
            if (down - c1 - c0 < k && k <= down) L.found = down - c1 >= k ? 2 * t : 2 * t + 1;
            L.counts[2 * t] = L.counts[2 * t + 1] = 0;
            __syncthreads();
            bin = L.found;
        } else if (turn >= 0 && !all_listed) {
            for (int b = 2 * t; b < 2 * t + 2; ++b) {
                const uint64_t lo_s = b ? L.sums[b - 1] : 0, lo_c = b ? L.counts[b - 1] : 0;
                if (by_count ? lo_c <= target && target < L.counts[b] : lo_s <= target && target < L.sums[b]) {
                    L.found = b;
                    L.found_before = lo_s;
                    L.found_count = lo_c;
                }
            }
            __syncthreads();
            bin = L.found;
        }
        bool listed = false;
        uint32_t key_lo = 0, key_hi = top;
        if (bin >= 0 && bin != in_list) {
            // the bin's lowest logit, and the lowest of the bins before it: by the even waves and the odd ones
            const int upto = bin - (wave & 1);
            const uint32_t key = upto >= 0 ? least_key(top, [&](float v) { return bin_of(row.distance(v)) <= upto; }) : top + 1;
            if (t == 0) L.bounds[0] = key;
            if (t == 64) L.bounds[1] = key;
            __syncthreads();
            key_lo = L.bounds[0];
            if (turn >= 0) {
                key_hi = L.bounds[1] - 1;
                before = L.found_before;
                before_count = L.found_count;
            }
            const float lo = value_of_key(key_lo), hi = value_of_key(key_hi);
            uint64_t prefix = 0;
            int shift = BITS;                           // places with this prefix above `shift` bits are in question
            while (true) {
                __syncthreads();
                if (t == 0) L.listed = 0;
                __syncthreads();
                // A bit for each of 64 logits; those that are in question, one or two of the 64 in most rows, are read again (put
                // down where they are met: 128 rows of 131071 53 us, so 49).
                uint64_t hits = 0;
                int bits = 0, from[4];
                auto put = [&] {
                    if (hits) {
                        uint32_t p = atomicAdd(&L.listed, (uint32_t)__popcll(hits));
                        do {
                            const int j = __builtin_ctzll(hits);
                            hits &= hits - 1;
                            constexpr int per = 16 / sizeof(T);     // of a load, 16 of a part
                            const int base = j < 32 ? j < 16 ? from[0] : from[1] : j < 48 ? from[2] : from[3];
                            const int i = base + j % 16 / per * (kThreads * per) + j % per;
                            if (p < kList) {
                                L.keys[p] = order_key((float)x[i]);
                                L.at[p] = i;
                            }
                            ++p;
                        } while (hits);
                    }
                    bits = 0;
                };
                for_parts<sizeof(T)>(x, n, [&](const auto& v, auto&& i, auto each) {
                    constexpr int E = decltype(each)::value;
                    static_assert(E == 16 || E == 1, "16 logits, or one of those beside the 16-byte borders");
                    uint32_t now = 0;
#pragma unroll
                    for (int j = 0; j < E; ++j) now |= (uint32_t)((v[j] >= lo) & (v[j] <= hi)) << j;    // (no branches)
                    if (shift < BITS && now) {
                        for (uint32_t rest = now; rest; rest &= rest - 1)
                            if (const int j = __builtin_ctz(rest); place((float)x[i(j)], i(j)) >> shift != prefix) now &= ~(1u << j);
                    }
                    hits |= (uint64_t)now << bits;
                    (bits < 32 ? bits < 16 ? from[0] : from[1] : bits < 48 ? from[2] : from[3]) = i(0);
                    bits += 16;
                    if (bits == 64) put();
                });
                put();
                __syncthreads();
                listed = L.listed <= kList;
                if (listed || turn < 0) break;
                // more than the list holds: by parts of eight bits of their places, which all differ
                const int next = max(shift - 8, 0);
                __syncthreads();
                L.part_sums[t] = 0;
                L.part_counts[t] = 0;
                __syncthreads();
                for_row<1>(x, n, [&](float v, int i) {
                    if (!(v >= lo && v <= hi) || place(v, i) >> shift != prefix) return;
                    const int p = (int)(place(v, i) >> next) & ((1 << (shift - next)) - 1);
                    atomicAdd(&L.part_counts[p], 1u);
                    add(L.part_sums[p], weight_of(row.distance(v)));
                });
                __syncthreads();
                const uint64_t s = L.part_sums[t];
                const uint32_t c = L.part_counts[t];
                uint64_t run = s, none;
                uint32_t runs = c, number;
                scan_threads(L, run, runs, none, number);
                const uint64_t rs = before + run, rc = before_count + runs;
                if (by_count ? rc - c <= target && target < rc : rs - s <= target && target < rs) {
                    L.found = t;
                    L.found_before = rs - s;
                    L.found_count = rc - c;
                }
                __syncthreads();
                prefix = prefix << (shift - next) | (uint64_t)L.found;
                shift = next;
                before = L.found_before;
                before_count = L.found_count;
            }
            if (shift < BITS) {                         // what the prefix leaves of the range
                const int low = shift - 20;             // bits of the key in question, none where the index is
                key_hi = ~(uint32_t)(low > 0 ? prefix << low : prefix >> -low);
                key_lo = low > 0 ? key_hi - ((1u << low) - 1) : key_hi;
            }
            in_list = shift == BITS && turn >= 0 ? bin : -1;
        }
        if (turn < 0) {
            all_listed = listed;
            if (listed) count = UINT64_MAX;
            else {
                // counts (where there is a top_k) and sums by bins; how many tokens min_p keeps does not matter, only their sum
                for_row<sizeof(T) / 2>(x, n, [&](float v, int) {
                    const double d = row.distance(v);
                    const int b = bin_of(d);
                    if (b >= kBins) return;
                    const uint64_t weight = weight_of(d);
                    if (weight >= least) kept += weight;
                    if (top_k > 0) atomicAdd(&L.counts[b], 1u);
                    add(L.sums[b], weight);
                });
                __syncthreads();
                const uint64_t s1 = L.sums[2 * t + 1];
                const uint32_t c1 = L.counts[2 * t + 1];
                uint64_t run = L.sums[2 * t] + s1;
                uint32_t runs = L.counts[2 * t] + c1, number;
                scan_threads(L, run, runs, sum, number);
                count = number;
                L.sums[2 * t] = run - s1;
                L.sums[2 * t + 1] = run;
                L.counts[2 * t] = runs - c1;
                L.counts[2 * t + 1] = runs;
            }
        }
        if (listed) {
            sorted = false;
            L.part_sums[t] = 0;
            L.part_counts[t] = 0;
            if (t == 0) L.few = 0;
            __syncthreads();
            const double each = (double)kThreads / (((double)(key_hi - key_lo) + 1.0) * n);
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int i = t + j * kThreads;
                w[j] = 0;
                part[j] = kThreads;
                if (i >= (int)L.listed) continue;
                const uint32_t key = L.keys[i];
                w[j] = weight_of(row.distance(value_of_key(key)));
                if (all_listed) kept += w[j] >= least ? w[j] : 0;
                part[j] = min((uint32_t)(((double)(key_hi - key) * n + L.at[i]) * each), (uint32_t)kThreads - 1);    // (keeps order)
                atomicAdd(&L.part_counts[part[j]], 1u);
                add(L.part_sums[part[j]], w[j]);
            }
            __syncthreads();
            uint64_t run = L.part_sums[t], here;
            uint32_t runs = L.part_counts[t], number;
            scan_threads(L, run, runs, here, number);
            L.part_sums[t] = run;
            L.part_counts[t] = runs;
            if (all_listed) sum = here;
        }
        if (turn < 0) {
            if (least) {                                // (of all that are listed: no less than of the kept ones, if those are fewer)
                uint32_t zero = 0, number;
                uint64_t mine = kept;
                scan_threads(L, mine, zero, kept, number);
            }
            continue;
        }

        // The token at which the running number of tokens (by_count) or the running sum passes `target`: to L.token, L.found_weight,
        // and the running sum with it to L.found_sum.  Where its part of the list has up to 64 tokens, one wave compares them all;
        // else the list is sorted.
        __syncthreads();
        const int tokens = (int)L.listed;
        if (!sorted) {
            const uint64_t hi_s = before + L.part_sums[t], lo_s = t ? before + L.part_sums[t - 1] : before;
            const uint64_t hi_c = before_count + L.part_counts[t], lo_c = t ? before_count + L.part_counts[t - 1] : before_count;
            if (by_count ? lo_c <= target && target < hi_c : lo_s <= target && target < hi_s) {
                L.found = t;
                L.found_before = lo_s;
                L.found_count = lo_c;
                L.found_tokens = hi_c - lo_c;
            }
            __syncthreads();
            if (L.found_tokens <= 64) {
#pragma unroll
                for (int j = 0; j < EACH; ++j)
                    if (part[j] == (uint32_t)L.found) {
                        const uint32_t p = atomicAdd(&L.few, 1u);
                        L.few_keys[p] = L.keys[t + j * kThreads];
                        L.few_at[p] = L.at[t + j * kThreads];
                    }
                __syncthreads();
                if (wave == 0) {
                    const int few = (int)L.found_tokens;
                    uint32_t key = lane < few ? L.few_keys[lane] : 0;
                    int at = lane < few ? L.few_at[lane] : INT32_MAX;
                    const uint64_t weight = lane < few ? weight_of(row.distance(value_of_key(key))) : 0;
                    // how many of them, and which sum, come before this one
                    uint64_t run = L.found_before, rank = L.found_count;
                    for (int i = 0; i < few; ++i) {
                        const uint32_t ki = (uint32_t)__builtin_amdgcn_readlane((int)key, i);
                        const int ai = __builtin_amdgcn_readlane(at, i);
                        const uint64_t wi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)weight, i) |
                                            (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(weight >> 32), i) << 32;
                        if (ki > key || (ki == key && ai < at)) {
                            run += wi;
                            ++rank;
                        }
                    }
                    if (lane < few && (by_count ? rank == target : run <= target && target < run + weight)) {
                        L.token = at;
                        L.found_weight = weight;
                        L.found_sum = run + weight;
                    }
                    if (lane == 0) L.few = 0;
                }
            } else {
                sort_list(L, tokens);
                sorted = true;
            }
        }
        if (sorted) {                                   // thread t has the tokens 4 t ..
            uint64_t v[EACH], mine = 0, none;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int i = t * EACH + j;
                v[j] = i < tokens ? weight_of(row.distance(value_of_key(L.keys[i]))) : 0;
                mine += v[j];
            }
            uint64_t run = mine;
            uint32_t zero = 0, number;
            scan_threads(L, run, zero, none, number);
            run += before - mine;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int i = t * EACH + j;
                if (i < tokens && (by_count ? before_count + i == target : run <= target && target < run + v[j])) {
                    L.token = L.at[i];
                    L.found_weight = v[j];
                    L.found_sum = run + v[j];
                }
                run += v[j];
            }
        }
        __syncthreads();
        if (turn < 2) sum = L.found_sum;
    }
    if (t == 0) answer(L.token, (float)((double)L.found_weight / (double)sum));
}

}  // namespace mq

using namespace mq;

extern "C" mq_status mq_sample(int rows, int vocab, mq_dtype type, const void* logits, int64_t ldx, const float* u,
                               const float* temperature, float temperature_all, const int32_t* top_k, int top_k_all,
                               const float* top_p, float top_p_all, const float* min_p, float min_p_all, int64_t* tokens,
                               float* probs, hipStream_t stream) {
    if (rows < 0 || vocab < 0 || (!mq_host::is_half_type(type) && type != MQ_FP32)) return MQ_ERR_INVALID_ARG;
    if ((!temperature && !(temperature_all >= 0.0f)) || (!top_p && !(top_p_all >= 0.0f)) || (!min_p && !(min_p_all >= 0.0f)))
        return MQ_ERR_INVALID_ARG;
    if (vocab < 1 || vocab > MQ_SAMPLE_MAX_VOCAB || ldx < vocab || !mq_host::launch_holds(rows, kThreads)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (rows == 0) return MQ_OK;
    if (!logits || !u || !tokens || !probs) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(logits, type == MQ_FP32 ? 4 : 2) || !mq_host::aligned(u, 4) || !mq_host::aligned(temperature, 4) ||
        !mq_host::aligned(top_k, 4) || !mq_host::aligned(top_p, 4) || !mq_host::aligned(min_p, 4) || !mq_host::aligned(tokens, 8) ||
        !mq_host::aligned(probs, 4))
        return MQ_ERR_MISALIGNED;
    const SampleArgs a{logits, ldx, rows, vocab, u, temperature, top_p, min_p, top_k, temperature_all, top_p_all, min_p_all, top_k_all,
                       tokens, probs};
    auto run = [&](auto z) {
        hipLaunchKernelGGL(sample_kernel<decltype(z)>, dim3(rows), dim3(kThreads), 0, stream, a);
        return mq_host::launch_status();
    };
    return type == MQ_FP32 ? run(float{}) : mq_host::with_half_type(type, run);
}
