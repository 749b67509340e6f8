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
//  2. with top_k, a logit that k are not below; if few enough are not, they are sorted in LDS, and the rest is done there;
//  3. otherwise counts and sums by bins of d = (max - x) log2(e) / T, kBinsPerUnit to a factor of two: a bin's tokens all
//     come before those of the next, and what has d >= kUnits has the weight 0 and no part in any of it.  Where the k-th
//     token, the end of top_p and the drawn token lie in their bins is found by sorting those bins' tokens.  A bin of more
//     than kList tokens is split by the logit's bits first (equal logits by the index's).
// A bin is a range of logits, found once, so passes that look for its tokens only compare.
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
    uint64_t part_sums[256];            // of a long bin's parts
    uint32_t part_counts[256];
    uint32_t keys[kList];               // the list: larger first
    int32_t at[kList];
    uint64_t scan[kThreads / 64];
    uint32_t listed, bounds[2];
    int found, token, nan;
    uint64_t found_before, found_count, found_tokens, found_sum, found_weight;
    float best[kThreads / 64];
};

// The least float x (as its key) with before(x), which holds for all from there to the key `top`: 64 keys at a time, by
// every wave.
template <typename F>
__device__ __forceinline__ uint32_t least_key(uint32_t top, F&& before) {
    const uint32_t lane = threadIdx.x & 63;
    uint64_t lo = order_key(-INFINITY), hi = (uint64_t)top + 1;     // the answer is in [lo, hi), and hi - 1 says yes
    while (hi - lo > 1) {
        const uint64_t step = (hi - lo + 63) / 64, k = lo + lane * step;
        const uint64_t yes = __ballot(k < hi && before(value_of_key((uint32_t)k)));
        const uint64_t no = yes ? (uint64_t)__builtin_ctzll(yes) : (hi - lo + step - 1) / step;     // lanes that say no
        if (yes) hi = lo + no * step + 1;
        if (no) lo += (no - 1) * step + 1;
    }
    return (uint32_t)(hi - 1);
}

// Inclusive running sums over the workgroup's threads, and the sum of all.
__device__ __forceinline__ uint64_t scan_threads(SampleLds& L, uint64_t v, uint64_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint64_t o = (uint64_t)__shfl_up((unsigned long long)v, m);
        if (lane >= m) v += o;
    }
    __syncthreads();
    if (lane == 63) L.scan[wave] = v;
    __syncthreads();
    uint64_t before = 0;
    all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += L.scan[w];
        all += L.scan[w];
    }
    return v + before;
}

// f(v, i, m) for the m <= EACH logits v of the row at i(j), j < m: all of them, by all threads, some loads at a time.
template <int AHEAD, typename T, typename F>
__device__ __forceinline__ void for_parts(const T* x, int n, F&& f) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int per = 16 / sizeof(T);
    // up to the first 16-byte border one by one
    const int head = min(n, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T)), body = (n - head) / per;
    const vec* v = reinterpret_cast<const vec*>(x + head);
    int c = threadIdx.x;
    for (; c + (AHEAD - 1) * kThreads < body; c += AHEAD * kThreads) {
        vec y[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) y[a] = v[c + a * kThreads];
        float z[AHEAD * per];
#pragma unroll
        for (int j = 0; j < AHEAD * per; ++j) z[j] = (float)y[j / per][j % per];
        f(z, [&](int j) { return head + (c + j / per * kThreads) * per + j % per; }, std::integral_constant<int, AHEAD * per>{});
    }
    for (; c < body; c += kThreads) {
        const vec y = v[c];
        float z[per];
#pragma unroll
        for (int j = 0; j < per; ++j) z[j] = (float)y[j];
        f(z, [&](int j) { return head + c * per + j; }, std::integral_constant<int, per>{});
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
                for (int j = min(k >> 1, most); j > 0; j >>= 1) {
                    const uint32_t ok = (uint32_t)__shfl_xor((int)key, j);
                    const int oa = __shfl_xor(at, j);
                    const bool other_first = ok > key || (ok == key && oa < at);
                    // the lower of the pair keeps the first where the stage ascends, the upper one the second
                    if (other_first == (((i & j) == 0) == ((i & k) == 0))) {
                        key = ok;
                        at = oa;
                    }
                }
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
    for_row<16 / sizeof(T)>(x, n, [&](float v, int) {
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

    // the tokens with logits lo <= x <= hi whose place above `shift` bits is `prefix`, sorted; false if they are more than kList
    // (a token's place in the order: 32 bits of its logit, the larger the lower, and 20 of its index)
    constexpr int BITS = 52;
    auto place = [](float v, int i) { return (uint64_t)~order_key(v) << 20 | (uint64_t)i; };
    auto make_list = [&](float lo, float hi, int shift, uint64_t prefix) {
        __syncthreads();
        if (t == 0) L.listed = 0;
        __syncthreads();
        for_parts<sizeof(T) == 4 ? 8 : 4>(x, n, [&](const auto& v, auto&& i, auto each) {
            constexpr int E = decltype(each)::value;
            static_assert(E <= 32, "a bit for each");
            uint32_t hits = 0;
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (v[j] >= lo && v[j] <= hi && (shift == BITS || place(v[j], i(j)) >> shift == prefix)) hits |= 1u << j;
            if (hits == 0) return;
            uint32_t p = atomicAdd(&L.listed, (uint32_t)__popc(hits));
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (hits >> j & 1) {
                    if (p < kList) {
                        L.keys[p] = order_key(v[j]);
                        L.at[p] = i(j);
                    }
                    ++p;
                }
        });
        __syncthreads();
        const uint32_t tokens = L.listed;
        if (tokens > kList) return false;
        sort_list(L, (int)tokens);
        return true;
    };
    // The weights of the list's first m tokens, and their running sums from `before` on, four tokens a thread; the sum of all
    // m, and of those that min_p keeps.
    constexpr int EACH = kList / kThreads;
    uint64_t w[EACH], runs[EACH];
    auto weigh = [&](int m, uint64_t before, uint64_t& sum, uint64_t& kept) {
        uint64_t mine = 0, keeps = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = t * EACH + j;
            w[j] = i < m ? weight_of(row.distance(value_of_key(L.keys[i]))) : 0;
            mine += w[j];
            keeps += w[j] >= least ? w[j] : 0;
        }
        runs[0] = before + scan_threads(L, mine, sum) - mine + w[0];
#pragma unroll
        for (int j = 1; j < EACH; ++j) runs[j] = runs[j - 1] + w[j];
        kept = sum;
        if (least) scan_threads(L, keeps, kept);
    };
    // Of them the one at which the running sum passes `target` (or the one in place `index`): to L.token, L.found_weight, and the
    // running sum with it to L.found_sum.
    auto pick = [&](uint64_t target, int index) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (index >= 0 ? t * EACH + j == index : runs[j] - w[j] <= target && target < runs[j]) {
                L.token = L.at[t * EACH + j];
                L.found_weight = w[j];
                L.found_sum = runs[j];
            }
        __syncthreads();
    };
    auto drawn = [&](uint64_t sum) { return u < 1.0f ? part_of<false>(fmaxf(u, 0.0f), sum) : sum - 1; };
    // the least beginning with a sum of top_p of it at least: it passes that less one
    auto cut = [&](uint64_t sum) { return max(part_of<true>(fmaxf(top_p, 0.0f), sum), (uint64_t)1) - 1; };
    static_assert(kBins == 2 * kThreads, "two bins a thread");
    uint64_t none;

    // 2. few tokens down to the k-th.  The k-th largest of the threads' two largest logits is no more than the k-th of all, so
    // its bin is the last in question.  Of logits in no order, k = 1000 of the 2048 are found among some 1130 tokens, 1536 among
    // 2070; where they are more than the list holds, all are looked at below.
    if (top_k > 0 && top_k <= 3 * kThreads / 2) {
        const float slope = (float)fmin(row.slope * kBinsPerUnit, 1e30);
        auto bin = [&](float v) { return v == best ? 0 : (int)fminf((best - v) * slope, (float)(kBins - 1)); };
        for (float v : {first, second})
            if (const int b = bin(v); b < kBins - 1) atomicAdd(&L.counts[b], 1u);
        if (t == 0) L.found = -1;
        __syncthreads();
        const uint32_t c0 = L.counts[2 * t], c1 = L.counts[2 * t + 1];
        const uint64_t down = scan_threads(L, (uint64_t)c0 + c1, none), k = (uint64_t)top_k;
        if (down - c1 - c0 < k && k <= down) L.found = down - c1 >= k ? 2 * t : 2 * t + 1;
        L.counts[2 * t] = L.counts[2 * t + 1] = 0;
        __syncthreads();
        const int last = L.found;
        if (last >= 0) {
            const uint32_t lo = least_key(top, [&](float v) { return bin(v) <= last; });
            if (make_list(value_of_key(lo), best, BITS, 0)) {
                uint64_t sum, kept;
                weigh(top_k, 0, sum, kept);
                if (top_p < 1.0f) {
                    pick(cut(sum), -1);
                    sum = L.found_sum;
                }
                sum = min(sum, kept);
                pick(drawn(sum), -1);
                if (t == 0) answer(L.token, (float)((double)L.found_weight / (double)sum));
                return;
            }
        }
    }

    // 3. counts and sums by bins; how many tokens min_p keeps does not matter, only their sum
    uint64_t kept = 0;
    for_row<sizeof(T) / 2>(x, n, [&](float v, int) {
        const double d = row.distance(v);
        const int b = bin_of(d);
        if (b >= kBins) return;
        const uint64_t w = weight_of(d);
        if (w >= least) kept += w;
        atomicAdd(&L.counts[b], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&L.sums[b]), (unsigned long long)w);
    });
    __syncthreads();
    uint64_t sum, count;
    {
        const uint64_t s0 = L.sums[2 * t], s1 = L.sums[2 * t + 1];
        const uint32_t c0 = L.counts[2 * t], c1 = L.counts[2 * t + 1];
        const uint64_t run = scan_threads(L, s0 + s1, sum), runs = scan_threads(L, (uint64_t)c0 + c1, count);
        scan_threads(L, kept, none);
        kept = none;
        L.sums[2 * t] = run - s1;
        L.sums[2 * t + 1] = run;
        L.counts[2 * t] = (uint32_t)(runs - c1);
        L.counts[2 * t + 1] = (uint32_t)runs;
        __syncthreads();
    }

    // in turn the k-th token, the end of top_p, the drawn token
    int in_list = -1;                                   // the bin that the list holds
#pragma unroll 1
    for (int turn = 0; turn < 3; ++turn) {
        const bool by_count = turn == 0;
        if (by_count ? top_k <= 0 || (uint64_t)top_k >= count : turn == 1 && !(top_p < 1.0f)) continue;
        if (turn == 2 && least) sum = min(sum, kept);
        const uint64_t target = by_count ? (uint64_t)top_k - 1 : turn == 1 ? cut(sum) : drawn(sum);
        __syncthreads();
        for (int b = 2 * t; b < 2 * t + 2; ++b) {
            const uint64_t lo_s = b ? L.sums[b - 1] : 0, lo_c = b ? L.counts[b - 1] : 0;
            if (by_count ? lo_c <= target && target < L.counts[b] : lo_s <= target && target < L.sums[b]) {
                L.found = b;
                L.found_before = lo_s;
                L.found_count = lo_c;
                L.found_tokens = L.counts[b] - lo_c;
            }
        }
        __syncthreads();
        const int bin = L.found;
        uint64_t before = L.found_before, before_count = L.found_count, tokens = L.found_tokens;
        if (in_list != bin) {
            // its lowest logit, and the lowest of the bins before it: by the even waves and the odd ones
            const int upto = bin - (wave & 1);
            const uint32_t key = upto >= 0 ? least_key(top, [&](float v) { return bin_of(row.distance(v)) <= upto; }) : top + 1;
            if (t == 0) L.bounds[0] = key;
            if (t == 64) L.bounds[1] = key;
            __syncthreads();
            const float lo = value_of_key(L.bounds[0]), hi = value_of_key(L.bounds[1] - 1);
            uint64_t prefix = 0;
            int shift = BITS;                           // places with this prefix above `shift` bits are in question
            while (tokens > kList) {                    // (each turn settles eight bits: places differ)
                const int next = max(shift - 8, 0);
                __syncthreads();
                if (t < 256) {
                    L.part_sums[t] = 0;
                    L.part_counts[t] = 0;
                }
                __syncthreads();
                for_row<1>(x, n, [&](float v, int i) {
                    if (!(v >= lo && v <= hi) || place(v, i) >> shift != prefix) return;
                    const int part = (int)(place(v, i) >> next) & ((1 << (shift - next)) - 1);
                    atomicAdd(&L.part_counts[part], 1u);
                    atomicAdd(reinterpret_cast<unsigned long long*>(&L.part_sums[part]), (unsigned long long)weight_of(row.distance(v)));
                });
                __syncthreads();
                const uint64_t ps = t < 256 ? L.part_sums[t] : 0, pc = t < 256 ? L.part_counts[t] : 0;
                const uint64_t rs = before + scan_threads(L, ps, none), rc = before_count + scan_threads(L, pc, none);
                if (by_count ? rc - pc <= target && target < rc : rs - ps <= target && target < rs) {
                    L.found = t;
                    L.found_before = rs - ps;
                    L.found_count = rc - pc;
                    L.found_tokens = pc;
                }
                __syncthreads();
                prefix = prefix << (shift - next) | (uint64_t)L.found;
                shift = next;
                before = L.found_before;
                before_count = L.found_count;
                tokens = L.found_tokens;
            }
            make_list(lo, hi, shift, prefix);           // (of `tokens`)
            in_list = shift == BITS ? bin : -1;
        }
        weigh((int)tokens, before, none, none);
        pick(target, by_count ? (int)(target - before_count) : -1);
        if (turn < 2) sum = L.found_sum;
    }
    if (t == 0) answer(L.token, (float)((double)L.found_weight / (double)sum));
}

}  // namespace mq

using namespace mq;

extern "C" size_t mq_sample_workspace_size(int rows, int vocab) {
    (void)rows;
    (void)vocab;
    return 0;
}

extern "C" mq_status mq_sample(int rows, int vocab, mq_dtype type, const void* logits, int64_t ldx, const float* u,
                               const float* temperature, float temperature_all, const int32_t* top_k, int top_k_all,
                               const float* top_p, float top_p_all, const float* min_p, float min_p_all, int64_t* tokens,
                               float* probs, void* workspace, size_t ws_bytes, hipStream_t stream) {
    if (rows < 0 || vocab < 0 || (!mq_host::is_half_type(type) && type != MQ_FP32)) return MQ_ERR_INVALID_ARG;
    if ((!temperature && !(temperature_all >= 0.0f)) || (!top_p && !(top_p_all >= 0.0f)) || (!min_p && !(min_p_all >= 0.0f)))
        return MQ_ERR_INVALID_ARG;
    if (vocab < 1 || vocab > MQ_SAMPLE_MAX_VOCAB || ldx < vocab || !mq_host::launch_holds(rows, kThreads)) return MQ_ERR_UNSUPPORTED_SHAPE;
    if (rows == 0) return MQ_OK;
    if (!logits || !u || !tokens || !probs) return MQ_ERR_INVALID_ARG;
    if (!mq_host::aligned(logits, type == MQ_FP32 ? 4 : 2) || !mq_host::aligned(u, 4) || !mq_host::aligned(temperature, 4) ||
        !mq_host::aligned(top_k, 4) || !mq_host::aligned(top_p, 4) || !mq_host::aligned(min_p, 4) || !mq_host::aligned(tokens, 8) ||
        !mq_host::aligned(probs, 4) || !mq_host::aligned(workspace, 16))
        return MQ_ERR_MISALIGNED;
    const size_t need = mq_sample_workspace_size(rows, vocab);
    if (need > 0 && (!workspace || ws_bytes < need)) return MQ_ERR_WORKSPACE;
    const SampleArgs a{logits, ldx, rows, vocab, u, temperature, top_p, min_p, top_k, temperature_all, top_p_all, min_p_all, top_k_all,
                       tokens, probs};
    auto run = [&](auto z) {
        hipLaunchKernelGGL(sample_kernel<decltype(z)>, dim3(rows), dim3(kThreads), 0, stream, a);
        return mq_host::launch_status();
    };
    return type == MQ_FP32 ? run(float{}) : mq_host::with_half_type(type, run);
}
