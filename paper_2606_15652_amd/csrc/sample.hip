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
//  2. counts and sums by bins of d = (max - x) log2(e) / T, kBinsPerUnit to a factor of two; a bin's tokens all come
//     before those of the next, and what has d >= kUnits has the weight 0 and no part in any of it;
//  3. the bin where the kept tokens end: its tokens, sorted, give the last of them, and the sum of all;
//  4. the bin where the running sum passes the target: its tokens, sorted, give the drawn one.
// A bin of more than kList tokens is split by the logit's bits instead (equal logits by the index's).
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
constexpr int kList = 2048;             // tokens of a bin that are sorted in LDS

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

// 2^-d in units of 2^-kShift for 0 <= d: of the fraction by its series (relative error below 2^-46), then rounded.
__device__ __forceinline__ uint64_t weight_of(double d) {
    if (!(d < kUnits)) return 0;                        // (infinite, too)
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
    return (uint64_t)(int64_t)rint(ldexp(y, kShift - (int)n));
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
    uint32_t listed;
    int found, token, nan;
    uint64_t found_before, found_sum, found_weight, found_count;
    float best[kThreads / 64];
    int best_at[kThreads / 64];
};

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

// f(x, i) for every logit of the row, by all threads.
template <typename T, typename F>
__device__ __forceinline__ void for_row(const T* x, int n, F&& f) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int per = 16 / sizeof(T);
    // up to the first 16-byte border one by one
    const int head = min(n, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T)), body = (n - head) / per;
    if ((int)threadIdx.x < head) f((float)x[threadIdx.x], (int)threadIdx.x);
    for (int c = threadIdx.x; c < body; c += kThreads) {
        const vec v = *reinterpret_cast<const vec*>(x + head + c * per);
#pragma unroll
        for (int j = 0; j < per; ++j) f((float)v[j], head + c * per + j);
    }
    const int tail = head + body * per + threadIdx.x;
    if (tail < n) f((float)x[tail], tail);
}

// Sorts the list (keys descending, index ascending among equals) and leaves it in order.
__device__ __forceinline__ void sort_list(SampleLds& L, int n) {
    int size = 1;
    while (size < n) size <<= 1;
    for (int i = n + threadIdx.x; i < size; i += kThreads) {
        L.keys[i] = 0;
        L.at[i] = INT32_MAX;
    }
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int p = threadIdx.x; p < size / 2; p += kThreads) {
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

    // 1. the maximum, the first of its places, and whether there is a NaN
    float best = -INFINITY;
    int best_at = INT32_MAX, nan = 0;
    for_row(x, n, [&](float v, int i) {
        if (v > best || (v == best && i < best_at)) {
            best = v;
            best_at = i;
        }
        nan |= v != v;
    });
    auto better = [](float a, int i, float b, int j) { return a > b || (a == b && i < j); };
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        const float o = __shfl_xor(best, m);
        const int oi = __shfl_xor(best_at, m);
        nan |= __shfl_xor(nan, m);
        if (better(o, oi, best, best_at)) {
            best = o;
            best_at = oi;
        }
    }
    if (t == 0) L.nan = 0;
    for (int i = t; i < kBins; i += kThreads) {
        L.sums[i] = 0;
        L.counts[i] = 0;
    }
    __syncthreads();
    if (lane == 0) {
        L.best[wave] = best;
        L.best_at[wave] = best_at;
        if (nan) L.nan = 1;
    }
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w)
        if (better(L.best[w], L.best_at[w], best, best_at)) {
            best = L.best[w];
            best_at = L.best_at[w];
        }
    auto answer = [&](int64_t token, float p) {
        a.tokens[r] = token;
        a.probs[r] = p;
    };
    if (L.nan || best == -INFINITY) {                   // nothing to draw from
        if (t == 0) answer(-1, L.nan ? __builtin_nanf("") : 0.0f);
        return;
    }
    if (!(temperature > 0.0f)) {
        if (t == 0) answer(best_at, 1.0f);
        return;
    }
    const Row row{1.4426950408889634074 / (double)temperature, (double)best};

    // 2. counts and sums by bins; how many tokens min_p keeps does not matter, only their sum
    const uint64_t least = min_p > 0.0f ? (uint64_t)ceil((double)fminf(min_p, 1.0f) * (double)(1ull << kShift)) : 0;
    uint64_t kept = 0;
    for_row(x, n, [&](float v, int) {
        const double d = row.distance(v);
        const int b = bin_of(d);
        if (b >= kBins) return;
        const uint64_t w = weight_of(d);
        if (w >= least) kept += w;
        atomicAdd(&L.counts[b], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&L.sums[b]), (unsigned long long)w);
    });
    __syncthreads();
    static_assert(kBins == 2 * kThreads, "two bins a thread");
    uint64_t sum, all, count;
    {
        const uint64_t s0 = L.sums[2 * t], s1 = L.sums[2 * t + 1];
        const uint32_t c0 = L.counts[2 * t], c1 = L.counts[2 * t + 1];
        uint64_t none;
        const uint64_t run = scan_threads(L, s0 + s1, all), runs = scan_threads(L, (uint64_t)c0 + c1, count);
        scan_threads(L, kept, none);
        kept = none;
        L.sums[2 * t] = run - s1;
        L.sums[2 * t + 1] = run;
        L.counts[2 * t] = (uint32_t)(runs - c1);
        L.counts[2 * t + 1] = (uint32_t)runs;
        __syncthreads();
    }

    // 3., 4. The token at which the running number of tokens (BY_COUNT), or the running sum, passes `target`, which the whole
    // row's does: L.token, its weight, and the running sum with it.
    int in_list = -1;                                   // the bin that the list holds
    auto locate = [&](auto by_count, uint64_t target) {
        constexpr bool COUNT = decltype(by_count)::value;
        __syncthreads();
        for (int b = 2 * t; b < 2 * t + 2; ++b) {
            const uint64_t lo_s = b ? L.sums[b - 1] : 0, lo_c = b ? L.counts[b - 1] : 0;
            if (COUNT ? lo_c <= target && target < L.counts[b] : lo_s <= target && target < L.sums[b]) {
                L.found = b;
                L.found_before = lo_s;
                L.found_sum = lo_c;
                L.found_count = L.counts[b] - lo_c;
            }
        }
        __syncthreads();
        const int bin = L.found;
        uint64_t before = L.found_before, before_count = L.found_sum, tokens = L.found_count;
        // a token's place in the order: 32 bits of its logit, the larger the lower, and 20 of its index
        constexpr int BITS = 52;
        auto place = [](float v, int i) { return (uint64_t)~order_key(v) << 20 | (uint64_t)i; };
        uint64_t prefix = 0;
        int shift = BITS;                               // places with this prefix above `shift` bits are in question
        while (tokens > kList) {                        // (each turn settles eight bits: places differ)
            const int next = max(shift - 8, 0);
            __syncthreads();
            if (t < 256) {
                L.part_sums[t] = 0;
                L.part_counts[t] = 0;
            }
            __syncthreads();
            for_row(x, n, [&](float v, int i) {
                const double d = row.distance(v);
                if (bin_of(d) != bin || place(v, i) >> shift != prefix) return;
                const int part = (int)(place(v, i) >> next) & ((1 << (shift - next)) - 1);
                atomicAdd(&L.part_counts[part], 1u);
                atomicAdd(reinterpret_cast<unsigned long long*>(&L.part_sums[part]), (unsigned long long)weight_of(d));
            });
            __syncthreads();
            const uint64_t ps = t < 256 ? L.part_sums[t] : 0, pc = t < 256 ? L.part_counts[t] : 0;
            uint64_t none;
            const uint64_t rs = before + scan_threads(L, ps, none), rc = before_count + scan_threads(L, pc, none);
            if (COUNT ? rc - pc <= target && target < rc : rs - ps <= target && target < rs) {
                L.found = t;
                L.found_before = rs - ps;
                L.found_sum = rc - pc;
                L.found_count = pc;
            }
            __syncthreads();
            prefix = prefix << (shift - next) | (uint64_t)L.found;
            shift = next;
            before = L.found_before;
            before_count = L.found_sum;
            tokens = L.found_count;
        }
        const int m = (int)tokens;
        if (shift != BITS || in_list != bin) {
            __syncthreads();
            if (t == 0) L.listed = 0;
            __syncthreads();
            for_row(x, n, [&](float v, int i) {
                if (bin_of(row.distance(v)) != bin || place(v, i) >> shift != prefix) return;
                const uint32_t p = atomicAdd(&L.listed, 1u);
                L.keys[p] = order_key(v);
                L.at[p] = i;
            });
            __syncthreads();
            sort_list(L, m);
            in_list = shift == BITS ? bin : -1;
        }
        uint64_t w[kList / kThreads] = {}, mine = 0, none;
#pragma unroll
        for (int j = 0; j < kList / kThreads; ++j) {
            const int i = t * (kList / kThreads) + j;
            if (i < m) w[j] = weight_of(row.distance(value_of_key(L.keys[i])));
            mine += w[j];
        }
        uint64_t run = before + scan_threads(L, mine, none) - mine;
#pragma unroll
        for (int j = 0; j < kList / kThreads; ++j) {
            const int i = t * (kList / kThreads) + j;
            if (i < m && (COUNT ? before_count + i == target : run <= target && target < run + w[j])) {
                L.token = L.at[i];
                L.found_weight = w[j];
                L.found_sum = run + w[j];
            }
            run += w[j];
        }
        __syncthreads();
    };
    sum = all;
    if (top_k > 0 && (uint64_t)top_k < count) {
        locate(std::true_type{}, (uint64_t)top_k - 1);
        sum = L.found_sum;
    }
    if (top_p < 1.0f) {
        // the least beginning with a sum of top_p of it at least: it passes that less one
        locate(std::false_type{}, max(part_of<true>(fmaxf(top_p, 0.0f), sum), (uint64_t)1) - 1);
        sum = L.found_sum;
    }
    if (least) sum = min(sum, kept);
    const uint64_t target = u < 1.0f ? part_of<false>(fmaxf(u, 0.0f), sum) : sum - 1;
    locate(std::false_type{}, target);
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
