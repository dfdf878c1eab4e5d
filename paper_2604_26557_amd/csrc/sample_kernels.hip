// The next token of every row of logits: temperature, top-k, top-p and min-p from given random numbers.
//
// Mathematics.  w_i = exp((l_i - max) / T) is held as an integer W_i of 2^-s, s = 62 - log2(n_vocab) or 51: sums are exact, whatever their order, so splits, histograms
// and prefix sums of any shape give one answer, and adding takes no care.  With tokens ordered by (l from the largest, index), each of the three cuts keeps a beginning of that order: what is kept
// is every token up to one, the border, in that order, and the token is found in order of indices: sums of tiles, of which one is gone over again.
//
// A workgroup has a row. It is read from HBM once, for its maximum, and from L2 after that.
//   Few of the largest (top_k up to 256): no fewer than k tokens reach the k-th largest of the threads' own maxima; a list of those that do is all there is to rank.
//   top_p alone: the sum of all, and a histogram over distances from the maximum. A token below (1 - p) / n_vocab of the sum is kept by none: a sample says about where that is, and only what is
//     above goes into the histogram (a quarter of the tokens in a usual case; an atomic of 64 bits for all of them takes longer than the exponentials). Then a list of what is kept for sure, and of the bin with the border.
//   min_p alone: a list of what is above.
//   What these have no room for, or larger top_k: histograms over the whole row, of its keys in the end, in as many rounds as they need.
// What bounds it: the exponentials in double precision where the sum of all is needed (23 instructions each), otherwise latencies of a pass.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "launch.hpp"
#include "plan.hpp"

namespace {

using namespace kvb;

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kTiles = 1024;     // of a row, each at least 512 tokens: what a wavefront loads at once is of one
constexpr int kExpTable = 256;
constexpr int kList = 16384;     // tokens of a list
constexpr int kRanked = 1024;    // tokens that are put into order one against all others

struct SampleParams {
    kv_sample_args_t a;
    int shift;   // log2 of the weights' unit
    int tile;    // log2 of the tokens of a tile
};

// A logit's bits as a number that grows with it; -0 is 0.
__device__ __forceinline__ unsigned key_of(float x)
{
    const unsigned b = __float_as_uint(x + 0.f);
    return b >> 31 ? ~b : b | 0x80000000u;
}

template <int DTYPE> constexpr int kVector = DTYPE == KV_F32 ? 4 : 8;   // logits of a load of 16 bytes

template <int DTYPE>
__device__ __forceinline__ float logit_at(const void *row, long long i)
{
    if constexpr (DTYPE == KV_F32) return ((const float *)row)[i];
    else if constexpr (DTYPE == KV_F16) return (float)((const _Float16 *)row)[i];
    else return __uint_as_float((unsigned)((const unsigned short *)row)[i] << 16);
}

struct Nothing {
    __device__ __forceinline__ void operator()(int) const {}
};
// f(logit, index) for the logits of a row that fall to this thread, several loads of 16 bytes at a time; what lies before the first aligned one, and after the last, goes to a thread each.
// loaded(first index) after each load.
template <int DTYPE, typename F, typename L = Nothing>
__device__ __forceinline__ void for_logits(const char *row, int V, int tid, const F &f, const L &loaded = L{})
{
    constexpr int E = kVector<DTYPE>, kBytes = 16 / E, kAhead = 4;
    const int before = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / kBytes), vectors = (V - before) / E, after = before + vectors * E;
    if (tid < before) f(logit_at<DTYPE>(row, tid), tid), loaded(tid);
    if (tid < V - after) f(logit_at<DTYPE>(row, after + tid), after + tid), loaded(after + tid);
    const uint4 *const at = (const uint4 *)(row + (long long)before * kBytes);
    for (int v0 = tid; v0 < vectors; v0 += kAhead * kThreads) {
        uint4 w[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (v0 + k * kThreads < vectors) w[k] = at[v0 + k * kThreads];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int v = v0 + k * kThreads;
            if (v >= vectors) break;
            const unsigned x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float l;
                if constexpr (DTYPE == KV_F32) l = __uint_as_float(x[e]);
                else if constexpr (DTYPE == KV_BF16) l = __uint_as_float(e % 2 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
                else l = (float)__builtin_bit_cast(_Float16, (unsigned short)(e % 2 ? x[e / 2] >> 16 : x[e / 2]));
                f(l, before + v * E + e);
            }
            loaded(before + v * E);
        }
    }
}

// Sum over the wavefront, in every lane.
__device__ __forceinline__ u64 wave_sum(u64 x)
{
#pragma unroll
    for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o);
    return x;
}
__device__ __forceinline__ u64 wave_sums_to(u64 x, int lane)   // of the lanes up to this one
{
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const u64 y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    return x;
}

struct Shared {
    double exps[kExpTable];
    u64 weight[kBins];
    unsigned count[kBins];
    u64 tile_weight[kTiles];
    unsigned list[kList];           // indices
    u64 ranked[kRanked];            // (key, ~index): what is larger comes first
    u64 ranked_weight[kRanked];
    unsigned n_list, n_ranked, n_kept;
    u64 wave_u64[kWaves];
    unsigned wave_u32[kWaves];
    float wave_max[kWaves];
    // what one thread tells the others
    u64 told_weight, told_all;
    unsigned told_bin, told_count;
};

// Where a token is in the order: larger ones come first. Keys are never zero.
__device__ __forceinline__ u64 place_of(unsigned key, int i) { return (u64)key << 32 | (unsigned)~i; }

template <int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_sample_kernel(SampleParams p)
{
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = p.a.n_vocab;
    const int b = blockIdx.x;
    const char *const row = (const char *)p.a.logits + (long long)b * p.a.stride * (DTYPE == KV_F32 ? 4 : 2);
    auto answer = [&](int token, float prob) {
        p.a.tokens[b] = token;
        if (p.a.probs) p.a.probs[b] = prob;
    };
    // Sum over the workgroup, in every thread.
    auto sum_of = [&](u64 x) {
        x = wave_sum(x);
        __syncthreads();
        if (lane == 0) s.wave_u64[wave] = x;
        __syncthreads();
        u64 all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += s.wave_u64[w];
        return all;
    };
    // Sum over the threads before this one.
    auto sum_before = [&](u64 x) {
        const u64 to = wave_sums_to(x, lane);
        __syncthreads();
        if (lane == 63) s.wave_u64[wave] = to;
        __syncthreads();
        u64 before = to - x;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) before += w < wave ? s.wave_u64[w] : 0;
        return before;
    };

    const float T = p.a.temperature ? p.a.temperature[b] : 1.f;
    const bool greedy = !(T > 0.f);
    const int k_asked = greedy ? 1 : p.a.top_k ? p.a.top_k[b] : 0;
    const unsigned k = k_asked <= 0 || k_asked > V ? (unsigned)V : (unsigned)k_asked;
    const bool cut_k = k < (unsigned)V;
    const float top_p = greedy || !p.a.top_p ? 1.f : p.a.top_p[b];
    const float min_p = greedy || !p.a.min_p ? 0.f : fminf(p.a.min_p[b], 1.f);
    const bool cut_p = top_p < 1.f;
    float u = p.a.u[b];
    u = u > 0.f ? u : 0.f;

    // The largest logit, its first index, and this thread's own; a NaN or +infinity makes it +infinity.
    if (tid < kExpTable) s.exps[tid] = exp2((double)tid / kExpTable);
    if (tid == 0) s.n_list = s.n_ranked = s.n_kept = 0;
    float top = -INFINITY, mine;
    for_logits<DTYPE>(row, V, tid, [&](float x, int) { top = x <= FLT_MAX ? fmaxf(top, x) : INFINITY; });
    mine = top;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) s.wave_max[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s.wave_max[w]);
    if (!(fabsf(top) <= FLT_MAX)) {
        if (tid == 0) answer(-1, 0.f);
        return;
    }

    // exp((l - max) / T) = 2^(n / 256 + g / 256) with |g| <= 1/2: a table, and e^(g ln 2 / 256) by its series (the next term is below 2^-54). What is below 2^-60 has no weight.
    const double per_unit = greedy ? 0. : 1.4426950408889634 * kExpTable / (double)T, top64 = top;
    auto scaled_weight = [&](float x, int shift) -> double {
        constexpr double c = 0.6931471805599453 / kExpTable;
        const double y = fmax(((double)x - top64) * per_unit, -60. * kExpTable);
        const double n = rint(y), g = y - n;
        const int at = (int)n;
        const double e = fma(g, fma(g, fma(g, fma(g, c * c * c * c / 24, c * c * c / 6), c * c / 2), c), 1.);
        return ldexp(s.exps[at & (kExpTable - 1)] * e, (at >> 8) + shift);
        static_assert(kExpTable == 256, "8 bits");
    };
    auto weight_of = [&](float x) { return x == -INFINITY ? 0. : scaled_weight(x, 0); };
    // to the nearest integer by adding 2^52, whose lowest bit is worth one
    auto units_of = [&](float x) { return x == -INFINITY ? 0 : (u64)__double_as_longlong(scaled_weight(x, p.shift) + 4503599627370496.) & 0xfffffffffffffull; };

    // The border: kept is what is not after it in the order (and weighs enough).
    u64 border = 0;
    // Tiles begin where loads of 16 bytes do; what is before that is of the first.
    const int before_loads = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / (DTYPE == KV_F32 ? 4 : 2)), n_tiles = max(1, ((V - before_loads - 1) >> p.tile) + 1);
    auto tile_of = [&](int i) { return max(0, i - before_loads) >> p.tile; };
    auto tile_begin = [&](int t) { return t == 0 ? 0 : before_loads + (t << p.tile); };
    auto tile_end = [&](int t) { return min(V, before_loads + ((t + 1) << p.tile)); };
    auto pick = [&] {   // tile_weight holds the sums of what is kept
        __syncthreads();
        const u64 own = tid < n_tiles ? s.tile_weight[tid] : 0, before = sum_before(own);
        u64 all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += s.wave_u64[w];
        const double at = (double)u * (double)all;
        const u64 target = min((u64)at, all - 1);   // the largest has a weight: all > 0
        if (before <= target && target < before + own) {
            s.told_bin = (unsigned)tid;
            s.told_weight = before;
        }
        __syncthreads();
        if (wave != 0) return;
        const int t = (int)s.told_bin, end = tile_end(t);
        u64 sum = s.told_weight;
        for (int i0 = tile_begin(t); i0 < end; i0 += 64) {
            const int i = i0 + lane;
            const float x = i < end ? logit_at<DTYPE>(row, i) : -INFINITY;
            const bool in = i < end && place_of(key_of(x), i) >= border && weight_of(x) >= (double)min_p;
            const u64 to = sum + wave_sums_to(in ? units_of(x) : 0, lane);
            const u64 hit = __ballot(to > target);
            if (hit != 0) {
                if (lane == __ffsll((long long)hit) - 1) answer(i, (float)(scaled_weight(x, p.shift) / (double)all));
                return;
            }
            sum = __shfl(to, 63);
        }
    };
    auto clear_tiles = [&] { s.tile_weight[tid] = 0; };
    static_assert(kTiles == kThreads, "a tile each");
    // Adds a token for sure kept to the list, for all lanes at once; false: no room.
    auto append = [&](bool is, unsigned value, unsigned *n, unsigned *to, unsigned room) {
        const u64 some = __ballot(is);
        if (some == 0) return;
        unsigned at = 0;
        if (lane == __ffsll((long long)some) - 1) at = atomicAdd(n, (unsigned)__popcll(some));
        at = (unsigned)__shfl((int)at, __ffsll((long long)some) - 1) + (unsigned)__popcll(some & ((1ull << lane) - 1));
        if (is && at < room) to[at] = value;
    };
    // s.ranked[0 .. n) and weights: the sum of weights (or the number) before each in the order
    auto before_in_order = [&](int n, auto by_weight) {
        u64 before = 0;
        if (tid < n) {
            const u64 own = s.ranked[tid];
            for (int j = 0; j < n; ++j) before += s.ranked[j] > own ? (decltype(by_weight)::value ? s.ranked_weight[j] : 1) : 0;
        }
        return before;
    };

    if (greedy) {   // the first of the largest
        int at = INT_MAX;
        if (mine == top) for_logits<DTYPE>(row, V, tid, [&](float x, int i) { at = x == top ? min(at, i) : at; });
#pragma unroll
        for (int o = 1; o < 64; o *= 2) at = min(at, __shfl_xor(at, o));
        if (lane == 0) s.wave_u64[wave] = (u64)at;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kWaves; ++w) at = min(at, (int)s.wave_u64[w]);
            answer(at, 1.f);
        }
        return;
    }
    // a logit that weighs min_p, less some units of its own rounding: what is below is not kept
    float least = min_p > 0.f ? (float)((double)top + log((double)min_p) * (double)T) - 1.0e-5f * (fabsf(top) + 1.f) - 1.0e-5f * T : -INFINITY;
    if (!(least == least)) least = -INFINITY;

    if (!cut_k && !cut_p && !(min_p > 0.f)) {   // nothing is cut off
        clear_tiles();
        __syncthreads();
        u64 sum = 0;
        for_logits<DTYPE>(
            row, V, tid, [&](float x, int) { sum += units_of(x); },
            [&](int i) {
                if (__ballot(1) == ~0ull) {   // 64 loads side by side are of one tile
                    sum = wave_sum(sum);
                    if (lane == 0) atomicAdd(&s.tile_weight[tile_of(i)], sum);
                } else {
                    atomicAdd(&s.tile_weight[tile_of(i)], sum);
                }
                sum = 0;
            });
        pick();
        return;
    }

    if (cut_k && k <= 256) {
        // at least k threads' maxima reach the lower end of the bin with the k-th of them
        s.count[tid] = 0;
        float lowest = mine == -INFINITY ? top : mine;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) lowest = fminf(lowest, __shfl_xor(lowest, o));
        __syncthreads();
        if (lane == 0) s.wave_max[wave] = lowest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) lowest = fminf(lowest, s.wave_max[w]);
        const float span = top - lowest, per = span > 0.f && span <= FLT_MAX ? 1023.f / span : 0.f;
        const int bin = mine == -INFINITY ? -1 : (int)fminf((top - mine) * per, 1023.f);
        if (bin >= 0) atomicAdd(&s.count[bin], 1u);
        __syncthreads();
        const u64 own = s.count[tid], before = sum_before(own);
        if (tid == 0) s.told_bin = kBins;
        __syncthreads();
        if (before < k && k <= before + own) s.told_bin = (unsigned)tid;
        __syncthreads();
        const unsigned last = s.told_bin;
        // by the same arithmetic as the bins: what is in one of the first `last` + 1
        auto reaches = [&](float x) { return x != -INFINITY && (top - x) * per < (float)(last + 1); };
        if (last < (unsigned)kBins && span <= FLT_MAX) {
            for_logits<DTYPE>(row, V, tid, [&](float x, int i) {
                if (__any(reaches(x))) append(reaches(x), (unsigned)i, &s.n_list, s.list, kList);
            });
            __syncthreads();
            const int n = (int)s.n_list;
            if (n <= kRanked) {
                float x = 0.f;
                if (tid < n) {
                    x = logit_at<DTYPE>(row, (long long)s.list[tid]);
                    s.ranked[tid] = place_of(key_of(x), (int)s.list[tid]);
                    s.ranked_weight[tid] = units_of(x);
                }
                __syncthreads();
                const u64 rank = before_in_order(n, std::false_type{});
                bool in = tid < n && rank < k;
                if (cut_p) {
                    // weights of what the first cut leaves out do not count
                    __syncthreads();
                    if (tid < n && !in) s.ranked_weight[tid] = 0;
                    __syncthreads();
                    const u64 sum = sum_of(in ? s.ranked_weight[tid] : 0);
                    const double want = ceil((double)(top_p > 0.f ? top_p : 0.f) * (double)sum);
                    const u64 target = max((u64)1, min((u64)want, sum));
                    in = in && before_in_order(n, std::true_type{}) < target;
                }
                in = in && weight_of(x) >= (double)min_p;
                clear_tiles();
                if (tid == 0) s.told_all = ~0ull;
                __syncthreads();
                if (in) {
                    atomicAdd(&s.tile_weight[tile_of((int)s.list[tid])], s.ranked_weight[tid]);
                    atomicMin(&s.told_all, s.ranked[tid]);
                }
                __syncthreads();
                border = s.told_all;
                pick();
                return;
            }
            __syncthreads();
            if (tid == 0) s.n_list = 0;
        }
        __syncthreads();
    }

    if (!cut_k && cut_p) {
        // Weights of every 1024th of the row give about the sum; the largest alone is 1.
        float sample = 0.f;
        const int take = min(V, 8 * kThreads);
        for (int j = 0; j < 8; ++j) {
            const int i = j * kThreads + tid;
            if (i < take) sample += __expf((logit_at<DTYPE>(row, (long long)i * V / take) - top) / T);
        }
#pragma unroll
        for (int o = 1; o < 64; o *= 2) sample += __shfl_xor(sample, o);
        __syncthreads();
        if (lane == 0) s.wave_max[wave] = sample;
        s.count[tid] = s.count[kThreads + tid] = 0;
        s.weight[tid] = s.weight[kThreads + tid] = 0;
        __syncthreads();
        sample = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sample += s.wave_max[w];
        sample = fmaxf(1.f, sample * (float)V / (float)take);
        // down to a quarter of what is looked for, in bins
        const float reach = fminf(T * __logf(4.f * (float)V / ((1.f - fmaxf(top_p, 0.f)) * sample)), T * 42.f), per = (float)kBins / reach;
        u64 sum = 0;
        if (reach > 0.f && reach <= FLT_MAX && per <= FLT_MAX) {
            for_logits<DTYPE>(row, V, tid, [&](float x, int) {
                const u64 w = units_of(x);
                sum += w;
                const float bin = (top - x) * per;
                if (bin < (float)kBins) {
                    atomicAdd(&s.count[(int)bin], 1u);
                    atomicAdd(&s.weight[(int)bin], w);
                }
            });
            sum = sum_of(sum);
            const double want = ceil((double)(top_p > 0.f ? top_p : 0.f) * (double)sum);
            const u64 target = max((u64)1, min((u64)want, sum));
            const u64 w0 = s.weight[2 * tid], w1 = s.weight[2 * tid + 1], before = sum_before(w0 + w1);
            if (tid == 0) s.told_bin = kBins;
            const u64 counts = (u64)s.count[2 * tid] + s.count[2 * tid + 1], counts_before = sum_before(counts);
            if (before < target && target <= before + w0 + w1) {
                const bool second = target > before + w0;
                s.told_bin = 2 * tid + second;
                s.told_weight = target - before - (second ? w0 : 0);   // of the bin itself
                s.told_count = (unsigned)min(counts_before + (second ? s.count[2 * tid] : 0), (u64)UINT_MAX);
            }
            __syncthreads();
            const unsigned bin = s.told_bin;
            const u64 in_bin = s.told_weight;
            if (bin < (unsigned)kBins && s.count[bin] <= (unsigned)kRanked && s.told_count <= (unsigned)kList) {
                const float from = (float)bin;
                for_logits<DTYPE>(row, V, tid, [&](float x, int i) {
                    const float at = (top - x) * per;
                    const bool sure = at < from && x >= least, maybe = at >= from && at < from + 1.f;
                    if (!__any(sure || maybe)) return;
                    append(sure, (unsigned)i, &s.n_list, s.list, kList);
                    append(maybe, (unsigned)i, &s.n_ranked, (unsigned *)s.ranked_weight + kRanked, kRanked);
                });
                __syncthreads();
                const int n = (int)s.n_ranked, n_sure = (int)s.n_list;
                unsigned i = 0;
                float x = 0.f;
                u64 w = 0;
                if (tid < n) {
                    i = ((unsigned *)s.ranked_weight)[kRanked + tid];
                    x = logit_at<DTYPE>(row, (long long)i);
                    w = units_of(x);
                    s.ranked[tid] = place_of(key_of(x), (int)i);
                }
                clear_tiles();
                if (tid == 0) s.told_all = ~0ull;
                __syncthreads();
                if (tid < n) s.ranked_weight[tid] = w;
                __syncthreads();
                if (tid < n && before_in_order(n, std::true_type{}) < in_bin) {
                    atomicMin(&s.told_all, s.ranked[tid]);
                    if (weight_of(x) >= (double)min_p) atomicAdd(&s.tile_weight[tile_of((int)i)], w);
                }
                for (int j = tid; j < n_sure; j += kThreads) {
                    const unsigned at = s.list[j];
                    const float y = logit_at<DTYPE>(row, (long long)at);
                    if (weight_of(y) >= (double)min_p) atomicAdd(&s.tile_weight[tile_of((int)at)], units_of(y));
                }
                __syncthreads();
                border = s.told_all;
                pick();
                return;
            }
        }
        __syncthreads();
    }

    if (!cut_k && !cut_p) {   // min_p alone
        for_logits<DTYPE>(row, V, tid, [&](float x, int i) {
            if (__any(x >= least)) append(x >= least, (unsigned)i, &s.n_list, s.list, kList);
        });
        clear_tiles();
        __syncthreads();
        const int n = (int)s.n_list;
        if (n <= kList) {
            for (int j = tid; j < n; j += kThreads) {
                const unsigned at = s.list[j];
                const float y = logit_at<DTYPE>(row, (long long)at);
                if (weight_of(y) >= (double)min_p) atomicAdd(&s.tile_weight[tile_of((int)at)], units_of(y));
            }
            pick();
            return;
        }
        __syncthreads();
    }

    // Anything: the key at which a count, or a sum of weights, is reached, going down: histograms over bins of falling keys, whose bin with the border becomes the next range. All keys above
    // `border_key` are kept, and of those that equal it the first `ties`.
    unsigned border_key = 0, ties = (unsigned)V;
    u64 kept = 0;   // weight of what the order's beginning up to there holds
    auto find_border = [&](auto by_weight, u64 target, unsigned from_key) {
        constexpr bool W = decltype(by_weight)::value;
        // keys in [low, high] are looked at; above them there are `above` tokens of weight `above_weight`
        unsigned low = from_key, high = key_of(top);
        u64 above = 0, above_weight = 0;
        for (bool by_distance = true;; by_distance = false) {
            int shift = 0;
            while (((high - low) >> shift) >= kBins) ++shift;
            // the first round's bins: 1/64 of a temperature's unit wide, the last one open
            const float bins_per = 64.f / fmaxf(T, 1.0e-30f);
            auto bin_of = [&](float x, unsigned key) -> unsigned {
                if (by_distance) return (unsigned)fminf((top - x) * bins_per, (float)(kBins - 1));
                return (high - key) >> shift;
            };
            __syncthreads();
            for (int i = tid; i < kBins; i += kThreads) s.weight[i] = 0, s.count[i] = 0;
            __syncthreads();
            for_logits<DTYPE>(row, V, tid, [&](float x, int) {
                const unsigned key = key_of(x);
                if (key < low || key > high) return;
                const unsigned at = bin_of(x, key);
                atomicAdd(&s.count[at], 1u);
                atomicAdd(&s.weight[at], units_of(x));
            });
            __syncthreads();
            // sums before each bin: a thread has two
            const u64 c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1], w0 = s.weight[2 * tid], w1 = s.weight[2 * tid + 1];
            const u64 counts = above + sum_before(c0 + c1), weights = above_weight + sum_before(w0 + w1);
            const u64 before = W ? weights : counts, first = W ? w0 : c0, both = W ? w0 + w1 : c0 + c1;
            if (tid == 0) s.told_bin = kBins;
            __syncthreads();
            if (before < target && target <= before + both) {
                const bool second = target > before + first;
                s.told_bin = 2 * tid + second;
                s.told_all = counts + (second ? c0 : 0);
                s.told_weight = weights + (second ? w0 : 0);
            }
            __syncthreads();
            const unsigned bin = s.told_bin;
            if (bin >= (unsigned)kBins) return;   // more is asked for than there is: all
            above = s.told_all;
            above_weight = s.told_weight;
            const unsigned in_bin = s.count[bin];
            const u64 bin_weight = s.weight[bin];
            if (by_distance) {
                // the keys that are in the bin
                unsigned least_key = ~0u, most_key = 0;
                for_logits<DTYPE>(row, V, tid, [&](float x, int) {
                    const unsigned key = key_of(x);
                    if (key >= low && key <= high && bin_of(x, key) == bin) least_key = min(least_key, key), most_key = max(most_key, key);
                });
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    least_key = min(least_key, (unsigned)__shfl_xor((int)least_key, o));
                    most_key = max(most_key, (unsigned)__shfl_xor((int)most_key, o));
                }
                __syncthreads();
                if (lane == 0) s.wave_u32[wave] = least_key, s.wave_u64[wave] = most_key;
                __syncthreads();
                low = ~0u, high = 0;
                for (int w = 0; w < kWaves; ++w) low = min(low, s.wave_u32[w]), high = max(high, (unsigned)s.wave_u64[w]);
            } else {
                const unsigned last = high - (bin << shift), width = (1u << shift) - 1;
                low = width > last - low ? low : last - width;
                high = last;
            }
            if (low == high) {   // one key: how many of its tokens, all of one weight
                border_key = low;
                const u64 each = in_bin ? bin_weight / in_bin : 0;
                if (W) ties = each == 0 ? in_bin : (unsigned)min((u64)in_bin, (target - above_weight + each - 1) / each);
                else ties = (unsigned)(target - above);
                kept = above_weight + (u64)ties * each;
                return;
            }
        }
    };
    if (cut_k) find_border(std::false_type{}, (u64)k, 0u);
    if (cut_p) {
        if (!cut_k) {   // the sum of all
            u64 sum = 0;
            for_logits<DTYPE>(row, V, tid, [&](float x, int) { sum += units_of(x); });
            kept = sum_of(sum);
        }
        // no more than the top-k's keys; what of its border's key is past k counts in no sum before the target, which is at most theirs
        const double want = ceil((double)(top_p > 0.f ? top_p : 0.f) * (double)kept);
        const u64 target = max((u64)1, min((u64)want, kept));
        const unsigned k_border = border_key, k_ties = ties;
        find_border(std::true_type{}, target, border_key);
        if (border_key == k_border && cut_k) ties = min(ties, k_ties);
    }

    // Tiles: sums of what is above the border's key, and how many have it; the last of these that is kept is the border.
    __syncthreads();
    s.count[tid] = 0;
    s.tile_weight[tid] = 0;
    __syncthreads();
    for (int t = wave; t < n_tiles; t += kWaves) {
        u64 sum = 0;
        unsigned equal = 0;
        const int end = tile_end(t);
        for (int i = tile_begin(t) + lane; i < end; i += 64) {
            const float x = logit_at<DTYPE>(row, i);
            const unsigned key = key_of(x);
            if (key > border_key && x >= least && weight_of(x) >= (double)min_p) sum += units_of(x);
            equal += key == border_key;
        }
        sum = wave_sum(sum);
        equal = (unsigned)wave_sum(equal);
        if (lane == 0) s.tile_weight[t] = sum, s.count[t] = equal;
    }
    __syncthreads();
    const float border_logit = __uint_as_float(border_key >> 31 ? border_key & 0x7fffffffu : ~border_key);
    const u64 each = border_key != 0 && weight_of(border_logit) >= (double)min_p ? units_of(border_logit) : 0;
    const u64 equal = s.count[tid], equal_before = sum_before(equal), taken = equal_before >= ties ? 0 : min(equal, ties - equal_before);
    s.tile_weight[tid] += taken * each;
    if (tid == 0) s.told_all = 0;
    __syncthreads();
    if (border_key != 0 && equal_before < ties && equal_before + equal >= ties) s.told_all = (u64)(ties - equal_before) << 32 | (unsigned)tid;   // the last one is in this tile
    __syncthreads();
    if (s.told_all != 0) {
        // every wavefront for itself
        unsigned left = (unsigned)(s.told_all >> 32);
        const int t = (int)(unsigned)s.told_all, end = tile_end(t);
        for (int i0 = tile_begin(t); i0 < end; i0 += 64) {
            const int i = i0 + lane;
            u64 is = __ballot(i < end && key_of(logit_at<DTYPE>(row, min(i, end - 1))) == border_key);
            const unsigned n = (unsigned)__popcll(is);
            if (n >= left) {
                for (; left > 1; --left) is &= is - 1;
                border = place_of(border_key, i0 + __ffsll((long long)is) - 1);
                break;
            }
            left -= n;
        }
    } else if (border_key != 0) {
        border = place_of(border_key, INT_MAX);
    }
    __syncthreads();
    pick();
}

}  // namespace

extern "C" size_t kv_sample_workspace(int n_rows, int n_vocab)
{
    if (n_rows < 0 || n_vocab < 0) return 0;
    return 16;
}

extern "C" int kv_sample(const kv_sample_args_t *a, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!a || !workspace || ((uintptr_t)workspace & 15)) return KV_EINVAL;
    if (a->dtype != KV_F16 && a->dtype != KV_BF16 && a->dtype != KV_F32) return KV_EINVAL;
    if (a->n_rows < 0 || a->n_vocab < 1 || a->stride < 0) return KV_EINVAL;
    if (ws_bytes < kv_sample_workspace(a->n_rows, a->n_vocab)) return KV_ENOSPC;
    if (a->n_rows == 0) return KV_OK;
    if (a->n_vocab > 1 << 24) return KV_ERANGE;
    if (!a->logits || !a->u || !a->tokens || ((uintptr_t)a->logits & (a->dtype == KV_F32 ? 3 : 1))) return KV_EINVAL;
    SampleParams p{};
    p.a = *a;
    int bits = 0;
    while ((1 << bits) < a->n_vocab) ++bits;
    p.shift = std::min(51, 62 - bits);
    p.tile = 9;
    while (((a->n_vocab - 1) >> p.tile) >= kTiles) ++p.tile;
    (void)launch_kernel(a->dtype == KV_F32 ? kv_sample_kernel<KV_F32> : a->dtype == KV_F16 ? kv_sample_kernel<KV_F16> : kv_sample_kernel<KV_BF16>, dim3((unsigned)a->n_rows),
                        dim3(kThreads), (hipStream_t)hip_stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
