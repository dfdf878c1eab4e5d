// The next token of every row of logits: temperature, top-k, top-p and min-p from given random numbers.
//
// Mathematics.  w_i = exp((l_i - max) / T) is held as an integer W_i of 2^-s, s = 62 - log2(n_vocab) or 51: sums are exact, whatever their order, so slices, histograms
// and prefix sums of any shape give one answer, and adding takes no care.  With tokens ordered by (l from the largest, index), each of the three cuts keeps a beginning of that order: what is kept
// is every token up to one, the border, in that order, and the token is found in order of indices: sums of tiles, of which one is gone over again.
//
// A workgroup has a row. It is read from HBM for its maximum, and again for the rest, from the caches where they hold it by then, and where few of the largest are wanted out of registers if it fits them.
//   Few of the largest (top_k up to 256): no fewer than k tokens reach the k-th largest of the threads' own maxima; a list of those that do is all there is to rank.
//   More of them, without top_p: a histogram of their number by distance from the maximum says which bin the k-th is in; what is above is kept, the bin is a list, which is ranked.  2 rows of 106775
//     in 32 bits, the largest 1000: 62 us; 115 by the rounds below.
//   top_p alone: the sum of all, and a histogram of weights by distance from the maximum.  Tokens below (1 - p) / n_vocab of the sum are not needed to get from p to the whole: a sample says about where
//     that is, and only what is above goes into the histogram (a third of the tokens in a usual case).  Then as before; or, where no more than 256 tokens can have what there is up to the border, as with
//     few: a row of 32000 of which a dozen have nine tenths of the weight 19.5 -> 17.0 us (with room for 1024 rows of 74 were ranked for longer than it saved: 64 of 128256 43 -> 48).
//   min_p alone: what is above it is kept.
//   What these have no room for, and top_k past 256 with top_p: histograms over the whole row, of its keys in the end, in as many rounds as they need.
// What bounds it: where the sum of all is needed, the row's second reading and some 35 vector instructions a token, many in double precision, which hide each other in part (256 rows of 50257 in 32 bits, nothing
// cut: 24.3 us; 97 MB, 19 us at the rate of a large copy; vector instructions in 67 % of the cycles); otherwise a pass' latencies.  So few rows of many tokens are shared by several workgroups for the
// maximum and for the weights, a launch each ahead of the rows' own: 64 rows of 128256 in 16 bits with top_p 43.5 us, 75 with a workgroup each (the sum's pass 16.2, vector instructions in 65 % of its
// cycles; that of what is kept 16.3, in 49 %; launches and what they wait for are the rest).  One row
// of 32000 in 32 bits with top_k and top_p takes 11.3 us: 3.2 until it is there, 2.6 for the threads' maxima, the rest what threads tell each other, one after the other.
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
constexpr int kThreads = 1024, kWaves = kThreads / 64;   // of a row: of one workgroup, or of several
constexpr int kBins = 2048;
constexpr int kTiles = 1024;     // of a row, each at least 512 tokens: what a wavefront loads at once is of one
constexpr int kExpTable = 256;
constexpr int kRanked = 1024;    // tokens that are put into order one against all others
constexpr int kMostSlices = 8;   // a row of 128256 with top_p: 38 us with up to 16, 33 with 8, 34 with 4; 16 rows 47, 40 and 38

// What the slices of a row leave for the next launch.
struct RowState {
    float maxima[kMostSlices][kThreads];   // of each thread; +infinity for a NaN or +infinity
    u64 tile_weight[kTiles];               // sums of what is kept for sure
    unsigned some[kRanked];                // of what may be kept: index, logit
    float some_logit[kRanked];
    u64 in_bin;                            // of the target, what its bin has to give
    float per;                             // bins per unit of a logit, of top_p rows
    unsigned n_some, fits, unused;         // fits: the above says it all, if n_some does not pass kRanked; 2: the list alone
};
// And each slice of a top_p row.
struct SliceState {
    u64 weight[kBins], sum, unused;
};

struct SampleParams {
    kv_sample_args_t a;
    RowState *rows;   // null: a workgroup a row does it all
    SliceState *slice_of;
    int slices;
    int shift;        // log2 of the weights' unit
    int tile;         // log2 of the tokens of a tile
};

// A logit's bits as a number that grows with it; -0 is 0.
__device__ __forceinline__ unsigned key_of(float x)
{
    const unsigned b = __float_as_uint(x + 0.f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(unsigned key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
// Where a token is in the order: larger ones come first. Keys are never zero.
__device__ __forceinline__ u64 place_of(unsigned key, int i) { return (u64)key << 32 | (unsigned)~i; }

template <int DTYPE> constexpr int kVector = DTYPE == KV_F32 ? 4 : 8;   // logits of a load of 16 bytes

template <int DTYPE>
__device__ __forceinline__ float logit_at(const void *row, long long i)
{
    if constexpr (DTYPE == KV_F32) return ((const float *)row)[i];
    else if constexpr (DTYPE == KV_F16) return (float)((const _Float16 *)row)[i];
    else return __uint_as_float((unsigned)((const unsigned short *)row)[i] << 16);
}

template <int DTYPE>
__device__ __forceinline__ void unpack(uint4 w, float (&l)[kVector<DTYPE>])
{
    const unsigned x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < kVector<DTYPE>; ++e) {
        if constexpr (DTYPE == KV_F32) l[e] = __uint_as_float(x[e]);
        else if constexpr (DTYPE == KV_BF16) l[e] = __uint_as_float(e % 2 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
        else l[e] = (float)__builtin_bit_cast(_Float16, (unsigned short)(e % 2 ? x[e / 2] >> 16 : x[e / 2]));
    }
}

// each(logits, first index, their number) for the loads of 16 bytes of a row that fall to thread `tid` of `threads`, AHEAD at a time; what lies before the first aligned one, and after the last,
// goes to a thread each. A wavefront's loads lie side by side; with some lanes missing in the end.
template <int DTYPE, int AHEAD, typename F>
__device__ __forceinline__ void for_loads(const char *row, int V, int tid, int threads, const F &each)
{
    constexpr int E = kVector<DTYPE>, kBytes = 16 / E;
    const int before = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / kBytes), vectors = (V - before) / E, after = before + vectors * E;
    if (tid < before + V - after) {   // at most 2 (E - 1)
        const int i = tid < before ? tid : after + tid - before;
        float l[E] = {};
        l[0] = logit_at<DTYPE>(row, i);
        each(l, i, 1);
    }
    const uint4 *const at = (const uint4 *)(row + (long long)before * kBytes);
    auto unpacked = [&](uint4 w, int v) {
        float l[E];
        unpack<DTYPE>(w, l);
        each(l, before + v * E, E);
    };
    int v = tid;
    if constexpr (AHEAD > 1) {
        for (; v + (AHEAD - 1) * threads < vectors; v += AHEAD * threads) {
            uint4 w[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) w[k] = at[v + k * threads];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) unpacked(w[k], v + k * threads);
        }
    }
    // the next one is loaded before one is worked on
    uint4 next = v < vectors ? at[v] : uint4{};
#pragma unroll 1
    for (; v < vectors; v += threads) {
        const uint4 w = next;
        if (v + threads < vectors) next = at[v + threads];
        unpacked(w, v);
    }
}
// f(logit, index) for each, of a workgroup's row.
template <int DTYPE, typename F>
__device__ __forceinline__ void for_logits(const char *row, int V, int tid, const F &f)
{
    for_loads<DTYPE, 1>(row, V, tid, kThreads, [&](const float (&l)[kVector<DTYPE>], int i, int n) {
#pragma unroll
        for (int e = 0; e < kVector<DTYPE>; ++e)
            if (e < n) f(l[e], i + e);
    });
}

// x moved by a data-parallel primitive (of which lanes without a source get 0)
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 x)
{
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)x, CTRL, ROWS, 0xf, false), hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(x >> 32), CTRL, ROWS, 0xf, false);
    return (u64)hi << 32 | lo;
}
// Sums over the lanes up to each: 1, 2, 4, 8 of a row of 16, then over rows. All lanes take part.
__device__ __forceinline__ u64 wave_sums_to(u64 x)
{
    x += moved<0x111, 0xf>(x);
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);
    x += moved<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ u64 of_lane(u64 x, int l)
{
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(x >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)x, l);
}
__device__ __forceinline__ u64 wave_sum(u64 x) { return of_lane(wave_sums_to(x), 63); }

// 2^(i / 256), by the series of e^x.
struct ExpTable {
    double of[kExpTable];
    constexpr ExpTable() : of()
    {
        for (int i = 0; i < kExpTable; ++i) {
            double sum = 1., term = 1.;
            for (int k = 1; k < 24; ++k) sum += term *= i * 0.6931471805599453 / kExpTable / k;
            of[i] = sum;
        }
    }
};
__device__ const ExpTable kExps{};

// A thread's sum of the logits from i on to their tile's: 64 loads side by side are of one.
template <typename R>
__device__ __forceinline__ void add_to_tile(const R &row, int i, u64 sum, u64 *weight)
{
    if (__ballot(1) == ~0ull) {
        sum = wave_sum(sum);
        if ((threadIdx.x & 63) == 0) atomicAdd(&weight[row.tile_of(i)], sum);
    } else {
        atomicAdd(&weight[row.tile_of(i)], sum);
    }
}

// A row, and what is asked of it.
template <int DTYPE>
struct Row {
    static constexpr int E = kVector<DTYPE>;
    const char *at;
    int V, shift, tile, before_loads, n_tiles;
    float T, top_p, min_p, top;
    unsigned k;
    bool greedy, cut_k, cut_p;
    float least;          // what is below does not weigh min_p
    double per_unit, top64;
    const double *exps;   // 2^(i / 256)

    __device__ __forceinline__ Row(const SampleParams &p, int b)
    {
        const kv_sample_args_t &a = p.a;
        at = (const char *)a.logits + (long long)b * a.stride * (16 / E);
        V = a.n_vocab;
        shift = p.shift;
        tile = p.tile;
        before_loads = min(V, (int)((16 - ((uintptr_t)at & 15)) & 15) / (16 / E));
        n_tiles = max(1, ((V - before_loads - 1) >> tile) + 1);
        T = a.temperature ? a.temperature[b] : 1.f;
        greedy = !(T > 0.f);
        const int asked = greedy ? 1 : a.top_k ? a.top_k[b] : 0;
        k = asked <= 0 || asked > V ? (unsigned)V : (unsigned)asked;
        cut_k = k < (unsigned)V;
        top_p = greedy || !a.top_p ? 1.f : a.top_p[b];
        cut_p = top_p < 1.f;
        min_p = greedy || !a.min_p ? 0.f : fminf(a.min_p[b], 1.f);
    }
    __device__ __forceinline__ void set_top(float t, const double *table)
    {
        top = t;
        top64 = t;
        per_unit = greedy ? 0. : 1.4426950408889634 * kExpTable / (double)T;
        exps = table;
        // less some units of its own rounding
        least = min_p > 0.f ? (float)(top64 + log((double)min_p) * (double)T) - 1.0e-5f * (fabsf(top) + 1.f) - 1.0e-5f * T : -INFINITY;
        if (!(least == least)) least = -INFINITY;
    }
    // exp((l - max) / T) * 2^shift = 2^(n / 256 + g / 256 + shift) with |g| <= 1/2: a table, and e^(g ln 2 / 256) by its series (the next term is below 2^-54). What is below 2^-60 counts as that.
    __device__ __forceinline__ double scaled_weight(float x, int by) const
    {
        static_assert(kExpTable == 256, "8 bits");
        constexpr double c = 0.6931471805599453 / kExpTable;
        const double y = fmax(((double)x - top64) * per_unit, -60. * kExpTable);   // the bound for an infinity times zero as well
        const double n = rint(y), g = y - n;
        const int i = (int)n;
        const double e = fma(g, fma(g, fma(g, fma(g, c * c * c * c / 24, c * c * c / 6), c * c / 2), c), 1.);
        return ldexp(exps[i & (kExpTable - 1)] * e, (i >> 8) + by);
    }
    __device__ __forceinline__ bool weighs(float x) const { return !(min_p > 0.f) || scaled_weight(x, 0) >= (double)min_p; }
    // to the nearest integer by adding 2^52, whose lowest bit is worth one
    __device__ __forceinline__ u64 units_of(float x) const { return (u64)__double_as_longlong(scaled_weight(x, shift) + 4503599627370496.) & 0xfffffffffffffull; }
    // Tiles begin where loads of 16 bytes do; what is before that is of the first.
    __device__ __forceinline__ int tile_of(int i) const { return max(0, i - before_loads) >> tile; }
    __device__ __forceinline__ int tile_begin(int t) const { return t == 0 ? 0 : before_loads + (t << tile); }
    __device__ __forceinline__ int tile_end(int t) const { return min(V, before_loads + ((t + 1) << tile)); }

    __device__ __forceinline__ float largest(int tid, int threads) const
    {
        float t = -INFINITY;
        for_loads<DTYPE, 8>(at, V, tid, threads, [&](const float (&l)[E], int, int n) {
            if (n == 1) {
                t = l[0] <= FLT_MAX ? fmaxf(t, l[0]) : INFINITY;
                return;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) t = l[e] <= FLT_MAX ? fmaxf(t, l[e]) : INFINITY;
        });
        return t;
    }
    // Every thread's part of a sample, a load of each of up to 1024, eights of which are a cache line, and how many logits that is in all: about the sum of the weights.
    __device__ __forceinline__ int sample_size() const { return min((V - before_loads) / E, kThreads) * E; }
    __device__ __forceinline__ float sampled(int i) const
    {
        const unsigned vectors = (unsigned)(V - before_loads) / E;
        float x = 0.f;
        if ((unsigned)i < vectors) {
            float l[E];
            unpack<DTYPE>(((const uint4 *)(at + (long long)before_loads * (16 / E)))[vectors > kThreads ? (unsigned)(i / 8) * vectors / (kThreads / 8) + i % 8 : i], l);
#pragma unroll
            for (int e = 0; e < E; ++e) x += __expf((l[e] - top) / T);
        }
        return x;
    }
    // Bins per unit of a logit: they reach down to a quarter of the weight that is looked for; the largest alone weighs 1. 0: no such thing.
    __device__ __forceinline__ float bins_per_unit(float sample) const
    {
        const int n = sample_size();
        const float sum = fmaxf(1.f, n > 0 ? sample * (float)V / (float)n : 1.f);
        const float reach = fminf(T * __logf(4.f * (float)V / ((1.f - fmaxf(top_p, 0.f)) * sum)), T * 42.f), per = (float)kBins / reach;
        return reach > 0.f && reach <= FLT_MAX && per <= FLT_MAX ? per : 0.f;
    }
    // Sum of this thread's weights, and the histogram.
    __device__ __forceinline__ u64 sum_and_bins(int tid, int threads, float per, u64 *weight) const
    {
        u64 sum = 0;
        for_loads<DTYPE, 1>(at, V, tid, threads, [&](const float (&l)[E], int, int n) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (e >= n) break;
                const u64 w = units_of(l[e]);
                sum += w;
                const float bin = (top - l[e]) * per;
                if (bin < (float)kBins) atomicAdd(&weight[(int)bin], w);
            }
        });
        return sum;
    }
    // The histogram of numbers of tokens.
    __device__ __forceinline__ void count_bins(int tid, int threads, float per, u64 *count) const
    {
        for_loads<DTYPE, 4>(at, V, tid, threads, [&](const float (&l)[E], int, int n) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float bin = (top - l[e]) * per;
                if (e < n && bin < (float)kBins) atomicAdd(&count[(int)bin], 1ull);
            }
        });
    }
    __device__ __forceinline__ void sum_tiles(int tid, int threads, u64 *weight) const
    {
        for_loads<DTYPE, 1>(at, V, tid, threads, [&](const float (&l)[E], int i, int n) {
            u64 sum = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) sum += e < n ? units_of(l[e]) : 0;
            add_to_tile(*this, i, sum, weight);
        });
    }
    __device__ __forceinline__ bool nothing_cut() const { return !greedy && !cut_k && !cut_p && !(min_p > 0.f); }
    __device__ __forceinline__ bool by_bins() const { return !cut_k && cut_p; }
    __device__ __forceinline__ bool few() const { return cut_k && k <= 256; }
    __device__ __forceinline__ bool by_counts() const { return cut_k && k > 256 && !cut_p; }
    __device__ __forceinline__ u64 target_of(u64 sum) const   // of top_p
    {
        const double want = ceil((double)(top_p > 0.f ? top_p : 0.f) * (double)sum);
        return max((u64)1, min((u64)want, sum));
    }
};

// A row that fits the registers of a workgroup's threads: eight loads of 16 bytes each, and what lies before and after the aligned ones. Read once instead of twice: 256 rows of 32000 in 32 bits 15.1 -> 13.9 us.
template <int DTYPE>
struct HeldRow {
    static constexpr int kLoads = 8, E = kVector<DTYPE>;
    uint4 w[kLoads];
    float odd;
    int odd_at, before, vectors;

    static __device__ __forceinline__ bool fits(const Row<DTYPE> &row) { return (row.V - row.before_loads) / E <= kLoads * kThreads; }
    // -infinity where there is nothing
    __device__ __forceinline__ void load(const Row<DTYPE> &row, int tid)
    {
        constexpr unsigned none = DTYPE == KV_F32 ? 0xff800000u : DTYPE == KV_F16 ? 0xfc00fc00u : 0xff80ff80u;
        before = row.before_loads;
        vectors = (row.V - before) / E;
        const int after = before + vectors * E;
        const uint4 *const at = (const uint4 *)(row.at + (long long)before * (16 / E));
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            if (k * kThreads >= vectors) break;
            const int v = tid + k * kThreads;
            w[k] = v < vectors ? at[v] : uint4{none, none, none, none};
        }
        odd_at = tid < before ? tid : after + tid - before;
        odd = tid < before + row.V - after ? logit_at<DTYPE>(row.at, odd_at) : -INFINITY;
    }
    // each(logits, first index, their number)
    template <typename F>
    __device__ __forceinline__ void for_loads(int tid, const F &each) const
    {
        float l[E] = {};
        l[0] = odd;
        each(l, odd_at, 1);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            if (k * kThreads >= vectors) break;
            unpack<DTYPE>(w[k], l);
            each(l, before + (tid + k * kThreads) * E, E);
        }
    }
    __device__ __forceinline__ float largest(int tid) const
    {
        float t = -INFINITY;
        for_loads(tid, [&](const float (&l)[E], int, int n) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < n) t = l[e] <= FLT_MAX ? fmaxf(t, l[e]) : INFINITY;
        });
        return t;
    }
};

struct Shared {
    double exps[kExpTable];
    u64 weight[kBins];
    unsigned count[kBins];
    u64 tile_weight[kTiles];
    u64 ranked[kRanked];            // (key, ~index): what is larger comes first
    u64 ranked_weight[kRanked];
    unsigned some[kRanked];
    float some_logit[kRanked];
    unsigned n_some;
    u64 wave_u64[kWaves];
    unsigned wave_u32[kWaves];
    float wave_f32[kWaves];
    // what one thread tells the others
    u64 told_weight, told_all, told_above;
    unsigned told_bin;
};

// A workgroup's steps that all of its threads take together.
struct Group {
    Shared &s;
    int tid, lane, wave;
    __device__ __forceinline__ explicit Group(Shared &shared) : s(shared), tid(threadIdx.x), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) {}

    __device__ __forceinline__ void begin()
    {
        if (tid < kExpTable) s.exps[tid] = kExps.of[tid];
        if (tid == 0) s.n_some = 0;
    }
    // Sums over the wavefronts up to each, in the lanes of their numbers.
    __device__ __forceinline__ u64 waves_to(u64 of_wave, int from_lane)
    {
        static_assert(kWaves == 16, "a row of lanes");
        __syncthreads();
        if (lane == from_lane) s.wave_u64[wave] = of_wave;
        __syncthreads();
        u64 x = s.wave_u64[lane & 15];
        x += moved<0x111, 0xf>(x);
        x += moved<0x112, 0xf>(x);
        x += moved<0x114, 0xf>(x);
        x += moved<0x118, 0xf>(x);
        return x;
    }
    // Sum, in every thread.
    __device__ __forceinline__ u64 sum_of(u64 x) { return of_lane(waves_to(wave_sums_to(x), 63), 15); }
    // Sum over the threads before this one, and of all.
    __device__ __forceinline__ u64 sum_before(u64 x, u64 *all = nullptr)
    {
        const u64 to = wave_sums_to(x), waves = waves_to(to, 63);
        if (all) *all = of_lane(waves, 15);
        return to - x + (wave > 0 ? of_lane(waves, max(wave - 1, 0)) : 0);
    }
    __device__ __forceinline__ float largest_of(float x)
    {
#pragma unroll
        for (int o = 1; o < 64; o *= 2) x = fmaxf(x, __shfl_xor(x, o));
        __syncthreads();
        if (lane == 0) s.wave_f32[wave] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x = fmaxf(x, s.wave_f32[w]);
        return x;
    }
    __device__ __forceinline__ float sum_of_f32(float x)
    {
#pragma unroll
        for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o);
        __syncthreads();
        if (lane == 0) s.wave_f32[wave] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += s.wave_f32[w];
        return x;
    }
    // Lists: `which` has a bit for each of this thread's logits that goes there; one counter's step for a wavefront's loads.
    template <int E>
    __device__ __forceinline__ void append(const float (&l)[E], int i, unsigned which, unsigned *n, unsigned *to, float *logits, unsigned room)
    {
        const u64 active = __ballot(1);
        if (__ballot(which != 0) == 0) return;
        unsigned at;
        const unsigned count = (unsigned)__popc(which);
        if (active == ~0ull) {
            const unsigned upto = (unsigned)wave_sums_to(count);
            unsigned first = 0;
            if (lane == 63) first = atomicAdd(n, upto);
            at = (unsigned)__builtin_amdgcn_readlane((int)first, 63) + upto - count;
        } else {
            at = count ? atomicAdd(n, count) : 0;
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (which >> e & 1) {
                if (at < room) to[at] = (unsigned)(i + e), logits[at] = l[e];
                ++at;
            }
    }
    // Adds up in s.tile_weight what of the row's share (tid of threads) is kept: logits from `sure` on, but none that is after `border` in the order or weighs too little. Those from `from` on and below
    // `sure` go to the list. Weights are taken where a wavefront has any: a dense list of what is kept, in LDS, took longer to write than the weights of idle lanes.
    template <int DTYPE>
    __device__ __forceinline__ void keep(const Row<DTYPE> &row, int tid, int threads, float sure, float from, u64 border)
    {
        constexpr int E = kVector<DTYPE>;
        for_loads<DTYPE, 1>(row.at, row.V, tid, threads, [&](const float (&l)[E], int i, int n) {
            unsigned some = 0;
            u64 sum = 0;
            bool any = false;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool is = e < n && l[e] >= from && l[e] >= row.least, certain = is && l[e] >= sure && place_of(key_of(l[e]), i + e) >= border;
                some |= is && l[e] < sure ? 1u << e : 0;
                if (__ballot(certain) == 0) continue;
                any = true;
                sum += certain && row.weighs(l[e]) ? row.units_of(l[e]) : 0;
            }
            if (any) add_to_tile(row, i, sum, s.tile_weight);
            append(l, i, some, &s.n_some, s.some, s.some_logit, kRanked);
        });
        __syncthreads();
    }
    // Where top_p ends, in the bin to which s.weight[.. bin] leads: all from `sure` on are kept, and of those from `from` on some, *in_bin of their weight. Or, as often where a few tokens have most of the
    // weight, no more than 256 tokens can have what there is from `from` on, none of which weighs less: then true, and *in_bin is of all of them.
    template <int DTYPE>
    __device__ __forceinline__ bool cut_at(const Row<DTYPE> &row, float per, unsigned bin, u64 *in_bin, float *sure, float *from)
    {
        const u64 above = s.told_above, here = s.weight[bin];
        *from = fmaxf(least_of(row, per, (float)bin + 1.f), row.least);
        if (above + here <= 256 * row.units_of(*from)) {
            *in_bin += above;
            return true;
        }
        if (bin > 0) *sure = least_of(row, per, (float)bin);
        return false;
    }
    // The list of those from `from` on alone.
    template <int DTYPE>
    __device__ __forceinline__ void list_from(const Row<DTYPE> &row, int tid, int threads, float from)
    {
        constexpr int E = kVector<DTYPE>;
        for_loads<DTYPE, 4>(row.at, row.V, tid, threads, [&](const float (&l)[E], int i, int n) {
            unsigned all = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) all |= e < n && l[e] >= from ? 1u << e : 0;
            append(l, i, all, &s.n_some, s.some, s.some_logit, kRanked);
        });
        __syncthreads();
    }
    template <int DTYPE>
    __device__ __forceinline__ void list_from(const HeldRow<DTYPE> &held, float from)
    {
        constexpr int E = kVector<DTYPE>;
        held.for_loads(tid, [&](const float (&l)[E], int i, int n) {
            unsigned all = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) all |= e < n && l[e] >= from ? 1u << e : 0;
            append(l, i, all, &s.n_some, s.some, s.some_logit, kRanked);
        });
        __syncthreads();
    }
    // Which bin of s.weight a sum of `target` is reached in, and what of it is the bin's to give; kBins: none.
    __device__ __forceinline__ unsigned bin_of_target(u64 target, u64 *in_bin)
    {
        const u64 w0 = s.weight[2 * tid], w1 = s.weight[2 * tid + 1], before = sum_before(w0 + w1);
        if (tid == 0) s.told_bin = kBins;
        __syncthreads();
        if (before < target && target <= before + w0 + w1) {
            const bool second = target > before + w0;
            s.told_bin = 2 * tid + second;
            s.told_above = before + (second ? w0 : 0);
            s.told_weight = target - s.told_above;
        }
        __syncthreads();
        *in_bin = s.told_weight;
        return s.told_bin;
    }
    // The least logit of a bin before `end`: a logit's bin never grows with it, so a search for the first finds it, 64 at a time.
    template <int DTYPE>
    __device__ __forceinline__ float least_of(const Row<DTYPE> &row, float per, float end) const
    {
        unsigned lo = key_of(-FLT_MAX), hi = key_of(row.top);   // hi is one of them, what is below lo is none
        while (lo < hi) {
            const unsigned step = (hi - lo) / 64 + 1, at = (unsigned)min((u64)lo + (u64)lane * step, (u64)hi);
            const u64 is = __ballot((row.top - logit_of(at)) * per < end);
            if (is == 0) {
                lo += 63 * step + 1;
                continue;
            }
            const int first = __ffsll((long long)is) - 1;
            hi = (unsigned)__builtin_amdgcn_readlane((int)at, first);
            if (first > 0) lo = (unsigned)__builtin_amdgcn_readlane((int)at, first - 1) + 1;
            else lo = hi;
        }
        return logit_of(hi);
    }
    // What the k-th largest is not below: at least k threads' maxima reach it. NaN: there are fewer.
    template <int DTYPE>
    __device__ __forceinline__ float reached_by(const Row<DTYPE> &row, float mine)
    {
        s.count[tid] = 0;
        const float lowest = -largest_of(-(mine == -INFINITY ? row.top : mine));
        const float span = row.top - lowest, per = span > 0.f && span <= FLT_MAX ? 1023.f / span : 0.f;
        if (mine != -INFINITY) atomicAdd(&s.count[(int)fminf((row.top - mine) * per, 1023.f)], 1u);
        __syncthreads();
        const u64 own = s.count[tid], before = sum_before(own);
        if (tid == 0) s.told_bin = kBins;
        __syncthreads();
        if (before < row.k && row.k <= before + own) s.told_bin = (unsigned)tid;
        __syncthreads();
        const unsigned last = s.told_bin;
        if (last >= (unsigned)kBins || !(span <= FLT_MAX)) return NAN;
        return least_of(row, per, (float)(last + 1));
    }
};

// The threads' maxima of a slice, and what the next launches add to.
template <int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_sample_max_kernel(SampleParams p)
{
    const Row<DTYPE> row(p, blockIdx.y);
    RowState &state = p.rows[blockIdx.y];
    const int tid = threadIdx.x;
    state.maxima[blockIdx.x][tid] = row.largest(blockIdx.x * kThreads + tid, p.slices * kThreads);
    if (blockIdx.x == 0) {
        state.tile_weight[tid] = 0;
        if (tid == 0) state.n_some = state.fits = 0;
    }
}
// The weights of a slice.
template <int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_sample_sum_kernel(SampleParams p)
{
    __shared__ Shared s;
    Row<DTYPE> row(p, blockIdx.y);
    if (!row.nothing_cut() && !row.by_bins()) return;
    RowState &state = p.rows[blockIdx.y];
    Group g(s);
    const int tid = threadIdx.x, threads = p.slices * kThreads;
    g.begin();
    float mine = -INFINITY;
    for (int j = 0; j < p.slices; ++j) mine = fmaxf(mine, state.maxima[j][tid]);
    const float top = g.largest_of(mine);
    if (!(fabsf(top) <= FLT_MAX)) return;
    row.set_top(top, s.exps);
    s.weight[tid] = s.weight[kThreads + tid] = 0;
    if (row.nothing_cut()) {
        if (blockIdx.x == 0 && tid == 0) state.fits = 1;
        row.sum_tiles(blockIdx.x * kThreads + tid, threads, state.tile_weight);
        return;
    }
    const float per = row.bins_per_unit(g.sum_of_f32(row.sampled(tid)));
    if (blockIdx.x == 0 && tid == 0) state.per = per;
    if (per == 0.f) return;
    SliceState &slice = p.slice_of[blockIdx.y * p.slices + blockIdx.x];
    const u64 sum = g.sum_of(row.sum_and_bins(blockIdx.x * kThreads + tid, threads, per, s.weight));
    if (tid == 0) slice.sum = sum;
    slice.weight[tid] = s.weight[tid];
    slice.weight[kThreads + tid] = s.weight[kThreads + tid];
}
// What of a slice is kept for sure, and what may be.
template <int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_sample_keep_kernel(SampleParams p)
{
    __shared__ Shared s;
    Row<DTYPE> row(p, blockIdx.y);
    if (row.greedy || row.nothing_cut() || (row.cut_k && !row.few())) return;
    RowState &state = p.rows[blockIdx.y];
    Group g(s);
    const int tid = threadIdx.x, threads = p.slices * kThreads;
    g.begin();
    float mine = -INFINITY;
    for (int j = 0; j < p.slices; ++j) mine = fmaxf(mine, state.maxima[j][tid]);
    const float top = g.largest_of(mine);
    if (!(fabsf(top) <= FLT_MAX)) return;
    row.set_top(top, s.exps);
    s.tile_weight[tid] = 0;
    float sure = INFINITY, from;
    bool whole = row.few();   // a list has all that may be kept
    if (row.few()) {
        from = g.reached_by(row, mine);
        if (!(from == from)) return;
    } else if (row.cut_p) {
        const float per = state.per;
        if (per == 0.f) return;
        const SliceState *const slices = p.slice_of + blockIdx.y * p.slices;
        u64 sum = 0, w[2] = {0, 0};
        for (int j = 0; j < p.slices; ++j) {
            w[0] += slices[j].weight[tid];
            w[1] += slices[j].weight[kThreads + tid];
            sum += slices[j].sum;
        }
        s.weight[tid] = w[0];
        s.weight[kThreads + tid] = w[1];
        __syncthreads();
        u64 in_bin;
        const unsigned bin = g.bin_of_target(row.target_of(sum), &in_bin);
        if (bin >= (unsigned)kBins) return;
        whole = g.cut_at(row, per, bin, &in_bin, &sure, &from);
        if (blockIdx.x == 0 && tid == 0) state.in_bin = in_bin;
    } else {
        sure = from = row.least;
    }
    if (blockIdx.x == 0 && tid == 0) state.fits = whole ? 2 : 1;
    __syncthreads();
    if (whole) g.list_from(row, blockIdx.x * kThreads + tid, threads, from);
    else g.keep(row, blockIdx.x * kThreads + tid, threads, sure, from, 0);
    const unsigned n = s.n_some;
    if (tid == 0) s.told_bin = n ? atomicAdd(&state.n_some, n) : 0;
    __syncthreads();
    if (const unsigned to = s.told_bin + tid; (unsigned)tid < n && to < (unsigned)kRanked) {
        state.some[to] = s.some[tid];
        state.some_logit[to] = s.some_logit[tid];
    }
    if (const u64 w = s.tile_weight[tid]; w != 0) atomicAdd(&state.tile_weight[tid], w);
}

template <int DTYPE>
__global__ void __launch_bounds__(kThreads) kv_sample_kernel(SampleParams p)
{
    __shared__ Shared s;
    Group g(s);
    const int tid = g.tid, lane = g.lane, wave = g.wave;
    const int b = blockIdx.x;
    Row<DTYPE> row(p, b);
    const RowState *const state = p.rows ? p.rows + b : nullptr;
    const int V = row.V;
    const float T = row.T;
    const unsigned k = row.k;
    auto answer = [&](int token, float prob) {
        p.a.tokens[b] = token;
        if (p.a.probs) p.a.probs[b] = prob;
    };
    float u = p.a.u[b];
    u = u > 0.f ? u : 0.f;

    // The largest logit, and this thread's own; a NaN or +infinity makes it +infinity.
    g.begin();
    float mine = -INFINITY;
    HeldRow<DTYPE> held;   // read once, where few of the largest are all that is wanted
    const bool is_held = !state && row.few() && HeldRow<DTYPE>::fits(row);
    if (state) {
        for (int j = 0; j < p.slices; ++j) mine = fmaxf(mine, state->maxima[j][tid]);
    } else if (is_held) {
        held.load(row, tid);
        mine = held.largest(tid);
    } else {
        mine = row.largest(tid, kThreads);
    }
    const float top = g.largest_of(mine);
    if (!(fabsf(top) <= FLT_MAX)) {
        if (tid == 0) answer(-1, 0.f);
        return;
    }
    row.set_top(top, s.exps);
    s.tile_weight[tid] = 0;

    // The border: kept is what is not after it in the order (and weighs enough).
    u64 border = 0;
    auto pick = [&] {   // tile_weight holds the sums of what is kept
        __syncthreads();
        u64 all;
        const u64 own = tid < row.n_tiles ? s.tile_weight[tid] : 0, before = g.sum_before(own, &all);
        const double at = (double)u * (double)all;
        const u64 target = min((u64)at, all - 1);   // the largest has a weight: all > 0
        if (before <= target && target < before + own) {
            s.told_bin = (unsigned)tid;
            s.told_weight = before;
        }
        __syncthreads();
        // a thread a token
        const int t = (int)s.told_bin, end = row.tile_end(t);
        u64 sum = s.told_weight;
        for (int i0 = row.tile_begin(t); i0 < end; i0 += kThreads) {
            const int i = i0 + tid;
            const float x = i < end ? logit_at<DTYPE>(row.at, i) : -INFINITY;
            const u64 w = i < end && place_of(key_of(x), i) >= border && row.weighs(x) ? row.units_of(x) : 0;
            u64 here;
            const u64 from = sum + g.sum_before(w, &here);
            if (from <= target && target < from + w) answer(i, (float)(row.scaled_weight(x, p.shift) / (double)all));
            sum += here;
            if (sum > target) return;
        }
    };
    static_assert(kTiles == kThreads, "a tile each");
    // Of s.ranked[0 .. n): the number, and the sum of weights, before each in the order.
    auto before_in_order = [&](int n, u64 *weight) {
        unsigned before = 0;
        *weight = 0;
        if (tid < n) {
            const u64 own = s.ranked[tid];
#pragma unroll 8
            for (int j = 0; j < n; ++j) {
                const u64 place = s.ranked[j], w = s.ranked_weight[j];   // both loaded, whatever the one says
                before += place > own;
                *weight += place > own ? w : 0;
            }
        }
        return before;
    };

    if (row.greedy) {   // the first of the largest
        int at = INT_MAX;
        if (mine == top) for_logits<DTYPE>(row.at, V, tid, [&](float x, int i) { at = x == top ? min(at, i) : at; });
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

    // What is kept for sure, in s.tile_weight, and what may be: s.some
    bool fits = false, whole = row.few();   // whole: s.some alone has all of it
    u64 in_bin = 0;
    if (state && !row.by_counts()) {
        fits = state->fits != 0 && state->n_some <= (unsigned)kRanked;
        if (fits) {
            whole = whole || state->fits == 2;
            s.tile_weight[tid] = state->tile_weight[tid];
            if (tid < (int)state->n_some) s.some[tid] = state->some[tid], s.some_logit[tid] = state->some_logit[tid];
            if (tid == 0) s.n_some = state->n_some;
            in_bin = state->in_bin;
        }
    } else if (row.nothing_cut()) {
        __syncthreads();
        row.sum_tiles(tid, kThreads, s.tile_weight);
        fits = true;
    } else if (row.few() || row.cut_p == false || row.by_bins()) {
        float sure = INFINITY, from = NAN;
        if (row.few()) {
            from = g.reached_by(row, mine);
        } else if (row.by_bins()) {
            s.weight[tid] = s.weight[kThreads + tid] = 0;
            const float per = row.bins_per_unit(g.sum_of_f32(row.sampled(tid)));
            if (per != 0.f) {
                const u64 sum = g.sum_of(row.sum_and_bins(tid, kThreads, per, s.weight));
                const unsigned bin = g.bin_of_target(row.target_of(sum), &in_bin);
                if (bin < (unsigned)kBins) whole = g.cut_at(row, per, bin, &in_bin, &sure, &from);
            }
        } else if (row.by_counts()) {
            s.weight[tid] = s.weight[kThreads + tid] = 0;
            __syncthreads();
            const float per = 64.f / T;
            if (per <= FLT_MAX) {
                row.count_bins(tid, kThreads, per, s.weight);
                __syncthreads();
                const unsigned bin = g.bin_of_target(k, &in_bin);
                if (bin < (unsigned)kBins) {
                    if (bin > 0) sure = g.least_of(row, per, (float)bin);
                    from = g.least_of(row, per, (float)bin + 1.f);
                }
            }
        } else if (!row.cut_k) {
            sure = from = row.least;
        }
        if (from == from) {
            __syncthreads();
            if (is_held) g.list_from(held, from);
            else if (whole) g.list_from(row, tid, kThreads, from);
            else g.keep(row, tid, kThreads, sure, from, 0);
            fits = s.n_some <= (unsigned)kRanked;
        }
    }
    if (fits) {
        __syncthreads();
        const int n = (int)s.n_some;
        if (whole && n <= 64) {
            // A wavefront has them all, a lane each, and needs nobody else (the largest 50 of 32000 with top_p: 15.6 -> 12.5 us, and 11.6 with the row held).
            if (wave != 0) return;
            const int i = lane < n ? (int)s.some[lane] : INT_MAX;
            const float x = lane < n ? s.some_logit[lane] : -INFINITY;
            const u64 own = lane < n ? place_of(key_of(x), i) : 0, weight = lane < n ? row.units_of(x) : 0;
            // Sums over those that are before this one, in the order, then by index. Of the first k all that are ahead of one are of them too.
            auto sums = [&](u64 place, u64 w, auto counts) {
                // what the lanes have read before is read, and what they write is there for all of them after: an order for the compiler, LDS keeps it by itself
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
                __builtin_amdgcn_wave_barrier();
                s.ranked[lane] = place;
                s.ranked_weight[lane] = w;
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
                __builtin_amdgcn_wave_barrier();
                for (int j0 = 0; j0 < n; j0 += 16) {
                    u64 at[16], of[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) at[j] = s.ranked[j0 + j], of[j] = s.ranked_weight[j0 + j];
#pragma unroll
                    for (int j = 0; j < 16; ++j) counts(at[j] > place, of[j]);
                }
            };
            unsigned ahead = 0;
            u64 before = 0;
            sums(own, weight, [&](bool is, u64 w) { ahead += is, before += is ? w : 0; });
            bool in = lane < n && ahead < k;
            if (row.cut_p) {   // all lanes take part in a sum
                const u64 sum = wave_sum(in ? weight : 0), target = row.few() ? row.target_of(sum) : in_bin;
                in = in && before < target;
            }
            const u64 kept = in && row.weighs(x) ? weight : 0, all = wave_sum(kept);
            const u64 target = min((u64)((double)u * (double)all), all - 1);   // the largest has a weight: all > 0
            before = 0;
            sums((u64)(unsigned)~i, kept, [&](bool is, u64 w) { before += is ? w : 0; });
            if (before <= target && target < before + kept) answer(i, (float)(row.scaled_weight(x, p.shift) / (double)all));
            return;
        }
        const float x = tid < n ? s.some_logit[tid] : 0.f;
        if (tid < n) {
            s.ranked[tid] = place_of(key_of(x), (int)s.some[tid]);
            s.ranked_weight[tid] = row.units_of(x);
        }
        if (tid == 0) s.told_all = n > 0 ? ~0ull : 0;
        __syncthreads();
        bool in = tid < n;
        u64 weight;
        const unsigned ahead = before_in_order(n, &weight);
        if (row.few()) {   // of the first k all that are ahead of one are of them too
            in = in && ahead < k;
            if (row.cut_p) {   // all threads take part in a sum
                const u64 target = row.target_of(g.sum_of(in ? s.ranked_weight[tid] : 0));
                in = in && weight < target;
            }
        } else {
            in = in && (row.by_counts() ? ahead : weight) < in_bin;
        }
        if (in) {
            atomicMin(&s.told_all, s.ranked[tid]);
            if (row.weighs(x)) atomicAdd(&s.tile_weight[row.tile_of((int)s.some[tid])], s.ranked_weight[tid]);
        }
        __syncthreads();
        border = s.told_all;
        pick();
        return;
    }
    __syncthreads();

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
            for_logits<DTYPE>(row.at, V, tid, [&](float x, int) {
                const unsigned key = key_of(x);
                if (key < low || key > high) return;
                const unsigned at = bin_of(x, key);
                atomicAdd(&s.count[at], 1u);
                atomicAdd(&s.weight[at], row.units_of(x));
            });
            __syncthreads();
            // sums before each bin: a thread has two
            const u64 c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1], w0 = s.weight[2 * tid], w1 = s.weight[2 * tid + 1];
            const u64 counts = above + g.sum_before(c0 + c1), weights = above_weight + g.sum_before(w0 + w1);
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
                for_logits<DTYPE>(row.at, V, tid, [&](float x, int) {
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
    if (row.cut_k) find_border(std::false_type{}, (u64)k, 0u);
    if (row.cut_p) {
        if (!row.cut_k) {   // the sum of all
            u64 sum = 0;
            for_logits<DTYPE>(row.at, V, tid, [&](float x, int) { sum += row.units_of(x); });
            kept = g.sum_of(sum);
        }
        // no more than the top-k's keys; what of its border's key is past k counts in no sum before the target, which is at most theirs
        const u64 target = row.target_of(kept);
        const unsigned k_border = border_key, k_ties = ties;
        find_border(std::true_type{}, target, border_key);
        if (border_key == k_border && row.cut_k) ties = min(ties, k_ties);
    }

    // Tiles: how many have the border's key; the last of these that is kept is the border.
    if (border_key != 0) {
        __syncthreads();
        s.count[tid] = 0;
        if (tid == 0) s.told_all = 0;
        __syncthreads();
        for_logits<DTYPE>(row.at, V, tid, [&](float x, int i) {
            if (key_of(x) == border_key) atomicAdd(&s.count[row.tile_of(i)], 1u);
        });
        __syncthreads();
        const u64 equal = s.count[tid], before = g.sum_before(equal);
        if (before < ties && before + equal >= ties) s.told_all = (u64)(ties - before) << 32 | (unsigned)tid;   // the last one is in this tile
        __syncthreads();
        border = place_of(border_key, INT_MAX);
        if (s.told_all != 0) {
            // every wavefront for itself
            unsigned left = (unsigned)(s.told_all >> 32);
            const int t = (int)(unsigned)s.told_all, end = row.tile_end(t);
            for (int i0 = row.tile_begin(t); i0 < end; i0 += 64) {
                const int i = i0 + lane;
                u64 is = __ballot(i < end && key_of(logit_at<DTYPE>(row.at, min(i, end - 1))) == border_key);
                const unsigned n = (unsigned)__popcll(is);
                if (n >= left) {
                    for (; left > 1; --left) is &= is - 1;
                    border = place_of(border_key, i0 + __ffsll((long long)is) - 1);
                    break;
                }
                left -= n;
            }
        }
    }
    __syncthreads();
    s.tile_weight[tid] = 0;
    __syncthreads();
    const float from = border_key != 0 ? logit_of(border_key) : -FLT_MAX;
    g.keep(row, tid, kThreads, from, from, border);
    pick();
}

}  // namespace

static int slices_of(int n_rows, int n_vocab)
{
    // 128 rows fill half of the card by themselves; short rows are over before another launch has begun
    if (n_rows < 1 || n_rows >= 128 || n_vocab <= 65536) return 1;
    int slices = kMostSlices;   // a power of two: equal shares of a row's threads
    while (slices * n_rows > 256) slices /= 2;
    return slices;
}

extern "C" size_t kv_sample_workspace(int n_rows, int n_vocab)
{
    if (n_rows < 0 || n_vocab < 0) return 0;
    // what fewer rows need as well: they may be shared by more slices
    size_t most = 16;
    for (int n = 1; n <= std::min(n_rows, 127); ++n)
        if (const int slices = slices_of(n, n_vocab); slices > 1) most = std::max(most, n * (sizeof(RowState) + slices * sizeof(SliceState)));
    return most;
}

extern "C" int kv_sample(const kv_sample_args_t *a, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!a || !workspace || ((uintptr_t)workspace & 15)) return KV_EINVAL;
    if (a->dtype != KV_F16 && a->dtype != KV_BF16 && a->dtype != KV_F32) return KV_EINVAL;
    if (a->n_rows < 0 || a->n_vocab < 1 || a->stride < 0) return KV_EINVAL;
    if (ws_bytes < kv_sample_workspace(a->n_rows, a->n_vocab)) return KV_ENOSPC;
    if (a->n_rows == 0) return KV_OK;
    if (a->n_vocab > 1 << 24 || (uint64_t)a->n_rows * kThreads >= 1ull << 32) return KV_ERANGE;   // threads of a launch
    if (!a->logits || !a->u || !a->tokens || ((uintptr_t)a->logits & (a->dtype == KV_F32 ? 3 : 1))) return KV_EINVAL;
    SampleParams p{};
    p.a = *a;
    int bits = 0;
    while ((1 << bits) < a->n_vocab) ++bits;
    p.shift = std::min(51, 62 - bits);
    p.tile = 9;
    while (((a->n_vocab - 1) >> p.tile) >= kTiles) ++p.tile;
    p.slices = slices_of(a->n_rows, a->n_vocab);
    p.rows = p.slices > 1 ? (RowState *)workspace : nullptr;
    p.slice_of = (SliceState *)((RowState *)workspace + a->n_rows);
    auto of = [&](auto f32, auto f16, auto bf16) { return a->dtype == KV_F32 ? f32 : a->dtype == KV_F16 ? f16 : bf16; };
    hipStream_t st = (hipStream_t)hip_stream;
    if (p.rows) {
        const dim3 grid((unsigned)p.slices, (unsigned)a->n_rows), block(kThreads);
        (void)launch_kernel(of(kv_sample_max_kernel<KV_F32>, kv_sample_max_kernel<KV_F16>, kv_sample_max_kernel<KV_BF16>), grid, block, st, p);
        (void)launch_kernel(of(kv_sample_sum_kernel<KV_F32>, kv_sample_sum_kernel<KV_F16>, kv_sample_sum_kernel<KV_BF16>), grid, block, st, p);
        if (a->top_p || a->top_k || a->min_p) (void)launch_kernel(of(kv_sample_keep_kernel<KV_F32>, kv_sample_keep_kernel<KV_F16>, kv_sample_keep_kernel<KV_BF16>), grid, block, st, p);
    }
    (void)launch_kernel(of(kv_sample_kernel<KV_F32>, kv_sample_kernel<KV_F16>, kv_sample_kernel<KV_BF16>), dim3((unsigned)a->n_rows), dim3(kThreads), st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
