// The next token of every row of logits: temperature, top-k, top-p and min-p from given random numbers.
//
// Mathematics.  w_i = exp((l_i - max) / T) is held as an integer W_i of 2^-s, s = 62 - log2(n_vocab): sums are exact, whatever their order, so splits, histograms
// and prefix sums of any shape give one answer, and adding takes no care.  With tokens ordered by (l from the largest, index), each of the three cuts keeps a beginning of that order, so together they are
// one key (a logit's bits, ordered like the logit) and a number of tokens of that key that are kept, the first by index: all keys above it are kept.  The key at which a count
// (top-k) or a sum of weights (top-p) is reached comes from histograms: first over distances from the maximum, then over the keys of the bin in which it is, as often as its keys
// need.  The token is found in order of indices: sums of tiles, of which one is gone over again.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>

#include "launch.hpp"
#include "plan.hpp"

namespace {

using namespace kvb;

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kTiles = 1024;     // of a row, each at least 256 tokens
constexpr int kExpTable = 64;

struct SampleParams {
    kv_sample_args_t a;
    int shift;   // log2 of the weights' unit
    int tile;    // tokens of a tile, a multiple of 256
};

// A logit's bits as a number that grows with it; -0 is 0.
__device__ __forceinline__ unsigned key_of(float x)
{
    const unsigned b = __float_as_uint(x + 0.f);
    return b >> 31 ? ~b : b | 0x80000000u;
}

template <int DTYPE>
__device__ __forceinline__ float logit_at(const void *row, long long i)
{
    if constexpr (DTYPE == KV_F32) return ((const float *)row)[i];
    else if constexpr (DTYPE == KV_F16) return (float)((const _Float16 *)row)[i];
    else return __uint_as_float((unsigned)((const unsigned short *)row)[i] << 16);
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
    unsigned tile_ties[kTiles];
    u64 wave_u64[kWaves];
    unsigned wave_u32[kWaves];
    float wave_max[kWaves];
    // what one thread tells the others
    u64 told_weight, told_all;
    unsigned told_bin, told_count;
};

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

    // The largest logit; a NaN or +infinity makes it +infinity.
    for (int i = tid; i < kExpTable; i += kThreads) s.exps[i] = exp2((double)i / kExpTable);
    float top = -INFINITY;
    for (int i = tid; i < V; i += kThreads) {
        const float x = logit_at<DTYPE>(row, i);
        top = x <= FLT_MAX ? fmaxf(top, x) : INFINITY;
    }
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

    const float T = p.a.temperature ? p.a.temperature[b] : 1.f;
    const bool greedy = !(T > 0.f);
    const double per_unit = greedy ? 0. : 1.4426950408889634 * kExpTable / (double)T;
    // exp((l - max) / T) = 2^(n / 64 + r) with |r| <= 1/128: a table, and e^(r ln 2) by its series (the next term is below 2^-54)
    auto weight_of = [&](float x) -> double {
        const double y = ((double)x - (double)top) * per_unit;
        if (!(y > -64. * kExpTable)) return 0.;   // -infinity too
        const double n = rint(y), g = (y - n) * (0.6931471805599453 / kExpTable);
        const int k = (int)n;
        const double e = fma(g, fma(g, fma(g, fma(g, fma(g, 1. / 120, 1. / 24), 1. / 6), 0.5), 1.), 1.);
        return ldexp(s.exps[k & (kExpTable - 1)] * e, k >> 6);
    };
    auto units_of = [&](double w) { return (u64)rint(ldexp(w, p.shift)); };

    const int k_asked = greedy ? 1 : p.a.top_k ? p.a.top_k[b] : 0;
    const unsigned k = k_asked <= 0 || k_asked > V ? (unsigned)V : (unsigned)k_asked;
    const float top_p = greedy || !p.a.top_p ? 1.f : p.a.top_p[b];
    const float min_p = greedy || !p.a.min_p ? 0.f : fminf(p.a.min_p[b], 1.f);
    const bool cut_p = top_p < 1.f;
    float u = p.a.u[b];
    u = u > 0.f ? u : 0.f;

    // All keys above `border` are kept, and of those that equal it the first `ties`.
    unsigned border = 0, ties = (unsigned)V;
    u64 kept = 0;   // weight of what the order's beginning up to there holds, where that is known

    // The key at which a count, or a sum of weights, is reached, going down: histograms over bins of falling keys, whose bin with the border becomes the next range.
    auto find_border = [&](auto by_weight, u64 target, unsigned from_key) {
        constexpr bool W = decltype(by_weight)::value;
        // keys in [low, high] are looked at; above them there are `above` tokens of weight `above_weight`
        unsigned low = from_key, high = key_of(top);
        u64 above = 0, above_weight = 0;
        for (int round = 0;; ++round) {
            const bool by_distance = round == 0;
            int shift = 0;
            while (((high - low) >> shift) >= kBins) ++shift;
            // the first round's bins: 1/64 of a temperature's unit wide, the last one open
            const float bins_per = 64.f / fmaxf(T, 1.0e-30f);
            auto bin_of = [&](float x, unsigned key) -> unsigned {
                if (by_distance) return (unsigned)fminf((top - x) * bins_per, (float)(kBins - 1));
                return (high - key) >> shift;
            };
            for (int i = tid; i < kBins; i += kThreads) s.weight[i] = 0, s.count[i] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += kThreads) {
                const float x = logit_at<DTYPE>(row, i);
                const unsigned key = key_of(x);
                if (key < low || key > high) continue;
                const unsigned at = bin_of(x, key);
                atomicAdd(&s.count[at], 1u);
                atomicAdd(&s.weight[at], units_of(weight_of(x)));
            }
            __syncthreads();
            // sums before each bin: a thread has two
            const u64 c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1], w0 = s.weight[2 * tid], w1 = s.weight[2 * tid + 1];
            const u64 own = W ? w0 + w1 : c0 + c1;
            u64 to = wave_sums_to(own, lane);
            if (lane == 63) s.wave_u64[wave] = to;
            __syncthreads();
            u64 before = to - own;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) before += w < wave ? s.wave_u64[w] : 0;
            before += W ? above_weight : above;
            if (tid == 0) s.told_bin = kBins;
            __syncthreads();
            const u64 first = W ? w0 : c0, second = W ? w1 : c1;
            if (before < target && target <= before + first) s.told_bin = 2 * tid;
            else if (before + first < target && target <= before + first + second) s.told_bin = 2 * tid + 1;
            __syncthreads();
            const unsigned bin = s.told_bin;
            if (bin >= (unsigned)kBins) {   // all there is: more is asked for than there is
                __syncthreads();
                return;
            }
            // both sums before the bin
            u64 counts = 0, weights = 0;
            for (unsigned i = tid; i < bin; i += kThreads) counts += s.count[i], weights += s.weight[i];
            counts = wave_sum(counts);
            if (lane == 0) s.wave_u64[wave] = counts;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) above += s.wave_u64[w];
            __syncthreads();
            weights = wave_sum(weights);
            if (lane == 0) s.wave_u64[wave] = weights;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) above_weight += s.wave_u64[w];
            const unsigned in_bin = s.count[bin];
            const u64 bin_weight = s.weight[bin];
            __syncthreads();
            if (by_distance) {
                // the keys that are in the bin
                unsigned least = ~0u, most = 0;
                for (int i = tid; i < V; i += kThreads) {
                    const float x = logit_at<DTYPE>(row, i);
                    const unsigned key = key_of(x);
                    if (key >= low && key <= high && bin_of(x, key) == bin) least = min(least, key), most = max(most, key);
                }
#pragma unroll
                for (int o = 1; o < 64; o *= 2) least = min(least, (unsigned)__shfl_xor((int)least, o)), most = max(most, (unsigned)__shfl_xor((int)most, o));
                if (lane == 0) s.wave_u32[wave] = least, s.wave_u64[wave] = most;
                __syncthreads();
                low = ~0u, high = 0;
                for (int w = 0; w < kWaves; ++w) low = min(low, s.wave_u32[w]), high = max(high, (unsigned)s.wave_u64[w]);
                __syncthreads();
            } else {
                const unsigned last = high - (bin << shift);
                const unsigned least = ((1u << shift) - 1) > last - low ? low : last - ((1u << shift) - 1);
                high = last;
                low = least;
            }
            if (low == high) {   // one key: how many of its tokens
                border = low;
                const u64 each = in_bin ? bin_weight / in_bin : 0;
                if (W) ties = each == 0 ? in_bin : (unsigned)min((u64)in_bin, (target - above_weight + each - 1) / each);
                else ties = (unsigned)(target - above);
                kept = above_weight + (u64)ties * each;
                return;
            }
        }
    };
    if (k < (unsigned)V) find_border(std::false_type{}, (u64)k, 0u);
    if (cut_p) {
        if (k >= (unsigned)V) {   // the sum of all
            u64 sum = 0;
            for (int i = tid; i < V; i += kThreads) sum += units_of(weight_of(logit_at<DTYPE>(row, i)));
            sum = wave_sum(sum);
            if (lane == 0) s.wave_u64[wave] = sum;
            __syncthreads();
            kept = 0;
            for (int w = 0; w < kWaves; ++w) kept += s.wave_u64[w];
            __syncthreads();
        }
        // no more than the top-k's keys; what of its border's key is past k counts in no sum before the target, which is at most theirs
        const double want = ceil((double)(top_p > 0.f ? top_p : 0.f) * (double)kept);
        const u64 target = max((u64)1, min((u64)want, kept));
        const unsigned k_border = border, k_ties = ties;
        find_border(std::true_type{}, target, border);
        if (border == k_border && k < (unsigned)V) ties = min(ties, k_ties);
    }

    // Sums of tiles over what is kept; the border's key apart, whose tokens are kept up to a number.
    const int n_tiles = (V + p.tile - 1) / p.tile;
    for (int t = wave; t < n_tiles; t += kWaves) {
        u64 sum = 0;
        unsigned equal = 0;
        const int end = min(V, (t + 1) * p.tile);
        for (int i = t * p.tile + lane; i < end; i += 64) {
            const float x = logit_at<DTYPE>(row, i);
            const unsigned key = key_of(x);
            if (key < border) continue;
            const double w = weight_of(x);
            if (key > border && w >= (double)min_p) sum += units_of(w);
            equal += key == border;
        }
        sum = wave_sum(sum);
        equal = (unsigned)wave_sum(equal);
        if (lane == 0) s.tile_weight[t] = sum, s.tile_ties[t] = equal;
    }
    __syncthreads();
    const float border_logit = __uint_as_float(border >> 31 ? border & 0x7fffffffu : ~border);
    const double border_w = border ? weight_of(border_logit) : 0.;
    const u64 border_weight = border_w >= (double)min_p ? units_of(border_w) : 0;
    // prefix sums over tiles, a thread each
    const unsigned my_equal = tid < n_tiles ? s.tile_ties[tid] : 0;
    u64 upto = wave_sums_to(my_equal, lane);
    if (lane == 63) s.wave_u64[wave] = upto;
    __syncthreads();
    u64 equal_before = upto - my_equal;
    for (int w = 0; w < wave; ++w) equal_before += s.wave_u64[w];
    __syncthreads();
    const u64 my_kept_ties = equal_before >= ties ? 0 : min((u64)my_equal, ties - equal_before);
    const u64 my_weight = tid < n_tiles ? s.tile_weight[tid] + my_kept_ties * border_weight : 0;
    upto = wave_sums_to(my_weight, lane);
    if (lane == 63) s.wave_u64[wave] = upto;
    __syncthreads();
    u64 before = upto - my_weight, all = 0;
    for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? s.wave_u64[w] : 0;
        all += s.wave_u64[w];
    }
    const double at = (double)u * (double)all;
    const u64 target = min((u64)at, all - 1);   // the largest has a weight: all > 0
    if (before <= target && target < before + my_weight) {
        s.told_bin = (unsigned)tid;
        s.told_weight = before;
        s.told_count = (unsigned)min(equal_before, (u64)UINT_MAX);
    }
    __syncthreads();
    if (wave != 0) return;
    const int t = (int)s.told_bin, end = min(V, (t + 1) * p.tile);
    u64 sum = s.told_weight;
    unsigned equal = s.told_count;
    for (int i0 = t * p.tile; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const float x = i < end ? logit_at<DTYPE>(row, i) : -INFINITY;
        const unsigned key = key_of(x);
        const bool is_equal = i < end && key == border;
        const u64 ballot = __ballot(is_equal);
        const unsigned rank = equal + (unsigned)__popcll(ballot & ((1ull << lane) - 1));
        const double w = weight_of(x);
        const bool in = i < end && w >= (double)min_p && (key > border || (is_equal && rank < ties));
        const u64 mine = in ? units_of(w) : 0, to = sum + wave_sums_to(mine, lane);
        const u64 hit = __ballot(to > target);
        if (hit != 0) {
            if (lane == __ffsll((long long)hit) - 1) answer(i, (float)(ldexp(w, p.shift) / (double)all));
            return;
        }
        sum = __shfl(to, 63);
        equal += (unsigned)__popcll(ballot);
    }
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
    p.shift = 62 - bits;
    p.tile = std::max(1, ((a->n_vocab + kTiles - 1) / kTiles + 255) / 256) * 256;
    (void)launch_kernel(a->dtype == KV_F32 ? kv_sample_kernel<KV_F32> : a->dtype == KV_F16 ? kv_sample_kernel<KV_F16> : kv_sample_kernel<KV_BF16>, dim3((unsigned)a->n_rows),
                        dim3(kThreads), (hipStream_t)hip_stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
