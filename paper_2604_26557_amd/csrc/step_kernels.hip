// Block tables and slot maps of a step, from the lengths of its requests.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <type_traits>

#include "launch.hpp"
#include "plan.hpp"

namespace {

using namespace kvb;

constexpr int kMostSequences = 8192;
constexpr int kSegment = 256;       // entries of a row that a wavefront goes over, where rows are copied
constexpr int kTokens = 2048;       // rows of the maps that a workgroup writes

struct TablesParams {
    kv_tables_args_t a;
    int segments;        // of a row; 1 in place
    int table_groups;    // workgroups that go over rows; the others write maps
    int in_place;
};

// What the lengths say of a sequence.
struct Request {
    long long len, need;
    int news, held, common, leader;
    bool ended;
};
__device__ __forceinline__ Request request_of(const kv_tables_args_t &a, int b, bool only_tokens = false)
{
    Request r{};
    const int t = a.new_lens[b];
    r.ended = t < 0;
    r.news = t < 0 ? 0 : t;
    r.len = max(a.seq_lens[b], 0);
    if (only_tokens) return r;   // nothing that a call in place changes
    r.need = r.ended ? 0 : (r.len + r.news + a.block_tokens - 1) / a.block_tokens;
    r.held = min(max(a.held[b], 0), a.max_blocks);
    r.leader = a.leader ? a.leader[b] : -1;
    if ((unsigned)r.leader >= (unsigned)a.batch || r.leader == b) r.leader = -1;
    r.common = r.leader >= 0 ? min(max(a.shared[b], 0), a.max_blocks) : 0;
    return r;
}
// Blocks that it takes from the free ones, and gives back.
__device__ __forceinline__ long long fresh_of(const Request &r) { return max(0ll, r.need - max(r.held, r.common)); }
__device__ __forceinline__ int gone_of(const Request &r) { return r.ended ? max(0, r.held - r.common) : 0; }

// The last b in [0, n) with first[b] <= x; first[0] = 0, ascending.
__device__ __forceinline__ int segment_of(const unsigned *first, int n, unsigned x)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Sums over the lanes up to each: 1, 2, 4, 8 of a row of 16, then over rows. All lanes take part.
__device__ __forceinline__ unsigned long long wave_sums_to(unsigned long long x)
{
    auto moved = [](unsigned long long x, auto ctrl, auto rows) {
        const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(x >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        return (unsigned long long)hi << 32 | lo;
    };
    using std::integral_constant;
    const integral_constant<int, 0xf> all;
    x += moved(x, integral_constant<int, 0x111>{}, all);
    x += moved(x, integral_constant<int, 0x112>{}, all);
    x += moved(x, integral_constant<int, 0x114>{}, all);
    x += moved(x, integral_constant<int, 0x118>{}, all);
    x += moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
    x += moved(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
    return x;
}

// Every workgroup sums up all lengths by itself (a few loads a thread), so that one launch does: the first ones go over rows of the table, a wavefront a row or a part of it, the others
// write the maps. In place it is one workgroup for the table, which looks everything up before it changes it. Bound by the launch and a chain of dependent loads: lengths, sums, the entry
// of the stack, the table: 64 requests of a token each 5.1 us, 384 with chunks of up to 768 tokens (128K rows of maps) 6.6; with 1024 threads for the 64, what the lengths say read again from memory
// and sums over LDS they took 12 and 14. In place 10.9 and 44: 16 wavefronts have all rows, and go over them twice.
template <int MOST, int kThreads>
__global__ void __launch_bounds__(kThreads) kv_step_tables_kernel(TablesParams p)
{
    constexpr int kWaves = kThreads / 64;
    constexpr bool kKept = MOST <= 1024;   // what a length says of its sequence, in LDS
    const kv_tables_args_t &a = p.a;
    const int B = a.batch, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    __shared__ unsigned first[MOST + 1], fresh[MOST + 1], gone[MOST + 1];
    __shared__ int4 kept[kKept ? MOST : 1];   // need (-1: ended), held, shared entries, leader
    __shared__ unsigned long long sums[3][kWaves];
    __shared__ int unfit[kWaves];
    const bool maps = (int)blockIdx.x >= p.table_groups;
    const int free_now = maps ? 0 : a.n_free[0];

    // Sums before each sequence: a thread has up to `per` neighbouring ones.
    const int per = (B + kThreads - 1) / kThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    unsigned long long mine[3] = {0, 0, 0};
    int over = 0;
    for (int b = b0; b < b1; ++b) {
        const Request r = request_of(a, b, maps);
        mine[0] += r.news;
        mine[1] += fresh_of(r);
        mine[2] += gone_of(r);
        over += r.need > a.max_blocks;
        if constexpr (kKept) kept[b] = int4{r.ended ? -1 : (int)min(r.need, (long long)INT_MAX), r.held, r.common, r.leader};
    }
    unsigned long long before[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const unsigned long long x = wave_sums_to(mine[k]);
        before[k] = x - mine[k];
        if (lane == 63) sums[k][wave] = x;
    }
    over = __popcll(__ballot(over > 0)) > 0 ? (int)wave_sums_to((unsigned long long)over) : 0;
    if (lane == 63) unfit[wave] = over;
    __syncthreads();
    unsigned long long all[3] = {0, 0, 0};
    over = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        over += unfit[w];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            before[k] += w < wave ? sums[k][w] : 0;
            all[k] += sums[k][w];
        }
    }
    auto count = [](unsigned long long x) { return (unsigned)min(x, (unsigned long long)INT_MAX); };
    // as the lengths, or LDS, have it
    auto request = [&](int b) {
        if constexpr (kKept) {
            const int4 k = kept[b];
            Request r{};
            r.need = max(k.x, 0);
            r.held = k.y;
            r.common = k.z;
            r.leader = k.w;
            r.ended = k.x < 0;
            return r;
        } else {
            return request_of(a, b);
        }
    };
    for (int b = b0; b < b1; ++b) {
        first[b] = count(before[0]);
        fresh[b] = count(before[1]);
        gone[b] = count(before[2]);
        if (b + 1 < b1) {
            const Request r = request_of(a, b, maps);
            before[0] += r.news;
            before[1] += fresh_of(r);
            before[2] += gone_of(r);
        }
    }
    if (tid == 0) first[B] = count(all[0]), fresh[B] = count(all[1]), gone[B] = count(all[2]);
    __syncthreads();

    if (maps) {
        // rows up to 2^31 - 1: the end of the last workgroup's is past 31 bits
        const unsigned t0 = (blockIdx.x - (unsigned)p.table_groups) * kTokens, t1 = min((unsigned)a.n_tok, t0 + kTokens);
        for (unsigned t = t0 + tid; t < t1; t += kThreads) {
            const bool there = t < first[B];
            const int b = there ? segment_of(first, B, t) : 0;
            a.tok_seq[t] = there ? b : -1;
            a.tok_slot[t] = there ? (int)(max(a.seq_lens[b], 0) + (t - first[b])) : -1;
        }
        return;
    }

    const unsigned n_free = (unsigned)min(max(free_now, 0), a.n_pool);
    const unsigned long long top = n_free + all[2];   // of the stack, with what ends
    const bool fine = all[1] <= top && over == 0;
    // The block that is taken after k others. What ends in this call is looked up in its row.
    auto taken = [&](unsigned k) {
        const unsigned long long i = top - 1 - k;
        if (i < n_free) return a.free_ids[i];
        const unsigned g = (unsigned)(i - n_free);
        const int b = segment_of(gone, B, g);
        const int common = request(b).common;
        return a.block_table[(long long)b * a.max_blocks + common + (int)(g - gone[b])];
    };
    // The entry i of row b as this call finds or fills it. Sequences without an offset of their own share it with the next: segment_of takes the last, which has some.
    auto filled = [&](const Request &r, int b, int i) {
        if (fine && !r.ended && i >= max(r.held, r.common) && i < r.need) return taken(fresh[b] + (unsigned)(i - max(r.held, r.common)));
        return a.block_table[(long long)b * a.max_blocks + i];
    };
    auto entry = [&](const Request &r, int b, int i) {
        if (r.ended) return -1;
        if (!(fine && i >= r.held && i < min((long long)r.common, r.need))) return filled(r, b, i);
        const Request l = request(r.leader);
        return l.ended || (i >= l.held && i < l.common) ? -1 : filled(l, r.leader, i);
    };

    if (!p.in_place) {
        const int items = B * p.segments;
        for (int item = blockIdx.x * kWaves + wave; item < items; item += p.table_groups * kWaves) {
            const int b = item / p.segments, i0 = (item - b * p.segments) * kSegment, i1 = min(i0 + kSegment, a.max_blocks);
            const Request r = request(b);
            for (int i = i0 + lane; i < i1; i += 64) {
                const long long at = (long long)b * a.max_blocks + i;
                if (r.ended && i >= r.common && i < r.held) {
                    const unsigned long long to = (unsigned long long)n_free + gone[b] + (unsigned)(i - r.common);
                    if (to < (unsigned)a.n_pool) a.free_ids[to] = a.block_table[at];
                }
                a.block_table_out[at] = entry(r, b, i);
            }
            if (i0 == 0 && lane == 0) a.held_out[b] = r.ended ? 0 : fine ? (int)max((long long)r.held, r.need) : r.held;
        }
    } else {
        // Fill and push, then clear: what ended is read until then. Its entries and what is filled are different places.
        for (int b = wave; b < B; b += kWaves) {
            const Request r = request(b);
            const int i0 = r.ended ? r.common : r.held, i1 = r.ended ? r.held : fine ? (int)r.need : 0;
            for (int i = i0 + lane; i < i1; i += 64) {
                const long long at = (long long)b * a.max_blocks + i;
                if (r.ended) {
                    const unsigned long long to = (unsigned long long)n_free + gone[b] + (unsigned)(i - r.common);
                    if (to < (unsigned)a.n_pool) a.free_ids[to] = a.block_table[at];
                } else {
                    a.block_table_out[at] = entry(r, b, i);
                }
            }
        }
        __syncthreads();
        for (int b = wave; b < B; b += kWaves) {
            const Request r = request(b);
            for (int i = lane; r.ended && i < a.max_blocks; i += 64) a.block_table_out[(long long)b * a.max_blocks + i] = -1;
        }
        __syncthreads();
        // each thread its own sequences: nobody else looks at what they held any more
        for (int b = b0; b < b1; ++b) {
            const Request r = request(b);
            a.held_out[b] = r.ended ? 0 : fine ? (int)max((long long)r.held, r.need) : r.held;
        }
    }
    if (blockIdx.x == 0) {
        for (int b = tid; b <= B; b += kThreads) a.tok_first[b] = (int)first[b];
        if (tid == 0) {
            a.n_free_out[0] = (int)min(top - (fine ? all[1] : 0), (unsigned long long)a.n_pool);   // fine: all[1] <= top
            a.status[0] = all[1] > top ? (int)count(all[1] - top) : 0;
            a.status[1] = over;
        }
    }
}

}  // namespace

extern "C" int kv_step_tables(const kv_tables_args_t *a, void *hip_stream)
{
    if (!a) return KV_EINVAL;
    if (a->batch < 1 || a->batch > kMostSequences || a->block_tokens < 1 || a->max_blocks < 0 || a->n_pool < 0 || a->n_tok < 0) return KV_EINVAL;
    if (!a->seq_lens || !a->new_lens || !a->held || !a->n_free || !a->held_out || !a->n_free_out || !a->tok_first || !a->status) return KV_EINVAL;
    if (!a->leader != !a->shared) return KV_EINVAL;
    if ((a->max_blocks > 0 && (!a->block_table || !a->block_table_out)) || (a->n_pool > 0 && !a->free_ids) || (a->n_tok > 0 && (!a->tok_seq || !a->tok_slot))) return KV_EINVAL;
    const bool in_place = a->held_out == a->held;
    if ((a->n_free_out == a->n_free) != in_place || (a->max_blocks > 0 && (a->block_table_out == a->block_table) != in_place)) return KV_EINVAL;
    if ((int64_t)a->batch * a->max_blocks > INT_MAX) return KV_ERANGE;
    TablesParams p{};
    p.a = *a;
    p.in_place = in_place;
    p.segments = in_place ? 1 : std::max(1, (a->max_blocks + kSegment - 1) / kSegment);
    // in place one workgroup has all rows: as many wavefronts as it may have
    const bool few = a->batch <= 1024 && !in_place;
    const int threads = !few ? 1024 : a->batch <= 256 ? 256 : 512, waves = threads / 64;   // a sequence each, for most
    p.table_groups = in_place ? 1 : std::min(few ? 1024 : 256, (a->batch * p.segments + waves - 1) / waves);
    const unsigned maps = (unsigned)((a->n_tok + (int64_t)kTokens - 1) / kTokens);
    (void)launch_kernel(threads == 256 ? kv_step_tables_kernel<1024, 256> : threads == 512 ? kv_step_tables_kernel<1024, 512> : a->batch <= 1024 ? kv_step_tables_kernel<1024, 1024> : kv_step_tables_kernel<kMostSequences, 1024>,
                        dim3((unsigned)p.table_groups + maps), dim3((unsigned)threads), (hipStream_t)hip_stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
