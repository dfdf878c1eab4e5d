// Attention of new tokens over a cache, for sequences that share prefixes and for scores that are capped, biased or bounded: the kernels are those of tree_attn.hpp, whose units of work are here
// a group's prefix with all rows of its sequences, and each sequence's own tokens with its rows. The partial results of both are joined like those of splits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <memory>
#include <new>

#include "group_cut.hpp"
#include "tree_combine.hpp"

namespace {

using namespace kvb;

template <int D>
__global__ void __launch_bounds__(64 * kCombineWaves) kv_group_combine_kernel(GroupParams p)
{
    const int b = blockIdx.y, lane = threadIdx.x & 63, Hq = p.H * p.G;
    const int r = __builtin_amdgcn_readfirstlane(blockIdx.x * kCombineWaves + (int)(threadIdx.x >> 6));
    const int first = load_uniform(p.tok_first + b), drafted = load_uniform(p.tok_first + b + 1) - first;
    int shared = 0;
    if (p.n_groups > 0 && !p.joined) {
        const bool of = lane < p.n_groups && b >= p.group_first[lane] && b < p.group_first[lane + 1];
        const unsigned long long which = __ballot(of);
        if (which != 0) shared = load_uniform(p.prefix + __ffsll((long long)which) - 1);
    }
    if (r >= drafted * Hq) return;
    const int total = max(shared, min(load_uniform(p.seq_lens + b), p.max_total - drafted)) + drafted;
    const int of_prefix = shared > 0 ? min(p.prefix_ns, (shared - 1) / p.prefix_tokens + 1) : 0;
    const int of_own = min(p.ns - p.prefix_ns, (total - (shared & ~31) - 1) / p.split_tokens + 1), skip = p.prefix_ns - of_prefix;
    combine_row<D>(p, first + r / Hq, r % Hq, of_prefix + of_own, lane, [=](int s) { return s < of_prefix ? s : s + skip; });
}

}  // namespace

extern "C" size_t kv_group_attn_workspace(const kv_plan_t *p, int n_tok, int max_len)
{
    if (!p || n_tok < 0 || max_len < 0) return 0;
    return (size_t)std::max<uint64_t>(16, group_workspace_bytes(tree_shape(p, 16, false), n_tok, (long long)max_len + n_tok));
}

extern "C" int kv_group_attn(const kv_plan_t *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const kv_tree_args_t *a, const kv_groups_t *groups,
                             const kv_scores_t *scores, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!p || !view || !a || !workspace || ((uintptr_t)workspace & 15)) return KV_EINVAL;
    if (p->D != 64 && p->D != 128 && p->D != 256) return KV_EINVAL;
    if (!view->seq_lens_host || !view->seq_lens_dev || !a->tok_first_host || !a->tok_first_dev) return KV_EINVAL;
    if (a->out_dtype != KV_OUT_F32 && a->out_dtype != KV_OUT_SAME) return KV_EINVAL;
    if (a->n_splits < 0 || a->n_splits > kMaxTreeSplits || !std::isfinite(a->scale)) return KV_EINVAL;
    if (p->B > 65535 || p->Hq > 65535 || p->Hq / p->H > 4095) return KV_EINVAL;
    if (a->tok_first_host[0] != 0) return KV_EINVAL;
    const int n_groups = groups ? groups->n_groups : 0;
    if (n_groups < 0 || n_groups > kMostGroups) return KV_EINVAL;
    if (n_groups > 0 && (!groups->first_host || !groups->first_dev || !groups->prefix_host || !groups->prefix_dev)) return KV_EINVAL;
    const int *const group_first = n_groups > 0 ? groups->first_host : nullptr, *const prefix = n_groups > 0 ? groups->prefix_host : nullptr;
    for (int g = 0; g < n_groups; ++g)
        if (group_first[g] < 0 || group_first[g + 1] < group_first[g] || group_first[g + 1] > p->B || prefix[g] < 0) return KV_EINVAL;
    if (scores) {
        if (!std::isfinite(scores->softcap) || scores->softcap < 0.f || (scores->slopes && !scores->positions)) return KV_EINVAL;
    }
    long long max_total = 0, most_new = 0;
    for (int b = 0, g = 0; b < p->B; ++b) {
        const int len = view->seq_lens_host[b], n = a->tok_first_host[b + 1] - a->tok_first_host[b];
        if (len < 0 || a->tok_first_host[b + 1] < a->tok_first_host[b]) return KV_EINVAL;
        while (g < n_groups && b >= group_first[g + 1]) ++g;
        if (g < n_groups && b >= group_first[g] && len < prefix[g]) return KV_EINVAL;
        if ((a->mask && n > KV_TREE_MAX) || (long long)len + n > 1 << 30) return KV_ERANGE;
        if (a->mask && n > 64ll * a->mask_words) return KV_ERANGE;
        max_total = std::max(max_total, (long long)len + n);
        most_new = std::max<long long>(most_new, n);
    }
    GroupParams t{};
    const int rc = cache_addr(p, view, blocks, layer, view->seq_lens_host, a->tok_first_host, &t.c);
    if (rc != KV_OK) return rc;
    // a row's scales are loaded at once
    if (blocks && (((uintptr_t)t.c.kz | (uintptr_t)t.c.vz | t.c.zb | t.c.zh | t.c.zs) & (p->D / kBlockElems - 1))) return KV_EINVAL;
    const int n_tok = a->tok_first_host[p->B];
    if (n_tok == 0) return KV_OK;
    if (t.c.table && t.c.n_pool < 1) return KV_ERANGE;
    if ((int64_t)n_tok * p->Hq > INT_MAX) return KV_ERANGE;
    if (!a->q || !a->out || ((uintptr_t)a->q & 15)) return KV_EINVAL;
    if (a->q_stride_t < 0 || a->q_stride_h < 0 || a->out_stride_t < 0 || a->out_stride_h < 0 || ((a->q_stride_t | a->q_stride_h) & 7)) return KV_EINVAL;
    const bool bf16 = p->dtype == KV_BF16;
    t.q = (const char *)a->q;
    t.out = a->out;
    t.q_st = a->q_stride_t; t.q_sh = a->q_stride_h; t.o_st = a->out_stride_t; t.o_sh = a->out_stride_h;
    t.seq_lens = view->seq_lens_dev;
    t.tok_first = a->tok_first_dev;
    t.mask = (const unsigned long long *)a->mask;
    t.words = a->mask_words;
    t.max_total = (int)max_total;
    t.H = p->H; t.G = p->Hq / p->H; t.B = p->B;
    const double scale = a->scale == 0.f ? 1 / std::sqrt((double)p->D) : std::fabs((double)a->scale);
    t.q_sign = a->scale < 0.f ? 0x80008000u : 0;
    t.out_mode = a->out_dtype == KV_OUT_F32 ? 0 : bf16 ? 2 : 1;
    t.scale = (float)scale;
    if (scores) {
        t.cap = scores->softcap;
        t.cap_in = t.cap > 0.f ? (float)(scale / t.cap) : 0.f;
        if (!std::isfinite(t.cap_in)) return KV_EINVAL;
        t.slopes = scores->slopes;
        t.positions = scores->positions;
        t.from = scores->sees_from;
        t.to = scores->sees_to;
    }
    const bool shaped = t.cap > 0.f || t.slopes;
    // the error of a cap by sigmoids grows with it: beyond 64 it would show in 16-bit results
    if (t.out_mode != 0 && t.cap > 0.f && t.cap <= 64.f) t.sigmoid_in = -2.88539008f * t.cap_in;
    // slopes without a cap are divided by the scale, unless that would leave the range of 32 bits: a multiplication of each score less
    const bool divided = !(t.cap > 0.f) && scale > 1e-6 && scale < 1e6;
    t.bias = divided ? (float)(1 / scale) : 1.f;
    t.prescale = divided || t.cap > 0.f ? 1.f : t.scale;
    t.scale_log2e = (float)(1.4426950408889634 * (!shaped || divided ? scale : t.sigmoid_in != 0.f && !t.slopes ? 2. * t.cap : 1.));

    const int format = blocks ? blocks->format : KV_FORMAT_16;
    const TreeShape shape = tree_shape(p, format_bits(format), t.c.table != nullptr);
    // prefixes and sequences, and sequences alone
    GroupUnit few[384];
    const size_t n_most = (size_t)n_groups + 2 * (size_t)p->B;
    const std::unique_ptr<GroupUnit[]> many(n_most > 384 ? new (std::nothrow) GroupUnit[n_most] : nullptr);
    if (n_most > 384 && !many) return KV_ENOSPC;
    GroupUnit *units = many ? many.get() : few;
    int n_units = 0;
    bool any_prefix = false;
    for (int i = 0, g = 0; i < n_groups + p->B; ++i) {
        const int b = i - n_groups;
        while (b >= 0 && g < n_groups && b >= group_first[g + 1]) ++g;
        const int shared = b >= 0 && g < n_groups && b >= group_first[g] ? prefix[g] : 0;
        const GroupUnit u = group_unit(i, n_groups, group_first, prefix, view->seq_lens_host, a->tok_first_host, shared);
        if (u.tokens <= 0 || u.span <= 0) continue;
        units[n_units++] = u;
        any_prefix = any_prefix || u.prefix;
    }
    if (any_prefix && ws_bytes < 2 * tree_split_bytes(shape, n_tok)) return KV_ENOSPC;
    GroupCut cut = cut_group(shape, units, n_units, !a->mask, t.from != nullptr, shaped, a->n_splits, ws_bytes, n_tok);
    if (any_prefix && a->n_splits == 0) {
        GroupUnit *const own = units + n_groups + p->B;
        int n_own = 0;
        for (int b = 0; b < p->B; ++b) {
            const GroupUnit u = group_unit(b, 0, nullptr, nullptr, view->seq_lens_host, a->tok_first_host, 0);
            if (u.tokens > 0 && u.span > 0) own[n_own++] = u;
        }
        const GroupCut joined = cut_group(shape, own, n_own, !a->mask, t.from != nullptr, shaped, 0, ws_bytes, n_tok);
        if (better_joined(joined, cut, !a->mask, n_tok, p->B)) {
            cut = joined;
            units = own;
            n_units = n_own;
            t.joined = 1;
        }
    }
    t.ns = cut.ns;
    t.prefix_ns = cut.prefix_ns;
    t.split_tokens = cut.split_tokens;
    t.prefix_tokens = cut.prefix_tokens;
    t.n_groups = any_prefix ? n_groups : 0;
    t.group_first = n_groups > 0 ? groups->first_dev : nullptr;
    t.prefix = n_groups > 0 ? groups->prefix_dev : nullptr;
    t.part_acc = (float *)workspace;
    t.part_ml = t.part_acc + (size_t)n_tok * p->Hq * cut.ns * p->D;
    t.bt_shift = -1;
    if (t.c.table && (t.c.bt & (t.c.bt - 1)) == 0) t.bt_shift = __builtin_ctz((unsigned)t.c.bt);
    uint64_t workgroups = 0;
    for (int i = 0; i < n_units; ++i) workgroups += unit_workgroups(shape, units[i], units[i].prefix ? cut.nb_prefix : cut.nb, units[i].prefix ? cut.prefix_tokens : cut.split_tokens);
    if (workgroups * kTreeThreads >= 1ull << 32) return KV_ERANGE;   // threads of a launch
    auto over = [](int d) { return (unsigned)(((1ull << 32) + d - 1) / d); };
    t.by_g = over(t.G); t.by_h = over(p->H); t.by_split = over(cut.split_tokens); t.by_prefix = over(cut.prefix_tokens);
    t.grouped = t.c.table ? t.c.bt % 16 == 0 && t.c.sb < 1ull << 32 && t.c.zb < 1ull << 32 && t.c.zs < (1ull << 32) / (uint64_t)t.c.bt
                          : t.c.ss < 1ull << 25 && t.c.zs < 1ull << 25;
    t.dense = t.c.ss == (uint64_t)p->D * format_bits(format) / 8;
    GroupKernel k = (format == KV_FORMAT_FP8 ? shaped ? shaped_kernel_fp8 : group_kernel_fp8
                     : format == KV_FORMAT_FP4 ? shaped ? shaped_kernel_fp4 : group_kernel_fp4 : shaped ? shaped_kernel_16 : group_kernel_16)(p->D, bf16, t.out_mode == 0, cut.nb, cut.nb_prefix != cut.nb);
    hipStream_t st = (hipStream_t)hip_stream;
    const dim3 cgrid((unsigned)((most_new * p->Hq + kCombineWaves - 1) / kCombineWaves), (unsigned)p->B);
    if (cut.ns > 1 && (uint64_t)cgrid.x * 64 * kCombineWaves >= 1ull << 32) return KV_ERANGE;
    (void)launch_kernel(k, dim3((unsigned)workgroups), dim3(kTreeThreads), st, t);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    if (cut.ns == 1) return KV_OK;
    (void)launch_kernel(p->D == 64 ? kv_group_combine_kernel<64> : p->D == 128 ? kv_group_combine_kernel<128> : kv_group_combine_kernel<256>, cgrid, dim3(64 * kCombineWaves), st, t);
    e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
