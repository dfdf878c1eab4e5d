// Attention of drafted tokens over a cache of 16, 8 or 4 bits:  out[t,hq,:] = softmax_j(q[t,hq,:] . K[b,h,j,:] * scale) V[b,h,j,:] over the
// context of the token's sequence and those drafted tokens whose bit is set in its mask.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "tree_attn.hpp"

namespace {

using namespace kvb;

// A wavefront joins the splits of one query row: out = sum_s 2^(ref_s - max) acc_s / sum_s 2^(ref_s - max) l_s.  A lane has the weight of a split (of two, beyond 64), so the
// exponentials take one instruction for the row, and the sums of up to 8 * 64 / (D / 4) splits are loaded at once, ahead of the weights.  Bound by its launch and two dependent reads: 4.0 us for 7
// splits of 512 rows, 5.8 for 16 of 2048 (17 MB).
constexpr int kCombineWaves = 4;
constexpr float kNothing = -1.f;   // weight of a split without anything
template <int D>
__global__ void __launch_bounds__(64 * kCombineWaves) kv_tree_combine_kernel(TreeParams p)
{
    constexpr int kLanes = D / 4, kTogether = 64 / kLanes, kRound = 8;   // lanes of a row; splits at a time; of them on their way
    const int b = blockIdx.y, lane = threadIdx.x & 63, Hq = p.H * p.G;
    const int r = __builtin_amdgcn_readfirstlane(blockIdx.x * kCombineWaves + (int)(threadIdx.x >> 6));
    const int first = load_uniform(p.tok_first + b), drafted = min(load_uniform(p.tok_first + b + 1) - first, KV_TREE_MAX);
    const int total = max(0, min(load_uniform(p.seq_lens + b), p.max_total - drafted)) + drafted;
    if (r >= drafted * Hq) return;
    const int t = first + r / Hq, hq = r % Hq;
    const int ns = min(p.ns, (total - 1) / p.split_tokens + 1);
    const long long row = (long long)t * Hq + hq;
    const f32x2 *const ml = (const f32x2 *)p.part_ml + row * p.ns;
    const int sub = lane / kLanes, d = lane % kLanes * 4;
    const float *const part = p.part_acc + row * p.ns * D + d;
    const f32x2 m0 = lane < ns ? ml[lane] : f32x2{kNoScore, 0.f}, m1 = 64 + lane < ns ? ml[64 + lane] : f32x2{kNoScore, 0.f};
    f32x4 y[kRound];
    auto load = [&](int s0) {
#pragma unroll
        for (int k = 0; k < kRound; ++k) {
            const int s = s0 + k * kTogether + sub;
            if (s0 + k * kTogether < ns) y[k] = *(const f32x4 *)&part[(long long)(s < ns ? s : 0) * D];
        }
    };
    load(0);
    float to = fmaxf(m0[0], m1[0]);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) to = fmaxf(to, __shfl_xor(to, o));
    const float w0 = m0[1] == 0.f ? kNothing : __builtin_amdgcn_exp2f(m0[0] - to), w1 = m1[1] == 0.f ? kNothing : __builtin_amdgcn_exp2f(m1[0] - to);
    float l = m0[1] * w0 + m1[1] * w1;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) l += __shfl_xor(l, o);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](auto some_are_zero) {
        for (int s0 = 0; s0 < ns; s0 += kRound * kTogether) {
            if (s0 > 0) load(s0);
#pragma unroll
            for (int k = 0; k < kRound; ++k) {
                const int s = s0 + k * kTogether + sub;
                if (s0 + k * kTogether >= ns) break;
                const float f = __shfl(s0 < 64 ? w0 : w1, s & 63);
                if (s < ns && f != kNothing) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)   // a weight too small for 32 bits still counts against an infinity
                        x[e] = fmaf(y[k][e], decltype(some_are_zero)::value && f == 0.f && !__builtin_isfinite(y[k][e]) ? 1.0e-37f : f, x[e]);
                }
            }
        }
    };
    if (__any(w0 == 0.f || w1 == 0.f)) add(std::true_type{});
    else add(std::false_type{});
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int o = kLanes; o < 64; o *= 2) x[e] += __shfl_xor(x[e], o);
    }
    if (sub == 0) store_four(p.out, t * p.o_st + hq * p.o_sh + d, p.out_mode, x * (l == 0.f ? 0.f : 1.f / l));
}

TreeShape shape_of(const kv_plan *p, int bits, bool paged)
{
    static int cus = 0;
    if (cus == 0) {
        int dev = 0, n = 0;
        cus = hipGetDevice(&dev) == hipSuccess && hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0 ? n : 256;
    }
    return TreeShape{p->D, p->H, p->Hq / p->H, bits, cus, paged};
}

}  // namespace

extern "C" int kv_tree_masks(const int32_t *parents, int n, int words, uint64_t *masks, int32_t *depths)
{
    if (!parents || n < 0 || words < 1) return KV_EINVAL;
    if (n > 64ll * words) return KV_ERANGE;
    for (int i = 0; i < n; ++i)
        if (parents[i] < -1 || parents[i] >= i) return KV_ERANGE;
    for (int i = 0; masks && i < n; ++i) {
        uint64_t *const row = masks + (size_t)i * words;
        for (int w = 0; w < words; ++w) row[w] = parents[i] >= 0 ? masks[(size_t)parents[i] * words + w] : 0;
        row[i / 64] |= 1ull << (i % 64);
    }
    // the depth of a parent is known before its children's
    for (int i = 0; depths && i < n; ++i) depths[i] = parents[i] >= 0 ? depths[parents[i]] + 1 : 0;
    return KV_OK;
}

extern "C" size_t kv_tree_attn_workspace(const kv_plan_t *p, int n_tok, int max_len)
{
    if (!p || n_tok < 0 || max_len < 0) return 0;
    return (size_t)std::max<uint64_t>(16, tree_workspace_bytes(shape_of(p, 16, false), n_tok, (long long)max_len + KV_TREE_MAX));
}

extern "C" int kv_tree_attn(const kv_plan_t *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const kv_tree_args_t *a, void *workspace,
                            size_t ws_bytes, void *hip_stream)
{
    if (!p || !view || !a || !workspace || ((uintptr_t)workspace & 15)) return KV_EINVAL;
    if (p->D != 64 && p->D != 128 && p->D != 256) return KV_EINVAL;
    if (!view->seq_lens_host || !view->seq_lens_dev || !a->tok_first_host || !a->tok_first_dev) return KV_EINVAL;
    if (a->out_dtype != KV_OUT_F32 && a->out_dtype != KV_OUT_SAME) return KV_EINVAL;
    if (a->n_splits < 0 || a->n_splits > 128 || !std::isfinite(a->scale)) return KV_EINVAL;
    if (p->B > 65535 || p->Hq > 65535 || p->Hq / p->H > 4095) return KV_EINVAL;   // a row's number times the group is divided in 32 bits
    if (a->tok_first_host[0] != 0) return KV_EINVAL;
    int max_total = 0, most_drafted = 0;
    for (int b = 0; b < p->B; ++b) {
        const int len = view->seq_lens_host[b], n = a->tok_first_host[b + 1] - a->tok_first_host[b];
        if (len < 0 || a->tok_first_host[b + 1] < a->tok_first_host[b]) return KV_EINVAL;
        if (n > KV_TREE_MAX || len > 1 << 30) return KV_ERANGE;   // the kernels look some thousand tokens past a sequence's end in 32 bits
        if (a->mask && n > 64ll * a->mask_words) return KV_ERANGE;
        max_total = std::max(max_total, len + n);
        most_drafted = std::max(most_drafted, n);
    }
    TreeParams t{};
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
    t.max_total = max_total;
    t.H = p->H; t.G = p->Hq / p->H; t.B = p->B;
    t.scale_log2e = (float)(1.4426950408889634 * (a->scale == 0.f ? 1 / std::sqrt((double)p->D) : std::fabs((double)a->scale)));
    t.q_sign = a->scale < 0.f ? 0x80008000u : 0;
    t.out_mode = a->out_dtype == KV_OUT_F32 ? 0 : bf16 ? 2 : 1;

    const int format = blocks ? blocks->format : KV_FORMAT_16;
    const TreeCut cut = cut_tree(shape_of(p, format_bits(format), t.c.table != nullptr), p->B, view->seq_lens_host, a->tok_first_host, a->n_splits, ws_bytes);
    t.ns = cut.ns;
    t.split_tokens = cut.split_tokens;
    t.row_blocks = cut.row_blocks;
    t.part_acc = (float *)workspace;
    t.part_ml = t.part_acc + (size_t)n_tok * p->Hq * cut.ns * p->D;
    t.bt_shift = -1;
    if (t.c.table && (t.c.bt & (t.c.bt - 1)) == 0) t.bt_shift = __builtin_ctz((unsigned)t.c.bt);
    // units (a split of a KV head) go in eights where they have several row blocks (the kernel's note on XCDs)
    auto in_eights = [&](uint64_t units) { return cut.row_blocks > 1 ? (units + 7) / 8 * 8 : units; };
    uint64_t groups = in_eights((uint64_t)p->B * p->H * cut.ns) * cut.row_blocks;
    if (p->B > 1 && p->B <= kCounted) {   // without those that have nothing to do, if there are any
        uint64_t some = 0;
        for (int b = 0; b < p->B; ++b) {
            const int n = a->tok_first_host[b + 1] - a->tok_first_host[b];
            if (n > 0) some += in_eights((uint64_t)((view->seq_lens_host[b] + n - 1) / cut.split_tokens + 1) * p->H) * ((n * t.G + 16 * cut.nb - 1) / (16 * cut.nb));
        }
        t.ragged = some < groups;
        if (t.ragged) groups = some;
    }
    if (groups * kTreeThreads >= 1ull << 32) return KV_ERANGE;   // threads of a launch
    auto over = [](int d) { return (unsigned)(((1ull << 32) + d - 1) / d); };
    t.by_g = over(t.G); t.by_ns = over(cut.ns); t.by_h = over(p->H); t.by_row_blocks = over(cut.row_blocks);
    t.by_split = over(cut.split_tokens);
    const bool f32 = t.out_mode == 0;
    // offsets within a block, or from one of a wavefront's steps to the next (128 tokens), fit 32 bits; blocks hold whole groups of 16
    t.grouped = t.c.table ? t.c.bt % 16 == 0 && t.c.sb < 1ull << 32 && t.c.zb < 1ull << 32 && t.c.zs < (1ull << 32) / (uint64_t)t.c.bt
                          : t.c.ss < 1ull << 25 && t.c.zs < 1ull << 25;
    t.dense = t.c.ss == (uint64_t)p->D * format_bits(format) / 8;
    TreeKernel k = (format == KV_FORMAT_FP8 ? tree_kernel_fp8 : format == KV_FORMAT_FP4 ? tree_kernel_fp4 : tree_kernel_16)(p->D, bf16, f32, cut.nb);
    hipStream_t st = (hipStream_t)hip_stream;
    (void)launch_kernel(k, dim3((unsigned)groups), dim3(kTreeThreads), st, t);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    if (cut.ns == 1) return KV_OK;
    const dim3 cgrid((unsigned)(((long long)most_drafted * p->Hq + kCombineWaves - 1) / kCombineWaves), (unsigned)p->B);
    (void)launch_kernel(p->D == 64 ? kv_tree_combine_kernel<64> : p->D == 128 ? kv_tree_combine_kernel<128> : kv_tree_combine_kernel<256>, cgrid, dim3(64 * kCombineWaves), st, t);
    e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
