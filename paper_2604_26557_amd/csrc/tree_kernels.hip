// Attention of drafted tokens over a cache of 16, 8 or 4 bits:  out[t,hq,:] = softmax_j(q[t,hq,:] . K[b,h,j,:] * scale) V[b,h,j,:] over the
// context of the token's sequence and those drafted tokens whose bit is set in its mask.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "cache.hpp"
#include "launch.hpp"

namespace {

using namespace kvb;

struct TreeParams {
    CacheAddr c;
    const char *q;
    void *out;
    long long q_st, q_sh, o_st, o_sh;  // elements
    const int *seq_lens, *tok_first;
    const unsigned long long *mask;
    int words, max_total, H, G, B;
    float scale;
    int out_mode;                      // 0 fp32, 1 fp16, 2 bf16
};

template <bool BF16, int FORMAT>
__device__ __forceinline__ f32x2 load2(const char *row, const char *scales, int d)
{
    unsigned w;
    if constexpr (FORMAT == KV_FORMAT_16) {
        w = *(const unsigned *)(row + 2 * d);
    } else {
        const float s = scale_operand((unsigned char)scales[d / kBlockElems]);
        if constexpr (FORMAT == KV_FORMAT_FP8) w = decode2<BF16, FORMAT, 0>(*(const unsigned short *)(row + d), s);
        else w = decode2<BF16, FORMAT, 0>((unsigned char)row[d / 2], s);
    }
    return unpack2<BF16>(w);
}

// One workgroup of four wavefronts per query row; a wavefront takes every fourth token, its lanes pairs of elements.
template <int D, bool BF16, int FORMAT>
__global__ void __launch_bounds__(256) kv_tree_attn_kernel(TreeParams p)
{
    constexpr int N = (D + 127) / 128;
    const int t = blockIdx.x, hq = blockIdx.y, h = hq / p.G, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool on = 2 * lane < D;
    int b = 0;
    while (b + 1 < p.B && p.tok_first[b + 1] <= t) ++b;
    const int i = t - p.tok_first[b], drafted = p.tok_first[b + 1] - p.tok_first[b], len = max(0, min(p.seq_lens[b], p.max_total - drafted));
    const char *const q = p.q + 2 * (t * p.q_st + hq * p.q_sh);
    f32x2 x[N], acc[N] = {};
    for (int k = 0; k < N; ++k) x[k] = on ? unpack2<BF16>(*(const unsigned *)(q + 2 * (128 * k + 2 * lane))) : f32x2{0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (int j = wave; j < len + drafted; j += 4) {
        const int n = j - len;
        if (n >= 0 && !(p.mask ? p.mask[(long long)t * p.words + n / 64] >> (n % 64) & 1 : n <= i)) continue;
        unsigned block, row;
        if (!find_row(p.c, b, j, &block, &row)) continue;
        const unsigned long long at = block * p.c.sb + h * p.c.sh + row * p.c.ss, z = block * p.c.zb + h * p.c.zh + row * p.c.zs;
        float s = 0.f;
        f32x2 v[N];
        for (int k = 0; k < N; ++k) {
            const int d = on ? 128 * k + 2 * lane : 0;
            const f32x2 y = load2<BF16, FORMAT>(p.c.k + at, p.c.kz + z, d);
            v[k] = load2<BF16, FORMAT>(p.c.v + at, p.c.vz + z, d);
            s += on ? x[k][0] * y[0] + x[k][1] * y[1] : 0.f;
        }
        for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
        s *= p.scale;
        const float mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - mn), w = expf(s - mn);
        m = mn;
        l = l * f + w;
        for (int k = 0; k < N; ++k) acc[k] = acc[k] * f + v[k] * w;
    }
    __shared__ float sm[4], sl[4];
    __shared__ f32x2 sa[4][N][64];
    if (lane == 0) { sm[wave] = m; sl[wave] = l; }
    for (int k = 0; k < N; ++k) sa[wave][k][lane] = acc[k];
    __syncthreads();
    if (wave > 0 || !on) return;
    float M = -INFINITY, L = 0.f;
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w]);
    f32x2 a[N] = {};
    for (int w = 0; w < 4; ++w) {
        if (sl[w] == 0.f) continue;
        const float f = expf(sm[w] - M);
        L += sl[w] * f;
        for (int k = 0; k < N; ++k) a[k] += sa[w][k][lane] * f;
    }
    for (int k = 0; k < N; ++k)
        for (int e = 0; e < 2; ++e) {
            const long long o = t * p.o_st + hq * p.o_sh + 128 * k + 2 * lane + e;
            const float r = L == 0.f ? 0.f : a[k][e] / L;
            if (p.out_mode == 0) ((float *)p.out)[o] = r;
            else if (p.out_mode == 1) ((_Float16 *)p.out)[o] = (_Float16)r;
            else ((unsigned short *)p.out)[o] = bf16_bits(r);
        }
}

typedef void (*TreeKernel)(TreeParams);
template <int D, bool BF16>
TreeKernel tree_kernel(int format)
{
    return format == KV_FORMAT_FP8 ? kv_tree_attn_kernel<D, BF16, KV_FORMAT_FP8> : format == KV_FORMAT_FP4 ? kv_tree_attn_kernel<D, BF16, KV_FORMAT_FP4>
                                                                                                      : kv_tree_attn_kernel<D, BF16, KV_FORMAT_16>;
}
template <int D>
TreeKernel tree_kernel(bool bf16, int format)
{
    return bf16 ? tree_kernel<D, true>(format) : tree_kernel<D, false>(format);
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
    return 16;
}

extern "C" int kv_tree_attn(const kv_plan_t *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const kv_tree_args_t *a, void *workspace,
                            size_t ws_bytes, void *hip_stream)
{
    if (!p || !view || !a || !workspace || ((uintptr_t)workspace & 15)) return KV_EINVAL;
    if (p->D != 64 && p->D != 128 && p->D != 256) return KV_EINVAL;
    if (!view->seq_lens_host || !view->seq_lens_dev || !a->tok_first_host || !a->tok_first_dev) return KV_EINVAL;
    if (a->out_dtype != KV_OUT_F32 && a->out_dtype != KV_OUT_SAME) return KV_EINVAL;
    if (a->n_splits < 0 || a->n_splits > 128 || !std::isfinite(a->scale)) return KV_EINVAL;
    if (p->B > 65535 || p->Hq > 65535) return KV_EINVAL;
    if (a->tok_first_host[0] != 0) return KV_EINVAL;
    int max_total = 0;
    for (int b = 0; b < p->B; ++b) {
        const int len = view->seq_lens_host[b], n = a->tok_first_host[b + 1] - a->tok_first_host[b];
        if (len < 0 || a->tok_first_host[b + 1] < a->tok_first_host[b]) return KV_EINVAL;
        if (n > KV_TREE_MAX || len > INT_MAX - KV_TREE_MAX) return KV_ERANGE;
        if (a->mask && n > 64ll * a->mask_words) return KV_ERANGE;
        max_total = std::max(max_total, len + n);
    }
    TreeParams t{};
    const int rc = cache_addr(p, view, blocks, layer, view->seq_lens_host, a->tok_first_host, &t.c);
    if (rc != KV_OK) return rc;
    // a row's scales are loaded at once
    if (blocks && (((uintptr_t)t.c.kz | (uintptr_t)t.c.vz | t.c.zb | t.c.zh | t.c.zs) & (p->D / kBlockElems - 1))) return KV_EINVAL;
    const int n_tok = a->tok_first_host[p->B];
    if (n_tok == 0) return KV_OK;
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
    t.scale = a->scale == 0.f ? (float)(1 / std::sqrt((double)p->D)) : a->scale;
    t.out_mode = a->out_dtype == KV_OUT_F32 ? 0 : bf16 ? 2 : 1;
    const int format = blocks ? blocks->format : KV_FORMAT_16;
    TreeKernel k = p->D == 64 ? tree_kernel<64>(bf16, format) : p->D == 128 ? tree_kernel<128>(bf16, format) : tree_kernel<256>(bf16, format);
    (void)launch_kernel(k, dim3((unsigned)n_tok, (unsigned)p->Hq), dim3(256), (hipStream_t)hip_stream, t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    return KV_OK;
}
