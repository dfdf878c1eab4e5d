// Rows of new tokens into a cache of 16, 8 or 4 bits (K rotated on its way), and rows of it back as 16-bit values.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "cache.hpp"
#include "launch.hpp"
#include "rope.hpp"

namespace {

using namespace kvb;

constexpr int kThreads = 256;

struct RowParams {
    CacheAddr c;
    char *k, *v;                       // rows of the call, 16-bit (read: const in all but name)
    long long k_st, k_sh, v_st, v_sh;  // bytes
    const int *tok_seq, *tok_slot;
    const float *table;                // rotary positions; null: none
    const int *positions;
    int n_pos, rot;
    int n_heads, vectors;              // vectors of 8 elements in a head's row
    int n_rows;
    unsigned n_items;                  // of K; as many of V in the grid's second row
};

// Maximum over the four lanes of a block.
__device__ __forceinline__ unsigned quad_max(unsigned x)
{
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false));        // quad_perm [1,0,3,2]
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false));     // quad_perm [2,3,0,1]
}

// One lane's eight elements of a block that four neighbouring lanes hold: codes, and the scale's byte (the same in all four).
template <bool BF16, int FORMAT>
__device__ __forceinline__ u32x2 encode8(u32x4 x, unsigned *scale)
{
    // magnitudes as 16-bit patterns: their order is that of whole numbers, and what is not finite lies above what is
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fffu, x[i] >> 16 & 0x7fffu));
    top = quad_max(top);
    constexpr unsigned kInf = BF16 ? 0x7f80u : 0x7c00u;
    // 1.875 or 1.5 times the largest power of two: what lies above rounds to the next one, which is no number of the type
    constexpr unsigned kMost = BF16 ? (FORMAT == KV_FORMAT_FP8 ? 0x7f70u : 0x7f40u) : (FORMAT == KV_FORMAT_FP8 ? 0x7b80u : 0x7a00u);
    const float most = unpack2<BF16>(kMost)[0];
    const bool fine = top < kInf;
    const unsigned bits = __float_as_uint(unpack2<BF16>(min(top, kMost))[0]);
    // the largest code is 1.75 * 2^8 or 1.5 * 2^2: one exponent more where the mantissa is larger
    constexpr unsigned kLargest = FORMAT == KV_FORMAT_FP8 ? 0x600000u : 0x400000u;
    const int e = (int)(bits >> 23) - (FORMAT == KV_FORMAT_FP8 ? 8 : 2) + ((bits & 0x7fffffu) > kLargest ? 1 : 0);
    const unsigned byte = fine ? (unsigned)max(e, 0) : 255u;
    *scale = byte;
    const float inv = __uint_as_float((254u - min(byte, 253u)) << 23);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 y = unpack2<BF16>(x[i]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f[2 * i + j] = fine ? fminf(fmaxf(y[j], -most), most) * inv : 0.f;
        }
    }
    if constexpr (FORMAT == KV_FORMAT_FP8) {
        unsigned a = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false), b = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], 0, false);
        a = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], a, true);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], b, true);
        return u32x2{a, b};
    } else {
        unsigned a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, f[0], f[1], 1.f, 0);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, f[2], f[3], 1.f, 1);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, f[4], f[5], 1.f, 2);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, f[6], f[7], 1.f, 3);
        return u32x2{a, 0};
    }
}

// A thread has a vector column of a row, found once, in HPT heads of K (blockIdx.y = 0) or V.  Neighbouring lanes have a row's vectors, then the next rows': what lies
// side by side in the call's rows or in the cache is read and written by one wavefront.  The four vectors of a block are neighbouring lanes: head_dim is a multiple of 32.
struct Item {
    unsigned v, h, t;
    bool is_v;
};
template <int HPT>
__device__ __forceinline__ bool item_of(const RowParams &p, Item *it)
{
    const unsigned i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.n_items) return false;
    const unsigned r = i / (unsigned)p.vectors, g = r / (unsigned)p.n_rows;   // head groups one after the other
    *it = Item{i - r * (unsigned)p.vectors, g * HPT, r - g * (unsigned)p.n_rows, blockIdx.y != 0};
    return true;
}

// Bytes of a vector of eight elements.
constexpr int vector_bytes(int format) { return format_bits(format); }

// Rows into the cache.  The largest magnitude of a block is formed over the four lanes that have it, by two exchanges within the wavefront; everything else is a lane's own.  Where
// halves of a head are turned against each other a lane reads the other half's vector as well (out of L2) rather than exchanging it.  Bound by memory: 8192 rows of 2 x 8 heads x 128 to 4 bits
// (33.6 MB read, 8.9 MB written, the table) in 13.0 us; a step's 126 rows in 3.8 us, the launch.
template <bool BF16, int FORMAT, bool PAIRS, int HPT>
__global__ void __launch_bounds__(kThreads) kv_cache_write_kernel(RowParams p)
{
    Item it;
    if (!item_of<HPT>(p, &it)) return;
    unsigned block, row;
    if (!find_row(p.c, p.tok_seq[it.t], p.tok_slot[it.t], &block, &row)) return;  // a block's lanes share the row: all leave or none
    const char *const src = (it.is_v ? p.v + it.t * p.v_st : p.k + it.t * p.k_st);
    const long long sh = it.is_v ? p.v_sh : p.k_sh;
    char *const dst = (char *)(it.is_v ? p.c.v : p.c.k) + block * p.c.sb + row * p.c.ss + vector_bytes(FORMAT) * it.v;
    char *const scales = (char *)(it.is_v ? p.c.vz : p.c.kz) + block * p.c.zb + row * p.c.zs + it.v / 4;
    const bool turned = p.table && !it.is_v && it.v < (unsigned)p.rot / 8;
    const unsigned half = (unsigned)p.rot / 16;   // vectors
    const bool second = it.v >= half;
    Angles<8> ang;
    if (turned) {
        const int pos = p.positions[it.t];
        if constexpr (PAIRS) {
            const Angles<4> a = load_angles<4>(p.table, p.n_pos, p.rot / 2, pos, 4 * it.v, 1.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) ang.c[k] = a.c[k], ang.s[k] = a.s[k];
        } else {
            ang = load_angles<8>(p.table, p.n_pos, p.rot / 2, pos, 8 * (second ? it.v - half : it.v), 1.f);
        }
    }
    u32x4 x[HPT], other[HPT];
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const char *const at = src + min(it.h + k, (unsigned)p.n_heads - 1) * sh;   // a head past the last one is not stored
        x[k] = *(const u32x4 *)(at + 16 * it.v);
        if (!PAIRS && turned) other[k] = *(const u32x4 *)(at + 16 * (second ? it.v - half : it.v + half));
    }
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const unsigned h = it.h + k;
        if (h >= (unsigned)p.n_heads) break;
        if (turned) {
            if constexpr (PAIRS) {
                turn_pairs<BF16>(x[k], ang, 0);
            } else {
                u32x4 a = second ? other[k] : x[k], b = second ? x[k] : other[k];
                turn_halves<BF16>(a, b, ang);
                x[k] = second ? b : a;
            }
        }
        if constexpr (FORMAT == KV_FORMAT_16) {
            *(u32x4 *)(dst + h * p.c.sh) = x[k];
        } else {
            unsigned byte;
            const u32x2 w = encode8<BF16, FORMAT>(x[k], &byte);
            if constexpr (FORMAT == KV_FORMAT_FP8) *(u32x2 *)(dst + h * p.c.sh) = w;
            else *(unsigned *)(dst + h * p.c.sh) = w[0];
            if (it.v % 4 == 0) scales[h * p.c.zh] = (char)byte;
        }
    }
}

// Rows out of the cache: a code times its block's power of two, which the conversion instructions do exactly.  Bound by memory, writes for the most part: 37.5K rows of 2 x 8 heads x 128 from
// 8 bits (79 MB read, 154 MB written) in 36.2 us = 6.4 TB/s; stores bypass the caches, as nothing reads them soon.
template <bool BF16, int FORMAT, bool, int HPT>
__global__ void __launch_bounds__(kThreads) kv_cache_read_kernel(RowParams p)
{
    Item it;
    if (!item_of<HPT>(p, &it)) return;
    unsigned block, row;
    if (!find_row(p.c, p.tok_seq[it.t], p.tok_slot[it.t], &block, &row)) return;
    const char *const src = (it.is_v ? p.c.v : p.c.k) + block * p.c.sb + row * p.c.ss + vector_bytes(FORMAT) * it.v;
    const char *const scales = (it.is_v ? p.c.vz : p.c.kz) + block * p.c.zb + row * p.c.zs + it.v / 4;
    char *const dst = (it.is_v ? p.v + it.t * p.v_st : p.k + it.t * p.k_st) + 16 * it.v;
    const long long sh = it.is_v ? p.v_sh : p.k_sh;
    u32x4 x[HPT];
    unsigned byte[HPT];
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const unsigned h = min(it.h + k, (unsigned)p.n_heads - 1);
        if constexpr (FORMAT == KV_FORMAT_16) {
            x[k] = *(const u32x4 *)(src + h * p.c.sh);
        } else if constexpr (FORMAT == KV_FORMAT_FP8) {
            const u32x2 w = *(const u32x2 *)(src + h * p.c.sh);
            x[k] = u32x4{w[0], w[1], 0, 0};
        } else {
            x[k] = u32x4{*(const unsigned *)(src + h * p.c.sh), 0, 0, 0};
        }
        if constexpr (FORMAT != KV_FORMAT_16) byte[k] = (unsigned char)scales[h * p.c.zh];
    }
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const unsigned h = it.h + k;
        if (h >= (unsigned)p.n_heads) break;
        if constexpr (FORMAT != KV_FORMAT_16) x[k] = decode8<BF16, FORMAT>(u32x2{x[k][0], x[k][1]}, scale_operand(byte[k]));
        __builtin_nontemporal_store(x[k], (u32x4 *)(dst + h * sh));
    }
}

typedef void (*RowKernel)(RowParams);
template <bool BF16, int HPT>
RowKernel kernel_of(bool write, int format, bool pairs)
{
    if (write) {
        if (format == KV_FORMAT_FP8) return pairs ? kv_cache_write_kernel<BF16, KV_FORMAT_FP8, true, HPT> : kv_cache_write_kernel<BF16, KV_FORMAT_FP8, false, HPT>;
        if (format == KV_FORMAT_FP4) return pairs ? kv_cache_write_kernel<BF16, KV_FORMAT_FP4, true, HPT> : kv_cache_write_kernel<BF16, KV_FORMAT_FP4, false, HPT>;
        return pairs ? kv_cache_write_kernel<BF16, KV_FORMAT_16, true, HPT> : kv_cache_write_kernel<BF16, KV_FORMAT_16, false, HPT>;
    }
    return format == KV_FORMAT_FP8   ? kv_cache_read_kernel<BF16, KV_FORMAT_FP8, false, HPT>
           : format == KV_FORMAT_FP4 ? kv_cache_read_kernel<BF16, KV_FORMAT_FP4, false, HPT>
                                     : kv_cache_read_kernel<BF16, KV_FORMAT_16, false, HPT>;
}
RowKernel kernel_of(bool bf16, int heads, bool write, int format, bool pairs)
{
    if (bf16) return heads == 1 ? kernel_of<true, 1>(write, format, pairs) : heads == 2 ? kernel_of<true, 2>(write, format, pairs) : kernel_of<true, 4>(write, format, pairs);
    return heads == 1 ? kernel_of<false, 1>(write, format, pairs) : heads == 2 ? kernel_of<false, 2>(write, format, pairs) : kernel_of<false, 4>(write, format, pairs);
}

// Checks of the rows of a call and the launch, shared by both directions; p holds the cache's place and the rotary table.
int launch_rows(const kv_plan *pl, RowParams &p, bool write, int format, bool pairs, const void *k, const void *v, int64_t k_st, int64_t k_sh, int64_t v_st, int64_t v_sh,
                const int32_t *tok_seq, const int32_t *tok_slot, const int32_t *positions, int n_tok, void *hip_stream)
{
    if (n_tok < 0 || k_st < 0 || k_sh < 0 || v_st < 0 || v_sh < 0 || ((k_st | k_sh | v_st | v_sh) & 7)) return KV_EINVAL;
    if (n_tok == 0) return KV_OK;
    if (!k || !v || !tok_seq || !tok_slot || (((uintptr_t)k | (uintptr_t)v) & 15)) return KV_EINVAL;
    p.k_st = 2 * k_st; p.k_sh = 2 * k_sh; p.v_st = 2 * v_st; p.v_sh = 2 * v_sh;
    p.n_heads = pl->H;
    p.vectors = pl->D / 8;
    const int heads = heads_per_thread(n_tok, p.n_heads, p.vectors), head_groups = (p.n_heads + heads - 1) / heads;
    const RowKernel kernel = kernel_of(pl->dtype == KV_BF16, heads, write, format, pairs);
    const long long per_tok = (long long)head_groups * p.vectors;
    const long long most = (1ll << 31) / per_tok;  // tokens of a launch: items are counted in 32 bits
    if (most < 1) return KV_ERANGE;
    for (long long t0 = 0; t0 < n_tok; t0 += most) {
        const long long n = std::min<long long>(most, n_tok - t0);
        p.k = (char *)k + t0 * p.k_st;
        p.v = (char *)v + t0 * p.v_st;
        p.tok_seq = tok_seq + t0;
        p.tok_slot = tok_slot + t0;
        p.positions = positions ? positions + t0 : nullptr;
        p.n_items = (unsigned)(n * per_tok);
        p.n_rows = (int)n;
        (void)launch_kernel(kernel, dim3((p.n_items + kThreads - 1) / kThreads, 2), dim3(kThreads), (hipStream_t)hip_stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    }
    return KV_OK;
}

}  // namespace

int kvb::cache_addr(const kv_plan *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const int *lens, const int *first, CacheAddr *c)
{
    *c = CacheAddr{};
    if (!view->k_layers || !view->v_layers || view->seq_off_host || view->seq_off_dev) return KV_EINVAL;
    if (layer < 0 || layer >= p->L || layer >= view->n_layers) return KV_ERANGE;
    const int format = blocks ? blocks->format : KV_FORMAT_16;
    if (blocks) {
        if (format != KV_FORMAT_FP8 && format != KV_FORMAT_FP4) return KV_EINVAL;
        if (!blocks->k_scales || !blocks->v_scales) return KV_EINVAL;
        if (layer >= blocks->n_layers) return KV_ERANGE;
        if (p->D % kBlockElems != 0) return KV_EINVAL;
        if (blocks->stride_b < 0 || blocks->stride_h < 0 || blocks->stride_s < 0) return KV_EINVAL;
    }
    c->k = (const char *)view->k_layers[layer];
    c->v = (const char *)view->v_layers[layer];
    if (!c->k || !c->v || (((uintptr_t)c->k | (uintptr_t)c->v) & 15)) return KV_EINVAL;
    if (blocks) {
        c->kz = (const char *)blocks->k_scales[layer];
        c->vz = (const char *)blocks->v_scales[layer];
        if (!c->kz || !c->vz) return KV_EINVAL;
        c->zb = (uint64_t)blocks->stride_b; c->zh = (uint64_t)blocks->stride_h; c->zs = (uint64_t)blocks->stride_s;
    }
    const uint64_t row = (uint64_t)p->D * format_bits(format) / 8, zrow = (uint64_t)p->D / kBlockElems;
    c->B = p->B;
    // no byte past the buffer's end; the sums are kept in 128 bits
    auto inside = [](uint64_t nb, uint64_t sb, uint64_t nh, uint64_t sh, uint64_t ns, uint64_t ss, uint64_t row_bytes, uint64_t bytes) {
        const unsigned __int128 end = (unsigned __int128)(nb - 1) * sb + (unsigned __int128)(nh - 1) * sh + (unsigned __int128)(ns - 1) * ss + row_bytes;
        return end <= bytes;
    };
    if (view->layout == KV_LAYOUT_BHSD) {
        if (view->stride_b < 0 || view->stride_h < 0 || view->stride_s < 0 || view->s_alloc < 0) return KV_EINVAL;
        if ((view->stride_b | view->stride_h | view->stride_s) & 7) return KV_EINVAL;
        c->sb = 2 * (uint64_t)view->stride_b; c->sh = 2 * (uint64_t)view->stride_h; c->ss = 2 * (uint64_t)view->stride_s;
        c->rows = view->s_alloc;
        for (int b = 0; b < p->B; ++b) {
            const int64_t n = lens ? (int64_t)lens[b] + (first[b + 1] - first[b]) : view->s_alloc;
            if (n > view->s_alloc) return KV_ERANGE;
            if (n < 1) continue;
            if (!inside(b + 1, c->sb, p->H, c->sh, n, c->ss, row, view->layer_bytes)) return KV_ERANGE;
            if (blocks && !inside(b + 1, c->zb, p->H, c->zh, n, c->zs, zrow, blocks->layer_bytes)) return KV_ERANGE;
        }
    } else if (view->layout == KV_LAYOUT_PAGED) {
        if (!view->block_table || view->block_tokens < 1 || view->n_pool_blocks < 0 || view->max_blocks_per_seq < 0) return KV_EINVAL;
        c->table = view->block_table;
        c->max_blocks = view->max_blocks_per_seq;
        c->bt = view->block_tokens;
        c->n_pool = view->n_pool_blocks;
        c->ss = row;
        c->sh = row * (uint64_t)c->bt;
        c->sb = c->sh * (uint64_t)p->H;
        if (c->n_pool > 0) {
            if (!inside(c->n_pool, c->sb, p->H, c->sh, c->bt, c->ss, row, view->layer_bytes)) return KV_ERANGE;
            if (blocks && !inside(c->n_pool, c->zb, p->H, c->zh, c->bt, c->zs, zrow, blocks->layer_bytes)) return KV_ERANGE;
        }
        for (int b = 0; lens && b < p->B; ++b)
            if (ceil_div((uint64_t)lens[b] + (uint64_t)(first[b + 1] - first[b]), (uint64_t)c->bt) > (uint64_t)c->max_blocks) return KV_ERANGE;
    } else {
        return KV_EINVAL;
    }
    return KV_OK;
}

extern "C" int kv_cache_write(const kv_plan_t *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const kv_write_args_t *a, void *hip_stream)
{
    if (!p || !view || !a || p->D % kBlockElems != 0) return KV_EINVAL;
    RowParams r{};
    int rc = cache_addr(p, view, blocks, layer, nullptr, nullptr, &r.c);
    if (rc != KV_OK) return rc;
    bool pairs = false;
    if (a->rope) {
        rc = check_rope(a->rope, p->D);
        if (rc != KV_OK) return rc;
        if (!a->positions && a->n_tok > 0) return KV_EINVAL;
        r.table = a->rope->table;
        r.n_pos = a->rope->n_pos;
        r.rot = a->rope->rot_dim;
        pairs = a->rope->style == KV_ROPE_PAIRS;
    }
    const int format = blocks ? blocks->format : KV_FORMAT_16;
    return launch_rows(p, r, true, format, pairs, a->k, a->v, a->k_stride_t,
                       a->k_stride_h, a->v_stride_t, a->v_stride_h, a->tok_seq, a->tok_slot, a->positions, a->n_tok, hip_stream);
}

extern "C" int kv_cache_read(const kv_plan_t *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const kv_read_args_t *a, void *hip_stream)
{
    if (!p || !view || !a || p->D % kBlockElems != 0) return KV_EINVAL;
    RowParams r{};
    const int rc = cache_addr(p, view, blocks, layer, nullptr, nullptr, &r.c);
    if (rc != KV_OK) return rc;
    const int format = blocks ? blocks->format : KV_FORMAT_16;
    return launch_rows(p, r, false, format, false, a->k, a->v, a->k_stride_t, a->k_stride_h,
                       a->v_stride_t, a->v_stride_h, a->tok_seq, a->tok_slot, nullptr, a->n_tok, hip_stream);
}
