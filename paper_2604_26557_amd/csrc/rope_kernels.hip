// Rotary positions: the table of a schedule of frequencies (host), and the rotation of rows on their own (kv_rope).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cache.hpp"
#include "launch.hpp"
#include "rope.hpp"

namespace {

using namespace kvb;

constexpr int kThreads = 256;

struct RopeParams {
    const float *table;
    const int *positions;
    const char *x;
    char *out;
    long long x_st, x_sh, o_st, o_sh;  // bytes
    float sign;
    int n_pos, rot, n_heads, chunks;   // chunks of 16 elements in a head
    unsigned n_items;
};

// An item is a chunk of HPT heads of a token: two vectors of eight elements, whose pairs are the same eight in both layouts (8 c .. 8 c + 7: first half
// and second half, or side by side), so in-place rows need no other thread's data.  The angles are looked up once for the HPT heads.  Bound by memory: an element is read and
// written once, 4 bytes: 8124 rows of 32 heads x 128 (135 MB) in 26.0 us = 5.2 TB/s, the rate of a plain copy; a decode step's 8 rows in 2.9 us, the launch.
template <bool BF16, bool PAIRS, int HPT>
__global__ void __launch_bounds__(kThreads) kv_rope_kernel(RopeParams p)
{
    const unsigned i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.n_items) return;
    const unsigned groups = (unsigned)(p.n_heads + HPT - 1) / HPT;
    const unsigned c = i % (unsigned)p.chunks, r = i / (unsigned)p.chunks, g = r % groups, t = r / groups;
    const bool turned = c < (unsigned)p.rot / 16;
    const unsigned va = PAIRS || !turned ? 2 * c : c, vb = PAIRS || !turned ? 2 * c + 1 : c + (unsigned)p.rot / 16;
    const char *const x = p.x + t * p.x_st;
    char *const out = p.out + t * p.o_st;
    u32x4 a[HPT], b[HPT];
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const unsigned h = min(g * HPT + k, (unsigned)p.n_heads - 1);  // a head past the last one is not stored
        a[k] = *(const u32x4 *)(x + h * p.x_sh + 16 * va);
        b[k] = *(const u32x4 *)(x + h * p.x_sh + 16 * vb);
    }
    if (turned) {
        const Angles<8> ang = load_angles<8>(p.table, p.n_pos, p.rot / 2, p.positions[t], 8 * c, p.sign);
#pragma unroll
        for (int k = 0; k < HPT; ++k) {
            if constexpr (PAIRS) {
                turn_pairs<BF16>(a[k], ang, 0);
                turn_pairs<BF16>(b[k], ang, 4);
            } else {
                turn_halves<BF16>(a[k], b[k], ang);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
        const unsigned h = g * HPT + k;
        if (h >= (unsigned)p.n_heads) break;
        *(u32x4 *)(out + h * p.o_sh + 16 * va) = a[k];
        *(u32x4 *)(out + h * p.o_sh + 16 * vb) = b[k];
    }
}

template <int HPT>
void launch(bool bf16, bool pairs, dim3 grid, hipStream_t st, const RopeParams &p)
{
    auto *const kernel = bf16 ? (pairs ? kv_rope_kernel<true, true, HPT> : kv_rope_kernel<true, false, HPT>)
                              : (pairs ? kv_rope_kernel<false, true, HPT> : kv_rope_kernel<false, false, HPT>);
    (void)launch_kernel(kernel, grid, dim3(kThreads), st, p);
}

}  // namespace

int kvb::check_rope(const kv_rope_t *r, int head_dim)
{
    if (!r->table || ((uintptr_t)r->table & 15) || r->n_pos < 1) return KV_EINVAL;
    if (r->rot_dim < 16 || r->rot_dim % 16 != 0 || r->rot_dim > head_dim) return KV_EINVAL;
    if (r->style != KV_ROPE_HALF && r->style != KV_ROPE_PAIRS) return KV_EINVAL;
    return KV_OK;
}

extern "C" int kv_rope_table(const kv_rope_desc_t *d, float *table, size_t bytes)
{
    if (!d || !table || d->n_pos < 1 || d->rot_dim < 16 || d->rot_dim % 16 != 0) return KV_EINVAL;
    if (d->scaling < KV_ROPE_PLAIN || d->scaling > KV_ROPE_INDEX) return KV_EINVAL;
    // written so that a NaN fails
    if (!(d->base > 1) || !std::isfinite(d->base) || !std::isfinite(d->magnitude)) return KV_EINVAL;
    if (d->scaling != KV_ROPE_PLAIN && (!(d->factor >= 1) || !std::isfinite(d->factor))) return KV_EINVAL;
    const bool mixed = d->scaling == KV_ROPE_WAVELENGTH || d->scaling == KV_ROPE_INDEX;
    if (mixed && (d->trained_pos < 1 || !(d->low > 0) || !(d->high > d->low) || !std::isfinite(d->high))) return KV_EINVAL;
    const int half = d->rot_dim / 2;
    if (bytes / sizeof(float) / d->rot_dim < (size_t)d->n_pos) return KV_ENOSPC;
    const double two_pi = 6.283185307179586476925, magnitude = d->magnitude == 0 ? 1 : d->magnitude;
    const double base = d->scaling == KV_ROPE_BASE ? d->base * std::pow(d->factor, d->rot_dim / (d->rot_dim - 2.0)) : d->base;
    // INDEX: the pair at which a frequency makes t turns within the trained context; there need be none of that number
    auto pair_of = [&](double t) { return half * std::log(d->trained_pos / (t * two_pi)) / std::log(base); };
    auto end_of = [&](double i) { return std::min(std::max(i, 0.0), d->rot_dim - 1.0); };
    const double first = mixed ? end_of(std::floor(pair_of(d->high))) : 0, last = mixed ? end_of(std::ceil(pair_of(d->low))) : 0;
    for (int i = 0; i < half; ++i) {
        double f = std::pow(base, -(double)i / half);
        if (d->scaling == KV_ROPE_LINEAR) f /= d->factor;
        if (mixed) {
            double keep;  // share of the frequency that is not stretched
            if (d->scaling == KV_ROPE_WAVELENGTH) keep = (d->trained_pos * f / two_pi - d->low) / (d->high - d->low);
            else keep = 1 - (i - first) / std::max(last - first, 1e-3);
            keep = std::min(std::max(keep, 0.0), 1.0);
            f = f * keep + f / d->factor * (1 - keep);
        }
        for (int n = 0; n < d->n_pos; ++n) {
            float *const at = table + ((size_t)n * half + i) * 2;
            at[0] = (float)(magnitude * std::cos(n * f));
            at[1] = (float)(magnitude * std::sin(n * f));
        }
    }
    return KV_OK;
}

extern "C" int kv_rope(const kv_rope_t *r, const kv_rope_args_t *a, void *hip_stream)
{
    if (!r || !a || a->n_tok < 0 || a->n_heads < 1 || a->head_dim < 16 || a->head_dim % 16 != 0) return KV_EINVAL;
    if (a->dtype != KV_F16 && a->dtype != KV_BF16) return KV_EINVAL;
    int rc = check_rope(r, a->head_dim);
    if (rc != KV_OK) return rc;
    if (a->n_tok == 0) return KV_OK;
    if (!a->x || !a->out || !a->positions || (((uintptr_t)a->x | (uintptr_t)a->out) & 15)) return KV_EINVAL;
    if ((a->x_stride_t | a->x_stride_h | a->out_stride_t | a->out_stride_h) & 7) return KV_EINVAL;
    if (a->x_stride_t < 0 || a->x_stride_h < 0 || a->out_stride_t < 0 || a->out_stride_h < 0) return KV_EINVAL;
    if (a->x == a->out && (a->x_stride_t != a->out_stride_t || a->x_stride_h != a->out_stride_h)) return KV_EINVAL;

    RopeParams p{};
    p.table = r->table;
    p.x_st = 2 * a->x_stride_t; p.x_sh = 2 * a->x_stride_h; p.o_st = 2 * a->out_stride_t; p.o_sh = 2 * a->out_stride_h;
    p.sign = a->transposed ? -1.f : 1.f;
    p.n_pos = r->n_pos; p.rot = r->rot_dim; p.n_heads = a->n_heads; p.chunks = a->head_dim / 16;
    const int heads = heads_per_thread(a->n_tok, a->n_heads, p.chunks);
    const long long per_tok = (long long)((a->n_heads + heads - 1) / heads) * p.chunks;
    const long long most = (1ll << 31) / per_tok;  // tokens of a launch: items are counted in 32 bits
    if (most < 1) return KV_ERANGE;
    for (long long t0 = 0; t0 < a->n_tok; t0 += most) {
        const long long n = std::min<long long>(most, a->n_tok - t0);
        p.x = (const char *)a->x + t0 * p.x_st;
        p.out = (char *)a->out + t0 * p.o_st;
        p.positions = a->positions + t0;
        p.n_items = (unsigned)(n * per_tok);
        const dim3 grid((p.n_items + kThreads - 1) / kThreads);
        (heads == 4 ? launch<4> : heads == 2 ? launch<2> : launch<1>)(a->dtype == KV_BF16, r->style == KV_ROPE_PAIRS, grid, (hipStream_t)hip_stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) { set_hip_error((int)e); return KV_EHIP; }
    }
    return KV_OK;
}
