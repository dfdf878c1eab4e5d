// Rotation of a head's elements, shared by kv_rope and by the cache write.
#pragma once

#include "cache.hpp"

namespace kvb {

// Cosines and sines of N neighbouring pairs of a position; NaN where the table does not have it.
template <int N>
struct Angles {
    float c[N], s[N];
};
template <int N>
__device__ __forceinline__ Angles<N> load_angles(const float *table, int n_pos, int half, int pos, unsigned pair, float sign)
{
    Angles<N> a;
    const bool known = (unsigned)pos < (unsigned)n_pos;
    const f32x4 *const at = (const f32x4 *)(table + ((unsigned long long)(known ? pos : 0) * half + pair) * 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const f32x4 w = at[i];
        a.c[2 * i] = known ? w[0] : __builtin_nanf("");
        a.s[2 * i] = known ? sign * w[1] : __builtin_nanf("");
        a.c[2 * i + 1] = known ? w[2] : __builtin_nanf("");
        a.s[2 * i + 1] = known ? sign * w[3] : __builtin_nanf("");
    }
    return a;
}

// (x, y) turned: each product and the sum are rounded on their own, so a result does not depend on what the compiler fuses, and blocks
// formed of rotated rows are the same wherever they are formed.  The products cost nothing next to the memory traffic.
__device__ __forceinline__ void turn(float x, float y, float c, float s, float *tx, float *ty)
{
#pragma clang fp contract(off)
    *tx = x * c - y * s;
    *ty = y * c + x * s;
}

// Two vectors of eight elements that pair up element by element.
template <bool BF16>
__device__ __forceinline__ void turn_halves(u32x4 &a, u32x4 &b, const Angles<8> &t)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 x = unpack2<BF16>(a[i]), y = unpack2<BF16>(b[i]);
        float x0, y0, x1, y1;
        turn(x[0], y[0], t.c[2 * i], t.s[2 * i], &x0, &y0);
        turn(x[1], y[1], t.c[2 * i + 1], t.s[2 * i + 1], &x1, &y1);
        a[i] = pack2<BF16>(x0, x1);
        b[i] = pack2<BF16>(y0, y1);
    }
}
// A vector of four pairs side by side; t holds them from `first` on.
template <bool BF16, int N>
__device__ __forceinline__ void turn_pairs(u32x4 &a, const Angles<N> &t, int first)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 x = unpack2<BF16>(a[i]);
        float x0, x1;
        turn(x[0], x[1], t.c[first + i], t.s[first + i], &x0, &x1);
        a[i] = pack2<BF16>(x0, x1);
    }
}

}  // namespace kvb
