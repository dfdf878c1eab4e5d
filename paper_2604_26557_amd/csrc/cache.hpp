// What the kernels over a cache of 16, 8 or 4 bits share: where a row lies, its checks on the host, and the conversions of its blocks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "plan.hpp"

namespace kvb {

constexpr int kBlockElems = 32;  // elements of a head's row that share a scale

// Where the rows of one layer lie.  Strides are bytes; the scales' (z) are zero in a 16-bit cache.
struct CacheAddr {
    const char *k, *v, *kz, *vz;
    unsigned long long sb, sh, ss;  // from sequence to sequence (paged: block to block), head to head, token to token
    unsigned long long zb, zh, zs;
    const int *table;               // paged: [B, max_blocks]; null: strided
    int max_blocks, bt, n_pool;
    int B, rows;                    // strided: token rows of a sequence
};

// Sequence's (paged: block's) number and the token's row in it; false where the cache has no such row.
__device__ __forceinline__ bool find_row(const CacheAddr &c, int seq, int slot, unsigned *block, unsigned *row)
{
    if ((unsigned)seq >= (unsigned)c.B || slot < 0) return false;
    if (!c.table) {
        *block = (unsigned)seq;
        *row = (unsigned)slot;
        return slot < c.rows;
    }
    const int i = slot / c.bt;
    if (i >= c.max_blocks) return false;
    const int id = c.table[(long long)seq * c.max_blocks + i];
    *block = (unsigned)id;
    *row = (unsigned)(slot - i * c.bt);
    return (unsigned)id < (unsigned)c.n_pool;
}

// Bits of an element in the cache.
constexpr int format_bits(int format) { return format == KV_FORMAT_16 ? 16 : format == KV_FORMAT_FP8 ? 8 : 4; }

// Checks a layer of a cache against the plan and fills c.  lens[b] + first[b + 1] - first[b], or without them s_alloc, is how many token rows of
// sequence b may be touched.
int cache_addr(const kv_plan *p, const kv_view_t *view, const kv_blocks_t *blocks, int layer, const int *lens, const int *first, CacheAddr *c);

// Heads of a row that a thread of the row kernels goes over: what it looks up of the row (its place, the angles of its position) serves all of them, but with few
// rows they are rather worked on side by side.  Four once that leaves 2048 wavefronts, two once it leaves 1024.  One against four heads: 37.5K rows of 8 heads x 128 read from 8 bits 71 -> 36 us,
// 8192 rows written to 4 bits and read back 25 -> 21; a step's hundred rows are the launch either way.
inline int heads_per_thread(long long n_tok, int n_heads, int vectors)
{
    const long long waves = n_tok * n_heads * vectors / 64;
    return n_heads >= 4 && waves >= 4 * 2048 ? 4 : n_heads >= 2 && waves >= 2 * 1024 ? 2 : 1;
}

// A rotary table that fits head_dim.
int check_rope(const kv_rope_t *r, int head_dim);

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned short bf16_bits(float f)
{
    return __builtin_bit_cast(unsigned short, (__bf16)f);  // to nearest even; a NaN stays one
}

// Two floats to a pair of 16-bit numbers, to nearest even.
template <bool BF16>
__device__ __forceinline__ unsigned pack2(float x, float y)
{
    if constexpr (BF16) return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x, y}, bf16x2));
    else return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x, y}, f16x2));
}
template <bool BF16>
__device__ __forceinline__ f32x2 unpack2(unsigned w)
{
    if constexpr (BF16) return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
    else return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
}

// A scale's byte as the operand that the conversions below take their exponent from: 255 gives NaN, 0 gives 2^-127 (all 256 bytes
// times all codes were compared with the definition on the card).
__device__ __forceinline__ float scale_operand(unsigned byte) { return __uint_as_float(byte << 23); }

// Two neighbouring codes to a pair of 16-bit numbers: code times scale, which is exact unless the 16-bit type runs out of exponent.
// FP8: codes 2 * SEL and 2 * SEL + 1 of w, SEL = 0 or 1; FP4: SEL = 0..3.
template <bool BF16, int FORMAT, int SEL>
__device__ __forceinline__ unsigned decode2(unsigned w, float scale)
{
    if constexpr (FORMAT == KV_FORMAT_FP8) {
        if constexpr (BF16) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, SEL != 0));
        else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, SEL != 0));
    } else {
        if constexpr (BF16) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
        else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL));
    }
}
// Eight neighbouring codes: FP8 from two words, FP4 from one.
template <bool BF16, int FORMAT>
__device__ __forceinline__ u32x4 decode8(u32x2 w, float scale)
{
    if constexpr (FORMAT == KV_FORMAT_FP8)
        return u32x4{decode2<BF16, FORMAT, 0>(w[0], scale), decode2<BF16, FORMAT, 1>(w[0], scale),
                     decode2<BF16, FORMAT, 0>(w[1], scale), decode2<BF16, FORMAT, 1>(w[1], scale)};
    else
        return u32x4{decode2<BF16, FORMAT, 0>(w[0], scale), decode2<BF16, FORMAT, 1>(w[0], scale),
                     decode2<BF16, FORMAT, 2>(w[0], scale), decode2<BF16, FORMAT, 3>(w[0], scale)};
}

}  // namespace kvb
