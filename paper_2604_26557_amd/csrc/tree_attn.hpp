// Kernels of kv_tree_attn, a translation unit for each cache format (tree_attn_16.hip, tree_attn_fp8.hip, tree_attn_fp4.hip).
//
// Mathematics.  A query row is one query head of one drafted token; the G query heads of a KV head share its K and V, so the rows of a sequence and KV head are
// T * G.  Each row has out = sum_j p_j V_j / sum_j p_j with p_j = exp2((q . K_j) scale log2(e) - ref), in one pass over the tokens: ref is any number near the running
// maximum, the same for all tokens that are added up, and sums are multiplied by exp2(old - new) when it moves.  Parts of the tokens with references of their own
// (wavefronts, then workgroups) are joined by the same factors.
//
// Work.  A workgroup has a split of a KV head's tokens and 16, 32 or 64 of its rows (NB row groups); its four wavefronts take every fourth step of 32 tokens, each for
// all the rows, so K and V are decoded once per workgroup, and join their sums at the end.  Both products are on the matrix cores (16 x 16 x 32): S^T = K q^T has K's
// rows as its first operand and query rows as columns, so that a lane ends up with eight scores of one row, which as they lie are the second operand of V^T P^T: no score
// changes lanes.  Sums of probabilities are one more product, with ones.
//
// What bounds it, and what was measured (MI355X, us per call, the second launch that joins splits included):
//   the bytes of K and V, where rows are few: 4 sequences of 8K x 16 heads x 256, 8-bit, 6 rows per head: 278 MB in 49.2 = 5.6 TB/s;
//   the vector ALU, where rows are many (an exponential for every row and token and its two parts, a conversion for every element of K and V, beside the matrix cores at 39 %): 32K
//   tokens x 8 heads x 128, 8-bit, 256 rows per head: 34.4 GFLOP in 67.4 = 510 TFLOP/s;
//   the start of a workgroup, its merge (3 to 5 us) and the second launch (4), where the call is short: 4K tokens x 8 heads x 128, 64 rows per head: 14.2.
// Why so:
//   K and V go through LDS, loaded there without passing registers: 16 KiB of a wavefront are on their way while it computes, without spilling what holds the sums.  When this was
//   changed: 307 -> 88 at the 32K case, 91 -> 73 at the 256-wide heads.
//   64 rows per workgroup where there are as many: the 32K case takes 68.6 with 64, 74.5 with 32 and 103.9 with 16, in 16 bits 66.9, 87.3 and 135.5, each with its best number of splits; where
//   there are but 16 (32K tokens, 16 bits, 4 drafted), 16 take 27.8, 32 28.9 and 64 33.1.  Which, and how many splits: cut_tree.  With 32-bit results of bf16 three instances of 64 rows spill
//   (D = 128; 8-bit rows most: 48 registers): 91 in the loop in which 16-bit results take 76.
//   Four wavefronts, merged by halves: what one gives another goes through LDS twice (half, then a quarter of the sums), and two workgroups share a compute unit: one
//   merges while the other reads.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "cache.hpp"
#include "launch.hpp"
#include "tree_cut.hpp"

namespace kvb {

struct TreeParams {
    CacheAddr c;
    const char *q;
    void *out;
    long long q_st, q_sh, o_st, o_sh;  // elements
    const int *seq_lens, *tok_first;
    const unsigned long long *mask;    // null: a chain
    float *part_acc, *part_ml;         // [n_tok * Hq, ns, D] and [n_tok * Hq, ns, 2]; not read where ns = 1
    float scale_log2e;                 // without its sign
    unsigned q_sign;                   // the scale's, for the two halves of a word of q
    int words, max_total, H, G, B, out_mode;  // out_mode: 0 fp32, 1 fp16, 2 bf16
    int ns, split_tokens, row_blocks;
    int bt_shift;                      // log2 of a block's tokens, or -1
    unsigned by_g, by_ns, by_h, by_row_blocks, by_split;  // 2^32 over G, ns, ..., rounded up (quotient)
    int ragged;                        // at most 64 sequences, of which some have fewer splits or row blocks than others
    int dense;                         // rows of a head lie side by side
    int grouped;                       // rows of context are looked up by groups of 16
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <bool BF16>
__device__ __forceinline__ f32x4 mfma32(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Maximum over the four row groups of lanes (n, n + 16, n + 32, n + 48), in every one of them.
__device__ __forceinline__ float groups_max(float x)
{
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

// mode: 0 fp32, 1 fp16, 2 bf16
__device__ __forceinline__ void store_one(void *out, long long i, int mode, float r)
{
    if (mode == 0) ((float *)out)[i] = r;
    else if (mode == 1) ((_Float16 *)out)[i] = (_Float16)r;
    else ((unsigned short *)out)[i] = bf16_bits(r);
}
__device__ __forceinline__ void store_four(void *out, long long i, int mode, f32x4 r)
{
    if (mode == 0 && !(((uintptr_t)out | (uintptr_t)(4 * i)) & 15)) {
        *(f32x4 *)((float *)out + i) = r;
    } else if (mode != 0 && !(((uintptr_t)out | (uintptr_t)(2 * i)) & 7)) {
        *(u32x2 *)((unsigned short *)out + i) = mode == 1 ? u32x2{pack2<false>(r[0], r[1]), pack2<false>(r[2], r[3])}
                                                          : u32x2{pack2<true>(r[0], r[1]), pack2<true>(r[2], r[3])};
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) store_one(out, i + k, mode, r[k]);
    }
}

// C columns side by side; at column 8 of 16, those of rows of 512 bytes go on 128 columns further
template <int C>
__device__ __forceinline__ void store_columns(void *out, long long i, int mode, const float (&x)[C])
{
    if constexpr (C >= 4) {
#pragma unroll
        for (int c = 0; c < C; c += 4) store_four(out, i + c, mode, f32x4{x[c], x[c + 1], x[c + 2], x[c + 3]});
    } else if constexpr (C == 2) {
        if (mode == 0 && !(((uintptr_t)out | (uintptr_t)(4 * i)) & 7)) *(f32x2 *)((float *)out + i) = f32x2{x[0], x[1]};
        else if (mode != 0 && !(((uintptr_t)out | (uintptr_t)(2 * i)) & 3)) *(unsigned *)((unsigned short *)out + i) = mode == 1 ? pack2<false>(x[0], x[1]) : pack2<true>(x[0], x[1]);
        else store_one(out, i, mode, x[0]), store_one(out, i + 1, mode, x[1]);
    } else {
        store_one(out, i, mode, x[0]);
    }
}

constexpr float kNoScore = -3.402823466e38f;   // reference of a row that has seen no score: no number is less
// A reference follows the running maximum when a probability passes 2^4 of it.
constexpr float kLargeRef = 1048576.f;  // beyond it the rounding of a reference would leave the range of the probabilities
// fp16 probabilities are taken of 2^11 times themselves (at most 2^15): what is lost lies below 2^-36 of the largest
template <bool BF16> constexpr float kLiftLog2 = BF16 ? 0.f : 11.f;
template <bool BF16> constexpr float kMostProbability = BF16 ? 16.f : 32768.f;   // 2^(4 + kLiftLog2)
// Probabilities as 16-bit operands: parts whose sum is the 32-bit value up to 2^-22 (fp16, two parts) or 2^-16 (bf16, two), or that value (bf16, three).  Two in bf16 go with
// bf16 results, whose own rounding, to 2^-8, is 256 times as coarse.  One part, rounded, would make the error of a 16-bit result 1.4 times that of its own rounding, for 56.2 instead of 67.3 us
// with 64 drafted tokens over 32K x 8 heads x 128 in 8 bits, 48.2 instead of 49.9 in a ragged batch of 8, 49.5 either way where HBM is the limit.
template <bool BF16, bool F32> constexpr int kParts = BF16 && F32 ? 3 : 2;

template <bool BF16, int N>
__device__ __forceinline__ void split_pair(float x, float y, unsigned (&out)[N])
{
    if constexpr (BF16) {
#pragma unroll
        for (int t = 0; t + 1 < N; ++t) {   // cut off, which takes one instruction for two
            const unsigned a = __float_as_uint(x), b = __float_as_uint(y);
            out[t] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            x -= __uint_as_float(a & 0xffff0000u);
            y -= __uint_as_float(b & 0xffff0000u);
        }
        out[N - 1] = pack2<BF16>(x, y);
    } else {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            out[t] = pack2<BF16>(x, y);
            if (t + 1 < N) {
                const f32x2 r = unpack2<BF16>(out[t]);
                x -= r[0];
                y -= r[1];
            }
        }
    }
}

constexpr int kTreeThreads = 256;

// The tile of a wavefront's step: 32 tokens, whose K and V pass through LDS as they lie in the cache.
template <int D, int FORMAT, int NB>
struct TreeTile {
    static constexpr int kBits = format_bits(FORMAT);
    static constexpr bool kBlocks = FORMAT != KV_FORMAT_16;
    static constexpr int kColumns = D / 16;           // columns of V that a lane works on
    static constexpr int kSteps = D / 32;             // products of 16 tokens' q K^T
    static constexpr int kRows = 16 * NB;             // query rows of a workgroup
    static constexpr bool kQStays = NB * D > 256;     // q is read from LDS at each step: more rows than their registers are worth
    static constexpr int kRow = D * kBits / 8;        // bytes of a token's row
    static constexpr int kPieces = kRow / 16;         // a row's pieces of 16 bytes: a lane's share of a load
    static constexpr int kTokens = 64 / kPieces;      // rows of a load (1 KiB)
    static constexpr int kLoads = 32 / kTokens;       // loads of a step's K, and as many of V
    static constexpr int kKPiece = kRow >= 64 ? 16 : 8;   // bytes of K that a lane reads from LDS at a time
    static constexpr int kKReads = kRow / 4 / kKPiece;
    static constexpr int kKElems = kKPiece * 8 / kBits;
    static constexpr int kVBytes = kColumns * kBits / 8;  // bytes of a token's row that a lane works on
    static constexpr int kKBytes = 32 * kRow;         // of a stage, and as many of V
    static constexpr int kZRow = D / kBlockElems;
    static constexpr int kZBytes = !kBlocks ? 0 : D == 256 ? 512 : 256;   // 32 rows' scales of K, then of V, each 4 (8) bytes apart
    static constexpr int kZLoads = !kBlocks ? 0 : D == 256 ? 2 : 1;
    static constexpr int kWaves = 4;                  // two workgroups and more on a compute unit: one merges while another reads
    static constexpr int kStage = 2 * kKBytes + kZBytes;
    static constexpr int kQBytes = NB * kSteps * 1024;
    static constexpr int kHalfLds = 80 * 1024;
    // Steps on their way while one is worked on: up to 16 KiB of a wavefront, as long as two workgroups fit a compute unit's LDS.  A wavefront's reads have some 2 us of
    // latency to cover.
    static constexpr int kStages = kWaves * 4 * kStage + kQBytes <= kHalfLds && kStage <= 4096 ? 4 : kWaves * 2 * kStage + kQBytes <= kHalfLds ? 2 : 1;
    static constexpr int kRing = kWaves * kStages * kStage;
    static constexpr int kMerge = kWaves * NB * kColumns / 2 * 1024, kStates = (2 * kWaves * kRows + kWaves) * 4;   // bytes
    static constexpr int kLds = kRing + kQBytes > kMerge + kStates ? kRing + kQBytes : kMerge + kStates;
    static_assert(kLds <= (D == 256 ? 2 : 1) * kHalfLds, "LDS of a compute unit");
    static constexpr int kQIssues = (NB * kSteps + kWaves - 1) / kWaves;

    // The first of the eight elements of d that a lane contributes to product s: any order will do that q follows as well.
    static __device__ __forceinline__ int q_at(int s, int group)
    {
        constexpr int per = kKElems / 8;  // products of a read
        return (s / per) * 4 * kKElems + group * kKElems + (s % per) * 8;
    }
    // K's pieces are exchanged within a row by a number of the token's, so that the 16 rows of which a read takes one piece lie in different banks.
    static __device__ __forceinline__ int k_turn(int token)
    {
        return kPieces >= 16 ? token & 15 : kPieces == 8 ? token >> 1 & 7 : kPieces == 4 ? token >> 2 & 3 : 0;
    }
    // Column of V (of d) behind row m of the product's result and the lane's column c: rows of 512 bytes are read in two halves.
    static __device__ __forceinline__ int v_column(int m, int c) { return kVBytes == 32 ? (c / 8) * 128 + 8 * m + c % 8 : kColumns * m + c; }
};

// 16 (4, 2) bytes per lane from memory to LDS, behind the wavefront's back: lane l's arrive at lds + 16 l (4 l).  Only counted waits (wait_loads) say when.
template <int BYTES, bool NT>
__device__ __forceinline__ void load_to_lds(const char *from, unsigned lds)
{
    if constexpr (BYTES == 16 && NT) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(from), "s"(lds) : "memory");
    else if constexpr (BYTES == 16) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(lds) : "memory");
    else if constexpr (BYTES == 4) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(lds) : "memory");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ushort %0, off" ::"v"(from), "s"(lds) : "memory");
}
// The same from a start that all lanes share and a lane's 32-bit offset.
template <bool NT>
__device__ __forceinline__ void load_to_lds16(unsigned long long start, unsigned offset, unsigned lds)
{
    // in scalar registers, wherever the compiler has it
    start = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)start) | (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(start >> 32)) << 32;
    if constexpr (NT) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(start), "s"(lds) : "memory");
    else asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(start), "s"(lds) : "memory");
}
// N of them (1, 2 or 4) with both ends a kilobyte further each; the q-th's lane offset is offset ^ (q * TURN & MASK).
template <bool NT, int N, int TURN, int MASK>
__device__ __forceinline__ void load_run(unsigned long long start, unsigned offset, unsigned lds)
{
    start = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)start) | (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(start >> 32)) << 32;
    const unsigned o1 = offset ^ (TURN & MASK), o2 = offset ^ (2 * TURN & MASK), o3 = offset ^ (3 * TURN & MASK);
#define KV_LOAD(O, OFFSET, HINT) "\n\tglobal_load_lds_dwordx4 " O ", %0 offset:" OFFSET HINT
#define KV_RUN(HINT)                                                                                                                                          \
    if constexpr (N == 1) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0" KV_LOAD("%2", "0", HINT)::"s"(start), "s"(lds), "v"(offset) : "memory");                   \
    else if constexpr (N == 2) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0" KV_LOAD("%2", "0", HINT) KV_LOAD("%3", "1024", HINT)::"s"(start), "s"(lds), "v"(offset), "v"(o1) : "memory"); \
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0" KV_LOAD("%2", "0", HINT) KV_LOAD("%3", "1024", HINT) KV_LOAD("%4", "2048", HINT) KV_LOAD("%5", "3072", HINT) \
                      ::"s"(start), "s"(lds), "v"(offset), "v"(o1), "v"(o2), "v"(o3) : "memory");
    if constexpr (NT) { KV_RUN(" nt") }
    else { KV_RUN("") }
#undef KV_RUN
#undef KV_LOAD
}
// x as if it was new here: what follows from it is computed where it is used, and not kept in registers that the loop has none of.
__device__ __forceinline__ int here(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
template <int N>
__device__ __forceinline__ void wait_loads()   // all but the last N
{
    static_assert(N < 64, "vmcnt");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// What was read from LDS has arrived: its place may be loaded into again.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Byte offsets of a token row of one sequence and head (the same for K and V), and of its scales.
struct RowAt {
    unsigned long long at, z;
    bool there;
};
__device__ __forceinline__ RowAt row_at(const CacheAddr &c, const int *table, unsigned long long base, unsigned long long zbase, int j)
{
    if (!c.table) return RowAt{base + j * c.ss, zbase + j * c.zs, true};
    const int i = j / c.bt, id = table[i], r = j - i * c.bt;
    const bool there = (unsigned)id < (unsigned)c.n_pool;
    const unsigned long long at = there ? id : 0;
    return RowAt{base + at * c.sb + r * c.ss, zbase + at * c.zb + r * c.zs, there};
}

// x / d by 2^32 / d, rounded up: the product may be one too large.
__device__ __forceinline__ unsigned quotient(unsigned x, unsigned d, unsigned by_d)
{
    if (d == 1) return x;
    const unsigned q = __umulhi(x, by_d);
    return q * d > x ? q - 1 : q;
}

// The drafted token of row r of a KV head's query rows: at most 256 G, so the product is never too large.
__device__ __forceinline__ int token_of(const TreeParams &p, int r) { return p.G == 1 ? r : (int)__umulhi((unsigned)r, p.by_g); }

// The kernel's arguments, loaded where they are needed: what is only used now and then, or after the loop, takes no scalar registers in it (there are too few: the
// others would be kept in lanes of a vector register and fetched from there at each step: when this was changed, 4 sequences of 8K x 16 heads x 256 of 8 bits went from 51.8 to 49.0 us).
__device__ __forceinline__ TreeParams arguments()
{
#if __HIP_DEVICE_COMPILE__
    typedef const __attribute__((address_space(4))) TreeParams *Args;
    unsigned long long at = (unsigned long long)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(Args)at;
#else
    return TreeParams{};   // the host's pass over this file knows no such address
#endif
}

// A value that all lanes load, through the scalar cache: nothing writes it while the kernel runs.
__device__ __forceinline__ int load_uniform(const int *at) { return *(const __attribute__((address_space(4))) int *)(unsigned long long)at; }

// Does row r of a KV head's query rows see token j of its sequence?
__device__ __forceinline__ bool row_sees(const TreeParams &p, int first, int r, int j, int len, int total)
{
    if (j < len) return true;
    if (j >= total || r >= (total - len) * p.G) return false;
    const int t = token_of(p, r), i = j - len;
    if (!p.mask) return i <= t;
    return (bool)(p.mask[(long long)(first + t) * p.words + (i >> 6)] >> (i & 63) & 1);
}

// The same of 32 tokens from j on, as bits.
__device__ __forceinline__ unsigned row_sees32(const TreeParams &p, int first, int r, int j, int len, int total)
{
    auto below = [](int x) { return x >= 32 ? ~0u : (1u << max(x, 0)) - 1u; };
    const unsigned context = below(len - j), drafted = below(total - j) & ~context;
    if (drafted == 0 || r >= (total - len) * p.G) return context;
    const int t = token_of(p, r), i = j - len;   // i > -32: a token's bit is i + its place
    unsigned long long bits;
    if (!p.mask) {
        bits = below(t + 1 - i);
    } else {
        const unsigned long long *const row = p.mask + (long long)(first + t) * p.words;
        const int w = max(i, 0) >> 6, shift = max(i, 0) & 63;
        bits = row[w] >> shift;
        if (shift > 32 && w + 1 < p.words) bits |= row[w + 1] << (64 - shift);
        if (i < 0) bits <<= -i;
    }
    return context | (drafted & (unsigned)bits);
}

// Four columns of a query row's sums: the result, or the partial result of a split.
template <int D>
__device__ __forceinline__ void store_sums(const TreeParams &p, unsigned h, int first, int r, unsigned split, int d, f32x4 x, float ref, float l)
{
    const int t = token_of(p, r), hq = (int)h * p.G + r - t * p.G;
    if (p.ns == 1) {
        store_four(p.out, (first + t) * p.o_st + hq * p.o_sh + d, p.out_mode, x * (l == 0.f ? 0.f : 1.f / l));
    } else {
        const long long at = ((long long)(first + t) * (p.H * p.G) + hq) * p.ns + split;
        *(f32x4 *)&p.part_acc[at * D + d] = x;
        if (d == 0) *(f32x2 *)&p.part_ml[at * 2] = f32x2{ref, l};
    }
}

// One query row over a split on the vector ALU, a token at a time: its largest score, then its sums.  Whatever the cache holds, nothing but what the row sees
// enters them.  A lane has four columns (of which several lanes may have the same).
template <int D, bool BF16, int FORMAT>
__device__ __forceinline__ void plain_row(const TreeParams &p, const int *table, unsigned long long base, unsigned long long zbase, unsigned h, int first, int r,
                                       int len, int total, int s0, int s1, unsigned split, int lane)
{
    const int t = token_of(p, r), hq = (int)h * p.G + r - t * p.G, at = lane % (D / 4);
    const u32x2 qw = *(const u32x2 *)(p.q + 2 * ((first + t) * p.q_st + hq * p.q_sh + 4 * at));
    const f32x2 q0 = unpack2<BF16>(qw[0] ^ p.q_sign), q1 = unpack2<BF16>(qw[1] ^ p.q_sign);
    auto row = [&](const char *rows, const char *scales, int j, bool *there) {
        const RowAt x = row_at(p.c, table, base, zbase, j);
        *there = x.there;
        u32x2 w;
        if constexpr (FORMAT == KV_FORMAT_16) {
            w = *(const u32x2 *)(rows + x.at + 8 * at);
        } else {
            const float z = scale_operand((unsigned char)scales[x.z + at / 8]);
            unsigned codes;
            if constexpr (FORMAT == KV_FORMAT_FP8) codes = *(const unsigned *)(rows + x.at + 4 * at);
            else codes = *(const unsigned short *)(rows + x.at + 2 * at);
            w = u32x2{decode2<BF16, FORMAT, 0>(codes, z), decode2<BF16, FORMAT, 1>(codes, z)};
        }
        const f32x2 a = unpack2<BF16>(w[0]), b = unpack2<BF16>(w[1]);
        return f32x4{a[0], a[1], b[0], b[1]};
    };
    auto score = [&](int j) {
        bool there;
        const f32x4 k = row(p.c.k, p.c.kz, j, &there);
        float s = fmaf(q0[0], k[0], fmaf(q0[1], k[1], fmaf(q1[0], k[2], q1[1] * k[3])));
#pragma unroll
        for (int o = 1; o < D / 4; o *= 2) s += __shfl_xor(s, o);
        return there ? s * p.scale_log2e : -INFINITY;
    };
    float top = -INFINITY, l = 0.f;
    for (int j = s0; j < s1; ++j)
        if (row_sees(p, first, r, j, len, total)) top = fmaxf(top, score(j));
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int j = s0; j < s1; ++j) {
        if (!row_sees(p, first, r, j, len, total)) continue;
        const float s = score(j);
        if (s == -INFINITY) continue;
        const float w = __builtin_amdgcn_exp2f(s - top);
        bool there;
        const f32x4 v = row(p.c.v, p.c.vz, j, &there);
        l += w;
#pragma unroll
        for (int k = 0; k < 4; ++k)   // a probability too small for 32 bits still counts against an infinity
            x[k] = fmaf(w == 0.f && !__builtin_isfinite(v[k]) ? 1.0e-37f : w, v[k], x[k]);
    }
    if (lane < D / 4) store_sums<D>(p, h, first, r, split, 4 * at, x, top == -INFINITY ? kNoScore : top, l);
}

template <int D, bool BF16, int FORMAT, int NB, bool F32>
__global__ void __launch_bounds__((64 * TreeTile<D, FORMAT, NB>::kWaves), (TreeTile<D, FORMAT, NB>::kLds <= TreeTile<D, FORMAT, NB>::kHalfLds ? 2 : 1)) kv_tree_partial_kernel(TreeParams p)
{
    using T = TreeTile<D, FORMAT, NB>;
    constexpr int kRows = T::kRows, kColumns = T::kColumns, kSteps = T::kSteps, kP = kParts<BF16, F32>, kWaves = T::kWaves, kStages = T::kStages;
    constexpr bool kNT = NB <= 2;   // with more rows other workgroups may read the same K and V out of L2

    // The arguments' cache lines at once, not each where the first of its values is needed.
    asm volatile("" ::"s"(p.c.k), "s"(p.c.kz), "s"(p.q), "s"(p.part_acc), "s"(p.scale_log2e), "s"(p.by_split));

    // Which sequence, KV head, split and row block.  Workgroups go round the eight XCDs; the row blocks of a split are a multiple of eight apart: they run at about the same
    // time on one XCD and share its L2.
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned b, h, split, rb = 0;
    int first, drafted, len;
    if (p.ragged) {
        // Only what there is, sequence after sequence (a lane each): workgroups that have nothing to do would take places from others, which then share a compute unit
        // while the next one is idle.
        int f = 0, n = 0, l = 0;
        unsigned units = 0;   // splits of heads, in eights where there may be row blocks
        if (lane < p.B) {
            f = p.tok_first[lane];
            n = min(p.tok_first[lane + 1] - f, KV_TREE_MAX);
            l = max(0, min(p.seq_lens[lane], p.max_total - n));
            units = n <= 0 ? 0 : (quotient((unsigned)(l + n - 1), (unsigned)p.split_tokens, p.by_split) + 1) * (unsigned)p.H;
            if (p.row_blocks > 1) units = (units + 7) & ~7u;
        }
        const unsigned all = units * ((unsigned)(n * p.G + kRows - 1) / kRows);
        unsigned end = all;   // of the sequence's workgroups
        end += (unsigned)__builtin_amdgcn_update_dpp(0, (int)end, 0x111, 0xf, 0xf, true);   // sums over the lanes below: 1, 2, 4, 8 of a row of 16, then over rows
        end += (unsigned)__builtin_amdgcn_update_dpp(0, (int)end, 0x112, 0xf, 0xf, true);
        end += (unsigned)__builtin_amdgcn_update_dpp(0, (int)end, 0x114, 0xf, 0xf, true);
        end += (unsigned)__builtin_amdgcn_update_dpp(0, (int)end, 0x118, 0xf, 0xf, true);
        end += (unsigned)__builtin_amdgcn_update_dpp(0, (int)end, 0x142, 0xa, 0xf, false);
        end += (unsigned)__builtin_amdgcn_update_dpp(0, (int)end, 0x143, 0xc, 0xf, false);
        b = (unsigned)__popcll(__ballot(end <= blockIdx.x));
        if (b >= (unsigned)p.B) return;
        first = __builtin_amdgcn_readlane(f, (int)b);
        drafted = __builtin_amdgcn_readlane(n, (int)b);
        len = __builtin_amdgcn_readlane(l, (int)b);
        units = (unsigned)__builtin_amdgcn_readlane((int)units, (int)b);
        unsigned unit = blockIdx.x - (unsigned)__builtin_amdgcn_readlane((int)(end - all), (int)b);
        if (unit >= units) {
            rb = unit / units;
            unit -= rb * units;
        }
        split = quotient(unit, (unsigned)p.H, p.by_h);
        h = unit - split * (unsigned)p.H;
    } else {
        unsigned unit = blockIdx.x;
        if (p.row_blocks > 1) {
            const unsigned turn = blockIdx.x / 8, eights = quotient(turn, (unsigned)p.row_blocks, p.by_row_blocks);
            rb = turn - eights * (unsigned)p.row_blocks;
            unit = eights * 8 + blockIdx.x % 8;
        }
        const unsigned bh = quotient(unit, (unsigned)p.ns, p.by_ns);
        split = unit - bh * (unsigned)p.ns;
        b = quotient(bh, (unsigned)p.H, p.by_h);
        h = bh - b * (unsigned)p.H;
        if (b >= (unsigned)p.B) return;
        const int next = load_uniform(p.tok_first + b + 1), l = load_uniform(p.seq_lens + b);
        first = load_uniform(p.tok_first + b);
        __builtin_amdgcn_sched_barrier(0);   // one wait for all three
        drafted = min(next - first, KV_TREE_MAX);
        len = max(0, min(l, p.max_total - drafted));
    }
    const int n_rows = drafted * p.G - (int)rb * kRows;   // of this block: the first kRows of them
    if (n_rows <= 0) return;
    const int total = len + drafted;
    if (!split_has_tokens(split, p.split_tokens, total)) return;
    const int s0 = (int)split * p.split_tokens, s1 = min(s0 + p.split_tokens, total);

    const int n = lane & 15, group = lane >> 4;
    const unsigned long long base = p.c.table ? h * p.c.sh : b * p.c.sb + h * p.c.sh;
    const unsigned long long zbase = p.c.table ? h * p.c.zh : b * p.c.zb + h * p.c.zh;
    const int *const table = p.c.table ? p.c.table + (long long)b * p.c.max_blocks : nullptr;

    // The ring of each wavefront's stages, then q; after the last step the merge's rows and states.
    __shared__ __attribute__((aligned(1024))) char lds[T::kLds];
    const unsigned ring_at = (unsigned)wave * (kStages * T::kStage);
    const unsigned lds_at = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char *)lds + ring_at;
    const char *const ring = lds + ring_at;

    const int n_steps = (s1 - s0 + 31) / 32;
    const int mine = (n_steps - wave + kWaves - 1) / kWaves;   // steps of this wavefront: wave, wave + kWaves, ...

    // Where a step's rows are.  16 rows lie stride by stride from a start that all lanes share, in a block pool from an id that some lane holds; blocks of other
    // sizes and rows far apart are looked up one by one.  A row past the end is the last one; what has no place in the cache is block 0 of the pool; neither is seen.
    unsigned long long at0 = 0, at1 = 0, z0 = 0, z1 = 0;   // starts
    unsigned long long lane_at = 0, lane_z = 0;            // where not all rows exist, or they are looked up: the row of token lane % 32
    unsigned next_there = ~0u;                             // a bit for each token that the cache has
    unsigned long long ids_at = 0, ids_z = 0, ids_there = 0;   // block pool, lane l: start of half l % 2 of the wavefront's step l / 2 (of 32 steps); whether it has one, by lanes
    bool groups = false;
    auto where = [&](int m) {   // this wavefront's m-th step; called for each in turn
        const int j0 = s0 + 32 * (wave + m * kWaves), left = total - 1 - j0;
        groups = p.grouped && left >= 31;
        next_there = ~0u;
        if (!p.grouped) {
            const CacheAddr c = arguments().c;
            const RowAt r = row_at(c, table, base, zbase, j0 + min(lane & 31, left));
            lane_at = r.at;
            lane_z = r.z;
            next_there = (unsigned)__ballot(r.there);
            return;
        }
        if (!p.c.table) {
            // from one step to the next a sum, not a product
            at0 = m == 0 ? base + (unsigned)j0 * p.c.ss : at0 + 32 * kWaves * (unsigned)p.c.ss;
            at1 = at0 + 16 * (unsigned)p.c.ss;
            if (T::kBlocks) {
                z0 = m == 0 ? zbase + (unsigned)j0 * p.c.zs : z0 + 32 * kWaves * (unsigned)p.c.zs;
                z1 = z0 + 16 * (unsigned)p.c.zs;
            }
        } else {
            if (m % 32 == 0) {   // the starts of 32 steps at a time, a lane each
                const TreeParams p = arguments();
                const int j = min(j0 + 32 * kWaves * (lane >> 1) + 16 * (lane & 1), total - 1) & ~15, at = p.bt_shift >= 0 ? j >> p.bt_shift : j / p.c.bt;
                unsigned id = (unsigned)table[at];
                const unsigned in = j - at * p.c.bt;
                ids_there = __ballot(id < (unsigned)p.c.n_pool);
                id = id < (unsigned)p.c.n_pool ? id : 0;
                ids_at = base + (unsigned long long)id * (unsigned)p.c.sb + in * (unsigned)p.c.ss;
                if (T::kBlocks) ids_z = zbase + (unsigned long long)id * (unsigned)p.c.zb + in * (unsigned)p.c.zs;
            }
            const int l = 2 * (m % 32);
            auto of_lane = [](unsigned long long x, int k) {
                return (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)x, k) |
                       (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(x >> 32), k) << 32;
            };
            at0 = of_lane(ids_at, l);
            at1 = of_lane(ids_at, l + 1);
            if (T::kBlocks) {
                z0 = of_lane(ids_z, l);
                z1 = of_lane(ids_z, l + 1);
            }
            const unsigned both = (unsigned)(ids_there >> l) & 3;
            next_there = both == 3 ? ~0u : both == 2 ? 0xffff0000u : both == 1 ? 0xffffu : 0;
        }
        if (!groups) {
            const int t = min(lane & 31, left);
            lane_at = (t & 16 ? at1 : at0) + (unsigned)(t & 15) * (unsigned)p.c.ss;
            lane_z = (t & 16 ? z1 : z0) + (unsigned)(t & 15) * (unsigned)p.c.zs;
        }
    };
    auto from_lane = [](unsigned long long x, int l) {
        return (unsigned long long)(unsigned)__shfl((int)(unsigned)x, l) | (unsigned long long)(unsigned)__shfl((int)(unsigned)(x >> 32), l) << 32;
    };
    // Loads of a step's K (is_v = false) or V into a stage.
    auto issue_rows = [&](unsigned stage, auto is_v) {
        constexpr bool V = decltype(is_v)::value;
        const char *const rows = V ? p.c.v : p.c.k;
        const unsigned to = lds_at + stage * T::kStage + (V ? T::kKBytes : 0);
        const int l = here(lane), piece = l % T::kPieces, slot = l / T::kPieces;   // of a load
        if (groups && p.dense && T::kTokens <= 16) {
            // rows side by side: what a load brings of a row is where the lane is, and both ends of the loads of 16 rows are a kilobyte apart
            constexpr int kHalf = T::kRow / 64, kRun = kHalf < 4 ? kHalf : 4;   // loads of 16 rows, and of them with one start
            constexpr int kTurn = V ? 0 : T::kPieces >= 16 ? 16 * T::kTokens : T::kPieces == 8 ? 64 : 0, kMask = 16 * (T::kPieces < 16 ? T::kPieces : 16) - 1;
            const unsigned from = 16 * (V ? l : l ^ T::k_turn(slot));
#pragma unroll
            for (int q = 0; q < 2 * kHalf; q += kRun)
                load_run<kNT, kRun, kTurn, kMask>((unsigned long long)rows + (q < kHalf ? at0 : at1) + q % kHalf * 1024, from ^ (q % kHalf * kTurn & kMask), to + q * 1024);
        } else if (groups) {
            const unsigned lane_row = (unsigned)slot * (unsigned)p.c.ss;
#pragma unroll
            for (int q = 0; q < T::kLoads; ++q) {
                const int token = q * T::kTokens + slot;
                const unsigned from = 16 * (V ? piece : piece ^ T::k_turn(token));
                if constexpr (T::kTokens <= 16) {
                    const unsigned long long start = (q * T::kTokens < 16 ? at0 : at1) + (q * T::kTokens & 15) * (unsigned)p.c.ss;
                    load_to_lds16<kNT>((unsigned long long)rows + start, lane_row + from, to + q * 1024);
                } else {   // both groups in one
                    load_to_lds<16, kNT>(rows + (slot & 16 ? at1 : at0) + ((slot & 15) * (unsigned)p.c.ss + from), to + q * 1024);
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < T::kLoads; ++q) {
                const int token = q * T::kTokens + slot;
                const int from = 16 * (V ? piece : piece ^ T::k_turn(token));
                load_to_lds<16, kNT>(rows + from_lane(lane_at, token) + from, to + q * 1024);
            }
        }
    };
    auto issue_scales = [&](unsigned stage) {
        if constexpr (T::kBlocks) {
            const unsigned to = lds_at + stage * T::kStage + 2 * T::kKBytes;
            const int l = here(lane);
#pragma unroll
            for (int q = 0; q < T::kZLoads; ++q) {
                const int token = D == 256 ? l >> 1 : l & 31, half = D == 256 ? (l & 1) * 4 : 0;
                const char *const scales = (D == 256 ? q : l >> 5) ? p.c.vz : p.c.kz;
                unsigned long long z;
                if (groups) z = (token & 16 ? z1 : z0) + (unsigned)(token & 15) * (unsigned)p.c.zs;
                else z = from_lane(lane_z, token);
                load_to_lds<D == 64 ? 2 : 4, false>(scales + z + half, to + 256 * q);
            }
        }
    };

    // Query rows: token-major, the G heads of a token side by side.  Those past the last one are copies of it, whose results go nowhere.  They go to LDS ahead of the steps'
    // K and V: loaded into registers behind these, they were there only when all of these were (when this was changed: 4K tokens, 16 drafted 15.0 -> 14.3 us; 48 single tokens 22.7 -> 21.6).
    auto row_token = [&](int r) { return token_of(p, (int)rb * kRows + r); };
    const u32x4 *const q_lds = (const u32x4 *)(lds + T::kRing);
    auto issue_q = [&] {   // a wavefront's share of them to LDS
        const unsigned to = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char *)lds + T::kRing;
#pragma unroll
        for (int k = 0; k < T::kQIssues; ++k) {
            const int i = wave + k * kWaves, nb = i / kSteps, s = i % kSteps;
            const int r = min(nb * 16 + n, n_rows - 1), t = row_token(r), g = (int)rb * kRows + r - t * p.G;
            if (i < NB * kSteps) load_to_lds<16, false>(p.q + 2 * ((first + t) * p.q_st + ((int)h * p.G + g) * p.q_sh + T::q_at(s, group)), to + i * 1024);
        }
    };
    u32x4 q_reg[T::kQStays ? 1 : NB][kSteps];
    f32x4 acc[NB][kColumns], sum[NB];
    float ref[NB];
    const u32x4 ones = BF16 ? u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u} : u32x4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};

    // Scores of 32 tokens: lane (n, group) gets those of tokens group, group + 4, ..., from each half four; rows n of K's operand are tokens n / 4 + 4 * (n % 4) (+ 16).
    struct KRead {
        u32x4 w[T::kKReads][2];
        unsigned z[T::kBlocks ? T::kKReads : 1][2];
    };
    constexpr int kHalves = T::kVBytes == 32 ? 2 : 1, kPairs = kColumns / 2 / kHalves, kBytes = T::kVBytes / kHalves;
    struct VRead {
        unsigned w[kHalves][8][kBytes < 4 ? 1 : kBytes / 4];
        unsigned z[T::kBlocks ? 8 : 1];
    };
    auto read_k = [&](const char *stage, KRead &x) {
        const char *const k = stage, *const z = stage + 2 * T::kKBytes;
#pragma unroll
        for (int r = 0; r < T::kKReads; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int token = (n >> 2) + 4 * (n & 3) + 16 * i;
                if constexpr (T::kKPiece == 16) {
                    x.w[r][i] = *(const u32x4 *)(k + token * T::kRow + 16 * ((4 * r + group) ^ T::k_turn(token)));
                } else {
                    const u32x2 v = *(const u32x2 *)(k + token * T::kRow + 8 * group);
                    x.w[r][i] = u32x4{v[0], v[1], 0, 0};
                }
                if constexpr (T::kBlocks) x.z[r][i] = (unsigned char)z[token * (D == 256 ? 8 : 4) + (4 * r + group) * T::kKElems / kBlockElems];
            }
    };
    auto read_v = [&](const char *stage, VRead &x) {
        const char *const v = stage + T::kKBytes, *const z = stage + 2 * T::kKBytes + (D == 256 ? 256 : 128);
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const char *const at = v + (group + 4 * j) * T::kRow + kBytes * n + half * 256;
                unsigned *const w = x.w[half][j];
                if constexpr (kBytes == 2) {
                    w[0] = *(const unsigned short *)at;
                } else if constexpr (kBytes == 4) {
                    w[0] = *(const unsigned *)at;
                } else if constexpr (kBytes == 8) {
                    const u32x2 y = *(const u32x2 *)at;
                    w[0] = y[0];
                    w[1] = y[1];
                } else {
                    const u32x4 y = *(const u32x4 *)at;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = y[e];
                }
            }
        if constexpr (T::kBlocks) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x.z[j] = (unsigned char)z[(group + 4 * j) * (D == 256 ? 8 : 4) + kColumns * n / kBlockElems];
        }
    };
    auto scores = [&](const KRead &x, f32x4 (&s)[NB][2]) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int per = T::kKElems / 8;
#pragma unroll
        for (int r = 0; r < T::kKReads; ++r)
#pragma unroll
            for (int e = 0; e < per; ++e) {
                u32x4 q[NB];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if constexpr (T::kQStays) q[nb] = q_lds[(nb * kSteps + r * per + e) * 64 + lane];
                    else q[nb] = q_reg[nb][r * per + e];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    u32x4 a;
                    if constexpr (!T::kBlocks) a = x.w[r][i];
                    else if constexpr (FORMAT == KV_FORMAT_FP8) a = decode8<BF16, FORMAT>(u32x2{x.w[r][i][2 * e], x.w[r][i][2 * e + 1]}, scale_operand(x.z[r][i]));
                    else a = decode8<BF16, FORMAT>(u32x2{x.w[r][i][e], 0}, scale_operand(x.z[r][i]));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) s[nb][i] = mfma32<BF16>(a, q[nb], s[nb][i]);
                }
            }
    };
    auto product = [&](const VRead &x, const u32x4 (&pr)[NB][kP]) {
#pragma unroll
        for (int t = 0; t < kP; ++t)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) sum[nb] = mfma32<BF16>(ones, pr[nb][t], sum[nb]);
        float scale[8];
        if constexpr (T::kBlocks) {
#pragma unroll
            for (int j = 0; j < 8; ++j) scale[j] = scale_operand(x.z[j]);
        }
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
            for (int c = 0; c < kPairs; ++c) {
                unsigned y[8];   // two columns of the eight tokens
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const unsigned *const w = x.w[half][j];
                    if constexpr (!T::kBlocks) y[j] = w[c];
                    else if constexpr (FORMAT == KV_FORMAT_FP8) y[j] = c % 2 ? decode2<BF16, FORMAT, 1>(w[c / 2], scale[j]) : decode2<BF16, FORMAT, 0>(w[c / 2], scale[j]);
                    else y[j] = c % 4 == 0 ? decode2<BF16, FORMAT, 0>(w[c / 4], scale[j]) : c % 4 == 1 ? decode2<BF16, FORMAT, 1>(w[c / 4], scale[j])
                              : c % 4 == 2 ? decode2<BF16, FORMAT, 2>(w[c / 4], scale[j]) : decode2<BF16, FORMAT, 3>(w[c / 4], scale[j]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const unsigned sel = e ? 0x07060302u : 0x05040100u;
                    const u32x4 a = {__builtin_amdgcn_perm(y[1], y[0], sel), __builtin_amdgcn_perm(y[3], y[2], sel),
                                     __builtin_amdgcn_perm(y[5], y[4], sel), __builtin_amdgcn_perm(y[7], y[6], sel)};
#pragma unroll
                    for (int t = 0; t < kP; ++t)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            f32x4 &to = acc[nb][(half * kPairs + c) * 2 + e];
                            to = mfma32<BF16>(a, pr[nb][t], to);
                        }
                }
            }
    };
    auto rescale = [&](int nb, float f) {
        sum[nb] *= f;
#pragma unroll
        for (int c = 0; c < kColumns; ++c) acc[nb][c] *= f;
    };
    // Probabilities against a reference that follows the running maximum lazily: only where a probability came out above 2^4 are maxima formed over the lanes, sums
    // rescaled and the probabilities formed again: most steps have no exchange between lanes and leave the sums alone.  What is added up stays below 2^4 times the number of
    // tokens, far from where 32 bits end.
    // Their sum is that of their parts, so the weights add up to one.
    auto softmax = [&](f32x4 (&s)[NB][2], u32x4 (&pr)[NB][kP]) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float x[8];
            auto exponentials = [&] {
                const float sub = kLiftLog2<BF16> - ref[nb];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(fmaf(s[nb][j / 4][j % 4], p.scale_log2e, sub));
                return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            };
            if (__any(exponentials() > kMostProbability<BF16>)) {
                float top = s[nb][0][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, s[nb][j / 4][j % 4]);
                const float to = fmaxf(ref[nb], groups_max(top) * p.scale_log2e);
                rescale(nb, __builtin_amdgcn_exp2f(ref[nb] - to));
                ref[nb] = to;
                (void)exponentials();
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned w[kP];
                split_pair<BF16, kP>(x[2 * j], x[2 * j + 1], w);
#pragma unroll
                for (int t = 0; t < kP; ++t) pr[nb][t][j] = w[t];
            }
        }
    };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        ref[nb] = kNoScore;
        sum[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kColumns; ++c) acc[nb][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Steps.  Loads come back in order: all but those issued later are waited for.
    // Early: K and V of a step are read from LDS at once and its place loaded again before anything is computed; else V is read after the softmax.  Codes are few registers:
    // early and late, us, 4 x 8K x 16 x 256, 8 bits, 16 rows 49.2, 51.8; a ragged step of 32 rows, 8 bits 47.3, 48.1; 48 single tokens, 4 bits 21.4, 21.6; 32 x 500-2000 x 8 x 128 24.6, 25.8.
    // 16-bit rows, and more rows at 256 columns, leave too few for the sums: 16 x 4K, 16 bits, 32 rows 60.5, 59.0; 4 x 8K x 16 x 256, 8 bits, 32 rows 59.9, 58.2; 64 rows spill: 32K tokens,
    // 8 bits 107, 67.4; a ragged batch of 16 bits 61.4, 50.4.  (32K tokens, 16 bits, 16 rows: 29.8 both ways.)
    constexpr int kKIssues = T::kLoads + T::kZLoads, kVIssues = T::kLoads;
    constexpr bool kEarly = T::kBlocks && NB * D <= 256;
    // From 32 rows on a wavefront goes ahead of the other one of its SIMD in its products, whose operands wait for conversions and permutes between them: neither product, the second, both, us:
    // 32K tokens x 8 heads x 128, 64 drafted, in 8 bits 70.1, 68.5, 67.4; in 16 bits, where K needs no conversion, 70.9, 68.7, 72.2; 32 rows of a ragged 8-bit step 49.8, 48.6, 47.4.  With 16 rows it
    // is as often slower (32 x 500-2000 tokens 24.7 -> 25.3) as faster (48 single tokens 21.4 -> 20.9).
    constexpr bool kFirst = NB >= 2, kFirstK = kFirst && T::kBlocks;
    unsigned there[kStages], stage = 0;
    issue_q();
#pragma unroll
    for (int m = 0; m < kStages; ++m) {
        there[m] = ~0u;
        if (m >= mine) continue;
        where(m);
        issue_rows(m, std::false_type{});
        issue_scales(m);
        issue_rows(m, std::true_type{});
        there[m] = next_there;
    }
    // q is there once everybody's share is; the steps' loads go on
    if (mine >= kStages) wait_loads<kStages * (kKIssues + kVIssues)>();
    else wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // A negative scale turns q's signs here: references and masks are those of a positive one.
    if (const unsigned sign = arguments().q_sign; sign != 0) {
#pragma unroll
        for (int k = 0; k < T::kQIssues; ++k) {
            const int i = wave + k * kWaves;
            if (i < NB * kSteps) ((u32x4 *)(lds + T::kRing))[i * 64 + lane] ^= sign;
        }
        __syncthreads();
    }
    if constexpr (!T::kQStays) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) q_reg[nb][s] = q_lds[(nb * kSteps + s) * 64 + lane];
    }

#pragma unroll 1
    for (int m = 0; m < mine; ++m) {
        const bool more = m + kStages < mine;
        if (more) where(m + kStages);
        const char *const here_now = ring + stage * T::kStage;
        const int j0 = s0 + 32 * (wave + m * kWaves);
        f32x4 s[NB][2];
        VRead v;
        // The stage is read and loaded again at once where K and V both fit the registers beside the sums; else each as it is needed.
        if (m + kStages <= mine) wait_loads<kEarly ? (kStages - 1) * (kKIssues + kVIssues) : kVIssues + (kStages - 1) * (kKIssues + kVIssues)>();
        else wait_loads<0>();
        {
            KRead k;
            read_k(here_now, k);
            if constexpr (kEarly) read_v(here_now, v);
            if constexpr (kFirstK) __builtin_amdgcn_s_setprio(1);
            scores(k, s);
            if constexpr (kFirstK) __builtin_amdgcn_s_setprio(0);
        }
        if (j0 + 32 > len || there[0] != ~0u) {
            // Branch-free, for the compiler's sake too: with a condition for every token, inlined, it lost the masks of some instances.
            const TreeParams p = arguments();
            const int row = (int)rb * kRows + here(n);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const unsigned seen = (there[0] & row_sees32(p, first, row + nb * 16, j0, len, total)) >> group;
#pragma unroll
                for (int j = 0; j < 8; ++j) s[nb][j / 4][j % 4] = seen >> 4 * j & 1 ? s[nb][j / 4][j % 4] : -INFINITY;
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // a phase's registers at a time
        if (more) {
            wait_reads();
            issue_rows(stage, std::false_type{});
            if constexpr (kEarly) {
                issue_scales(stage);
                issue_rows(stage, std::true_type{});
            }
        }
        u32x4 pr[NB][kP];
        __builtin_amdgcn_sched_barrier(0);
        softmax(s, pr);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kEarly) {
            if (more) wait_loads<(kStages - 1) * (kKIssues + kVIssues) + T::kLoads>();
            else wait_loads<0>();
            read_v(here_now, v);
        }
        if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
        product(v, pr);
        if constexpr (kFirst) __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kEarly) {
            if (more) {
                wait_reads();
                issue_scales(stage);
                issue_rows(stage, std::true_type{});
            }
        }
#pragma unroll
        for (int k = 0; k + 1 < kStages; ++k) there[k] = there[k + 1];
        there[kStages - 1] = more ? next_there : ~0u;
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }

    // What is not finite may be none of a row's business (a probability of zero times it), and references may have grown too large:
    // then the workgroup does its split again, row by row.
    float finite[4] = {0.f, 0.f, 0.f, 0.f};   // zeros, or NaN
    bool bad = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        finite[0] = fmaf(sum[nb][0], 0.f, finite[0]);
#pragma unroll
        for (int c = 0; c < kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) finite[i] = fmaf(acc[nb][c][i], 0.f, finite[i]);
        bad = bad || (fabsf(ref[nb]) > kLargeRef && ref[nb] != kNoScore);
    }
    bad = bad || !((finite[0] + finite[1]) + (finite[2] + finite[3]) == 0.f);

    // Merge: the wavefronts' references and sums become factors of their accumulators; these are added by halves: a wavefront gives the one that is not in its keeping to
    // another and gets that one's half of what is, twice.  In the end each has a quarter of the sums of all four.
    const TreeParams a = arguments();
    static_assert(kWaves == 4 && NB * kColumns % 4 == 0, "halves of halves");
    constexpr int kTiles = NB * kColumns;
    f32x4 *const give = (f32x4 *)lds;                                                                // [kWaves][kTiles / 2][64]
    float *const ref_lds = (float *)(lds + T::kMerge), *const sum_lds = ref_lds + kWaves * kRows;   // [kWaves][kRows]
    float *const bad_lds = sum_lds + kWaves * kRows;                                                // [kWaves]
    __syncthreads();   // the rings are done with
    if (group == 0) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            ref_lds[wave * kRows + nb * 16 + n] = ref[nb];
            sum_lds[wave * kRows + nb * 16 + n] = sum[nb][0];
        }
    }
    const bool wave_bad = __any(bad);
    if (lane == 0) bad_lds[wave] = wave_bad ? 1.f : 0.f;
    __syncthreads();
    if ((bad_lds[0] + bad_lds[1]) + (bad_lds[2] + bad_lds[3]) != 0.f) {
        for (int r = wave; r < min(n_rows, kRows); r += kWaves)
            plain_row<D, BF16, FORMAT>(a, table, base, zbase, h, first, (int)rb * kRows + r, len, total, s0, s1, split, lane);
        return;
    }
    float to[NB], total_sum[NB];
    f32x4 tiles[kTiles];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float r[kWaves], l[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            r[w] = ref_lds[w * kRows + nb * 16 + n];
            l[w] = sum_lds[w * kRows + nb * 16 + n];
        }
        to[nb] = fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]));
        total_sum[nb] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total_sum[nb] += l[w] == 0.f ? 0.f : l[w] * __builtin_amdgcn_exp2f(r[w] - to[nb]);
        float f = sum[nb][0] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ref[nb] - to[nb]);
        if (a.ns == 1) f = total_sum[nb] == 0.f ? 0.f : f / total_sum[nb];
#pragma unroll
        for (int c = 0; c < kColumns; ++c) tiles[nb * kColumns + c] = acc[nb][c] * f;
    }
    const bool upper = wave & 2, odd = wave & 1;
    f32x4 half[kTiles / 2], mine_now[kTiles / 4];
#pragma unroll
    for (int t = 0; t < kTiles / 2; ++t) {
        half[t] = upper ? tiles[kTiles / 2 + t] : tiles[t];
        give[(wave * (kTiles / 2) + t) * 64 + lane] = upper ? tiles[t] : tiles[kTiles / 2 + t];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles / 2; ++t) half[t] += give[((wave ^ 2) * (kTiles / 2) + t) * 64 + lane];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles / 4; ++t) {
        mine_now[t] = odd ? half[kTiles / 4 + t] : half[t];
        give[(wave * (kTiles / 4) + t) * 64 + lane] = odd ? half[t] : half[kTiles / 4 + t];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles / 4; ++t) mine_now[t] += give[((wave ^ 1) * (kTiles / 4) + t) * 64 + lane];

    // The wavefront's quarter is a row group's columns from c0 on; of these a lane has those of rows 4 * group + i of the product.
    constexpr int kShare = kTiles / 4;
    static_assert(kColumns % kShare == 0, "of one row group");
    const int nb = kShare * wave / kColumns, c0 = kShare * wave % kColumns, r = nb * 16 + n;
    if (r >= n_rows) return;
    const int t = token_of(a, (int)rb * kRows + r), hq = (int)h * a.G + (int)rb * kRows + r - t * a.G;
    const long long part = ((long long)(first + t) * (a.H * a.G) + hq) * a.ns + split, at = a.ns == 1 ? (first + t) * a.o_st + hq * a.o_sh : part * D;
    if (a.ns > 1 && group == 0 && c0 == 0) {
        float ml[2] = {to[0], total_sum[0]};
#pragma unroll
        for (int k = 1; k < NB; ++k) {
            ml[0] = k == nb ? to[k] : ml[0];
            ml[1] = k == nb ? total_sum[k] : ml[1];
        }
        *(f32x2 *)&a.part_ml[part * 2] = f32x2{ml[0] - kLiftLog2<BF16>, ml[1]};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long o = at + T::v_column(4 * group + i, c0);
        float x[kShare];
#pragma unroll
        for (int c = 0; c < kShare; ++c) x[c] = mine_now[c][i];
        if (a.ns > 1) store_columns<kShare>(a.part_acc, o, 0, x);
        else store_columns<kShare>(a.out, o, a.out_mode, x);
    }
}

typedef void (*TreeKernel)(TreeParams);
template <int FORMAT, int D, int NB>
TreeKernel tree_kernel_of(bool bf16, bool f32)
{
    return !bf16 ? kv_tree_partial_kernel<D, false, FORMAT, NB, false> : f32 ? kv_tree_partial_kernel<D, true, FORMAT, NB, true> : kv_tree_partial_kernel<D, true, FORMAT, NB, false>;
}
template <int FORMAT>
TreeKernel tree_kernel_for(int D, bool bf16, bool f32, int nb)
{
    if (D == 256) return nb == 1 ? tree_kernel_of<FORMAT, 256, 1>(bf16, f32) : tree_kernel_of<FORMAT, 256, 2>(bf16, f32);
    if (D == 128)
        return nb == 1 ? tree_kernel_of<FORMAT, 128, 1>(bf16, f32) : nb == 2 ? tree_kernel_of<FORMAT, 128, 2>(bf16, f32) : tree_kernel_of<FORMAT, 128, 4>(bf16, f32);
    return nb == 1 ? tree_kernel_of<FORMAT, 64, 1>(bf16, f32) : nb == 2 ? tree_kernel_of<FORMAT, 64, 2>(bf16, f32) : tree_kernel_of<FORMAT, 64, 4>(bf16, f32);
}
// In a translation unit each.
TreeKernel tree_kernel_16(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_fp8(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_fp4(int D, bool bf16, bool f32, int nb);

}  // namespace kvb
