// Kernels of kv_tree_attn, a translation unit for each cache format and layout (tree_attn_16.hip, tree_attn_16_paged.hip, ...).
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>

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
    float scale_log2e;
    int words, max_total, H, G, B, out_mode;  // out_mode: 0 fp32, 1 fp16, 2 bf16
    int ns, split_tokens, row_blocks;
    int bt_shift;                      // log2 of a block's tokens, or -1
    int grouped;                       // rows of context are looked up by groups of eight
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

constexpr int kTreeWaves = 8, kTreeThreads = 64 * kTreeWaves;
constexpr float kNoScore = -1.0e30f;    // reference of a row that has seen no score
constexpr float kTreeRise = 4.f;        // a reference follows the running maximum when a score passes it by this (log2)
constexpr float kLargeRef = 1048576.f;  // beyond it the rounding of a reference would leave the range of the probabilities
// fp16 probabilities are taken of 2^11 times themselves (at most 2^15): what is lost lies below 2^-36 of the largest
template <bool BF16> constexpr float kLiftLog2 = BF16 ? 0.f : 11.f;
template <bool BF16, bool F32> constexpr int kParts = F32 ? (BF16 ? 3 : 2) : 1;

// Probabilities as 16-bit operands: rounded once, or as parts whose sum is the 32-bit value (bf16) or that value up to 2^-22 (fp16).
template <bool BF16, int N>
__device__ __forceinline__ void split_pair(float x, float y, unsigned (&out)[N])
{
    if constexpr (BF16 && N == 3) {
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            const unsigned a = __float_as_uint(x), b = __float_as_uint(y);
            out[t] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            x -= __uint_as_float(a & 0xffff0000u);
            y -= __uint_as_float(b & 0xffff0000u);
        }
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

template <typename T, bool NT>
__device__ __forceinline__ T load_as(const char *p)
{
    if constexpr (NT) return __builtin_nontemporal_load((const T *)p);
    else return *(const T *)p;
}

// How rows of context alone are addressed (in groups of eight tokens): a strided cache, scalar bases and 32-bit offsets of the lanes; a block pool of multiples of
// eight tokens, a pointer per lane and constant offsets.  Everything else is looked up row by row.
constexpr int kTreeStrided = 0, kTreePaged = 1;

// A step of a wavefront is 32 tokens.  Where their K and V are few bytes, four wavefronts a SIMD keep enough of them in flight, elsewhere two do.
template <int D, int FORMAT, int NB> constexpr int kTreeWavesPerSimd = NB == 1 && D * format_bits(FORMAT) <= 512 ? 4 : 2;

template <int D, bool BF16, int FORMAT, int NB, bool F32>
struct TreeTile {
    static constexpr int kColumns = D / 16;           // columns of V that a lane loads of a token
    static constexpr int kSteps = D / 32;             // products of a tile of q K^T
    static constexpr int kRows = 16 * NB;             // query rows of a workgroup
    static constexpr int kBits = format_bits(FORMAT);
    static constexpr bool kBlocks = FORMAT != KV_FORMAT_16;
    static constexpr bool kQInLds = NB * D > 256;   // more rows than their registers are worth
    static constexpr bool kNT = NB <= 2;              // more rows: other workgroups may read the same K and V out of L2
    static constexpr int kP = kParts<BF16, F32>;
    // K: a lane holds a quarter of a token's row, as pieces of 16 bytes (8 where the row is 32 bytes long)
    static constexpr int kQuarter = D * kBits / 32;   // bytes
    static constexpr int kPiece = kQuarter < 16 ? kQuarter : 16;
    static constexpr int kPieces = kQuarter / kPiece;
    static constexpr int kPieceElems = kPiece * 8 / kBits;
    static constexpr int kVBytes = kColumns * kBits / 8;
    static constexpr int kVWords = kVBytes < 4 ? 1 : kVBytes / 4;

    struct K {
        u32x4 w[kPieces];
        unsigned z[kBlocks ? kPieces : 1];
    };
    struct V {
        unsigned w[8][kVWords];
        unsigned z[kBlocks ? 8 : 1];
    };

    // The first of the eight elements of d that a lane contributes to product s: any order will do that q follows as well.
    static __device__ __forceinline__ int q_at(int s, int group)
    {
        constexpr int per = kPieceElems / 8;  // products of a piece
        return (s / per) * 4 * kPieceElems + group * kPieceElems + (s % per) * 8;
    }

    static __device__ __forceinline__ void load_k(K &k, const char *row, const char *zrow, int group) { load_k(k, row, 0, zrow, 0, group); }
    // Rows at a base that all lanes share and an offset of the lane's.
    static __device__ __forceinline__ void load_k(K &k, const char *row, unsigned lane_at, const char *zrow, unsigned lane_z, int group)
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const char *const at = row + 4 * kPiece * i + (lane_at + kPiece * group);
            if constexpr (kPiece == 16) {
                k.w[i] = load_as<u32x4, kNT>(at);
            } else {
                const u32x2 w = load_as<u32x2, kNT>(at);
                k.w[i] = u32x4{w[0], w[1], 0, 0};
            }
            if constexpr (kBlocks) k.z[i] = (unsigned char)(zrow + i * 4 * kPieceElems / kBlockElems)[lane_z + group * kPieceElems / kBlockElems];
        }
    }
    static __device__ __forceinline__ u32x4 k_operand(const K &k, int s)
    {
        if constexpr (!kBlocks) {
            return k.w[s];
        } else {
            constexpr int per = kPieceElems / 8;
            const u32x4 w = k.w[s / per];
            const float z = scale_operand(k.z[s / per]);
            if constexpr (FORMAT == KV_FORMAT_FP8) return decode8<BF16, FORMAT>(u32x2{w[2 * (s % per)], w[2 * (s % per) + 1]}, z);
            else return decode8<BF16, FORMAT>(u32x2{w[s % per], 0}, z);
        }
    }
    // Token j of the lane's eight.
    static __device__ __forceinline__ void load_v(V &v, int j, const char *row, const char *zrow, int n) { load_v(v, j, row, 0, zrow, 0, n); }
    static __device__ __forceinline__ void load_v(V &v, int j, const char *row, unsigned lane_at, const char *zrow, unsigned lane_z, int n)
    {
        const char *const at = row + (lane_at + kVBytes * n);
        if constexpr (kVBytes == 2) {
            v.w[j][0] = load_as<unsigned short, kNT>(at);
        } else if constexpr (kVBytes == 4) {
            v.w[j][0] = load_as<unsigned, kNT>(at);
        } else if constexpr (kVBytes == 8) {
            const u32x2 w = load_as<u32x2, kNT>(at);
            v.w[j][0] = w[0];
            v.w[j][1] = w[1];
        } else {
#pragma unroll
            for (int i = 0; i < kVBytes / 16; ++i) {
                const u32x4 w = load_as<u32x4, kNT>(at + 16 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) v.w[j][4 * i + e] = w[e];
            }
        }
        if constexpr (kBlocks) v.z[j] = (unsigned char)zrow[lane_z + kColumns * n / kBlockElems];
    }
    // Columns 2 * i and 2 * i + 1 of token j as 16-bit numbers.
    static __device__ __forceinline__ unsigned v_pair(const V &v, int j, int i)
    {
        if constexpr (!kBlocks) {
            return v.w[j][i];
        } else {
            const float z = scale_operand(v.z[j]);
            if constexpr (FORMAT == KV_FORMAT_FP8)
                return i % 2 ? decode2<BF16, FORMAT, 1>(v.w[j][i / 2], z) : decode2<BF16, FORMAT, 0>(v.w[j][i / 2], z);
            else
                return i % 4 == 0 ? decode2<BF16, FORMAT, 0>(v.w[j][i / 4], z) : i % 4 == 1 ? decode2<BF16, FORMAT, 1>(v.w[j][i / 4], z)
                     : i % 4 == 2 ? decode2<BF16, FORMAT, 2>(v.w[j][i / 4], z) : decode2<BF16, FORMAT, 3>(v.w[j][i / 4], z);
        }
    }
};

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

// Does row r of a KV head's query rows see token j of its sequence?
__device__ __forceinline__ bool row_sees(const TreeParams &p, int first, int r, int j, int len, int total)
{
    if (j < len) return true;
    if (j >= total || r >= (total - len) * p.G) return false;
    const int t = r / p.G, i = j - len;
    if (!p.mask) return i <= t;
    return (bool)(p.mask[(long long)(first + t) * p.words + (i >> 6)] >> (i & 63) & 1);
}

// The same of eight tokens from j on, as bits.
__device__ __forceinline__ unsigned row_sees8(const TreeParams &p, int first, int r, int j, int len, int total)
{
    auto below = [](int x) { return x >= 8 ? 0xffu : (1u << max(x, 0)) - 1u; };
    const unsigned context = below(len - j), drafted = below(total - j) & ~context;
    if (drafted == 0 || r >= (total - len) * p.G) return context;
    const int t = r / p.G, i = j - len;   // i > -8: a token's bit is i + its place
    unsigned long long bits;
    if (!p.mask) {
        bits = below(t + 1 - i);
    } else {
        const unsigned long long *const row = p.mask + (long long)(first + t) * p.words;
        const int w = max(i, 0) >> 6, shift = max(i, 0) & 63;
        bits = row[w] >> shift;
        if (shift > 56 && w + 1 < p.words) bits |= row[w + 1] << (64 - shift);
        if (i < 0) bits <<= -i;
    }
    return context | (drafted & (unsigned)bits);
}

// Four columns of a query row's sums: the result, or the partial result of a split.
template <int D>
__device__ __forceinline__ void store_sums(const TreeParams &p, unsigned h, int first, int r, unsigned split, int d, f32x4 x, float ref, float l)
{
    const int t = r / p.G, hq = (int)h * p.G + r - t * p.G;
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
    using T = TreeTile<64, BF16, FORMAT, 1, false>;   // four columns of a lane, sixteen lanes: here D / 4 lanes
    const int t = r / p.G, hq = (int)h * p.G + r - t * p.G, at = lane % (D / 4);
    const u32x2 qw = *(const u32x2 *)(p.q + 2 * ((first + t) * p.q_st + hq * p.q_sh + 4 * at));
    const f32x2 q0 = unpack2<BF16>(qw[0]), q1 = unpack2<BF16>(qw[1]);
    auto row = [&](const char *rows, const char *scales, int j, bool *there) {
        const RowAt x = row_at(p.c, table, base, zbase, j);
        *there = x.there;
        typename T::V v;
        T::load_v(v, 0, rows + x.at, scales + x.z, at);
        const f32x2 a = unpack2<BF16>(T::v_pair(v, 0, 0)), b = unpack2<BF16>(T::v_pair(v, 0, 1));
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

template <int D, bool BF16, int FORMAT, int NB, bool F32, int LAYOUT>
__global__ void __launch_bounds__(kTreeThreads, (kTreeWavesPerSimd<D, FORMAT, NB>)) kv_tree_partial_kernel(TreeParams p)
{
    using T = TreeTile<D, BF16, FORMAT, NB, F32>;
    constexpr int kRows = T::kRows, kColumns = T::kColumns, kSteps = T::kSteps, kP = T::kP;

    // Workgroups go round the eight XCDs: the row blocks of a split follow each other on one of them and share its L2.
    const unsigned xcd = blockIdx.x % 8, turn = blockIdx.x / 8;
    const unsigned rb = turn % (unsigned)p.row_blocks, unit = turn / (unsigned)p.row_blocks * 8 + xcd;
    const unsigned split = unit % (unsigned)p.ns, bh = unit / (unsigned)p.ns, b = bh / (unsigned)p.H, h = bh % (unsigned)p.H;
    if (b >= (unsigned)p.B) return;
    const int first = p.tok_first[b], drafted = min(p.tok_first[b + 1] - first, KV_TREE_MAX);
    const int n_rows = drafted * p.G - (int)rb * kRows;   // of this block: the first kRows of them
    if (n_rows <= 0) return;
    const int len = max(0, min(p.seq_lens[b], p.max_total - drafted)), total = len + drafted;
    const int s0 = (int)split * p.split_tokens, s1 = min(s0 + p.split_tokens, total);
    if (s0 >= total) return;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, group = lane >> 4;
    const unsigned long long base = p.c.table ? h * p.c.sh : b * p.c.sb + h * p.c.sh;
    const unsigned long long zbase = p.c.table ? h * p.c.zh : b * p.c.zb + h * p.c.zh;
    const int *const table = p.c.table ? p.c.table + (long long)b * p.c.max_blocks : nullptr;

    // Query rows: token-major, the G heads of a token side by side.  Rows past the last one are zeros.
    auto row_token = [&](int r) { return ((int)rb * kRows + r) / p.G; };
    __shared__ __attribute__((aligned(16))) u32x4 q_lds[T::kQInLds ? NB * kSteps * 64 : 1];
    u32x4 q_reg[T::kQInLds ? 1 : NB][kSteps];
    auto load_q = [&](int nb, int s) {
        const int r = nb * 16 + n;
        if (r >= n_rows) return u32x4{0, 0, 0, 0};
        const int t = row_token(r), g = (int)rb * kRows + r - t * p.G;
        return *(const u32x4 *)(p.q + 2 * ((first + t) * p.q_st + ((int)h * p.G + g) * p.q_sh + T::q_at(s, group)));
    };
    if constexpr (T::kQInLds) {
        for (int i = wave; i < NB * kSteps; i += kTreeWaves) q_lds[i * 64 + lane] = load_q(i / kSteps, i % kSteps);
        __syncthreads();
    } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) q_reg[nb][s] = load_q(nb, s);
    }

    f32x4 acc[NB][kColumns], sum[NB];
    float ref[NB];
    const u32x4 ones = BF16 ? u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u} : u32x4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};

    // Scores of 32 tokens: lane (n, group) gets those of tokens 8 * group + 0..3 from the first tile and + 4..7 from the second.
    auto scores = [&](const typename T::K (&k)[2], f32x4 (&s)[NB][2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[nb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                const u32x4 a = T::k_operand(k[i], st);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    u32x4 q;
                    if constexpr (T::kQInLds) q = q_lds[(nb * kSteps + st) * 64 + lane];
                    else q = q_reg[nb][st];
                    s[nb][i] = mfma32<BF16>(a, q, s[nb][i]);
                }
            }
    };
    auto product = [&](const typename T::V &v, const u32x4 (&pr)[NB][kP]) {
#pragma unroll
        for (int t = 0; t < kP; ++t)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) sum[nb] = mfma32<BF16>(ones, pr[nb][t], sum[nb]);
#pragma unroll
        for (int c = 0; c < kColumns; c += 2) {
            unsigned w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = T::v_pair(v, j, c / 2);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const unsigned sel = e ? 0x07060302u : 0x05040100u;
                const u32x4 a = {__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel),
                                 __builtin_amdgcn_perm(w[5], w[4], sel), __builtin_amdgcn_perm(w[7], w[6], sel)};
#pragma unroll
                for (int t = 0; t < kP; ++t)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) acc[nb][c + e] = mfma32<BF16>(a, pr[nb][t], acc[nb][c + e]);
            }
        }
    };
    auto rescale = [&](int nb, float f) {
        sum[nb] *= f;
#pragma unroll
        for (int c = 0; c < kColumns; ++c) acc[nb][c] *= f;
    };
    // Probabilities against a reference that follows the running maximum lazily.
    auto softmax = [&](f32x4 (&s)[NB][2], u32x4 (&pr)[NB][kP]) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const f32x4 a = s[nb][0], b4 = s[nb][1];
            const float top = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b4[0], b4[1]), fmaxf(b4[2], b4[3]))) * p.scale_log2e;
            if (__any(top > ref[nb] + kTreeRise)) {
                const float to = fmaxf(ref[nb], groups_max(top));
                rescale(nb, __builtin_amdgcn_exp2f(ref[nb] - to));
                ref[nb] = to;
            }
            const float sub = kLiftLog2<BF16> - ref[nb];
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_exp2f(fmaf(s[nb][j / 4][j % 4], p.scale_log2e, sub));
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

    const int n_steps = (s1 - s0 + 31) / 32;
    const int grouped = p.grouped ? max(0, min(len, s1) - s0) / 32 : 0;   // steps of context alone, looked up by groups of eight rows
    constexpr int kRow = D * T::kBits / 8, kZRow = D / kBlockElems;      // a pool's rows lie side by side
    const unsigned lane_k = LAYOUT == kTreePaged ? (n & 3) * kRow : (8 * (n >> 2) + (n & 3)) * (unsigned)p.c.ss;
    const unsigned lane_zk = LAYOUT == kTreePaged ? (n & 3) * kZRow : (8 * (n >> 2) + (n & 3)) * (unsigned)p.c.zs;
    const unsigned lane_v = LAYOUT == kTreePaged ? 0 : 8 * group * (unsigned)p.c.ss, lane_zv = LAYOUT == kTreePaged ? 0 : 8 * group * (unsigned)p.c.zs;
    auto block_of = [&](int j) { return p.bt_shift >= 0 ? j >> p.bt_shift : j / p.c.bt; };
    unsigned id_k = 0, id_v = 0;
    auto look_up = [&](int i) {
        if (LAYOUT == kTreePaged && i < grouped) {
            id_k = (unsigned)table[block_of(s0 + 32 * i + 8 * (n >> 2))];
            id_v = (unsigned)table[block_of(s0 + 32 * i + 8 * group)];
        }
    };
    look_up(wave);
    for (int i = wave; i < n_steps; i += kTreeWaves) {
        const int j0 = s0 + 32 * i;
        typename T::K k[2];
        typename T::V v;
        unsigned there = 0xff;
        // the lanes of K look all four groups up
        const bool one_by_one = i >= grouped || (LAYOUT == kTreePaged && __any(id_k >= (unsigned)p.c.n_pool));
        if (one_by_one) {
            // where a sequence ends, drafted tokens begin, a block has no place, or blocks are no multiples of eight tokens
            there = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const RowAt r = row_at(p.c, table, base, zbase, min(j0 + 8 * (n >> 2) + (n & 3) + 4 * t, total - 1));
                T::load_k(k[t], p.c.k + r.at, p.c.kz + r.z, group);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const RowAt r = row_at(p.c, table, base, zbase, min(j0 + 8 * group + j, total - 1));
                T::load_v(v, j, p.c.v + r.at, p.c.vz + r.z, n);
                there |= (unsigned)r.there << j;
            }
        } else if constexpr (LAYOUT == kTreePaged) {
            const int jk = j0 + 8 * (n >> 2), jv = j0 + 8 * group;
            const int in_k = jk - block_of(jk) * p.c.bt, in_v = jv - block_of(jv) * p.c.bt;
            const char *const rk = p.c.k + base + id_k * p.c.sb + in_k * kRow + lane_k, *const zk = p.c.kz + zbase + id_k * p.c.zb + in_k * kZRow + lane_zk;
            const char *const rv = p.c.v + base + id_v * p.c.sb + in_v * kRow, *const zv = p.c.vz + zbase + id_v * p.c.zb + in_v * kZRow;
            T::load_k(k[0], rk, zk, group);
            T::load_k(k[1], rk + 4 * kRow, zk + 4 * kZRow, group);
#pragma unroll
            for (int j = 0; j < 8; ++j) T::load_v(v, j, rv + j * kRow, zv + j * kZRow, n);
        } else {
            const unsigned long long at = base + j0 * p.c.ss, z = zbase + j0 * p.c.zs;
#pragma unroll
            for (int t = 0; t < 2; ++t) T::load_k(k[t], p.c.k + (at + 4 * t * p.c.ss), lane_k, p.c.kz + (z + 4 * t * p.c.zs), lane_zk, group);
#pragma unroll
            for (int j = 0; j < 8; ++j) T::load_v(v, j, p.c.v + (at + j * p.c.ss), lane_v, p.c.vz + (z + j * p.c.zs), lane_zv, n);
        }
        look_up(i + kTreeWaves);
        f32x4 s[NB][2];
        scores(k, s);
        if (one_by_one) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const unsigned seen = there & row_sees8(p, first, (int)rb * kRows + nb * 16 + n, j0 + 8 * group, len, total);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[nb][j / 4][j % 4] = seen >> j & 1 ? s[nb][j / 4][j % 4] : -INFINITY;
            }
        }
        u32x4 pr[NB][kP];
        softmax(s, pr);
        product(v, pr);
    }

    // What is not finite may be none of a row's business (a probability of zero times it), and references may have grown too large:
    // then the workgroup does its split again, row by row.
    bool bad = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float worst = fabsf(sum[nb][0]);
#pragma unroll
        for (int c = 0; c < kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) worst = fabsf(acc[nb][c][i]) < INFINITY ? worst : INFINITY;
        bad = bad || !(worst < INFINITY) || (fabsf(ref[nb]) > kLargeRef && ref[nb] != kNoScore);
    }
    if (__syncthreads_or(bad)) {
        for (int r = wave; r < min(n_rows, kRows); r += kTreeWaves)
            plain_row<D, BF16, FORMAT>(p, table, base, zbase, h, first, (int)rb * kRows + r, len, total, s0, s1, split, lane);
        return;
    }

    // Merge: the wavefronts' references and sums of each row, then their accumulators in two rounds.
    constexpr int kPad = D + 4;
    __shared__ __attribute__((aligned(16))) float rows_lds[4][kRows][kPad];
    __shared__ float ref_lds[kTreeWaves][kRows], sum_lds[kTreeWaves][kRows];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
        if (group == 0) {
            ref_lds[wave][nb * 16 + n] = ref[nb] - kLiftLog2<BF16>;
            sum_lds[wave][nb * 16 + n] = sum[nb][0];
        }
    __syncthreads();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float to = kNoScore;
#pragma unroll
        for (int w = 0; w < kTreeWaves; ++w) to = fmaxf(to, ref_lds[w][nb * 16 + n]);
        const float f = sum[nb][0] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ref[nb] - kLiftLog2<BF16> - to);
#pragma unroll
        for (int c = 0; c < kColumns; ++c) acc[nb][c] *= f;
    }
    auto put = [&](int buf, bool add) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < kColumns; c += 4) {
                    f32x4 *const at = (f32x4 *)&rows_lds[buf][nb * 16 + n][kColumns * (4 * group + i) + c];
                    f32x4 x = {acc[nb][c][i], acc[nb][c + 1][i], acc[nb][c + 2][i], acc[nb][c + 3][i]};
                    if (add) x += *at;
                    *at = x;
                }
    };
    if (wave >= 4) put(wave - 4, false);
    __syncthreads();
    if (wave < 4) put(wave, true);
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * (D / 4); i += kTreeThreads) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        if (r >= n_rows) break;
        float to = kNoScore, l = 0.f;
#pragma unroll
        for (int w = 0; w < kTreeWaves; ++w) to = fmaxf(to, ref_lds[w][r]);
#pragma unroll
        for (int w = 0; w < kTreeWaves; ++w) l += sum_lds[w][r] == 0.f ? 0.f : sum_lds[w][r] * __builtin_amdgcn_exp2f(ref_lds[w][r] - to);
        f32x4 x = *(const f32x4 *)&rows_lds[0][r][d] + *(const f32x4 *)&rows_lds[1][r][d];
        x += *(const f32x4 *)&rows_lds[2][r][d] + *(const f32x4 *)&rows_lds[3][r][d];
        store_sums<D>(p, h, first, (int)rb * kRows + r, split, d, x, to, l);
    }
}

typedef void (*TreeKernel)(TreeParams);
template <int FORMAT, int LAYOUT, int D, int NB>
TreeKernel tree_kernel_of(bool bf16, bool f32)
{
    return bf16 ? (f32 ? kv_tree_partial_kernel<D, true, FORMAT, NB, true, LAYOUT> : kv_tree_partial_kernel<D, true, FORMAT, NB, false, LAYOUT>)
                : (f32 ? kv_tree_partial_kernel<D, false, FORMAT, NB, true, LAYOUT> : kv_tree_partial_kernel<D, false, FORMAT, NB, false, LAYOUT>);
}
template <int FORMAT, int LAYOUT>
TreeKernel tree_kernel_for(int D, bool bf16, bool f32, int nb)
{
    if (D == 256) return nb == 1 ? tree_kernel_of<FORMAT, LAYOUT, 256, 1>(bf16, f32) : tree_kernel_of<FORMAT, LAYOUT, 256, 2>(bf16, f32);
    if (D == 128)
        return nb == 1 ? tree_kernel_of<FORMAT, LAYOUT, 128, 1>(bf16, f32) : nb == 2 ? tree_kernel_of<FORMAT, LAYOUT, 128, 2>(bf16, f32)
                                                                                     : tree_kernel_of<FORMAT, LAYOUT, 128, 4>(bf16, f32);
    return nb == 1 ? tree_kernel_of<FORMAT, LAYOUT, 64, 1>(bf16, f32) : nb == 2 ? tree_kernel_of<FORMAT, LAYOUT, 64, 2>(bf16, f32)
                                                                                : tree_kernel_of<FORMAT, LAYOUT, 64, 4>(bf16, f32);
}
// In a translation unit each.
TreeKernel tree_kernel_16(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_16_paged(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_fp8(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_fp8_paged(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_fp4(int D, bool bf16, bool f32, int nb);
TreeKernel tree_kernel_fp4_paged(int D, bool bf16, bool f32, int nb);

}  // namespace kvb
