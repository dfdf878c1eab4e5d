// The second launch of kv_tree_attn and kv_group_attn: the partial results of a row joined.
#pragma once

#include "tree_attn.hpp"

namespace kvb {

// A wavefront joins the splits of one query row: out = sum_s 2^(ref_s - max) acc_s / sum_s 2^(ref_s - max) l_s.  A lane has the weight of a split (of two, beyond 64), so the
// exponentials take one instruction for the row, and the sums of up to 8 * 64 / (D / 4) splits are loaded at once, ahead of the weights.  Bound by its launch and two dependent reads: 4.0 us for 7
// splits of 512 rows, 5.8 for 16 of 2048 (17 MB).
constexpr int kCombineWaves = 4;
constexpr float kNothing = -1.f;   // weight of a split without anything
// slot(i) is the place of a row's i-th partial result, of ns.
template <int D, typename Slot>
__device__ __forceinline__ void combine_row(const TreeParams &p, int t, int hq, int ns, int lane, const Slot &slot)
{
    constexpr int kLanes = D / 4, kTogether = 64 / kLanes, kRound = 8;   // lanes of a row; splits at a time; of them on their way
    const long long row = (long long)t * (p.H * p.G) + hq;
    const f32x2 *const ml = (const f32x2 *)p.part_ml + row * p.ns;
    const int sub = lane / kLanes, d = lane % kLanes * 4;
    const float *const part = p.part_acc + row * p.ns * D + d;
    const f32x2 m0 = lane < ns ? ml[slot(lane)] : f32x2{kNoScore, 0.f}, m1 = 64 + lane < ns ? ml[slot(64 + lane)] : f32x2{kNoScore, 0.f};
    f32x4 y[kRound];
    auto load = [&](int s0) {
#pragma unroll
        for (int k = 0; k < kRound; ++k) {
            const int s = s0 + k * kTogether + sub;
            if (s0 + k * kTogether < ns) y[k] = *(const f32x4 *)&part[(long long)slot(s < ns ? s : 0) * D];
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

// The plan's shape, on the current device.
TreeShape tree_shape(const kv_plan *p, int bits, bool paged);

}  // namespace kvb
