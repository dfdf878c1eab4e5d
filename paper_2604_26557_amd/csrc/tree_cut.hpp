// How a kv_tree_attn launch shares its work out: query rows per workgroup and token splits.  Host arithmetic only, for groups of at most 4095 heads and contexts of at
// most 2^30 tokens.
#pragma once

#include <algorithm>
#include <cstdint>

namespace kvb {

constexpr int kMaxTreeSplits = 128;

struct TreeShape {
    int D, H, G, bits, cus;  // bits of an element in the cache
    bool paged;
};
struct TreeCut {
    int nb;            // 16-row groups of a workgroup: 1, 2 or 4 (at head_dim 256 no more than 2: four groups' sums do not fit the registers)
    int row_blocks;    // workgroups that share a KV head's rows of the sequence with the most
    int ns;            // splits of the longest sequence
    int split_tokens;  // a multiple of 32
};

// No more splits than this for n_tok drafted tokens: so many that a compute unit gets about four workgroups of 64 rows.
inline int tree_most_splits(const TreeShape &s, long long n_tok)
{
    const long long blocks = std::max<long long>(1, (n_tok * s.G + 63) / 64) * s.H;
    return (int)std::min<long long>(kMaxTreeSplits, std::max<long long>(1, 4ll * s.cus / blocks));
}

inline uint64_t tree_split_bytes(const TreeShape &s, long long n_tok) { return (uint64_t)n_tok * s.H * s.G * (s.D + 2) * sizeof(float); }

// Both choices go by an estimate of the time in us, fitted to what 15 shapes took with 3 row groups times 16 split counts each (head_dim 64 to 256, the three formats, 1 to
// 64 drafted tokens, contexts of 256 to 32K):
//   a workgroup's start and merge, and its wavefronts' steps of 32 tokens; every further workgroup on a compute unit adds 39 % of the one and 56 % of the other;
//   the whole cache through HBM once;  where there are splits a second launch, and partial results written and read.
// Its choice was within 5 % of a shape's best on 11 of the 15 and within 20 % on all; 64 rows and 256 workgroups for every shape were up to 40 % off.
// At least one token is drafted.
inline TreeCut cut_tree(const TreeShape &s, int B, const int *lens, const int *first, int n_splits, uint64_t ws_bytes)
{
    int rows = 0, longest = 0;
    bool uniform = true;
    double blocks[3] = {0, 0, 0}, tokens[3] = {0, 0, 0}, context = 0;  // by row groups: workgroups without splits, and the tokens they go over
    for (int b = 0; b < B; ++b) {
        const int t = first[b + 1] - first[b], total = lens[b] + t;
        if (t == 0) continue;
        uniform = uniform && (longest == 0 || longest == total);
        rows = std::max(rows, t * s.G);
        longest = std::max(longest, total);
        context += total;
        for (int k = 0; k < 3; ++k) {
            const int n = (t * s.G + (16 << k) - 1) / (16 << k);
            blocks[k] += n;
            tokens[k] += (double)n * total;
        }
    }
    const long long n_tok = first[B];
    const int fit = (int)std::min<uint64_t>(kMaxTreeSplits, ws_bytes / tree_split_bytes(s, n_tok));
    const int most = std::max(1, std::min(fit, n_splits > 0 ? n_splits : tree_most_splits(s, n_tok)));
    const double hbm = context * s.H * 2.0 * s.D * s.bits / 8 / 7.0e6, part = 2.0 * n_tok * s.H * s.G * s.D * 4 / 2.1e6;
    constexpr int kCounted = 16;   // sequences whose workgroups are counted one by one: for more, and split, half a workgroup each is added
    TreeCut best{};
    double least = 1e30;
    for (int k = 0; k < (s.D == 256 ? 2 : 3); ++k) {
        const int nb = 1 << k;
        if (k > 0 && rows <= 8 * nb) break;   // half of the rows would be none
        const double step = (s.D == 256 ? 0.75 : 0.9) + 0.19 * nb * s.D / 128 * (s.D == 256 ? 2.6 : 1) + (s.paged ? 0.25 : 0), start = 3.0 + 0.9 * nb;
        for (int ns = n_splits > 0 ? most : 1; ns <= most; ns = ns < 8 ? ns + 1 : ns < 16 ? ns + 2 : ns < 32 ? ns + 4 : ns < 64 ? ns + 8 : ns + 32) {
            const int st = ((longest + ns - 1) / ns + 31) / 32 * 32;
            double items = blocks[k];
            if (ns > 1 && uniform) {
                items *= (longest - 1) / st + 1;
            } else if (ns > 1 && B <= kCounted) {
                items = 0;
                for (int b = 0; b < B; ++b) {
                    const int t = first[b + 1] - first[b];
                    items += (double)((t * s.G + 16 * nb - 1) / (16 * nb)) * ((lens[b] + t - 1) / st + 1);
                }
            } else if (ns > 1) {
                items = tokens[k] / st + 0.5 * blocks[k];
            }
            items *= s.H;
            double turns = std::max(1.0, items / s.cus);   // workgroups of the fullest compute unit
            if (uniform) turns = (double)(long long)(turns + 0.9);
            else if (turns > 1) turns += 0.25;
            const double us = std::max(hbm + 0.8 * start, start * (1 + 0.39 * (turns - 1)) + (st + 127) / 128 * step * (1 + 0.56 * (turns - 1))) + (ns > 1 ? 4.4 + ns * (part + 0.01) : 0);
            if (us < least) {
                least = us;
                best.nb = nb;
                best.split_tokens = st;
            }
        }
    }
    best.row_blocks = (rows + 16 * best.nb - 1) / (16 * best.nb);
    best.ns = (longest - 1) / best.split_tokens + 1;
    return best;
}

}  // namespace kvb
