// How a kv_tree_attn launch shares its work out: query rows per workgroup and token splits.  Host arithmetic only, for groups of at most 4095 heads and contexts of at
// most 2^30 tokens.
#pragma once

#include <algorithm>
#include <cmath>
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

// The numbers of splits that are considered.
constexpr int next_splits(int ns) { return ns < 8 ? ns + 1 : ns < 16 ? ns + 2 : ns < 32 ? ns + 4 : ns < 64 ? ns + 8 : ns + 32; }

// Room for whatever is chosen for up to n_tok drafted tokens over up to `tokens` of a sequence, drafted ones included.  Fewer tokens may be split more often: the most is wanted by n_tok or by
// as many as just fill some number of 64-row blocks.
inline uint64_t tree_workspace_bytes(const TreeShape &s, long long n_tok, long long tokens)
{
    int cap = 1;
    while (cap < (tokens + 31) / 32 && cap < kMaxTreeSplits) cap = next_splits(cap);
    auto room = [&](long long n) { return tree_split_bytes(s, n) * (uint64_t)std::min(tree_most_splits(s, n), cap); };
    uint64_t most = room(n_tok);
    for (long long blocks = 1, n = 0; (n = 64 * blocks / s.G) < n_tok; ++blocks) {
        if (n > 0) most = std::max(most, room(n));
        if (n > 0 && tree_most_splits(s, n) == 1) break;   // from there on more tokens take more room
    }
    return most;
}

// Sequences up to which a ragged batch's launch leaves out the workgroups that have nothing to do, and up to which they are counted one by one here: a lane of a wavefront each.
constexpr int kCounted = 64;

// Whether a split has any of a sequence's tokens.  Where units go in eights a workgroup's split may be up to 7 past the last one: with tokens of a split as many as a context's, that
// passes 32 bits.
constexpr bool split_has_tokens(unsigned split, int split_tokens, int total) { return (uint64_t)split * (unsigned)split_tokens < (uint64_t)total; }

// Both choices go by an estimate of the time in us, fitted to what 36 shapes took with 3 row groups times 20 split counts each (head_dim 64 to 256, the three formats, 1 to
// 48 sequences of equal or ragged lengths, 1 to 64 drafted tokens, contexts of 48 to 32K):
//   a workgroup's start and merge, and its wavefronts' steps of 32 tokens; every further workgroup on the fullest compute unit adds 40 % of the one and 41 to 50 % of the other;
//   the whole cache through HBM once, and again through L2 for further row blocks;
//   where there are splits a second launch, and partial results written and read.
// The fit was to kernels with one part to a probability of a 16-bit result.  With the present ones its choice is 7 % from a shape's best on average, within 5 % on 26 of the 36, within 10 %
// on 28 and 70 % off on the worst (many short sequences of unequal length, whose workgroups it takes for equals), where it was 6 %, 26, 28 and 70 %; the times themselves it gives to 13 % on average.
// At least one token is drafted.
inline TreeCut cut_tree(const TreeShape &s, int B, const int *lens, const int *first, int n_splits, uint64_t ws_bytes)
{
    int rows = 0, longest = 0;
    double blocks[3] = {0, 0, 0}, tokens[3] = {0, 0, 0}, context = 0;  // by row groups: workgroups without splits, and the tokens they go over
    float totals[kCounted], drafts[kCounted], groups[kCounted][3];     // of sequences that are counted
    int counted = 0;
    for (int b = 0; b < B; ++b) {
        const int t = first[b + 1] - first[b], total = lens[b] + t;
        if (t == 0) continue;
        rows = std::max(rows, t * s.G);
        longest = std::max(longest, total);
        context += total;
        for (int k = 0; k < 3; ++k) {
            const int n = (t * s.G + (16 << k) - 1) / (16 << k);
            blocks[k] += n;
            tokens[k] += (double)n * total;
            if (counted < kCounted) groups[counted][k] = (float)n;
        }
        if (counted < kCounted) {
            totals[counted] = (float)(total - 1);
            drafts[counted] = (float)t;
        }
        ++counted;
    }
    const long long n_tok = first[B];
    const int fit = (int)std::min<uint64_t>(kMaxTreeSplits, ws_bytes / tree_split_bytes(s, n_tok));
    const int most = std::max(1, std::min(fit, n_splits > 0 ? n_splits : tree_most_splits(s, n_tok)));
    const double row = s.H * 2.0 * s.D * s.bits / 8, hbm = context * row / 7.4e6, part = 2.0 * s.H * s.G * s.D * 4 / 2.0e6;
    TreeCut best{};
    double least = 1e30;
    for (int ns = n_splits > 0 ? most : 1; ns <= most; ns = next_splits(ns)) {
        const int st = ((longest + ns - 1) / ns + 31) / 32 * 32;
        float splits[3] = {0, 0, 0}, parts = 0;   // workgroups of a KV head, and partial results of a query head
        if (counted <= kCounted) {
            const float per = 1.f / (float)st;
            for (int b = 0; b < counted; ++b) {
                const float n = (float)((int)(totals[b] * per) + 1);
                for (int k = 0; k < 3; ++k) splits[k] += groups[b][k] * n;
                parts += drafts[b] * n;
            }
        } else {   // half a workgroup more each than their tokens fill
            for (int k = 0; k < 3; ++k) splits[k] = (float)(ns > 1 ? tokens[k] / st + 0.5 * blocks[k] : blocks[k]);
            parts = (float)n_tok * (float)ns;
        }
        for (int k = 0; k < (s.D == 256 ? 2 : 3); ++k) {
            const int nb = 1 << k;
            if (k > 0 && rows <= 8 * nb) break;   // half of the rows would be none
            const double step = 0.95 + 0.18 * nb * s.D / 128 * (s.D == 256 ? 1.4 : 1) + (s.paged ? 0.05 : 0), start = 2.6 + 0.6 * nb;
            const double further = std::max(0.0, std::ceil((double)splits[k] * s.H / s.cus) - 1);   // workgroups beside the first on the fullest compute unit
            const double us = std::max(hbm + (tokens[k] - context) * row / 25e6 + 1.06 * start, start * (1 + 0.4 * further) + (st + 127) / 128 * step * (1 + (0.53 - 0.03 * nb) * further)) +
                              (ns > 1 ? 3.9 + parts * part + 0.03 * ns : 0);
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
