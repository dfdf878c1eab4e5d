// How a kv_tree_attn launch shares its work out: query rows per workgroup and token splits.  Host arithmetic only.
#pragma once

#include <algorithm>
#include <cstdint>

namespace kvb {

constexpr int kMaxTreeSplits = 128;

struct TreeShape {
    int D, H, G, bits, cus;  // bits of an element in the cache
};
struct TreeCut {
    int nb;            // 16-row groups of a workgroup: 1, 2 or 4
    int row_blocks;    // workgroups that share a KV head's rows of the sequence with the most
    int ns;            // splits of the longest sequence
    int split_tokens;  // a multiple of 32
};

// 16-row groups of a workgroup that has up to `rows` query rows of a KV head.  At head_dim 256 four groups' sums do not fit the registers.
inline int tree_row_groups(int D, int rows) { return rows <= 16 ? 1 : rows <= 32 || D == 256 ? 2 : 4; }

// Workgroups that the card holds at a time.
inline int tree_slots(const TreeShape &s, int nb) { return s.cus; }

// More splits than this are never made for n_tok drafted tokens: so many that each slot gets two workgroups.
inline int tree_most_splits(const TreeShape &s, long long n_tok)
{
    const long long blocks = std::max<long long>(1, (n_tok * s.G + 63) / 64) * s.H;
    return (int)std::min<long long>(kMaxTreeSplits, std::max<long long>(1, 4ll * s.cus / blocks));
}

inline uint64_t tree_split_bytes(const TreeShape &s, long long n_tok) { return (uint64_t)n_tok * s.H * s.G * (s.D + 2) * sizeof(float); }

inline TreeCut cut_tree(const TreeShape &s, int B, const int *lens, const int *first, int n_splits, uint64_t ws_bytes)
{
    int rows = 0, longest = 0;
    for (int b = 0; b < B; ++b) {
        const int t = first[b + 1] - first[b];
        if (t == 0) continue;
        rows = std::max(rows, t * s.G);
        longest = std::max(longest, lens[b] + t);
    }
    TreeCut c{};
    c.nb = tree_row_groups(s.D, rows);
    const int block = 16 * c.nb;
    c.row_blocks = (rows + block - 1) / block;
    double blocks = 0, tokens = 0;  // workgroups without splits, and the tokens they go over
    for (int b = 0; b < B; ++b) {
        const int t = first[b + 1] - first[b], n = (t * s.G + block - 1) / block;
        blocks += n;
        tokens += (double)n * (lens[b] + t);
    }
    blocks *= s.H;
    tokens *= s.H;
    const long long n_tok = first[B];
    const int fit = (int)std::min<uint64_t>(kMaxTreeSplits, ws_bytes / tree_split_bytes(s, n_tok));
    const int most = std::max(1, std::min(fit, n_splits > 0 ? n_splits : tree_most_splits(s, n_tok)));
    int best = most;
    if (n_splits == 0) {
        // us: what HBM needs for the whole, or the fullest slot for its workgroups (each 32 tokens of a wavefront, bytes or products), and the second launch
        const int slots = tree_slots(s, c.nb);
        const double row = 2.0 * s.D * s.bits / 8, hbm = tokens / std::max(1, c.row_blocks) * row / 6.0e6;
        const double token = std::max(row / 50e3, 4.0 * block * s.D / 2.5e6) * (slots / s.cus);
        double least = 1e30;
        for (int ns = 1; ns <= most; ns = ns < 4 ? ns + 1 : ns + ns / 4) {
            const int st = (longest + ns - 1) / ns;
            const double items = ns == 1 ? blocks : tokens / st + 0.5 * blocks, turns = std::max(1.0, items / slots);
            const double us = std::max(hbm, std::max(std::max<double>(st, 256) * token, turns * st * token)) + (ns > 1 ? 3.0 + 0.02 * ns : 0);
            if (us < least) least = us, best = ns;
        }
    }
    c.split_tokens = ((longest + best - 1) / best + 31) / 32 * 32;
    c.ns = std::max(1, (longest + c.split_tokens - 1) / std::max(1, c.split_tokens));
    return c;
}

}  // namespace kvb
