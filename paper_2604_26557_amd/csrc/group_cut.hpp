// How a kv_group_attn launch shares its work out: query rows per workgroup and tokens per split, of prefixes and of sequences' own tokens.  Host arithmetic only.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "tree_cut.hpp"

namespace kvb {

constexpr int kMostGroups = 64;   // a lane each

// Prefixes, and sequences' own tokens: new tokens whose rows go over them, and how many they are.
struct GroupUnit {
    int tokens, span;
    bool prefix;
};
struct GroupCut {
    int nb, nb_prefix;                // 16-row groups of a workgroup, and of a prefix' workgroup: as many, or the most where the others have one
    int prefix_tokens, split_tokens;  // of a split, multiples of 32
    int prefix_ns, ns;                // partial results of a row: of its prefix, and in all
};

inline int splits_of(int span, int split_tokens) { return span <= 0 ? 0 : (span - 1) / split_tokens + 1; }

// Workgroups of a unit: its splits of all heads, in eights where it has several row blocks, times these.
inline uint64_t unit_workgroups(const TreeShape &s, const GroupUnit &u, int nb, int split_tokens)
{
    if (u.tokens <= 0 || u.span <= 0) return 0;
    const uint64_t rows = (uint64_t)u.tokens * s.G, blocks = (rows + 16 * nb - 1) / (16 * nb);
    uint64_t units = (uint64_t)splits_of(u.span, split_tokens) * s.H;
    if (blocks > 1) units = (units + 7) / 8 * 8;
    return units * blocks;
}

// Unit i of groups, then sequences: span of a sequence's own tokens begins at a multiple of 32.
inline GroupUnit group_unit(int i, int n_groups, const int *group_first, const int *prefix, const int *lens, const int *first, int shared)
{
    if (i < n_groups) return GroupUnit{first[group_first[i + 1]] - first[group_first[i]], prefix[i], true};
    const int b = i - n_groups, t = first[b + 1] - first[b];
    return GroupUnit{t, t > 0 ? lens[b] + t - (shared & ~31) : 0, false};
}

inline uint64_t group_workspace_bytes(const TreeShape &s, long long n_tok, long long tokens)
{
    return std::max(tree_workspace_bytes(s, n_tok, tokens + 64), 2 * tree_split_bytes(s, n_tok));
}

// By an estimate of the time in us, with the costs of cut_tree: what the workgroups take that a compute unit gets, two side by side, at least as long as one of them; the cache through HBM once; where there are
// splits a second launch and partial results. units: those of up to `counted` with work; chains without a mask see half of their new tokens.
inline GroupCut cut_group(const TreeShape &s, const GroupUnit *units, int n, bool chain, int n_splits, uint64_t ws_bytes, long long n_tok)
{
    int longest = 0, longest_prefix = 0;
    long long rows = 0, prefix_rows = 0;
    double context = 0;
    for (int i = 0; i < n; ++i) {
        if (units[i].tokens <= 0 || units[i].span <= 0) continue;
        (units[i].prefix ? longest_prefix : longest) = std::max(units[i].prefix ? longest_prefix : longest, units[i].span);
        rows = std::max(rows, (long long)units[i].tokens * s.G);
        if (units[i].prefix) prefix_rows = std::max(prefix_rows, (long long)units[i].tokens * s.G);
        context += units[i].span;
    }
    const uint64_t fit = ws_bytes / tree_split_bytes(s, n_tok);
    const int least_ns = longest_prefix > 0 ? 2 : 1;   // one of each kind: the caller has checked for their room
    const int room = (int)std::max<uint64_t>(least_ns, std::min<uint64_t>(fit, kMaxTreeSplits));
    const int most = n_splits > 0 ? room : std::min(room, std::max(least_ns, tree_most_splits(s, n_tok)));
    const int span = std::max(longest, longest_prefix);
    const double row = s.H * 2.0 * s.D * s.bits / 8, hbm = context * row / 7.4e6, part = 2.0 * s.H * s.G * s.D * 4 / 2.0e6;
    auto tokens_of = [&](int ns) { return (int)((((long long)span + ns - 1) / ns + 31) / 32 * 32); };
    auto results_of = [&](int ns) { return splits_of(longest_prefix, tokens_of(ns)) + splits_of(longest, tokens_of(ns)); };
    int only = n_splits;
    while (only > 1 && results_of(only) > most) --only;
    GroupCut best{};
    double least = 1e30;
    for (int ns = only > 0 ? only : 1; ns <= kMaxTreeSplits; ns = next_splits(ns)) {
        if (results_of(ns) > most) break;
        const int st = tokens_of(ns), of_prefix = splits_of(longest_prefix, st), of_own = splits_of(longest, st);
        const int most_nb = s.D == 256 ? 2 : 4;
        for (int k = 0; k < 4; ++k) {   // 1, 2, 4 of both; the most of prefixes alone
            const int nb = k == 3 ? 1 : 1 << k, nb_prefix = k == 3 ? most_nb : nb;
            if (nb > most_nb || (k == 3 && longest_prefix == 0)) continue;
            if (k > 0 && (k == 3 ? prefix_rows : rows) <= 8 * nb_prefix) continue;   // half of the rows would be none
            auto step = [&](int n) { return 0.95 + 0.18 * n * s.D / 128 * (s.D == 256 ? 1.4 : 1) + (s.paged ? 0.05 : 0); };
            double groups = 0, work = 0, parts = 0, longest_one = 0;
            for (int i = 0; i < n; ++i) {
                if (units[i].tokens <= 0 || units[i].span <= 0) continue;
                const int mine = units[i].prefix ? nb_prefix : nb;
                const double start = 2.6 + 0.6 * mine, blocks = std::ceil((double)units[i].tokens * s.G / (16 * mine)), splits = splits_of(units[i].span, st);
                const double seen = !units[i].prefix && chain ? units[i].span - 0.5 * units[i].tokens : units[i].span;
                groups += blocks * splits * s.H;
                work += blocks * s.H * (splits * start + seen / 128 * step(mine));
                parts += units[i].tokens * splits;
                longest_one = std::max(longest_one, start + std::min(st, units[i].span) / 128.0 * step(mine));
            }
            const double us = std::max({hbm + 3.4, groups > s.cus ? 1.45 * longest_one : longest_one, work / (s.cus * 1.4)}) +
                              (of_prefix + of_own > 1 ? 3.9 + parts * part + 0.03 * (of_prefix + of_own) : 0);
            if (us < least) {
                least = us;
                best = GroupCut{nb, nb_prefix, st, st, of_prefix, of_prefix + of_own};
            }
        }
        if (only > 0) break;
    }
    return best;
}

}  // namespace kvb
