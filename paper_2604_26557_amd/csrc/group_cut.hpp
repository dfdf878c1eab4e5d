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
    double us;                        // the estimate of its time
};

inline int splits_of(int span, int split_tokens) { return span <= 0 ? 0 : (span - 1) / split_tokens + 1; }

// Workgroups of a unit: its splits of all heads, times its row blocks.
inline uint64_t unit_workgroups(const TreeShape &s, const GroupUnit &u, int nb, int split_tokens)
{
    if (u.tokens <= 0 || u.span <= 0) return 0;
    const uint64_t rows = (uint64_t)u.tokens * s.G, blocks = (rows + 16 * nb - 1) / (16 * nb);
    return (uint64_t)splits_of(u.span, split_tokens) * s.H * blocks;
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

// What all units of a kind come to. By row groups of a workgroup, 1, 2 and 4: row blocks, the tokens that they go over, and those of them that they see.
struct GroupWork {
    int units = 0, longest = 0;
    long long rows = 0;          // the most of a unit
    double blocks[3] = {0, 0, 0}, over[3] = {0, 0, 0}, seen[3] = {0, 0, 0}, tokens = 0, parts = 0, context = 0;

    void add(const TreeShape &s, const GroupUnit &u, double of_span)   // of_span: what of its tokens a row sees
    {
        ++units;
        longest = std::max(longest, u.span);
        rows = std::max(rows, (long long)u.tokens * s.G);
        for (int k = 0; k < 3; ++k) {
            const double n = std::ceil((double)u.tokens * s.G / (16 << k));
            blocks[k] += n;
            over[k] += n * u.span;
            seen[k] += n * of_span;
        }
        tokens += u.tokens;
        parts += (double)u.tokens * u.span;
        context += of_span;
    }
};

// Which cut: by an estimate of the time in us, made of the longest workgroup, of all of them shared out to the places for them, of the rounds that those of prefixes take, and of
// what the bytes of K and V take, read once and again by further row blocks; where there are splits of the second launch and partial results. Its numbers were fitted to choose well rather than to
// tell the time: to 20 shapes (1 to 64 sequences, up to 4 prefixes of 300 to 16K tokens, 1 to 900 new tokens, every format and head_dim), each with 10 to 300 of the cuts below; what it
// chose there took 2 % longer than the best on average, 10 % at most (a common length of all splits, by cut_tree's numbers: 13 % and 45 %).
// One length of splits for sequences' own tokens, one for prefixes, and as many partial results for every row, whose sum is bounded: a chunk of a prompt in the batch leaves the contexts beside it in few splits.
// One token at 32K beside a chunk of 2048 (8 x 4 x 128, 16 bits) takes 490 us, as two calls 31 + 79; 32 single tokens at 8K beside it 239, 166 + 79; 48 at 300 to 2000 beside a chunk of 700 123, 43 + 25, where
// the second launch has workgroups for the chunk's rows in every sequence.
// chain: without a mask a sequence sees half of its new tokens; bounded: rows see only some tokens, how many only the GPU knows: half is taken. At least one unit has work.
inline GroupCut cut_group(const TreeShape &s, const GroupUnit *units, int n, bool chain, bool bounded, bool shaped, int n_splits, uint64_t ws_bytes, long long n_tok)
{
    GroupWork own, prefix;
    for (int i = 0; i < n; ++i) {
        const GroupUnit &u = units[i];
        if (u.tokens <= 0 || u.span <= 0) continue;
        (u.prefix ? prefix : own).add(s, u, (u.span - (chain && !u.prefix ? 0.5 * u.tokens : 0)) * (bounded ? 0.5 : 1));
    }
    const uint64_t fit = ws_bytes / tree_split_bytes(s, n_tok);
    const int least_ns = prefix.longest > 0 ? 2 : 1;   // one of each kind: the caller has checked for their room
    const int room = (int)std::max<uint64_t>(least_ns, std::min<uint64_t>(fit, kMaxTreeSplits));
    const int most = n_splits > 0 ? room : std::min(room, std::max(least_ns, tree_most_splits(s, n_tok)));
    const double row = s.H * 2.0 * s.D * s.bits / 8e6, part = 2.0 * s.H * s.G * s.D * 4 / 1e6;
    // Of one kind: its workgroups, what they take in us together and the longest of them, rows that K and V are read for again, and partial results.
    struct Part {
        double groups = 0, work = 0, longest = 0, again = 0, parts = 0;
    };
    auto part_of = [&](const GroupWork &w, int nb, int tokens) {
        Part x;
        if (w.units == 0) return x;
        const int rows16 = 1 << nb;
        const double step = (1.039 + 0.16 * rows16 * s.D / 128 * (s.D == 256 ? 2.837 : 1) + (s.bits < 16 ? 0.045 : 0) + (shaped ? 0.144 * rows16 : 0)) / 128, start = 3.0 + 1.55 * rows16;
        // about as many splits as there are: half a one more of each unit than its tokens fill
        const double splits = w.longest <= tokens ? w.blocks[nb] : std::max(w.blocks[nb], w.over[nb] / tokens + 0.5 * w.blocks[nb]);
        x.longest = start + std::min(tokens, w.longest) * (bounded ? 0.5 : 1) * step;
        x.groups = splits * s.H;
        x.work = (splits * start + w.seen[nb] * step) * s.H;
        x.again = w.seen[nb] - w.context;
        x.parts = w.longest <= tokens ? w.tokens : std::max(w.tokens, w.parts / tokens + 0.5 * w.tokens);
        return x;
    };
    GroupCut best{};
    double least = 1e30;
    const int most_nb = s.D == 256 ? 1 : 2;   // of 0, 1, 2
    auto consider = [&](int st, int pt, const Part (&of_own_rows)[3], const Part (&of_prefix_rows)[3]) {
        const int of_prefix = splits_of(prefix.longest, pt), of_own = splits_of(own.longest, st), ns = of_prefix + of_own;
        if (ns > most) return;
        for (int k = 0; k < 4; ++k) {   // 1, 2, 4 row groups of both kinds; the most for prefixes alone
            const int of = k == 3 ? 0 : k, of_p = k == 3 ? most_nb : k;
            if (of > most_nb || (k == 3 && prefix.units == 0)) continue;
            if (k > 0 && (k == 3 ? prefix.rows : std::max(own.rows, prefix.rows)) <= 8 << of_p) continue;   // half of the rows would be none
            // workgroups that a compute unit holds, by their LDS
            const bool one_each = s.D == 256 && (s.bits == 16 || (s.bits == 8 && of_p == 1));
            const double slots = one_each ? s.cus : 2 * s.cus, slower = one_each ? 1 : 1.256;
            const Part &o = of_own_rows[of], &f = of_prefix_rows[of_p];
            const double groups = o.groups + f.groups, work = o.work + f.work, longest = std::max(o.longest, f.longest), again = o.again + f.again, parts = o.parts + f.parts;
            // prefixes go first, and others fill what they leave; one kind alone, of unequal lengths, is over a little earlier
            double rounds = 0;
            auto in_rounds = [&](const Part &x, double by) {
                const double r = x.groups / slots;
                rounds = std::max(rounds, (r < 4 ? std::ceil(r - 0.02) : r + 0.5) * x.longest * slower * by);
            };
            if (prefix.units > 0) in_rounds(f, 1);
            else in_rounds(o, 0.8);
            const double memory = (own.context + prefix.context) * row / 10.3 + again * row / 15.8 + 0.345 * longest;
            const double us = (groups <= s.cus ? std::max(longest, memory) : std::max({work * slower / slots + 0.355 * longest, rounds, memory})) +
                              (ns > 1 ? 6.1 + parts * part / 4.37 + 0.047 * ns : 0);
            if (us < least) {
                least = us;
                best = GroupCut{1 << of, 1 << of_p, pt, st, of_prefix, ns, us};
            }
        }
    };
    auto parts_of = [&](const GroupWork &w, int tokens, Part (&to)[3]) {
        for (int nb = 0; nb <= most_nb; ++nb) to[nb] = part_of(w, nb, tokens);
    };
    const int span = std::max(own.longest, prefix.longest);
    auto even = [&](int ns) { return (int)((((long long)span + ns - 1) / ns + 31) / 32 * 32); };
    if (n_splits > 0) {
        for (int ns = n_splits; best.nb == 0 && ns >= 1; --ns) {
            Part o[3], f[3];
            parts_of(own, even(ns), o);
            parts_of(prefix, even(ns), f);
            consider(even(ns), even(ns), o, f);
        }
        return best;
    }
    // lengths of which those past twice a kind's longest say nothing new; the last is the whole
    static constexpr int kLengths[] = {128, 256, 384, 512, 768, 1024, 1536, 2048, 2816, 4096, 8192, 16384};
    constexpr int kN = sizeof(kLengths) / sizeof(*kLengths);
    Part of_prefix_rows[kN + 1][3];
    int n_prefix = 0;
    for (;; ++n_prefix) {
        const bool whole = n_prefix == kN || kLengths[n_prefix] >= prefix.longest;
        parts_of(prefix, whole ? even(1) : kLengths[n_prefix], of_prefix_rows[n_prefix]);
        if (whole) break;
    }
    for (int i = 0; i <= kN; ++i) {
        const bool whole = i == kN || kLengths[i] >= own.longest;
        const int st = whole ? even(1) : kLengths[i];
        Part of_own_rows[3];
        parts_of(own, st, of_own_rows);
        for (int j = 0; j <= n_prefix; ++j) consider(st, j == n_prefix ? even(1) : kLengths[j], of_own_rows, of_prefix_rows[j]);
        if (whole) break;
    }
    return best;
}

// Whether sequences go over their prefixes each for itself, by the estimates of both cuts: K and V of a prefix that several read come out of caches then, and its partial results are spared.
// The estimate misjudges the two by some 15 %, in favour of joined ones where rows are few (17 sequences of 8 to 12 tokens behind 6K: 97 us joined, 76 apart, estimated as 51 and 58), of
// others in long prompts (18 of 429 tokens behind 4K to 10K: 349 and 415 us, 270 and 318). Over 120 drawn batches this choice took 1.1 % longer than the better of both; always apart 15 %,
// always joined 9 %. The largest differences: 10 prompts of 447 to 710 tokens behind 473, 374 us apart and 229 joined; 43 tokens behind two prefixes of 1.2K to 1.6K, 21 and 47.
inline bool better_joined(const GroupCut &joined, const GroupCut &apart, bool chain, long long n_tok, int batch)
{
    return joined.us < (chain && n_tok > 128ll * batch ? 1.15 : 0.85) * apart.us;
}

}  // namespace kvb
