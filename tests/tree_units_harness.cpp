// Which workgroups of a ragged kv_tree_attn launch have tokens to go over, without a GPU.  One call per line of the input:
//   D H G n_splits ws_splits B len_0 .. len_{B-1} drafted_0 .. drafted_{B-1}
// One line of the output each: workgroups, those without tokens, and the tokens of the others, summed over sequences, heads and row blocks.
#include <algorithm>
#include <cstdio>
#include <vector>

#include "tree_cut.hpp"

int main()
{
    kvb::TreeShape s{};
    int n_splits = 0, ws_splits = 0, B = 0;
    s.bits = 8;
    s.cus = 256;
    while (std::scanf("%d %d %d %d %d %d", &s.D, &s.H, &s.G, &n_splits, &ws_splits, &B) == 6) {
        std::vector<int> lens((size_t)B), first((size_t)B + 1);
        for (auto &n : lens)
            if (std::scanf("%d", &n) != 1) return 1;
        for (int b = 0; b < B; ++b) {
            if (std::scanf("%d", &first[(size_t)b + 1]) != 1) return 1;
            first[(size_t)b + 1] += first[(size_t)b];
        }
        const kvb::TreeCut c = kvb::cut_tree(s, B, lens.data(), first.data(), n_splits, kvb::tree_split_bytes(s, first[(size_t)B]) * (uint64_t)ws_splits);
        long long groups = 0, idle = 0, tokens = 0;
        for (int b = 0; b < B; ++b) {
            const int n = first[(size_t)b + 1] - first[(size_t)b], total = lens[(size_t)b] + n;
            if (n == 0) continue;
            unsigned units = ((unsigned)(total - 1) / (unsigned)c.split_tokens + 1) * (unsigned)s.H;
            if (c.row_blocks > 1) units = (units + 7) & ~7u;
            const int blocks = (n * s.G + 16 * c.nb - 1) / (16 * c.nb);
            for (unsigned unit = 0; unit < units; ++unit) {
                const unsigned split = unit / (unsigned)s.H;
                groups += blocks;
                if (!kvb::split_has_tokens(split, c.split_tokens, total)) {
                    idle += blocks;
                    continue;
                }
                const int s0 = (int)split * c.split_tokens, s1 = std::min(s0 + c.split_tokens, total);   // as the kernel has them
                tokens += (long long)(s1 - s0) * blocks;
            }
        }
        std::printf("%lld %lld %lld %d %d\n", groups, idle, tokens, c.nb, c.split_tokens);
    }
    return 0;
}
