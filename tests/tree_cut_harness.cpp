// Drives the choice of rows and splits of kv_tree_attn without a GPU.  One call per line of the input:
//   D H G bits cus paged B n_splits ws_splits len_0 .. len_{B-1} drafted_0 .. drafted_{B-1}
// ws_splits: the workspace holds that many splits (-1: as many as are ever chosen).  One line of the output each:
//   nb row_blocks ns split_tokens most
#include <cstdio>
#include <vector>

#include "tree_cut.hpp"

int main()
{
    kvb::TreeShape s{};
    int paged = 0, B = 0, n_splits = 0, ws_splits = 0;
    while (std::scanf("%d %d %d %d %d %d %d %d %d", &s.D, &s.H, &s.G, &s.bits, &s.cus, &paged, &B, &n_splits, &ws_splits) == 9) {
        s.paged = paged != 0;
        std::vector<int> lens((size_t)B), first((size_t)B + 1);
        for (auto &n : lens)
            if (std::scanf("%d", &n) != 1) return 1;
        for (int b = 0; b < B; ++b) {
            if (std::scanf("%d", &first[(size_t)b + 1]) != 1) return 1;
            first[(size_t)b + 1] += first[(size_t)b];
        }
        const int most = kvb::tree_most_splits(s, first[(size_t)B]);
        const uint64_t ws = kvb::tree_split_bytes(s, first[(size_t)B]) * (uint64_t)(ws_splits >= 0 ? ws_splits : most);
        const kvb::TreeCut c = kvb::cut_tree(s, B, lens.data(), first.data(), n_splits, ws);
        std::printf("%d %d %d %d %d\n", c.nb, c.row_blocks, c.ns, c.split_tokens, most);
    }
    return 0;
}
