// Drives the choice of rows and splits of kv_group_attn without a GPU.  One call per line of the input:
//   D H G bits paged chain n_splits ws_splits B n_groups len.. new.. group_first.. (n_groups + 1) prefix..
// ws_splits: the workspace holds that many partial results of a row (-1: kv_group_attn_workspace's).  One line of the output each:
//   nb prefix_tokens split_tokens prefix_ns ns fit workgroups covered, the last the units whose splits hold all of their tokens.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "group_cut.hpp"

int main()
{
    kvb::TreeShape s{};
    int paged = 0, chain = 0, B = 0, n_groups = 0, n_splits = 0, ws_splits = 0;
    s.cus = 256;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &s.D, &s.H, &s.G, &s.bits, &paged, &chain, &n_splits, &ws_splits, &B, &n_groups) == 10) {
        s.paged = paged != 0;
        auto read = [](int n) {
            std::vector<int> v((size_t)n);
            for (auto &x : v)
                if (std::scanf("%d", &x) != 1) std::abort();
            return v;
        };
        const std::vector<int> lens = read(B), news = read(B), group_first = read(n_groups + 1), prefix = read(n_groups);
        std::vector<int> first((size_t)B + 1);
        int longest = 0;
        for (int b = 0; b < B; ++b) {
            first[(size_t)b + 1] = first[(size_t)b] + news[(size_t)b];
            longest = std::max(longest, lens[(size_t)b]);
        }
        std::vector<kvb::GroupUnit> units;
        for (int i = 0; i < n_groups + B; ++i) {
            int shared = 0;
            for (int g = 0; g < n_groups; ++g)
                if (i - n_groups >= group_first[(size_t)g] && i - n_groups < group_first[(size_t)g + 1]) shared = prefix[(size_t)g];
            const kvb::GroupUnit u = kvb::group_unit(i, n_groups, group_first.data(), prefix.data(), lens.data(), first.data(), shared);
            if (u.tokens > 0 && u.span > 0) units.push_back(u);
        }
        const long long n_tok = first[(size_t)B];
        const uint64_t one = kvb::tree_split_bytes(s, n_tok), ws = ws_splits >= 0 ? one * (uint64_t)ws_splits : kvb::group_workspace_bytes(s, n_tok, (long long)longest + n_tok);
        const kvb::GroupCut c = kvb::cut_group(s, units.data(), (int)units.size(), chain != 0, n_tok % 2 != 0, n_tok % 3 == 0, n_splits, ws, n_tok);
        uint64_t groups = 0, covered = 0;
        for (const auto &u : units) {
            const int st = u.prefix ? c.prefix_tokens : c.split_tokens, most = u.prefix ? c.prefix_ns : c.ns - c.prefix_ns;
            groups += kvb::unit_workgroups(s, u, u.prefix ? c.nb_prefix : c.nb, st);
            covered += kvb::splits_of(u.span, st) <= most;
        }
        std::printf("%d %d %d %d %d %d %llu %llu %d\n", c.nb, c.prefix_tokens, c.split_tokens, c.prefix_ns, c.ns, (int)std::min<uint64_t>(ws / one, 1u << 30), (unsigned long long)groups,
                    (unsigned long long)covered, (int)units.size());
    }
    return 0;
}
