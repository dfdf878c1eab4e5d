// Tells without a GPU which kernels of kv_group_attn a call takes, from the same choice as the call's.  One call per line of the input:
//   D H G bits paged chain bounded shaped n_splits B n_groups len.. new.. group_first.. (n_groups + 1) prefix..
// One line of the output each:
//   path nb nb_prefix ns prefix_ns, path: 0 no prefix that anybody shares, 1 prefixes apart, 2 each sequence over its own.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "group_cut.hpp"

int main()
{
    kvb::TreeShape s{};
    int paged = 0, chain = 0, bounded = 0, shaped = 0, n_splits = 0, B = 0, n_groups = 0;
    s.cus = 256;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d", &s.D, &s.H, &s.G, &s.bits, &paged, &chain, &bounded, &shaped, &n_splits, &B, &n_groups) == 11) {
        s.paged = paged != 0;
        auto read = [](int n) {
            std::vector<int> v((size_t)n);
            for (auto &x : v)
                if (std::scanf("%d", &x) != 1) std::abort();
            return v;
        };
        const std::vector<int> lens = read(B), news = read(B), group_first = read(n_groups + 1), prefix = read(n_groups);
        std::vector<int> first((size_t)B + 1);
        for (int b = 0; b < B; ++b) first[(size_t)b + 1] = first[(size_t)b] + news[(size_t)b];
        const long long n_tok = first[(size_t)B];
        const int longest = *std::max_element(lens.begin(), lens.end());
        // the workspace that a caller is told to bring, for rows of 16 bits
        const uint64_t ws = kvb::group_workspace_bytes(kvb::TreeShape{s.D, s.H, s.G, 16, s.cus, false}, n_tok, (long long)longest + n_tok);
        std::vector<kvb::GroupUnit> units, own;
        bool any_prefix = false;
        for (int i = 0; i < n_groups + B; ++i) {
            int shared = 0;
            for (int g = 0; g < n_groups; ++g)
                if (i - n_groups >= group_first[(size_t)g] && i - n_groups < group_first[(size_t)g + 1]) shared = prefix[(size_t)g];
            const kvb::GroupUnit u = kvb::group_unit(i, n_groups, group_first.data(), prefix.data(), lens.data(), first.data(), shared);
            if (u.tokens > 0 && u.span > 0) {
                units.push_back(u);
                any_prefix = any_prefix || u.prefix;
            }
        }
        for (int b = 0; b < B; ++b) {
            const kvb::GroupUnit u = kvb::group_unit(b, 0, nullptr, nullptr, lens.data(), first.data(), 0);
            if (u.tokens > 0 && u.span > 0) own.push_back(u);
        }
        kvb::GroupCut c = kvb::cut_group(s, units.data(), (int)units.size(), chain != 0, bounded != 0, shaped != 0, n_splits, ws, n_tok);
        int path = any_prefix ? 1 : 0;
        if (any_prefix && n_splits == 0) {
            const kvb::GroupCut joined = kvb::cut_group(s, own.data(), (int)own.size(), chain != 0, bounded != 0, shaped != 0, 0, ws, n_tok);
            if (kvb::better_joined(joined, c, chain != 0, n_tok, B)) {
                c = joined;
                path = 2;
            }
        }
        std::printf("%d %d %d %d %d\n", path, c.nb, c.nb_prefix, c.ns, c.prefix_ns);
    }
    return 0;
}
