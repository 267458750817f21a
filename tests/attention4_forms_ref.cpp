// The form that attention over a cache held in 4 bits takes, for calls read from stdin as attention4_plan_ref.cpp does:
// prints many, the padded head size, the rows of a tile, whether stretches end where sequences end (few rows), and whether some
// sequence is cut into parts that are joined.
#include <cstdio>
#include <vector>

#include "../paper_2609_21858_amd/csrc/psd_attention_plan.hpp"

using namespace psd;

int main() {
    int bf16, H, masked, window;
    CacheArgs c = {};
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d", &bf16, &H, &c.G, &c.D, &c.P, &c.rows, &c.max_new, &c.max_kv, &window,
                      &masked, &c.B) == 11) {
        std::vector<int32_t> start(c.B + 1), kv(c.B);
        for (auto& x : start)
            if (std::scanf("%d", &x) != 1) return 1;
        for (auto& x : kv)
            if (std::scanf("%d", &x) != 1) return 1;
        c.new_start = start.data();
        c.kv_len = kv.data();
        c.table_width = (c.max_kv + c.P - 1) / c.P;
        const int span = window > 0 ? (int)std::min<long>(c.max_kv, (long)window + c.max_new - 1) : c.max_kv;
        Plan p = make_plan(c, H, bf16, span, true);
        if (plan_bytes(p, c, H) > attention4_workspace(c, H, bf16)) p = make_plan(c, H, bf16, c.max_kv, true);
        const int items = c.B * p.tiles;
        int aligned = 0, joined = 0;
        if (p.many) {
            for (int i = 0; i < items; ++i) {
                const Seq s = load_seq(c, i / p.tiles);
                const Tile t = item_tile(p, s, i % p.tiles);
                if (t.rows <= 0) continue;
                const Range r = tile_range(masked, window, s, t.i_lo, t.i_hi);
                joined |= r.hi - r.lo > p.chunk;
            }
        } else {
            std::vector<int> before(items + 1, 0);
            int longest = 0;
            for (int i = 0; i < items; ++i) {
                const int n = item_units(masked, window, p, load_seq(c, i / p.tiles), i % p.tiles);
                before[i + 1] = before[i] + n;
                longest = std::max(longest, n);
            }
            const int units = before[items], least = join_units4(bf16);
            const int length = items <= 64 * kWaves4 ? aligned_length(units, items, longest, p.wgs, least, slack4(bf16, padded(c.D))) : 0;
            const Division cut = divide(units, p.wgs, least_units4(least, longest));
            aligned = length > 0;
            for (int i = 0; i < items; ++i)
                if (before[i] < before[i + 1])
                    joined |= aligned ? longest > length && before[i + 1] - before[i] > length
                                      : cut.owner(before[i]) != cut.owner(before[i + 1] - 1);
        }
        std::printf("%d %d %d %d %d\n", p.many, padded(c.D), p.tile_rows, aligned, joined);
    }
}
