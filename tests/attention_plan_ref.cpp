// Walks the few-row attention kernel's work as its workgroups do, for calls read from stdin:
//   bf16 H G D page rows max_new max_kv window masked B, then new_start[B + 1], kv_len[B].
// Prints many tile_rows tiles parts wgs, the items worked on, those of them without rows, the highest packed
// row whose query is read (-1: none) and the units that are not worked on exactly once.
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
        const Plan p = make_plan(c, H, bf16, span);
        long worked = 0, empty = 0, read = -1, wrong = 0;
        if (!p.many) {
            const int DP = padded(c.D), NT = 64 * stream_waves(DP, p.tile_rows / 16);
            const int items = c.B * p.tiles, each = (items + NT - 1) / NT;
            std::vector<int> n(items), before_chunk(NT + 1, 0);
            int units = 0, longest = 0;
            for (int t = 0; t < NT; ++t) {
                for (int i = t * each; i < std::min((t + 1) * each, items); ++i) {
                    n[i] = item_units(masked, window, p, load_seq(c, i / p.tiles), i % p.tiles);
                    units += n[i];
                    longest = std::max(longest, n[i]);
                }
                before_chunk[t + 1] = units;
            }
            const int least = join_units(bf16);
            const Division cut = divide(units, p.wgs, least);
            const bool whole = each == 1 && items <= p.wgs && longest <= units / p.wgs + 1 + least;
            auto at = [&](int w) { return whole ? before_chunk[std::min(w, items)] : cut.start(w); };
            std::vector<int> done(units, 0);
            for (int wg = 0; wg < (whole ? items : cut.wgs); ++wg) {
                const int u0 = at(wg), u1 = at(wg + 1);
                if (u0 == u1) continue;
                int chunk = 0;
                while (!(before_chunk[chunk] <= u0 && u0 < before_chunk[chunk + 1])) ++chunk;
                int item = chunk * each, before = before_chunk[chunk];
                for (int n_units; before < u1; before += n_units, ++item) {
                    n_units = n[item];
                    if (!works_on(before, n_units, u0)) continue;
                    const Seq s = load_seq(c, item / p.tiles);
                    const Tile t = item_tile(p, s, item % p.tiles);
                    ++worked;
                    empty += t.rows <= 0;
                    read = std::max(read, (long)s.row0 + std::max(t.i_lo, t.rows > 0 ? t.i_hi : 0));
                    for (int u = std::max(u0, before); u < std::min(u1, before + n_units); ++u) ++done[u];
                }
            }
            for (int x : done) wrong += x != 1;
        }
        std::printf("%d %d %d %d %d %ld %ld %ld %ld\n", p.many, p.tile_rows, p.tiles, p.parts, p.wgs, worked, empty, read, wrong);
    }
}
