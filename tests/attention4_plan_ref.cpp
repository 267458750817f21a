// Walks the few-row kernel's work over a cache held in 4 bits as its workgroups do, for calls read from stdin:
//   bf16 H G D page rows max_new max_kv window masked B, then new_start[B + 1], kv_len[B].
// Prints many tile_rows wgs aligned, the items worked on, those of them without rows, the highest packed row whose query is
// read (-1: none), the units not worked on exactly once, the parts that the join would look for elsewhere, and the bytes
// of workspace past those that are asked for.
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
        const size_t have = attention4_workspace(c, H, bf16);
        Plan p = make_plan(c, H, bf16, span, true);
        if (plan_bytes(p, c, H) > have) p = make_plan(c, H, bf16, c.max_kv, true);
        long worked = 0, empty = 0, read = -1, wrong = 0, lost = 0, past = (long)plan_bytes(p, c, H) - (long)have;
        int aligned = 0;
        if (!p.many) {
            const int DP = padded(c.D), NT = 64 * kWaves4;
            const int items = c.B * p.tiles, each = (items + NT - 1) / NT, least = join_units4(bf16);
            std::vector<int> n(items), before_chunk(NT + 1, 0), unit_start(items + 1, 0);
            int units = 0, longest = 0;
            for (int t = 0; t < NT; ++t) {
                for (int i = t * each; i < std::min((t + 1) * each, items); ++i) {
                    n[i] = item_units(masked, window, p, load_seq(c, i / p.tiles), i % p.tiles);
                    unit_start[i] = units;
                    units += n[i];
                    longest = std::max(longest, n[i]);
                }
                before_chunk[t + 1] = units;
            }
            unit_start[items] = units;
            const Division cut = divide(units, p.wgs, least_units4(least, longest));
            const int length = each == 1 ? aligned_length(units, items, longest, p.wgs, least, slack4(bf16, DP)) : 0;
            aligned = length > 0;
            std::vector<int> done(units, 0);
            // (item, from, to) of every part, by workgroup
            struct Part {
                int item, from, to;
            };
            std::vector<std::vector<Part>> parts(p.wgs);
            std::vector<int> first(items, 0), count(items, 0);
            if (aligned) {
                int w = 0;
                for (int i = 0; i < items; ++i) {
                    first[i] = w;
                    count[i] = longest <= length ? 1 : aligned_parts(n[i], length);
                    for (int k = 0; k < count[i]; ++k, ++w) {
                        if (w >= p.wgs) {
                            ++wrong;
                            continue;
                        }
                        const int u0 = unit_start[i] + k * length, u1 = std::min(u0 + length, unit_start[i + 1]);
                        if (u0 < u1) parts[w].push_back({i, u0, u1});
                    }
                }
            } else {
                for (int wg = 0; wg < cut.wgs; ++wg) {
                    const int u0 = cut.start(wg), u1 = cut.start(wg + 1);
                    if (u0 == u1) continue;
                    int chunk = 0;
                    while (!(before_chunk[chunk] <= u0 && u0 < before_chunk[chunk + 1])) ++chunk;
                    int item = chunk * each, before = before_chunk[chunk];
                    for (int n_units; before < u1; before += n_units, ++item) {
                        n_units = n[item];
                        if (!works_on(before, n_units, u0)) continue;
                        parts[wg].push_back({item, std::max(u0, before), std::min(u1, before + n_units)});
                    }
                }
                for (int i = 0; i < items; ++i)
                    if (n[i] > 0) {
                        first[i] = cut.owner(unit_start[i]);
                        count[i] = cut.owner(unit_start[i] + n[i] - 1) - first[i] + 1;
                    }
            }
            std::vector<int> found(items, 0);
            for (int wg = 0; wg < p.wgs; ++wg) {
                // two slots: of the item that a stretch begins with, and of one that begins later and goes on
                int later = 0;
                for (const Part& x : parts[wg]) {
                    const Seq s = load_seq(c, x.item / p.tiles);
                    const Tile t = item_tile(p, s, x.item % p.tiles);
                    ++worked;
                    empty += t.rows <= 0;
                    read = std::max(read, (long)s.row0 + std::max(t.i_lo, t.rows > 0 ? t.i_hi : 0));
                    for (int u = x.from; u < x.to; ++u) ++done[u];
                    ++found[x.item];
                    const bool cut_item = x.from != unit_start[x.item] || x.to != unit_start[x.item + 1];
                    if (cut_item && (wg < first[x.item] || wg >= first[x.item] + count[x.item])) ++lost;
                    if (cut_item && x.from != parts[wg][0].from && ++later > 1) ++lost;
                }
            }
            for (int i = 0; i < items; ++i) lost += n[i] > 0 && found[i] != count[i];
            for (int x : done) wrong += x != 1;
            if ((long)p.wgs * c.G > kCounters) ++wrong;
        }
        std::printf("%d %d %d %d %ld %ld %ld %ld %ld %ld\n", p.many, p.tile_rows, p.wgs, aligned, worked, empty, read, wrong, lost,
                    std::max(past, 0L));
    }
}
