// psd_attention_plan.hpp -- how a call over the paged cache is cut: its sequences with the host's bounds
// applied, the attention's tiles and parts, and the division of the few-row kernel's work among its
// workgroups (host and device; internal to libpsd).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "psd_layout.hpp"

#ifdef __HIPCC__
#define PSD_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define PSD_HOST_DEVICE inline
#endif

namespace psd {

PSD_HOST_DEVICE int lesser(int a, int b) { return a < b ? a : b; }
PSD_HOST_DEVICE int greater(int a, int b) { return a > b ? a : b; }

// Where a sequence's cached tokens lie (psd_cache, psd_seqs of the C ABI).
struct CacheArgs {
    void* k;
    void* v;
    int64_t stride_layer, stride_page, stride_token, stride_head;  // elements
    int G, D, P, pages, layers;
    int B, rows, max_new, max_kv, table_width;
    int64_t table_stride;
    const int32_t* new_start;
    const int32_t* kv_len;
    const int32_t* table;
};

// One sequence of the call, with the host's bounds applied.
struct Seq {
    int row0;   // packed row of its first new token
    int n;      // new tokens computed (at most max_new, rows inside the call's)
    int first;  // cache position of its first new token (may be negative)
    int kv;     // cached tokens that can be seen (positions [0, kv))
    int total;  // its new tokens, computed or not
};
PSD_HOST_DEVICE Seq load_seq(const CacheArgs& c, int b) {
    // lengths that no call can have are cut, so that positions and their differences stay inside 32 bits
    Seq s;
    const int lo = greater(c.new_start[b], 0), hi = lesser(c.new_start[b + 1], 1 << 24);
    const int len = lesser(greater(c.kv_len[b], 0), 1 << 30);
    const int total = greater(hi - lo, 0);
    s.total = total;
    s.row0 = lo;
    s.n = lesser(lesser(total, c.max_new), greater(c.rows - s.row0, 0));
    s.first = len - total;
    const long width = (long)c.table_width * c.P;
    const int held = width < c.max_kv ? (int)width : c.max_kv;
    s.kv = greater(lesser(lesser(len, c.max_kv), held), 0);
    return s;
}

// How a call is cut, by the host's bounds alone.
struct Plan {
    int h;          // rows per new token: H / G
    int tile_rows;  // rows of a workgroup
    int tiles;      // row tiles of the longest sequence
    int wgs;        // few rows: workgroups of each key/value head
    bool many;      // many rows: tile_kernel, with
    int parts;      // parts of the longest range of cached tokens and
    int chunk;      // cached tokens of a part
    int page_shift; // log2 of the page size, or -1
};

constexpr int kUnit = 128;  // cached tokens: a block of each wave (two in float32)
// Units that a workgroup has at least, if it has to join: leaving and joining the parts of an item
// takes as long as about so many (4 bfloat16 sequences of up to 512 tokens 13 us, with 2 units 20; under a
// far bound 8 sequences of 5 rows, up to 1500 tokens 28, with 8 units 40).  A float32 unit takes so much longer that
// joins pay from one on (37 tokens of 12 heads 38 us, with 4 units 49).
constexpr int join_units(bool bf16) { return bf16 ? 4 : 1; }

// Threads of the few-row kernel: one workgroup a CU, two waves a SIMD, or one where the rows' outputs take
// the registers of two.
constexpr int stream_waves(int DP, int RB) { return RB * DP >= 512 || DP == 256 ? 4 : 8; }

struct Range {
    int lo, hi;  // cached positions that some row of a tile sees
};

// Rows of new tokens [i_lo, i_hi] of a sequence see positions [lo, hi) at most.
PSD_HOST_DEVICE Range tile_range(bool masked, int window, const Seq& s, int i_lo, int i_hi) {
    Range r;
    r.lo = 0;
    r.hi = s.kv;
    if (!masked) {
        r.hi = greater(lesser(s.kv, s.first + i_hi + 1), 0);
        if (window > 0) r.lo = lesser(greater(s.first + i_lo - window + 1, 0), r.hi);
    }
    return r;
}

// An item of the few-row kernel: row tile `tile` of a sequence.
struct Tile {
    int row0, rows;  // rows <= 0: the sequence has none there
    int i_lo, i_hi;  // new tokens
};
PSD_HOST_DEVICE Tile item_tile(const Plan& p, const Seq& s, int tile) {
    Tile t;
    t.row0 = tile * p.tile_rows;
    t.rows = lesser(s.n * p.h - t.row0, p.tile_rows);
    t.i_lo = t.row0 / p.h;
    t.i_hi = (t.row0 + t.rows - 1) / p.h;
    return t;
}

// Its length in units; 0 without rows, and at least 1 with them.
PSD_HOST_DEVICE int item_units(bool masked, int window, const Plan& p, const Seq& s, int tile) {
    const Tile t = item_tile(p, s, tile);
    if (t.rows <= 0) return 0;
    const Range range = tile_range(masked, window, s, t.i_lo, t.i_hi);
    return greater((range.hi - range.lo + kUnit - 1) / kUnit, 1);
}

// All items' units in a row, cut into stretches of the same length: of R workgroups the first W mod R
// have W / R + 1 units.
struct Division {
    int wgs, share, more;
    PSD_HOST_DEVICE int start(int w) const { return w * share + lesser(w, more); }
    PSD_HOST_DEVICE int owner(int u) const {
        return u < more * (share + 1) ? u / (share + 1) : more + (u - more * (share + 1)) / share;
    }
};
PSD_HOST_DEVICE Division divide(int units, int wgs, int least_units) {
    Division d;
    d.wgs = lesser(wgs, greater(units / least_units, 1));
    d.share = units / d.wgs;
    d.more = units - d.share * d.wgs;
    return d;
}

// Does a workgroup whose stretch begins at unit u0 work on an item that begins at unit `before`, below the
// stretch's end?  An item without units has no rows, wherever it lies.
PSD_HOST_DEVICE bool works_on(int before, int n_units, int u0) { return n_units > 0 && before + n_units > u0; }

constexpr int kMaxParts = 64;   // join_kernel holds a part's weight in a lane
constexpr int kMinChunk = 256;  // tile_kernel: cached tokens of a part at least
// A block's time in 8 waves of one workgroup to that in 4 of each of two (D=128, 2048 tokens behind 14336:
// 568 us and 624; D=64: 388 and 402; 8 x 512 behind 1536: 110 and 114; 4 x 2048 behind none: 118 and 115,
// where the wider tile's triangle costs more).
constexpr double kWide = 0.9;
constexpr int kCus = 256;

inline int padded(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

inline Plan make_plan(const CacheArgs& c, int H, bool bf16, int span) {
    Plan p;
    p.h = H / c.G;
    const long most = (long)c.max_new * p.h;
    // tile_kernel for more rows than the other has registers for, and for fewer over a cache of up to 2^19
    // tokens of all key/value heads (2^20 with more than 32 rows; a fourth of either where a head's outputs
    // leave one workgroup a CU), which end before the other's division and joins pay.  D=128, G=8, us here
    // and there: 4 rows, 8 x 1500 18 and 24, 2 x 8000 20 and 25, 16 x 4096 43 and 42, 32 x 4096 74 and 66;
    // 20 rows, 64 x 1024 39 and 54, 16 x 4096 43 and 45, 32 x 4096 78 and 70; 48 rows, 64 x 1024 44 and 79,
    // 64 x 4096 163 and 160; D=256, G=4, 48 rows, 16 x 4096 70 and 99, 4 rows 65 and 43.  Up to 32 rows stay
    // there where it has a workgroup for each sequence and no more to gain by joins: 4 rows, 4 x 512 15 and
    // 13, 32 x 1000 31 and 23 (64 x 512, two sequences a workgroup: 24 and 33).  With one or two heads tile_kernel
    // has 64 or 128 parts for 256 CUs and is ahead all the same, since one workgroup joins a long item there: 8 rows,
    // G=1, 1 x 8192 15 and 22, 1 x 131072 59 and 107, 4 x 131072 59 and 68; G=2, 1 x 131072 59 and 73; 48 rows, G=1,
    // 1 x 131072 60 and 245.
    const long tokens = (long)c.B * c.G * span * (c.D > 128 ? 4 : 1);
    const long units = (span + kUnit - 1) / kUnit;
    const bool alone = (long)c.B * c.G <= kCus && units <= units * c.B * c.G / kCus + 5;
    p.many = bf16 && (most > 64 || (most > 32 ? tokens <= 1 << 20 : tokens <= 1 << 19 && !alone));
    p.wgs = p.parts = p.chunk = 0;
    if (!p.many) {
        // float32 rows in tiles of 32 while tiles of 64 would leave CUs without one (12 heads of 80, 37 tokens
        // of 6 sequences: 40 us and 45; 1024 new of 4096 tokens of 16 heads, CUs full: 450 and 408)
        const bool few = !bf16 && c.D > 64 && (long)c.B * c.G * ((most + 63) / 64) < kCus;
        const int limit = c.D > 128 || few ? 32 : 64;
        p.tile_rows = most <= 16 ? 16 : most <= 32 ? 32 : limit;
        p.tiles = (int)((most + p.tile_rows - 1) / p.tile_rows);
        p.wgs = std::max(kCus / c.G, 1);  // one a CU
    } else {
        // Rows of a workgroup and parts of the longest range, by the time they take in 64-token blocks:
        // every round of resident workgroups takes a part and about 3 blocks to start and end; the join of
        // 2 parts of 512 groups of 128 rows took as long as 13 blocks.
        double best = -1;
        for (int rows = 128; rows <= (c.D > 128 ? 128 : 256); rows *= 2) {
            const long tiles = (most + rows - 1) / rows, groups = (long)c.B * c.G * tiles;
            const long resident = kCus * (c.D > 128 || rows == 256 ? 1 : 2);
            for (int parts = 1; parts <= kMaxParts && (parts - 1) * kMinChunk < span; ++parts) {
                const int chunk = ((span + parts - 1) / parts + kMinChunk - 1) / kMinChunk * kMinChunk;
                const double rounds = (double)((groups * parts + resident - 1) / resident);
                const double join = parts > 1 ? 1.5 + groups * parts * (rows / 128) * (13.0 / 1024) : 0;
                const double cost = rounds * (chunk / 64.0 + 3) * (rows == 256 ? kWide : 1.0) + join;
                if (best >= 0 && cost >= best) continue;
                best = cost;
                p.tile_rows = rows;
                p.tiles = (int)tiles;
                p.chunk = chunk;
            }
        }
        p.parts = (span + p.chunk - 1) / p.chunk;
    }
    p.page_shift = -1;
    for (int k = 0; k <= 16; ++k)
        if (c.P == 1 << k) p.page_shift = k;
    return p;
}

// The workspace: a counter for each workgroup of the few-row kernel (zero between calls), then
// what workgroups leave for the join.
constexpr int kCounters = 1024;
constexpr int kCounterFloats = kCounters;

inline size_t plan_bytes(const Plan& p, const CacheArgs& c, int H) {
    if (!p.many)
        return align256(kCounterFloats * 4 + (size_t)p.wgs * c.G * 2 * p.tile_rows * (padded(c.D) + 2) * 4);
    return p.parts == 1 ? 0 : align256(kCounterFloats * 4 + (size_t)p.parts * c.rows * H * (c.D + 2) * 4);
}

inline size_t attention_workspace(const CacheArgs& c, int H, bool bf16) { return plan_bytes(make_plan(c, H, bf16, c.max_kv), c, H); }

// The launch stays inside a grid's limits.
inline bool attention_fits(const CacheArgs& c, int H, bool bf16) {
    const Plan p = make_plan(c, H, bf16, c.max_kv);
    if (!p.many) return (long)c.B * p.tiles * (c.max_kv / kUnit + 2) < 1L << 30;  // units
    return (long)c.B * c.G * p.tiles * p.parts < 1L << 23;
}

}  // namespace psd
