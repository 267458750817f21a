// psd_attention.hip -- attention of a block's new tokens over a paged cache (gfx950).
//
//   s_j = scale q . k_j over the cached tokens j that a row sees,
//   out = sum_j exp(s_j - lse) v_j,  lse = ln sum_j exp(s_j),
// in one pass over the cache with a running maximum m and sum l of the softmax: a new maximum
// m' rescales the sum and the output by exp(m - m').  Scores are kept in units of ln 2.
//
// The query heads of one key/value head and the new tokens are the rows of one matrix: row r of
// (sequence b, head g) is head g * h + r % h of new token r / h, h = H / G.  So a key or value
// that is read serves every row, and a block of drafted tokens costs little more than one.
//
// Both products keep the rows in the columns of their result, so that the softmax
// weights come out of the first product where the second wants them:
//   S^T = K Q^T      (A = keys, B = queries):   lane (r, q) of a 16x16 tile holds row r's scores of
//                                               tokens 4q .. 4q + 3
//   O^T = V^T P^T    (A = values, B = weights): wants from lane (r, q) row r's weights of 8 tokens;
//                                               a sum's order is free, so these are the tokens the
//                                               lane has, and only V is arranged to match.
// A lane then rescales its own column: maximum, sum and output of a row share its lanes.
#include <hip/hip_runtime.h>

#include "psd_attention_device.hpp"
#include "psd_attention_tile.hpp"

namespace psd {

namespace {

// A block's softmax weights of this lane's row as a B operand.  In bfloat16 they are rounded to it, since the
// matrix instructions take both operands in one type, and a second product of what the rounding left out would
// double the half of the products that are O^T = V^T P^T.  Each weight errs by 2^-8 of itself at most; maxima, sums
// (of the weights before they are rounded), lse and outputs stay in float32.  Normally distributed inputs: outputs
// 2.3e-3 of their size from those of 64 bits, where the rounding of the result alone is 1.7e-3.
template <bool BF16>
struct Weights {
    u32x4 all;
    __device__ void take(const f32x4 (&w)[BF16 ? 2 : 1]) {
        if constexpr (BF16)
            all = u32x4{pack_bf16(w[0][0], w[0][1]), pack_bf16(w[0][2], w[0][3]), pack_bf16(w[1][0], w[1][1]),
                        pack_bf16(w[1][2], w[1][3])};
        else
            all = __builtin_bit_cast(u32x4, w[0]);
    }
};

// 16 bytes of a bfloat16 value, which one workgroup reads for all its rows, once: a whole row at a time,
// it need not stay in a cache.  (A key's 128-byte line is read by two instructions, so keys stay.
// 32 x up to 16384 tokens: 236 us; neither 256, both 250.)  Float32 rows may be several tiles.
template <bool BF16>
__device__ __forceinline__ u32x4 stream_load(const char* at) {
    if constexpr (BF16) return __builtin_nontemporal_load((const u32x4*)at);
    return *(const u32x4*)at;
}

// ---------------------------------------------------------------- few rows

// Up to 16 RB rows of one (sequence, key/value head) over a stretch of its cache.  The waves of
// a workgroup take blocks of TOK tokens in turn, each with a softmax of its own, joined at the
// end; no wave waits for another in between.  Keys go from memory straight into the A operand
// (a lane's 16 bytes are consecutive dimensions of one token); values pass through the wave's own
// LDS, where bfloat16 is transposed by ds_read_b64_tr_b16 (16 lanes read a 4-token by 16-dimension
// tile and each gets one dimension's 4 tokens).  While a block is computed, the next one's
// keys and values are on their way into registers.
//
// Lengths are known on the device alone, so the device divides the work: an item is a row tile of a
// sequence, its length the 128-token units it sees, and each of a head's R workgroups (one a CU)
// takes an equal stretch of all items' W units in a row.  An item
// inside one workgroup's stretch is finished by it; of an item that is cut, every workgroup leaves its
// output, maximum and sum in the workspace, and the one that leaves last joins them.
//
// Memory bounds it, a key/value element for every 2 RB x 16 products: H=32, G=8, D=128, bfloat16, 32 sequences
// of one new token and up to 16384 cached, 1.37 GB: 237 us, 5.75 TB/s (a plain read of memory in the same
// order reads 5.9 - 6.2); 5 new tokens of 64 sequences, up to 4096 cached, 676 MB: 137 us.  One token of 4
// sequences, up to 512 cached: 13 us, of them 2 to divide the work, 2 to the first key, 5 in the loop and
// 2 to join.
// Float32, one token of 32 sequences, up to 4096 cached, 683 MB: 131 us; up to 16384: 452, 6.0 TB/s, memory again.
// More rows: 5 tokens of 32 sequences, up to 4096 cached, 239; 1024 new of 4096 804, 75 TFLOP/s (a library
// product 153).  Tiles of 32 and 64 rows spill there: DP=128 43 - 63 registers, DP=256 126 - 161, DP=64 with 64 rows 5 - 14
// (in bfloat16 DP=256 with 32 rows, 26 - 59).  12 heads of 80, 37 tokens, window 700: 38 us with the products busy 13 %
// of it.  About 25 are the same for any length (without a window 300 cached tokens take 26, 3000 65, 6000 105): starts of
// stretches of one or two units, 135 KB of the waves' outputs joined through LDS, parts.  Heads of 64, unpadded: 25.
template <bool BF16, int DP>
struct StreamShape {
    static constexpr int TOK = BF16 ? 32 : 16;
    static constexpr int TT = TOK / 16;                  // 16-token tiles of a block
    static constexpr int VEC = BF16 ? 8 : 4;             // elements of 16 bytes
    static constexpr int KSTEP = 4 * VEC;                // dimensions that a 16-byte piece per lane covers
    static constexpr int KK = DP / KSTEP;
    static constexpr int LPR = DP / VEC;                 // lanes of a value row
    static constexpr int TPI = 64 / LPR;                 // value rows of one load
    static constexpr int NV = TOK / TPI;
    // row pitch of the values in LDS (elements): the 16 rows that a transposing read touches
    // (bfloat16, 32 bytes each), or the 4 (float32, 64 bytes each), fall on all 64 banks evenly
    static constexpr int PITCH = BF16 ? DP + 16 : DP + 4;
    static constexpr int V_BYTES = TOK * PITCH * (BF16 ? 2 : 4);
};

// The waves' values; at an item's end, their outputs (rows of DP + 4 floats: the 16 rows of a store
// fall on different banks).
template <bool BF16, int DP, int RB>
constexpr int stream_lds() {
    using S = StreamShape<BF16, DP>;
    constexpr int values = stream_waves(DP, RB) * S::V_BYTES;
    constexpr int join = stream_waves(DP, RB) * 16 * RB * (DP + 4) * 4;
    return values > join ? values : join;
}

template <bool BF16, int DP, int RB, bool FULL>
__global__ __launch_bounds__(64 * stream_waves(DP, RB), 1) void stream_kernel(AttentionArgs a, Plan p) {
    using S = StreamShape<BF16, DP>;
    using E = Elem<BF16>;
    constexpr int DB = DP / 16;
    constexpr int NW = stream_waves(DP, RB), NT = 64 * NW;
    constexpr int ROWS = 16 * RB;
    __shared__ __align__(16) char s_mem[stream_lds<BF16, DP, RB>()];
    __shared__ int64_t s_off[NW][2][S::TOK];
    __shared__ StreamShared<NT, ROWS> sh;

    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int r = lane & 15, q = lane >> 4;
    const int g = blockIdx.x % c.G, wg = blockIdx.x / c.G;

    const Stretch st = find_stretch<0>(a, p, sh, wg, join_units(BF16));
    if (st.u0 == st.u1) return;
    const float sc = a.scale * kLog2e;
    const int64_t head_at = (int64_t)g * c.stride_head;
    char* s_v = s_mem + wave * S::V_BYTES;

    int item = st.item, before = st.before;
    for (int n_units; before < st.u1; before += n_units, ++item) {
        const Seq s = uniform(st.each == 1 ? sh.seq[item] : load_seq(c, item / p.tiles));
        n_units = st.each == 1 ? uniform(sh.units[item + 1]) - before
                               : uniform(item_units(a.mask != nullptr, a.window, p, s, item % p.tiles));
        if (!works_on(before, n_units, st.u0)) continue;
        const int b = item / p.tiles, tile = item - b * p.tiles;
        const Tile its = item_tile(p, s, tile);
        const int row0 = its.row0, rows = its.rows;
        const int i_lo = uniform(its.i_lo), i_hi = uniform(its.i_hi);
        const Range range = tile_range(a, s, i_lo, i_hi);
        const int from = max(st.u0, before), to = min(st.u1, before + n_units);
        const int c0 = range.lo + (from - before) * kUnit, c1 = min(range.lo + (to - before) * kUnit, range.hi);
        const int blocks = (c1 - c0 + S::TOK - 1) / S::TOK;
        const int32_t* table = c.table + (int64_t)b * c.table_stride;

        auto clamp = [&](int d) { return FULL ? d : min(d, c.D - S::VEC); };
        // this lane's rows, and their queries as B operands
        int row_i[RB];
        u32x4 qf[RB][S::KK];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int rr = row0 + rb * 16 + r;
            const bool on = rb * 16 + r < rows;
            row_i[rb] = on ? rr / p.h : i_lo;
            const int head = g * p.h + (on ? rr - row_i[rb] * p.h : 0);
            const char* src = (const char*)a.q.data +
                              ((int64_t)(s.row0 + row_i[rb]) * a.q.stride_row + (int64_t)head * a.q.stride_head) * E::kBytes;
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) {
                const int d = kk * S::KSTEP + q * S::VEC;
                qf[rb][kk] = *(const u32x4*)(src + clamp(d) * E::kBytes);
            }
        }
        // (unconditional loads; rows and dimensions that are not there count as zero)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) {
                const bool none = rb * 16 + r >= rows || kk * S::KSTEP + q * S::VEC >= c.D;
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[rb][kk][e] = none ? 0u : qf[rb][kk][e];
            }

        f32x4 o[RB][DB];
        float m[RB], l[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            m[rb] = kNoScore;
            l[rb] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // A block's tokens: lane t < TOK finds token t's place; -1: nothing there.  The page number is loaded
        // a block before it is used, so that no load in between has to be waited for with it.
        auto token_of = [&](int blk) { return c0 + blk * S::TOK + lane; };
        auto page_of = [&](int blk) {
            const int j = token_of(blk);
            const int at = lane < S::TOK && j < c1 ? j : 0;
            return table[p.page_shift >= 0 ? at >> p.page_shift : at / c.P];
        };
        auto place = [&](int blk, int page) -> int64_t {
            const int j = token_of(blk);
            const int pi = p.page_shift >= 0 ? j >> p.page_shift : j / c.P;
            if (lane >= S::TOK || j >= c1 || (unsigned)page >= (unsigned)c.pages) return -1;
            return (int64_t)page * c.stride_page + (int64_t)(j - pi * c.P) * c.stride_token;
        };
        // Loads are unconditional: a token that is not there reads the pool's first one instead, whose
        // scores are masked and whose values are zeroed, and a piece past the head's end reads its
        // last piece, which counts as zero in a key and goes to no output in a value.
        // float32 products bound their kernel, so those past the head's end are left out
        auto in_head = [&](int d) { return FULL || BF16 || d < c.D; };
        u32x4 kf[S::TT][S::KK], vf[S::NV];
        auto load_keys = [&](int slot) {
#pragma unroll
            for (int t = 0; t < S::TT; ++t) {
                const char* src = (const char*)c.k + (s_off[wave][slot][16 * t + r] + head_at) * E::kBytes;
#pragma unroll
                for (int kk = 0; kk < S::KK; ++kk)
                    kf[t][kk] = *(const u32x4*)(src + clamp(kk * S::KSTEP + q * S::VEC) * E::kBytes);
            }
        };
        auto load_values = [&](int slot) {
            const int d = clamp((lane % S::LPR) * S::VEC);
            const char* src = (const char*)c.v + (head_at + d) * E::kBytes;
#pragma unroll
            for (int k = 0; k < S::NV; ++k)
                vf[k] = stream_load<BF16>(src + s_off[wave][slot][k * S::TPI + lane / S::LPR] * E::kBytes);
        };
        auto wave_sync = [&]() {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };

        int64_t off = place(wave, page_of(wave));
        int page_next = page_of(wave + NW);
        if (lane < S::TOK) s_off[wave][0][lane] = max(off, (int64_t)0);
        wave_sync();
        load_keys(0);
        __builtin_amdgcn_sched_barrier(0);  // keys before values, as in the loop: their wait counts on it
        load_values(0);
        int slot = 0;
        for (int round = 0; round < blocks; round += NW, slot ^= 1) {
            // The CU serves its older waves first; left alone, they would be done in half the time, and the
            // others could not keep memory busy.  The next blocks' loads are in flight meanwhile.
            __builtin_amdgcn_s_barrier();
            const int blk = round + wave;
            if (blk >= blocks) continue;
            const int j0 = c0 + blk * S::TOK;
            const uint32_t there = (uint32_t)__ballot(lane < S::TOK && off >= 0);
            // every row sees the whole block, or bits say which tokens
            const uint32_t every = S::TOK == 32 ? ~0u : (1u << S::TOK) - 1u;
            const bool whole = there == every &&
                               (a.mask ? j0 + S::TOK <= s.first
                                       : j0 + S::TOK - 1 <= s.first + i_lo && (a.window == 0 || j0 > s.first + i_hi - a.window));
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) {
                if (FULL || ((kk + 1) * S::KSTEP <= DP / 2 && DP > 64)) continue;  // D > DP / 2 there
                const bool past = kk * S::KSTEP + q * S::VEC >= c.D;
#pragma unroll
                for (int t = 0; t < S::TT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) kf[t][kk][e] = past ? 0u : kf[t][kk][e];
            }
            Weights<BF16> w[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                f32x4 sv[S::TT];
#pragma unroll
                for (int t = 0; t < S::TT; ++t) {
                    sv[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk < S::KK; ++kk)
                        if (in_head(kk * S::KSTEP)) sv[t] = multiply<BF16>(kf[t][kk], qf[rb][kk], sv[t]);
                }
                if (rb == RB - 1) {
                    // the next block's keys set out
                    off = place(blk + NW, page_next);
                    if (lane < S::TOK) s_off[wave][slot ^ 1][lane] = max(off, (int64_t)0);
                    wave_sync();
                    load_keys(slot ^ 1);
                    page_next = page_of(blk + 2 * NW);
                }
                float top = kNoScore;
#pragma unroll
                for (int t = 0; t < S::TT; ++t) sv[t] *= sc;
                if (!whole) {
                    // this lane's tokens 4q .. 4q + 3 of each tile
                    const uint32_t bits = (there & row_bits(a, s, row_i[rb], s.row0 + row_i[rb], j0)) >> (4 * q);
#pragma unroll
                    for (int t = 0; t < S::TT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            sv[t][e] = bits & (1u << (16 * t + e)) ? sv[t][e] : kNoScore;
                }
#pragma unroll
                for (int t = 0; t < S::TT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, sv[t][e]);
                if (__any(top > m[rb] + kSlack)) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float next = fmaxf(m[rb], top);
                    const float by = next == kNoScore ? 1.f : exp2_hw(m[rb] - next);
                    m[rb] = next;
                    l[rb] *= by;
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[rb][db] *= by;
                }
                const float from = m[rb] == kNoScore ? 0.f : m[rb];
#pragma unroll
                for (int t = 0; t < S::TT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sv[t][e] = exp2_hw(sv[t][e] - from);
                        l[rb] += sv[t][e];
                    }
                w[rb].take(sv);
            }

            // Values.  A row's weight 0 times an infinite or NaN value that the row does not see would be
            // NaN: where rows differ in what they see, such elements are taken out, and a second
            // product of the largest finite numbers puts infinity where a row does see one.
            bool odd = false;
            if (!whole) {
                bool any = false;
#pragma unroll
                for (int k = 0; k < S::NV; ++k) {
                    const bool gone = !((there >> (k * S::TPI + lane / S::LPR)) & 1u);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (gone) vf[k][e] = 0;
                        any |= odd_lo<BF16>(vf[k][e]) || odd_hi(vf[k][e]);
                    }
                }
                odd = __any(any);
                if (odd) {
#pragma unroll
                    for (int k = 0; k < S::NV; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (odd_lo<BF16>(vf[k][e])) vf[k][e] &= 0xFFFF0000u;
                            if (odd_hi(vf[k][e])) vf[k][e] &= BF16 ? 0xFFFFu : 0u;
                        }
                }
            }
            auto piece_at = [&](int k) {
                return (u32x4*)(s_v + ((k * S::TPI + lane / S::LPR) * S::PITCH + (lane % S::LPR) * S::VEC) * E::kBytes);
            };
            // o += V^T of 16 dimensions (this lane's dimension of the tokens of its weights) times the weights
            auto add_values = [&]() {
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    if (!in_head(16 * db)) break;
                    u32x4 v;
                    if constexpr (BF16) {
                        char* at = s_v + ((4 * q + r / 4) * S::PITCH + db * 16 + (r % 4) * 4) * 2;
                        union {
                            s16x4 half[2];
                            u32x4 all;
                        } both;
                        both.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
                        both.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (__attribute__((address_space(3))) s16x4*)(at + 16 * S::PITCH * 2));
                        v = both.all;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = *(const uint32_t*)(s_v + ((4 * q + e) * S::PITCH + db * 16 + r) * 4);
                    }
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][db] = multiply<BF16>(v, w[rb].all, o[rb][db]);
                }
            };
#pragma unroll
            for (int k = 0; k < S::NV; ++k) *piece_at(k) = vf[k];
            wave_sync();
            load_values(slot ^ 1);
            add_values();
            wave_sync();
            if (odd) {
                constexpr uint32_t kLo = BF16 ? 0x7F7Fu : 0u, kHi = BF16 ? 0x7F7F0000u : 0x7F7FFFFFu;  // largest finite
                const int ol = again(lane);
                const int d = clamp((ol % S::LPR) * S::VEC);
#pragma unroll 1
                for (int k = 0; k < S::NV; ++k) {
                    const int t = k * S::TPI + ol / S::LPR;
                    u32x4 v = *(const u32x4*)((const char*)c.v + (head_at + d + s_off[wave][slot][t]) * E::kBytes);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = there >> t & 1u ? (odd_lo<BF16>(v[e]) ? kLo : 0u) | (odd_hi(v[e]) ? kHi : 0u) : 0u;
                    *piece_at(k) = v;
                }
                wave_sync();
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const uint32_t bits = (there & row_bits(a, s, row_i[rb], s.row0 + row_i[rb], j0)) >> (4 * q);
                    f32x4 one[S::TT];
#pragma unroll
                    for (int t = 0; t < S::TT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) one[t][e] = bits & (1u << (16 * t + e)) ? kHuge : 0.f;
                    w[rb].take(one);
                }
                add_values();
                wave_sync();
            }
        }

        finish_item<BF16, DP, RB, NT>(a, p, sh, s_mem, st, Item{s, row0, rows, before, n_units, from, to}, wg, g, o, m, l);
    }
}

// Joins tile_kernel's parts of each (row, head): one wave each, the weights of up to 64 parts in its lanes.
__global__ __launch_bounds__(kThreads) void join_kernel(AttentionArgs a, Plan p) {
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (item >= (int64_t)c.rows * a.H) return;
    const int t = (int)(item / a.H), head = (int)(item - (int64_t)t * a.H);
    const int b = find_seq(c.new_start, c.B, t);
    if (b >= c.B) return;
    const Seq s = load_seq(c, b);
    const int i = t - s.row0;
    if (i < 0 || i >= s.n) return;
    const int g = head / p.h;
    const int row0 = (i * p.h + head - g * p.h) / p.tile_rows * p.tile_rows;
    const int rows = min(s.n * p.h - row0, p.tile_rows);
    const Range range = tile_range(a, s, row0 / p.h, (row0 + rows - 1) / p.h);
    const int n_parts = max((range.hi - range.lo + p.chunk - 1) / p.chunk, 1);
    if (n_parts == 1) return;
    const float2* ml = (const float2*)((const float*)a.workspace + kCounterFloats + (int64_t)p.parts * c.rows * a.H * c.D);
    const int64_t step = (int64_t)c.rows * a.H;
    float2 mine = make_float2(kNoScore, 0.f);
    if (lane < n_parts) mine = ml[lane * step + item];
    float top = mine.x;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float by = mine.x == kNoScore ? 0.f : exp2_hw(mine.x - top);
    float total = mine.y * by;  // (NaN stays NaN)
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) total += __shfl_xor(total, k);
    const bool none = top == kNoScore && total == 0.f;
    // 4 dimensions a lane, and the parts in turn over what groups of lanes that leaves, four loads in flight each
    const int span = c.D <= 64 ? 16 : c.D <= 128 ? 32 : 64, groups = 64 / span;
    const int d = lane % span * 4, group = lane / span;
    const float* src = (const float*)a.workspace + kCounterFloats + item * c.D + min(d, c.D - 4);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < n_parts; k0 += 4 * groups) {
        f32x4 x[4];
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = k0 + i * groups + group;
            x[i] = *(const f32x4*)(src + min(k, n_parts - 1) * step * c.D);
            w[i] = __shfl(by, min(k, 63));  // 0 past the parts
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o += x[i] * w[i];
    }
    for (int k = span; k < 64; k <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], k);
    if (group == 0 && d < c.D) {
        const f32x4 y = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.f / total);
        char* dst = (char*)a.out.data + ((int64_t)t * a.out.stride_row + (int64_t)head * a.out.stride_head + d) * 2;
        *(uint2*)dst = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
    }
    if (lane == 0 && a.lse) a.lse[item] = none ? kNoScore : (top + log2f(total)) * kLn2;
}

template <bool BF16, int DP, bool FULL>
void launch_stream(const AttentionArgs& a, const Plan& p, dim3 grid, hipStream_t stream) {
    if (p.tile_rows == 16)
        hipLaunchKernelGGL((stream_kernel<BF16, DP, 1, FULL>), grid, dim3(64 * stream_waves(DP, 1)), 0, stream, a, p);
    else if (p.tile_rows == 32)
        hipLaunchKernelGGL((stream_kernel<BF16, DP, 2, FULL>), grid, dim3(64 * stream_waves(DP, 2)), 0, stream, a, p);
    else if constexpr (DP <= 128)
        hipLaunchKernelGGL((stream_kernel<BF16, DP, 4, FULL>), grid, dim3(64 * stream_waves(DP, 4)), 0, stream, a, p);
}

template <bool BF16, int DP>
void launch_stream(const AttentionArgs& a, const Plan& p, dim3 grid, hipStream_t stream) {
    if (a.c.D == DP)
        launch_stream<BF16, DP, true>(a, p, grid, stream);
    else
        launch_stream<BF16, DP, false>(a, p, grid, stream);
}

template <int DP>
void launch_tiles(const AttentionArgs& a, const Plan& p, dim3 grid, hipStream_t stream) {
    if (p.tile_rows == 256)
        hipLaunchKernelGGL((tile_kernel<false, DP, 8>), grid, dim3(512), 0, stream, a, p);
    else
        hipLaunchKernelGGL((tile_kernel<false, DP, 4>), grid, dim3(256), 0, stream, a, p);
}

}  // namespace

hipError_t launch_attention(const AttentionArgs& a, bool bf16, hipStream_t stream) {
    const CacheArgs& c = a.c;
    // a windowed row sees at most `window` positions, a tile's rows together max_new - 1 more
    const int span = a.window > 0 ? (int)std::min<long>(c.max_kv, (long)a.window + c.max_new - 1) : c.max_kv;
    Plan p = make_plan(c, a.H, bf16, span);
    // the caller's workspace is sized for max_kv: a window's parts may want more of it than there is
    if (plan_bytes(p, c, a.H) > a.workspace_bytes) p = make_plan(c, a.H, bf16, c.max_kv);
    const dim3 grid((unsigned)(p.many ? (long)c.B * c.G * p.tiles * p.parts : (long)p.wgs * c.G));
    if (p.many) {
        if (c.D <= 64)
            launch_tiles<64>(a, p, grid, stream);
        else if (c.D <= 128)
            launch_tiles<128>(a, p, grid, stream);
        else
            hipLaunchKernelGGL((tile_kernel<false, 256, 4>), grid, dim3(256), 0, stream, a, p);
    } else if (bf16) {
        if (c.D <= 64)
            launch_stream<true, 64>(a, p, grid, stream);
        else if (c.D <= 128)
            launch_stream<true, 128>(a, p, grid, stream);
        else
            launch_stream<true, 256>(a, p, grid, stream);
    } else {
        if (c.D <= 64)
            launch_stream<false, 64>(a, p, grid, stream);
        else if (c.D <= 128)
            launch_stream<false, 128>(a, p, grid, stream);
        else
            launch_stream<false, 256>(a, p, grid, stream);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || p.parts <= 1 ? e : launch_attention_join(a, p, stream);
}

hipError_t launch_attention_join(const AttentionArgs& a, const Plan& p, hipStream_t stream) {
    const dim3 joins((unsigned)(((long)a.c.rows * a.H + kWaves - 1) / kWaves));
    hipLaunchKernelGGL(join_kernel, joins, dim3(kThreads), 0, stream, a, p);
    return hipGetLastError();
}

}  // namespace psd
