// psd_attention_tile.hpp -- attention of many rows over the paged caches: one kernel for bfloat16 pools and for pools
// of 4-bit codes (device; internal to libpsd).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "psd_attention_device.hpp"
#include "psd_quant4.hpp"

namespace psd {

__device__ __forceinline__ const AttentionArgs& rows_of(const AttentionArgs& a) { return a; }
__device__ __forceinline__ const AttentionArgs& rows_of(const Attention4Args& a) { return a.a; }

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// One workgroup: 32 NW rows of one (sequence, key/value head), 32 a wave, over one part of its cache.
// Blocks of 64 tokens go through LDS, which all waves read: 32x32x16 products, 64 x 32
// scores a wave in 32 registers, the outputs in D/2 more.  Two buffers, one barrier a block: while
// block n is computed, block n + 1 is on its way into registers, and is stored behind the
// arithmetic.  Two waves a SIMD, so one wave's exponentials overlap the other's products: one
// workgroup of 8 waves a CU, which loads and stores half as much a row, or two of 4 for fewer rows.
// 2048 new tokens behind 14336, H=32, G=8, D=128: 544 - 570 us, 904 - 948 TFLOP/s (a large library product
// reaches 1370), the products busy 44 % of it; without its loads and stores of keys and values 440.  In LDS two
// buffers of 20 KB of values and 17 of keys.  Other heads, the same tokens: D=64 368 - 418 us; D=80, 96 and 112, padded to
// 128, 534 - 557; D=192, padded to 256, 1652; D=256 1625 - 1672 (one workgroup a CU, 24 registers spilled).  Window 4096,
// D=128: 157.  One token of 64 sequences, up to 4096 cached, window 1000, 263 MB: 46.
//
// Q4, over a cache held in 4 bits: a thread's pieces are a group's 16 bytes of codes and its scale byte, which become
// 64 bytes of bfloat16 on their way into LDS; from there on everything is the same.  2048 new tokens behind 14336: D=128
// 511 - 529 us, 974 - 1010 TFLOP/s, products busy 44 %; D=64 367; D=256 1407.
template <bool Q4, int DP, int NW>
struct TileShape {
    static constexpr int TOK = 64;
    static constexpr int NT = 64 * NW;
    static constexpr int ROWS = 32 * NW;
    static constexpr int LPR = DP / 8;              // 16-byte pieces of a token
    static constexpr int TPP = NT / LPR;      // tokens of one load of the workgroup
    static constexpr int N = TOK / TPP;             // loads a block
    static constexpr int GROUPS = DP / 32;          // Q4: groups of a token,
    static constexpr int PIECES = 2 * TOK * GROUPS; // of a block, keys first,
    static constexpr int N4 = (PIECES + NT - 1) / NT;  // of a thread
    // Row pitches (elements): 8 lanes reading 16 bytes of 8 consecutive keys, and the 4-token by
    // 64-byte tiles of the transposing reads, fall on different banks.
    static constexpr int KP = DP + 8, VP = DP + 32;
    static constexpr int BYTES = TOK * (KP + VP) * 2;
};

template <bool Q4, int DP, int NW>
__global__ __launch_bounds__(64 * NW, (DP == 256 || NW == 8 ? 1 : 2)) void tile_kernel(
    std::conditional_t<Q4, Attention4Args, AttentionArgs> args, Plan p) {
    using S = TileShape<Q4, DP, NW>;
    const AttentionArgs& a = rows_of(args);
    constexpr int KK = DP / 16, DB = DP / 32;
    __shared__ __align__(16) char s_mem[2 * S::BYTES];  // two buffers of keys and values
    __shared__ int64_t s_off[4][S::TOK];                // written two blocks ahead, read in two
    __shared__ int64_t s_scale[4][Q4 ? S::TOK : 1];
    __shared__ uint64_t s_there[4];
    __shared__ int s_odd[2];

    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int r = lane & 31, hi = lane >> 5;
    int x = blockIdx.x;
    const int g = x % c.G;
    x /= c.G;
    const int tile = p.tiles - 1 - x % p.tiles;  // causal rows: the longest first
    x /= p.tiles;
    const int b = x % c.B, part = x / c.B;

    const Seq s = uniform(load_seq(c, b));
    const int row0 = tile * S::ROWS;
    const int rows = min(s.n * p.h - row0, S::ROWS);
    if (rows <= 0) return;
    const int i_lo = uniform(row0 / p.h), i_hi = uniform((row0 + rows - 1) / p.h);
    const Range range = tile_range(a, s, i_lo, i_hi);
    const int n_parts = max((range.hi - range.lo + p.chunk - 1) / p.chunk, 1);
    if (part >= n_parts) return;
    const int c0 = range.lo + part * p.chunk, c1 = min(c0 + p.chunk, range.hi);
    const int blocks = (c1 - c0 + S::TOK - 1) / S::TOK;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;

    // this wave's rows: new tokens [w_lo, w_hi]; a wave without rows keeps company with zeros
    const int mine = min(max(rows - wave * 32, 0), 32);
    const int w_lo = uniform((row0 + min(wave * 32, rows - 1)) / p.h), w_hi = uniform((row0 + min(wave * 32 + 31, rows - 1)) / p.h);
    const bool on = r < mine;
    const int rr = row0 + wave * 32 + r;
    const int row_i = on ? rr / p.h : w_lo;
    const int head = g * p.h + (on ? rr - row_i * p.h : 0);
    const int64_t t_row = s.row0 + row_i;
    // scores in units of ln 2; a negative scale goes into the queries' signs, so that a maximum
    // of products is a maximum of scores
    const float sc = fmaxf(fabsf(a.scale) * kLog2e, 1.17549435e-38f);
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
    u32x4 qf[KK];
    {
        const char* src = (const char*)a.q.data + (t_row * a.q.stride_row + (int64_t)head * a.q.stride_head) * 2;
        // unconditional loads; rows and dimensions that are not there count as zero
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[kk] = *(const u32x4*)(src + min(kk * 16 + hi * 8, c.D - 8) * 2);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const bool none = !on || kk * 16 + hi * 8 >= c.D;
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[kk][e] = none ? 0u : qf[kk][e] ^ sign;
        }
    }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
    float m = kNoScore, l = 0.f;  // m: of products, scaled at the end

    const int64_t head_at = (int64_t)g * c.stride_head;
    const int piece = tid % S::LPR, token = tid / S::LPR;
    const int d_piece = min(piece * 8, c.D - 8);
    const bool past = piece * 8 >= c.D;  // keys past the head's end count as zero
    const char* k_src = (const char*)c.k + (head_at + d_piece) * 2;
    const char* v_src = (const char*)c.v + (head_at + d_piece) * 2;

    // Wave 0 finds the tokens' places; a page number is loaded a block before it is used.
    auto page_of = [&](int blk) {
        const int j = c0 + blk * S::TOK + lane;
        const int at = j < c1 ? j : 0;
        return table[p.page_shift >= 0 ? at >> p.page_shift : at / c.P];
    };
    auto place = [&](int blk, int page) -> int64_t {
        const int j = c0 + blk * S::TOK + lane;
        const int pi = p.page_shift >= 0 ? j >> p.page_shift : j / c.P;
        const bool none = j >= c1 || (unsigned)page >= (unsigned)c.pages;
        if constexpr (Q4)
            s_scale[blk & 3][lane] = none ? 0 : (int64_t)page * args.s.page + (int64_t)(j - pi * c.P) * args.s.token;
        if (none) return -1;
        return (int64_t)page * c.stride_page + (int64_t)(j - pi * c.P) * c.stride_token;
    };
    auto publish = [&](int blk, int page) {
        const int64_t off = place(blk, page);
        s_off[blk & 3][lane] = max(off, (int64_t)0);
        const uint64_t bits = __ballot(off >= 0);
        if (lane == 0) s_there[blk & 3] = bits;
    };
    auto there_of = [&](int blk) {
        const uint64_t bits = s_there[blk & 3];
        return (uint64_t)(uint32_t)uniform((int)(uint32_t)bits) | (uint64_t)(uint32_t)uniform((int)(bits >> 32)) << 32;
    };
    // Q4: this thread's piece k is of keys or values, of a token and a group (past the head's end: its last
    // group again, whose keys meet zeros and whose values go to no output)
    auto of_values = [&](int k) { return k * S::NT + tid >= S::PIECES / 2; };
    auto token_of = [&](int k) { return (k * S::NT + tid) / S::GROUPS % S::TOK; };
    auto group_of = [&](int k) { return (k * S::NT + tid) % S::GROUPS; };
    auto held_group = [&](int k) { return min(group_of(k), (c.D + 31) / 32 - 1); };
    auto has_piece = [&](int k) { return S::PIECES >= S::NT || tid < S::PIECES; };
    auto scale_at = [&](int blk, int k) -> uint32_t {
        if constexpr (Q4) {
            const uint8_t* at = (const uint8_t*)(of_values(k) ? args.s.v : args.s.k);
            return at[(int64_t)g * args.s.head + held_group(k) + s_scale[blk & 3][token_of(k)]];
        }
        return 0;
    };
    struct Rows16 {
        u32x4 k[S::N], v[S::N];
    };
    // Eight lanes store together: groups of a token begin 64 bytes apart, the next token's 16 (keys) or 64 (values) bytes
    // further on, of 128 in a round of the banks.  2048 tokens behind 14336, D=256 1550 us without turns, 1407 with them,
    // D=128 537 and 529: a fourth of all LDS cycles was waiting for banks, none is.
    auto turn_of = [&](int k) {
        if (DP == 256) return group_of(k) >> 1 & 3;
        if (of_values(k)) return DP == 64 ? token_of(k) & 3 : (group_of(k) & 2) | (token_of(k) & 1);
        return DP == 64 ? 0 : group_of(k) & 2;
    };
    struct Rows4 {
        u32x4 code[S::N4];
        uint32_t scale[S::N4];
    };
    using Stage = std::conditional_t<Q4, Rows4, Rows16>;
    auto load = [&](int blk, Stage& x) {
        if constexpr (Q4) {
#pragma unroll
            for (int k = 0; k < S::N4; ++k) {
                if (!has_piece(k)) continue;
                const char* at = (const char*)(of_values(k) ? c.v : c.k) + head_at + held_group(k) * 16;
                x.code[k] = *(const u32x4*)(at + s_off[blk & 3][token_of(k)]);
                x.scale[k] = scale_at(blk, k);
            }
            return;
        } else {
#pragma unroll
        for (int k = 0; k < S::N; ++k) {
            const int64_t at = s_off[blk & 3][k * S::TPP + token] * 2;
            x.k[k] = *(const u32x4*)(k_src + at);
            x.v[k] = *(const u32x4*)(v_src + at);
        }
        }
    };
    // Does every row of new tokens [lo, hi] see the whole block?
    auto whole = [&](int blk, int lo, int top) {
        const int j0 = c0 + blk * S::TOK;
        if (there_of(blk) != ~0ull) return false;
        if (a.mask) return j0 + S::TOK <= s.first;
        return j0 + S::TOK - 1 <= s.first + lo && (a.window == 0 || j0 > s.first + top - a.window);
    };
    auto key_at = [&](int blk) { return s_mem + (blk & 1) * S::BYTES; };
    auto value_at = [&](int blk) { return s_mem + (blk & 1) * S::BYTES + S::TOK * S::KP * 2; };
    // Into LDS.  Where rows differ in what they see, values of tokens that are not there are zeroed
    // and infinite or NaN values taken out (a weight 0 times them is NaN for rows that do not see them).
    auto store = [&](int blk, Stage& x) {
        if constexpr (Q4) {
            const bool all = whole(blk, i_lo, i_hi);
            const uint64_t there = there_of(blk);
#pragma unroll
            for (int k = 0; k < S::N4; ++k) {
                if (!has_piece(k)) continue;
                u32x4 w = x.code[k];
                uint32_t s8 = x.scale[k];
                if (!all && of_values(k)) {
                    const bool gone = !((there >> token_of(k)) & 1u), nan = s8 > quant4::kMost;
                    if (nan && !gone) s_odd[blk & 1] = blk + 1;
                    if (nan || gone) {
                        w = u32x4{0, 0, 0, 0};
                        s8 = 127;
                    }
                }
                const float by = quant4::scale_value(s8);
                char* to = (of_values(k) ? value_at(blk) + token_of(k) * S::VP * 2 : key_at(blk) + token_of(k) * S::KP * 2) +
                           group_of(k) * 64;
                quant4::decode_group(to, w, by, turn_of(k));
            }
            return;
        } else {
        if (past)
#pragma unroll
            for (int k = 0; k < S::N; ++k) x.k[k] = u32x4{0, 0, 0, 0};
        if (!whole(blk, i_lo, i_hi)) {
            const uint64_t there = there_of(blk);
            bool odd = false;
#pragma unroll
            for (int k = 0; k < S::N; ++k) {
                const bool gone = !((there >> (k * S::TPP + token)) & 1u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t w = gone ? 0u : x.v[k][e];
                    const bool lo_odd = odd_lo<true>(w), hi_odd = odd_hi(w);
                    odd |= lo_odd || hi_odd;
                    if (lo_odd) w &= 0xFFFF0000u;
                    if (hi_odd) w &= 0xFFFFu;
                    x.v[k][e] = w;
                }
            }
            if (odd) s_odd[blk & 1] = blk + 1;
        }
        char* keys = key_at(blk);
        char* values = value_at(blk);
#pragma unroll
        for (int k = 0; k < S::N; ++k) {
            *(u32x4*)(keys + ((k * S::TPP + token) * S::KP + piece * 8) * 2) = x.k[k];
            *(u32x4*)(values + ((k * S::TPP + token) * S::VP + piece * 8) * 2) = x.v[k];
        }
        }
    };
    // this lane's dimension of 32 db + .., tokens 16 ks + {4 hi .., 8 + 4 hi ..}, as an A operand
    const int v_lane = ((4 * hi + (lane & 15) / 4) * S::VP + ((lane >> 4) & 1) * 16 + (lane & 3) * 4) * 2;
    typedef __attribute__((address_space(3))) char lds_char;
    auto value = [&](lds_char* mine, int db, int ks) -> bf16x8 {  // mine: the block's values + v_lane
        lds_char* at = mine + (16 * ks * S::VP + db * 32) * 2;
        union {
            s16x4 half[2];
            bf16x8 all;
        } v;
        v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * S::VP * 2));
        return v.all;
    };

    // Blocks on their way into registers: one, or two where a workgroup of 8 waves has the registers (a block
    // takes it about as long as memory takes to answer).
    constexpr int AHEAD = NW == 8 ? 2 : 1;
    if (tid < 2) s_odd[tid] = 0;
    int pages[AHEAD + 2];
#pragma unroll
    for (int n = 0; n < AHEAD + 2; ++n) pages[n] = page_of(n);
    if (wave == 0)
#pragma unroll
        for (int n = 0; n <= AHEAD; ++n) publish(n, pages[n]);
    int page = pages[AHEAD + 1];
    __syncthreads();
    Stage first, second;
    load(0, first);
    if (blocks > 0) store(0, first);
    if (AHEAD == 2) load(1, first);
    // Block `blk`, which is in LDS, while `into` is loaded; then block blk + 1 goes from `from` into LDS.
    auto step = [&](int blk, Stage& from_stage, Stage& into) {
        __syncthreads();
        const int j0 = c0 + blk * S::TOK;
        const bool more = blk + 1 < blocks;
        load(blk + AHEAD, into);  // (past the end: the pool's first tokens, which nothing uses)
        const bool seen_by_all = whole(blk, w_lo, w_hi);
        const uint64_t there = there_of(blk);
        // nothing of the block lies before this wave's last row's end (or behind its window)
        const bool idle = mine == 0 || (!a.mask && (j0 > s.first + w_hi ||
                                                    (a.window > 0 && j0 + S::TOK - 1 <= s.first + w_lo - a.window)));
        uint32_t bits[2] = {~0u, ~0u};
        if (!idle) {
            const char* keys = key_at(blk);
            lds_char* values = (lds_char*)value_at(blk) + v_lane;
            // Scores: four keys' pieces are read from LDS while the last four are multiplied.
            f32x16 sv[2];
            u32x4 kb[2][4];
            constexpr int CH = KK / 4;  // groups of four pieces of 32 keys
            auto read_keys = [&](int n, u32x4 (&into)[4]) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    into[i] = *(const u32x4*)(keys + ((32 * (n / CH) + r) * S::KP + (n % CH * 4 + i) * 16 + hi * 8) * 2);
            };
            read_keys(0, kb[0]);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int n = 0; n < 2 * CH; ++n) {
                if (n + 1 < 2 * CH) read_keys(n + 1, kb[(n + 1) & 1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (n % CH == 0 && i == 0)
#pragma unroll
                        for (int e = 0; e < 16; ++e) sv[n / CH][e] = 0.f;
                    sv[n / CH] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kb[n & 1][i]),
                                                                        __builtin_bit_cast(bf16x8, qf[n % CH * 4 + i]), sv[n / CH], 0,
                                                                        0, 0);
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);                         // one product,
                    if (n + 1 < 2 * CH) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // one read
                }
            }
            if (!seen_by_all) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    // this lane's tokens: 8 (e / 4) + 4 hi + e % 4
                    bits[t] = ((uint32_t)(there >> (32 * t)) & row_bits(a, s, row_i, (int)t_row, j0 + 32 * t)) >> (4 * hi);
#pragma unroll
                    for (int e = 0; e < 16; ++e) sv[t][e] = bits[t] & (1u << (8 * (e / 4) + e % 4)) ? sv[t][e] : kNoScore;
                }
                if (a.mask) __builtin_amdgcn_s_waitcnt(0x0F70);  // no load of this branch is pending behind it
            }
            float top = sv[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, sv[t][e]);
            float from = m * sc;
            if (__any(top * sc > from + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float next = fmaxf(m, top);
                const float by = next == kNoScore ? 1.f : exp2_hw((m - next) * sc);
                m = next;
                from = m * sc;
                l *= by;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db] *= by;
            }
            // The exponent is fma(sv, sc, -from): a row's weights have the rounding of `from` in common, which the
            // division by their sum takes out, but which is no rounding error any more where scores are so large
            // that it reaches float32's range of exponents.  There the maximum is taken out before the scale.
            const bool none = from == kNoScore;
            from = none ? 0.f : from;
            if (__any(fabsf(from) > kFar)) {
                const float base = none ? 0.f : m;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sv[t][e] -= base;
                from -= from;  // (a maximum that is infinite when scaled: NaN)
            }
            // Weights of 16 tokens at a time, and their product with the values, whose pieces are read 16 tokens ahead:
            // exponentials and reads go between the products.  Weights are rounded to bfloat16, 2^-8 of each at most, since both
            // operands of a product have one type; their sum is that of the unrounded ones.  Outputs 2.3e-3 of their size from 64
            // bits, where the result's own rounding is 1.7e-3.
            auto weights = [&](int ks) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float w0 = exp2_hw(__builtin_fmaf(sv[ks / 2][8 * (ks % 2) + e], sc, -from));
                    const float w1 = exp2_hw(__builtin_fmaf(sv[ks / 2][8 * (ks % 2) + e + 1], sc, -from));
                    l += w0;
                    l += w1;
                    w[e / 2] = pack_bf16(w0, w1);
                }
                return w;
            };
            bf16x8 vb[2][DB];
            auto read_values = [&](int ks, bf16x8 (&into)[DB]) {
#pragma unroll
                for (int db = 0; db < DB; ++db) into[db] = value(values, db, ks);
            };
            read_values(0, vb[0]);
            u32x4 w = weights(0);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                u32x4 w_next = w;
                if (ks < 3) {
                    read_values(ks + 1, vb[(ks + 1) & 1]);
                    w_next = weights(ks + 1);
                }
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[ks & 1][db], __builtin_bit_cast(bf16x8, w), o[db], 0, 0, 0);
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                }
                w = w_next;
            }
        }
        if (uniform(s_odd[blk & 1]) == blk + 1) {
            // infinite or NaN values were taken out of this block: a product of the largest finite
            // numbers puts infinity where a row sees one
            char* values = value_at(blk);
            if constexpr (Q4) {
                __syncthreads();
#pragma unroll
                for (int k = 0; k < S::N4; ++k) {
                    if (!has_piece(k) || !of_values(k)) continue;
                    const bool nan = there >> token_of(k) & 1u && scale_at(blk, k) > quant4::kMost;
                    const uint32_t one = nan ? 0x7F7F7F7Fu : 0u;
                    char* to = values + token_of(k) * S::VP * 2 + group_of(k) * 64;
#pragma unroll
                    for (int e = 0; e < 4; ++e) *(u32x4*)(to + 16 * e) = u32x4{one, one, one, one};
                }
            } else {
            u32x4 again[S::N];
#pragma unroll
            for (int k = 0; k < S::N; ++k) again[k] = *(const u32x4*)(v_src + s_off[blk & 3][k * S::TPP + token] * 2);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < S::N; ++k) {
                const bool gone = !((there >> (k * S::TPP + token)) & 1u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t v = again[k][e];
                    again[k][e] = gone ? 0u : (odd_lo<true>(v) ? 0x7F7Fu : 0u) | (odd_hi(v) ? 0x7F7F0000u : 0u);
                }
                *(u32x4*)(values + ((k * S::TPP + token) * S::VP + piece * 8) * 2) = again[k];
            }
            }
            __syncthreads();
            if (!idle) {
                lds_char* ones = (lds_char*)value_at(blk) + v_lane;
                u32x4 w[4];
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const int bit = 16 * (ks & 1) + 8 * (e / 4) + e % 4;
                        w[ks][e / 2] = (bits[ks / 2] >> bit & 1u ? 0x7F7Fu : 0u) | (bits[ks / 2] >> (bit + 1) & 1u ? 0x7F7F0000u : 0u);
                    }
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(ones, db, ks), __builtin_bit_cast(bf16x8, w[ks]),
                                                                        o[db], 0, 0, 0);
            }
        }
        if (more) store(blk + 1, from_stage);
        if (wave == 0) publish(blk + 1 + AHEAD, page);
        page = page_of(blk + 2 + AHEAD);
    };
    for (int blk = 0; blk < blocks; blk += AHEAD) {
        step(blk, first, AHEAD == 2 ? second : first);
        if (AHEAD == 2 && blk + 1 < blocks) step(blk + 1, second, first);
    }

    l += __shfl_xor(l, 32);
    m *= sc;
    if (!on) return;
    if (n_parts == 1) {
        const bool none = m == kNoScore && l == 0.f;
        const float by = 1.f / l;
        char* dst = (char*)a.out.data + (t_row * a.out.stride_row + (int64_t)head * a.out.stride_head) * 2;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = db * 32 + 2 * e + 4 * hi;
                if (d >= c.D) continue;
                uint2 y = make_uint2(0, 0);
                if (!none)
                    y = make_uint2(pack_bf16(o[db][e] * by, o[db][e + 1] * by), pack_bf16(o[db][e + 2] * by, o[db][e + 3] * by));
                *(uint2*)(dst + d * 2) = y;
            }
        if (hi == 0 && a.lse) a.lse[t_row * a.H + head] = none ? kNoScore : (m + log2f(l)) * kLn2;
    } else {
        const int64_t at = ((int64_t)part * c.rows + t_row) * a.H + head;
        float* dst = (float*)a.workspace + kCounterFloats + at * c.D;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = db * 32 + 2 * e + 4 * hi;
                if (d < c.D) *(f32x4*)(dst + d) = f32x4{o[db][e], o[db][e + 1], o[db][e + 2], o[db][e + 3]};
            }
        if (hi == 0) {
            float2* ml = (float2*)((float*)a.workspace + kCounterFloats + (int64_t)p.parts * c.rows * a.H * c.D);
            ml[at] = make_float2(m, l);
        }
    }
}

}  // namespace

}  // namespace psd
