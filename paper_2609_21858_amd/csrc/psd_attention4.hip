// psd_attention4.hip -- attention over a paged cache held in 4 bits (gfx950).
//
// The values that codes stand for are exact in bfloat16 (two significant bits and a power of two), so both products
// run on the bfloat16 matrix instructions over converted codes, and nothing of the cache is rounded.  bfloat16
// rows are one operand; a float32 query or softmax weight is the sum of three bfloat16 terms of 8 bits each,
// whose products with codes are exact and summed in float32.  Tiles of many rows are tile_kernel's.
#include <hip/hip_runtime.h>

#include "psd_attention_device.hpp"
#include "psd_attention_tile.hpp"
#include "psd_quant4.hpp"

namespace psd {

namespace {

// x as bfloat16 terms that sum to it (float32: each the next 8 bits, cut towards zero, so that none overflows; infinite and
// NaN ones come out NaN).
template <int TERMS>
__device__ __forceinline__ void split(float x, float (&t)[TERMS]) {
    if constexpr (TERMS == 1) {
        t[0] = x;
    } else {
#pragma unroll
        for (int i = 0; i < TERMS; ++i) {
            t[i] = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
            x -= t[i];
        }
    }
}

// Upper halves of two words, as a pair of bfloat16.
__device__ __forceinline__ uint32_t upper(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Few rows: stream_kernel's scheme with blocks of 64 tokens a wave.  The keys' dimensions are summed in the order that
// gives each lane whole pieces of codes: of a token, lane q of four has the 4 DP / 32 words from dimension
// DP / 4 q on (DP = 256: 32 dimensions from 32 q and from 128 + 32 q on), one scale byte to each 32 dimensions, and the
// queries are laid out to match.  Values become bfloat16 on their way into the wave's LDS, 32 tokens at a time.
//
// Memory bounds long caches, (D/2 + D/32) 2 G bytes a token, and a chain of dependent loads short ones (start, division,
// places, keys, join of waves).  H=32, G=8, D=128: 1 token of 32 sequences, up to 16384 cached, 363 MB, 80 us, 4.5 TB/s,
// float32 rows 86 - 96; heads of 64 52, 4 heads of 256 83 - 92.  1 token of 64 sequences, up to 4096, 52 us, 5 tokens
// 62 - 70, float32 96 - 103; 1 token of 4 sequences, up to 512, 8.4 (the chain); behind 131072 46.  Of the 80 us, each
// token more goes by at 5.85 TB/s, the chain takes 8, and 10 are not accounted for: half of the vector loads move one byte a
// lane (scales), a third of the active LDS cycles wait for banks, products are busy 13 %.  float32 rows are bound by products,
// three for one: 4 x 512 tokens to 2048 264 us, 433 TFLOP/s of bfloat16 products.
// Four waves a workgroup and two workgroups a CU, so that one's chain lies under the other's loads; 143 - 256 registers a
// lane (heads of 256: one workgroup, with 356 - 512).  Tiles of 32 bfloat16 rows spill 10 of them, 50 with heads of 256;
// 64 - 117 scalar ones are spilled into lanes of vector registers in every form.
template <int DP>
struct Stream4Shape {
    static constexpr int TOK = 64;
    static constexpr int TT = TOK / 16;        // 16-token tiles of a block
    static constexpr int KK = DP / 32;         // products of a tile: words of codes of a lane
    static constexpr int NS = DP == 256 ? 2 : 1;  // groups of a lane
    static constexpr int GROUPS = DP / 32;     // groups of a token
    static constexpr int TPI = 64 / GROUPS;    // values: tokens of one load
    static constexpr int NV = TOK / TPI;       // loads of a block
    static constexpr int PITCH = DP + 16;      // of a token's values in LDS
    static constexpr int V_BYTES = 32 * PITCH * 2;
};

// The waves' values and two blocks' places, and in their stead, behind the loop, the outputs of the join.
template <int DP, int RB>
constexpr int stream4_lds() {
    using S = Stream4Shape<DP>;
    constexpr int loop = kWaves4 * (S::V_BYTES + 2 * 2 * 8 * S::TOK), join = kWaves4 * 16 * RB * (DP + 4) * 4;
    return loop > join ? loop : join;
}

template <bool BF16, int DP, int RB>
__global__ __launch_bounds__(64 * kWaves4, stream4_resident(DP, RB)) void stream4_kernel(Attention4Args args, Plan p) {
    using S = Stream4Shape<DP>;
    using E = Elem<BF16>;
    constexpr int TERMS = BF16 ? 1 : 3;
    constexpr int DB = DP / 16;
    constexpr int NW = kWaves4, NT = 64 * NW;
    constexpr int ROWS = 16 * RB;
    __shared__ __align__(16) char s_mem[stream4_lds<DP, RB>()];
    __shared__ StreamShared<NT, ROWS> sh;

    const AttentionArgs& a = args.a;
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int r = lane & 15, q = lane >> 4;
    const int g = blockIdx.x % c.G, wg = blockIdx.x / c.G;
    const Stretch st = find_stretch<slack4(BF16, DP)>(a, p, sh, wg, join_units4(BF16));
    if (st.u0 == st.u1) return;

    const bool younger = stream4_resident(DP, RB) > 1 && blockIdx.x >= gridDim.x / 2;
    const float sc = a.scale * kLog2e;
    const int last_group = (c.D + 31) / 32 - 1;
    char* s_v = s_mem + wave * S::V_BYTES;
    int64_t(*s_off)[S::TOK] = (int64_t(*)[S::TOK])(s_mem + NW * S::V_BYTES) + wave * 4;
    int64_t(*s_scale)[S::TOK] = s_off + 2;
    // this lane's codes of a key: groups past the head's end are its last one again, which meets zeros
    int key_at[S::NS], key_group[S::NS];
#pragma unroll
    for (int n = 0; n < S::NS; ++n) {
        key_group[n] = min(DP == 64 ? q / 2 : q + 4 * n, last_group);
        key_at[n] = DP == 64 ? min(q, 2 * last_group + 1) * 8 : key_group[n] * 16;
    }
    auto dim_of = [&](int kk) { return DP == 64 ? 16 * q + 8 * kk : 32 * (q + 4 * (kk / 4)) + 8 * (kk % 4); };
    const int v_group = lane % S::GROUPS, v_token = lane / S::GROUPS;
    const int v_held = min(v_group, last_group);
    // (eight lanes store together: all groups of a token, 64 bytes apart, of 128 in a round of the banks; 32 sequences of up
    // to 16384 tokens 84.5 us, in one order 92.  Two tokens of 4 groups lose less to the banks than turning them takes: 32 float32
    // rows, 98 us and 101)
    const int v_turn = DP == 256 ? v_group >> 1 & 3 : 0;
    const char* k_src = (const char*)c.k + (int64_t)g * c.stride_head;
    const char* v_src = (const char*)c.v + (int64_t)g * c.stride_head + v_held * 16;
    const uint8_t* ks_src = (const uint8_t*)args.s.k + (int64_t)g * args.s.head;
    const uint8_t* vs_src = (const uint8_t*)args.s.v + (int64_t)g * args.s.head + v_held;

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

        // A block's tokens: lane t finds token t's place; -1: nothing there.  The page number is loaded a block before
        // it is used, so that no load in between has to be waited for with it.
        auto token_of = [&](int blk) { return c0 + blk * S::TOK + lane; };
        auto page_of = [&](int blk) {
            const int j = token_of(blk);
            const int at = j < c1 ? j : 0;
            return table[p.page_shift >= 0 ? at >> p.page_shift : at / c.P];
        };
        const int first_page = page_of(wave);  // (set out first: the first keys wait for it)
        int page = page_of(wave + NW);
        // this lane's rows, and their queries as B operands (unconditional loads; what is not there counts as zero)
        int row_i[RB];
        u32x4 qf[RB][TERMS][S::KK];
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
                const int d = dim_of(kk);
                const bool none = !on || d >= c.D;
                const char* at = src + min(d, c.D - 8) * E::kBytes;
                if constexpr (BF16) {
                    const u32x4 w = *(const u32x4*)at;
#pragma unroll
                    for (int e = 0; e < 4; ++e) qf[rb][0][kk][e] = none ? 0u : w[e];
                } else {
                    const u32x4 lo = *(const u32x4*)at, hi = *(const u32x4*)(at + 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x[TERMS], y[TERMS];
                        split(__uint_as_float(none ? 0u : e < 2 ? lo[2 * e] : hi[2 * e - 4]), x);
                        split(__uint_as_float(none ? 0u : e < 2 ? lo[2 * e + 1] : hi[2 * e - 3]), y);
#pragma unroll
                        for (int i = 0; i < TERMS; ++i) qf[rb][i][kk][e] = upper(x[i], y[i]);
                    }
                }
            }
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
        auto wave_sync = [&]() {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        // publishes the places of block `blk`; a token that is not there reads the pool's first one, whose score is masked
        // and whose values are zeroed
        auto publish = [&](int blk, int page, int slot) {
            const int j = token_of(blk);
            const int pi = p.page_shift >= 0 ? j >> p.page_shift : j / c.P;
            const bool there = j < c1 && (unsigned)page < (unsigned)c.pages;
            const int64_t place = j - (int64_t)pi * c.P;
            s_off[slot][lane] = there ? (int64_t)page * c.stride_page + place * c.stride_token : 0;
            s_scale[slot][lane] = there ? (int64_t)page * args.s.page + place * args.s.token : 0;
            const uint64_t bits = __ballot(there);
            wave_sync();
            return bits;
        };
        struct Block {
            uint64_t there;
            uint32_t kc[S::TT][S::KK];
            u32x4 vc[S::NV];
            // (bytes as loaded: widened to words here, they would be waited for a round early)
            uint8_t ks[S::TT][S::NS], vs[S::NV];
        };
        auto load_keys = [&](int slot, Block& x) {
#pragma unroll
            for (int t = 0; t < S::TT; ++t) {
                const char* src = k_src + s_off[slot][16 * t + r];
                const uint8_t* scale = ks_src + s_scale[slot][16 * t + r];
                if constexpr (DP == 64) {
                    const uint2 w = *(const uint2*)(src + key_at[0]);
                    x.kc[t][0] = w.x;
                    x.kc[t][1] = w.y;
                } else {
#pragma unroll
                    for (int n = 0; n < S::NS; ++n) {
                        const u32x4 w = *(const u32x4*)(src + key_at[n]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x.kc[t][4 * n + e] = w[e];
                    }
                }
#pragma unroll
                for (int n = 0; n < S::NS; ++n) x.ks[t][n] = scale[key_group[n]];
            }
        };
        auto load_values = [&](int slot, Block& x) {
#pragma unroll
            for (int k = 0; k < S::NV; ++k) {
                x.vc[k] = *(const u32x4*)(v_src + s_off[slot][k * S::TPI + v_token]);
                x.vs[k] = vs_src[s_scale[slot][k * S::TPI + v_token]];
            }
        };

        Block x;
        x.there = publish(wave, first_page, 0);
        load_keys(0, x);
        __builtin_amdgcn_sched_barrier(0);  // keys before values, as in the loop: their wait counts on it
        load_values(0, x);
        __builtin_amdgcn_sched_barrier(0);
        // Block `blk` is in x, its places in `slot`; x takes the wave's next one as it becomes free.
        for (int blk = wave, slot = 0; blk < blocks; blk += NW, slot ^= 1) {
            // A CU serves its older waves first: its first workgroup would end 7 of 45 us before its second (32 x 8192 tokens).
            // The second goes first in every other block, which leaves 3.
            if (younger) {
                if (blk / NW & 1)
                    __builtin_amdgcn_s_setprio(1);
                else
                    __builtin_amdgcn_s_setprio(0);
            }
            const uint64_t there = x.there;
            const int j0 = c0 + blk * S::TOK;
            // every row sees the whole block, or bits say which tokens
            const bool whole = there == ~0ull &&
                               (a.mask ? j0 + S::TOK <= s.first
                                       : j0 + S::TOK - 1 <= s.first + i_lo && (a.window == 0 || j0 > s.first + i_hi - a.window));
            f32x4 sv[RB][S::TT];
#pragma unroll
            for (int t = 0; t < S::TT; ++t) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) sv[rb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < S::KK; ++kk) {
                    const u32x4 keys = quant4::decode8(x.kc[t][kk], quant4::scale_value(x.ks[t][S::NS == 2 ? kk / 4 : 0]));
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                        for (int i = 0; i < TERMS; ++i) sv[rb][t] = multiply<true>(keys, qf[rb][i][kk], sv[rb][t]);
                }
            }
            // the next block's keys set out
            x.there = publish(blk + NW, page, slot ^ 1);
            load_keys(slot ^ 1, x);
            page = page_of(blk + 2 * NW);
            // A row's weight 0 times a NaN value that the row does not see would be NaN: where rows differ in what they see,
            // such groups are taken out, and a second product puts infinity where a row does see one.
            bool odd = false;
            if (!whole) {
                bool any = false;
#pragma unroll
                for (int k = 0; k < S::NV; ++k) {
                    const bool gone = !((there >> (k * S::TPI + v_token)) & 1u), nan = x.vs[k] > quant4::kMost;
                    any |= nan && !gone;
                    if (gone || nan) {
                        x.vc[k] = u32x4{0, 0, 0, 0};
                        x.vs[k] = 127;
                    }
                }
                odd = __any(any);
            }
            auto piece_at = [&](int k) {  // of the half's buffer
                return s_v + ((k % (S::NV / 2) * S::TPI + v_token) * S::PITCH + v_group * 32) * 2;
            };
            auto write_values = [&](int h) {
#pragma unroll
                for (int k = h * S::NV / 2; k < (h + 1) * S::NV / 2; ++k) {
                    quant4::decode_group(piece_at(k), x.vc[k], quant4::scale_value(x.vs[k]), v_turn);
                }
                wave_sync();
            };
            write_values(0);  // beside the softmax
            u32x4 w[RB][2][TERMS];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float top = kNoScore;
#pragma unroll
                for (int t = 0; t < S::TT; ++t) sv[rb][t] *= sc;
                if (!whole) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // this lane's tokens 4q .. 4q + 3 of each tile
                        const uint32_t bits =
                            ((uint32_t)(there >> (32 * h)) & row_bits(a, s, row_i[rb], s.row0 + row_i[rb], j0 + 32 * h)) >> (4 * q);
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                sv[rb][2 * h + t][e] = bits & (1u << (16 * t + e)) ? sv[rb][2 * h + t][e] : kNoScore;
                    }
                }
#pragma unroll
                for (int t = 0; t < S::TT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, sv[rb][t][e]);
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
                const float base = m[rb] == kNoScore ? 0.f : m[rb];
                f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < S::TT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sv[rb][t][e] = exp2_hw(sv[rb][t][e] - base);
                        sum[e] += sv[rb][t][e];
                    }
                l[rb] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float w0 = sv[rb][2 * h + e / 2][2 * (e % 2)], w1 = sv[rb][2 * h + e / 2][2 * (e % 2) + 1];
                        if constexpr (BF16) {
                            // Weights are rounded as psd_attention's, 2^-8 of each at most: a second term would be a second
                            // product.  Outputs 2.1e-3 to 2.3e-3 of their size from 64 bits (the result's own rounding: 1.7e-3).
                            w[rb][h][0][e] = pack_bf16(w0, w1);
                        } else {
                            float u[TERMS], v[TERMS];
                            split(w0, u);
                            split(w1, v);
#pragma unroll
                            for (int i = 0; i < TERMS; ++i) w[rb][h][i][e] = upper(u[i], v[i]);
                        }
                    }
            }

            // o += V^T of 16 dimensions (this lane's dimension of the tokens of its weights) times the weights of half h;
            // LANES pieces of values are on their way from LDS while those before them are multiplied
            constexpr int LANES = DB < 4 ? DB : 4;
            auto add_values = [&](int h) {
                u32x4 v[2][LANES];
                auto read = [&](int group, u32x4 (&into)[LANES]) {
#pragma unroll
                    for (int i = 0; i < LANES; ++i) {
                        char* at = s_v + ((4 * q + r / 4) * S::PITCH + (group * LANES + i) * 16 + (r % 4) * 4) * 2;
                        union {
                            s16x4 half[2];
                            u32x4 all;
                        } both;
                        both.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
                        both.half[1] =
                            __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 16 * S::PITCH * 2));
                        into[i] = both.all;
                    }
                };
                read(0, v[0]);
#pragma unroll
                for (int n = 0; n < DB / LANES; ++n) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (n + 1 < DB / LANES) read(n + 1, v[(n + 1) & 1]);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < LANES; ++i)
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                            for (int t = 0; t < TERMS; ++t)
                                o[rb][n * LANES + i] = multiply<true>(v[n & 1][i], w[rb][h][t], o[rb][n * LANES + i]);
                }
            };
            add_values(0);
            wave_sync();
            write_values(1);
            load_values(slot ^ 1, x);
            add_values(1);
            wave_sync();
            if (odd) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll 1
                    for (int k = h * S::NV / 2; k < (h + 1) * S::NV / 2; ++k) {
                        const int t = k * S::TPI + v_token;
                        const bool nan = there >> t & 1u && vs_src[s_scale[slot][t]] > quant4::kMost;
                        const uint32_t one = nan ? 0x7F7F7F7Fu : 0u;  // the largest finite number, or nearly
#pragma unroll
                        for (int e = 0; e < 4; ++e) *(u32x4*)(piece_at(k) + 16 * e) = u32x4{one, one, one, one};
                    }
                    wave_sync();
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const uint32_t bits =
                            ((uint32_t)(there >> (32 * h)) & row_bits(a, s, row_i[rb], s.row0 + row_i[rb], j0 + 32 * h)) >> (4 * q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int bit = 16 * (e / 2) + 2 * (e % 2);
                            w[rb][h][0][e] = (bits >> bit & 1u ? 0x7F7Fu : 0u) | (bits >> (bit + 1) & 1u ? 0x7F7F0000u : 0u);
#pragma unroll
                            for (int i = 1; i < TERMS; ++i) w[rb][h][i][e] = 0u;
                        }
                    }
                    add_values(h);
                    wave_sync();
                }
            }
        }
        finish_item<BF16, DP, RB, NT, 4>(a, p, sh, s_mem, st, Item{s, row0, rows, before, n_units, from, to}, wg, g, o, m, l);
    }
}

template <bool BF16, int DP>
void launch_stream4(const Attention4Args& a, const Plan& p, dim3 grid, hipStream_t stream) {
    if constexpr (tile_limit4(BF16, DP) == 32)
        if (p.tile_rows == 32) {
            hipLaunchKernelGGL((stream4_kernel<BF16, DP, 2>), grid, dim3(64 * kWaves4), 0, stream, a, p);
            return;
        }
    hipLaunchKernelGGL((stream4_kernel<BF16, DP, 1>), grid, dim3(64 * kWaves4), 0, stream, a, p);
}

template <int DP>
void launch_tiles4(const Attention4Args& a, const Plan& p, dim3 grid, hipStream_t stream) {
    if (p.tile_rows == 256)
        hipLaunchKernelGGL((tile_kernel<true, DP, 8>), grid, dim3(512), 0, stream, a, p);
    else
        hipLaunchKernelGGL((tile_kernel<true, DP, 4>), grid, dim3(256), 0, stream, a, p);
}

}  // namespace

hipError_t launch_attention4(const Attention4Args& args, bool bf16, hipStream_t stream) {
    const AttentionArgs& a = args.a;
    const CacheArgs& c = a.c;
    // a windowed row sees at most `window` positions, a tile's rows together max_new - 1 more
    const int span = a.window > 0 ? (int)std::min<long>(c.max_kv, (long)a.window + c.max_new - 1) : c.max_kv;
    Plan p = make_plan(c, a.H, bf16, span, true);
    // the caller's workspace is sized for max_kv: a window's parts may want more of it than there is
    if (plan_bytes(p, c, a.H) > a.workspace_bytes) p = make_plan(c, a.H, bf16, c.max_kv, true);
    const dim3 grid((unsigned)(p.many ? (long)c.B * c.G * p.tiles * p.parts : (long)p.wgs * c.G));
    if (p.many) {
        if (c.D <= 64)
            launch_tiles4<64>(args, p, grid, stream);
        else if (c.D <= 128)
            launch_tiles4<128>(args, p, grid, stream);
        else
            hipLaunchKernelGGL((tile_kernel<true, 256, 4>), grid, dim3(256), 0, stream, args, p);
    } else if (bf16) {
        if (c.D <= 64)
            launch_stream4<true, 64>(args, p, grid, stream);
        else if (c.D <= 128)
            launch_stream4<true, 128>(args, p, grid, stream);
        else
            launch_stream4<true, 256>(args, p, grid, stream);
    } else {
        if (c.D <= 64)
            launch_stream4<false, 64>(args, p, grid, stream);
        else if (c.D <= 128)
            launch_stream4<false, 128>(args, p, grid, stream);
        else
            launch_stream4<false, 256>(args, p, grid, stream);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || p.parts <= 1 ? e : launch_attention_join(a, p, stream);
}

}  // namespace psd
