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

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kNoScore = -__builtin_inff();
// A running maximum is raised only when a score passes it by this much: weights stay below
// 2^8, sums exact to float32 as before, and most blocks need no exchange between lanes.
constexpr float kSlack = 8.f;
constexpr float kHuge = 3e38f;
// Scores above this (units of ln 2) are taken from the maximum before they are scaled, see tile_kernel.
constexpr float kFar = 1 << 20;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ Range tile_range(const AttentionArgs& a, const Seq& s, int i_lo, int i_hi) {
    return tile_range(a.mask != nullptr, a.window, s, i_lo, i_hi);
}

// Bit t of the result: the row of new token i sees position j0 + t (causal, window or mask; the end
// of the cache and its pages aside).
__device__ __forceinline__ uint32_t row_bits(const AttentionArgs& a, const Seq& s, int i, int row, int j0) {
    if (a.mask) {
        const int n0 = j0 - s.first;
        if (n0 <= -32) return ~0u;
        const uint32_t* words = a.mask + (int64_t)row * a.mask_words;
        auto word = [&](int w) { return w < a.mask_words ? words[w] : 0u; };
        if (n0 < 0) return (word(0) << -n0) | ((1u << -n0) - 1u);
        const int w = n0 / 32, shift = n0 % 32;
        return (uint32_t)(((uint64_t)word(w + 1) << 32 | word(w)) >> shift);
    }
    const int seen = s.first + i - j0 + 1;  // positions of the block up to the row's own
    uint32_t bits = seen >= 32 ? ~0u : seen <= 0 ? 0u : (1u << seen) - 1u;
    if (a.window > 0) {
        const int gone = seen - a.window;
        if (gone > 0) bits = gone >= 32 ? 0u : bits & (~0u << gone);
    }
    return bits;
}

// Infinite or NaN: the upper (float32: the) element of a word, and the lower one of two bfloat16.
__device__ __forceinline__ bool odd_hi(uint32_t w) { return (w & 0x7F800000u) == 0x7F800000u; }
template <bool BF16>
__device__ __forceinline__ bool odd_lo(uint32_t w) {
    return BF16 && (w & 0x7F80u) == 0x7F80u;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Sums of weights with maxima m and m2 as one with maximum `top` of both.  Maxima pass over NaN, sums do
// not: a row that sees nothing but NaN scores has no maximum and a NaN sum, one that sees nothing sum 0.
__device__ __forceinline__ float add_sums(float l, float m, float l2, float m2, float top) {
    return top == kNoScore ? l + l2 : l * exp2_hw(m - top) + l2 * exp2_hw(m2 - top);
}

// acc += A B of 16 x 16 results: 16 bytes of A's row and of B's column from each lane (32 products
// a result in bfloat16, 16 in float32, where element e of all lanes makes one instruction).
template <bool BF16>
__device__ __forceinline__ f32x4 multiply(const u32x4 x, const u32x4 y, f32x4 acc) {
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[e]), __uint_as_float(y[e]), acc, 0, 0, 0);
        return acc;
    }
}

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

// Values that are the same in all lanes, into scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Seq uniform(const Seq& s) {
    return Seq{uniform(s.row0), uniform(s.n), uniform(s.first), uniform(s.kv), uniform(s.total)};
}

// A value anew, so that what rare code computes from it is not kept in registers through the common.
__device__ __forceinline__ int again(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// What workgroups leave for each other: written through and read past the caches that are not
// shared (relaxed accesses of agent scope), so that no fence has to empty those.
__device__ __forceinline__ void leave2(float* at, float x, float y) {
    const uint64_t w = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
    __hip_atomic_store((uint64_t*)at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 fetch2(const float* at) {
    const uint64_t w = __hip_atomic_load((const uint64_t*)at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
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
    __shared__ float s_m[NW][ROWS], s_l[NW][ROWS], s_top[ROWS], s_sum[ROWS];
    __shared__ int s_units[NT + 1], s_wave[NW], s_longest[NW];
    __shared__ Seq s_seq[NT];  // of the items, while there are no more than threads
    __shared__ int s_chunk, s_last;

    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int r = lane & 15, q = lane >> 4;
    const int g = blockIdx.x % c.G, wg = blockIdx.x / c.G;

    // units before each thread's items, by a scan over the workgroup
    const int items = c.B * p.tiles;
    const int each = (items + NT - 1) / NT;
    auto seq_at = [&](int i) { return load_seq(c, i / p.tiles); };
    auto units_at = [&](int i, const Seq& s) { return item_units(a.mask != nullptr, a.window, p, s, i % p.tiles); };
    int mine = 0, longest = 0;
    for (int i = tid * each; i < min((tid + 1) * each, items); ++i) {
        const Seq s = seq_at(i);
        const int n = units_at(i, s);
        s_seq[tid] = s;
        mine += n;
        longest = max(longest, n);
    }
    int upto = mine;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int below = __shfl_up(upto, k);
        if (lane >= k) upto += below;
        longest = max(longest, __shfl_xor(longest, k));
    }
    if (lane == 63) {
        s_wave[wave] = upto;
        s_longest[wave] = longest;
    }
    __syncthreads();
    for (int w = 0; w < NW; ++w) {
        if (w < wave) upto += s_wave[w];
        longest = max(longest, s_longest[w]);
    }
    s_units[tid + 1] = upto;
    if (tid == 0) s_units[0] = 0;
    __syncthreads();
    const int units = uniform(s_units[NT]);
    // While no item is much longer than a stretch, each workgroup takes one item whole and none is joined.
    constexpr int kMinUnits = join_units(BF16);
    const Division cut = divide(units, p.wgs, kMinUnits);
    const bool whole_items = each == 1 && items <= p.wgs && uniform(longest) <= units / p.wgs + 1 + kMinUnits;
    auto start = [&](int w) { return whole_items ? s_units[min(w, items)] : cut.start(w); };
    if (wg >= (whole_items ? items : cut.wgs)) return;
    const int u0 = uniform(start(wg)), u1 = uniform(start(wg + 1));  // this workgroup's
    if (u0 == u1) return;
    if (s_units[tid] <= u0 && u0 < s_units[tid + 1]) s_chunk = tid;
    __syncthreads();
    const int chunk = uniform(s_chunk);
    int item = chunk * each, before = uniform(s_units[chunk]);
    constexpr int kSlot = ROWS * DP + 2 * ROWS;  // floats of what a workgroup leaves of an item
    auto slot_of = [&](int w, int second) {
        return (float*)a.workspace + kCounterFloats + (((int64_t)w * c.G + g) * 2 + second) * kSlot;
    };
    const float sc = a.scale * kLog2e;
    const int64_t head_at = (int64_t)g * c.stride_head;
    char* s_v = s_mem + wave * S::V_BYTES;

    for (int n_units; before < u1; before += n_units, ++item) {
        const Seq s = uniform(each == 1 ? s_seq[item] : seq_at(item));
        n_units = each == 1 ? uniform(s_units[item + 1]) - before : uniform(units_at(item, s));
        if (!works_on(before, n_units, u0)) continue;
        const int b = item / p.tiles, tile = item - b * p.tiles;
        const Tile its = item_tile(p, s, tile);
        const int row0 = its.row0, rows = its.rows;
        const int i_lo = uniform(its.i_lo), i_hi = uniform(its.i_hi);
        const Range range = tile_range(a, s, i_lo, i_hi);
        const int from = max(u0, before), to = min(u1, before + n_units);
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

        // Join the waves: a common maximum, then the outputs through LDS, summed by all threads, each for NP
        // pairs of neighbouring dimensions.
        constexpr int NP = ROWS * DP / 2 / NT;
        constexpr int OP = DP + 4;
        const int el = again(lane), et = again(tid), er = el & 15, eq = el >> 4;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            l[rb] += __shfl_xor(l[rb], 16);
            l[rb] += __shfl_xor(l[rb], 32);
            if (eq == 0) {
                s_m[wave][rb * 16 + er] = m[rb];
                s_l[wave][rb * 16 + er] = l[rb];
            }
        }
        __syncthreads();
        float* s_o = (float*)s_mem;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = rb * 16 + er;
            float top = kNoScore;
            for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[w][row]);
            const float by = m[rb] == kNoScore ? 0.f : exp2_hw(m[rb] - top);
#pragma unroll
            for (int db = 0; db < DB; ++db) *(f32x4*)(s_o + (wave * ROWS + row) * OP + db * 16 + 4 * eq) = o[rb][db] * by;
            if (wave == 0 && eq == 0) {
                float sum = 0.f;
                for (int w = 0; w < NW; ++w) sum = add_sums(sum, top, s_l[w][row], s_m[w][row], top);
                s_top[row] = top;
                s_sum[row] = sum;
            }
        }
        __syncthreads();
        float2 y[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = (i * NT + et) * 2;
            y[i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float2 x = *(const float2*)(s_o + (w * ROWS + e / DP) * OP + e % DP);
                y[i].x += x.x;
                y[i].y += x.y;
            }
        }
        if (from != before || to != before + n_units) {
            // A part of an item.  What a workgroup leaves of an item that its stretch begins with goes to
            // its first slot, of one that begins later to its second.
            const int w_first = cut.owner(before), n_parts = cut.owner(before + n_units - 1) - w_first + 1;
            float* dst = slot_of(wg, from == u0 ? 0 : 1);
#pragma unroll
            for (int i = 0; i < NP; ++i) leave2(dst + (i * NT + et) * 2, y[i].x, y[i].y);
            if (et < ROWS) leave2(dst + ROWS * DP + 2 * et, s_top[et], s_sum[et]);
            // all of it is written when the counter goes up: the workgroup that counts last finds every part
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (et == 0) {
                unsigned* counter = (unsigned*)a.workspace + w_first * c.G + g;
                const unsigned was = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = was == (unsigned)(n_parts - 1);
                if (s_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (!s_last) continue;  // s_last is written again two barriers later at the earliest
            // the parts' common maximum and sum of each row, then their outputs, kBatch parts at a time
            constexpr int kSubs = NT / ROWS, kBatch = 2048 / ROWS;
            float* s_red = (float*)s_mem;         // [kSubs][ROWS][2]
            float* s_fac = s_red + 2 * NT;  // [kBatch][ROWS]: the parts' factors
            const int first_slot = before == start(w_first) ? 0 : 1;
            auto part_slot = [&](int k) { return slot_of(w_first + k, k == 0 ? first_slot : 0); };
            const int row = et % ROWS;
            float mm = kNoScore, ll = 0.f;
            for (int k = et / ROWS; k < n_parts; k += kSubs) {
                const float2 x = fetch2(part_slot(k) + ROWS * DP + 2 * row);
                const float up = fmaxf(mm, x.x);
                ll = add_sums(ll, mm, x.y, x.x, up);
                mm = up;
            }
            s_red[2 * et] = mm;
            s_red[2 * et + 1] = ll;
            __syncthreads();
            if (et < ROWS) {
                for (int k = 1; k < kSubs; ++k) {
                    const float xm = s_red[2 * (k * ROWS + et)], xl = s_red[2 * (k * ROWS + et) + 1];
                    const float up = fmaxf(mm, xm);
                    ll = add_sums(ll, mm, xl, xm, up);
                    mm = up;
                }
                s_top[et] = mm;
                s_sum[et] = ll;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NP; ++i) y[i] = make_float2(0.f, 0.f);
            for (int k0 = 0; k0 < n_parts; k0 += kBatch) {
                const int nk = min(kBatch, n_parts - k0);
                for (int i = et; i < nk * ROWS; i += NT) {
                    const float pm = fetch2(part_slot(k0 + i / ROWS) + ROWS * DP + 2 * (i % ROWS)).x;
                    s_fac[i] = pm == kNoScore ? 0.f : exp2_hw(pm - s_top[i % ROWS]);
                }
                __syncthreads();
                // all of a part's loads set out before one is waited for, and the next part's before this one is added
                float2 x[NP], x_next[NP];
                auto fetch = [&](int k, float2 (&into)[NP]) {
                    const float* src = part_slot(k0 + k) + 2 * et;
#pragma unroll
                    for (int i = 0; i < NP; ++i) into[i] = fetch2(src + 2 * i * NT);
                };
                fetch(0, x);
                for (int k = 0; k < nk; ++k) {
                    fetch(min(k + 1, nk - 1), x_next);
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const float f = s_fac[k * ROWS + (i * NT + et) * 2 / DP];
                        y[i].x += x[i].x * f;
                        y[i].y += x[i].y * f;
                        x[i] = x_next[i];
                    }
                }
                __syncthreads();
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = (i * NT + et) * 2;
            const int row = e / DP, d = e % DP;
            if (row >= rows || d >= c.D) continue;
            const int rr = row0 + row, ri = rr / p.h;
            const int head = g * p.h + rr - ri * p.h;
            const int64_t t = s.row0 + ri;
            const bool none = s_top[row] == kNoScore && s_sum[row] == 0.f;
            const float by = none ? 0.f : 1.f / s_sum[row];
            const float y0 = none ? 0.f : y[i].x * by, y1 = none ? 0.f : y[i].y * by;
            char* dst = (char*)a.out.data + (t * a.out.stride_row + (int64_t)head * a.out.stride_head + d) * E::kBytes;
            if constexpr (BF16)
                *(uint32_t*)dst = pack_bf16(y0, y1);
            else
                *(float2*)dst = make_float2(y0, y1);
            if (d == 0 && a.lse) a.lse[t * a.H + head] = none ? kNoScore : (s_top[row] + log2f(s_sum[row])) * kLn2;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- many rows

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
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DP, int NW>
struct TileShape {
    static constexpr int TOK = 64;
    static constexpr int NT = 64 * NW;
    static constexpr int ROWS = 32 * NW;
    static constexpr int LPR = DP / 8;              // 16-byte pieces of a token
    static constexpr int TPP = NT / LPR;      // tokens of one load of the workgroup
    static constexpr int N = TOK / TPP;             // loads a block
    // Row pitches (elements): 8 lanes reading 16 bytes of 8 consecutive keys, and the 4-token by
    // 64-byte tiles of the transposing reads, fall on different banks.
    static constexpr int KP = DP + 8, VP = DP + 32;
    static constexpr int BYTES = TOK * (KP + VP) * 2;
};

template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, (DP == 256 || NW == 8 ? 1 : 2)) void tile_kernel(AttentionArgs a, Plan p) {
    using S = TileShape<DP, NW>;
    constexpr int KK = DP / 16, DB = DP / 32;
    __shared__ __align__(16) char s_mem[2 * S::BYTES];  // two buffers of keys and values
    __shared__ int64_t s_off[4][S::TOK];                // written two blocks ahead, read in two
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
        if (j >= c1 || (unsigned)page >= (unsigned)c.pages) return -1;
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
    struct Stage {
        u32x4 k[S::N], v[S::N];
    };
    auto load = [&](int blk, Stage& x) {
#pragma unroll
        for (int k = 0; k < S::N; ++k) {
            const int64_t at = s_off[blk & 3][k * S::TPP + token] * 2;
            x.k[k] = *(const u32x4*)(k_src + at);
            x.v[k] = *(const u32x4*)(v_src + at);
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
            // exponentials and reads go between the products.
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
            u32x4 again[S::N];
#pragma unroll
            for (int k = 0; k < S::N; ++k) again[k] = *(const u32x4*)(v_src + s_off[blk & 3][k * S::TPP + token] * 2);
            __syncthreads();
            char* values = value_at(blk);
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
        hipLaunchKernelGGL((tile_kernel<DP, 8>), grid, dim3(512), 0, stream, a, p);
    else
        hipLaunchKernelGGL((tile_kernel<DP, 4>), grid, dim3(256), 0, stream, a, p);
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
            hipLaunchKernelGGL((tile_kernel<256, 4>), grid, dim3(256), 0, stream, a, p);
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
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts <= 1) return e;
    const dim3 joins((unsigned)(((long)c.rows * a.H + kWaves - 1) / kWaves));
    hipLaunchKernelGGL(join_kernel, joins, dim3(kThreads), 0, stream, a, p);
    return hipGetLastError();
}

}  // namespace psd
