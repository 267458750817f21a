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

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// How a call is cut, by the host's bounds alone.
struct Plan {
    int h;          // rows per new token: H / G
    int tile_rows;  // rows of a workgroup
    int tiles;      // row tiles of the longest sequence
    int parts;      // parts of the longest range of cached tokens
    int chunk;      // cached tokens of a part
    int page_shift; // log2 of the page size, or -1
};

struct Range {
    int lo, hi;  // cached positions that some row of a tile sees
};

// Rows [row0, row0 + rows) of a sequence see positions [lo, hi) at most.
__device__ __forceinline__ Range tile_range(const AttentionArgs& a, const Seq& s, int i_lo, int i_hi) {
    Range r;
    r.lo = 0;
    r.hi = s.kv;
    if (!a.mask) {
        r.hi = max(min(s.kv, s.first + i_hi + 1), 0);
        if (a.window > 0) r.lo = min(max(s.first + i_lo - a.window + 1, 0), r.hi);
    }
    return r;
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

__device__ __forceinline__ int64_t token_offset(const CacheArgs& c, const Plan& p, const int32_t* table, int j) {
    const int pi = p.page_shift >= 0 ? j >> p.page_shift : j / c.P;
    const int page = table[pi];
    if ((unsigned)page >= (unsigned)c.pages) return -1;
    return (int64_t)page * c.stride_page + (int64_t)(j - pi * c.P) * c.stride_token;
}

// Infinite or NaN: the upper (float32: the) element of a word, and the lower one of two bfloat16.
__device__ __forceinline__ bool odd_hi(uint32_t w) { return (w & 0x7F800000u) == 0x7F800000u; }
template <bool BF16>
__device__ __forceinline__ bool odd_lo(uint32_t w) {
    return BF16 && (w & 0x7F80u) == 0x7F80u;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

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

// A block's softmax weights of this lane's row as a B operand.
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

// ---------------------------------------------------------------- few rows

// One workgroup: up to 16 RB rows of one (sequence, key/value head) over one part of its cache.
// Its waves take blocks of TOK tokens in turn, each with a softmax of its own, joined at the
// end; no wave waits for another in between.  Keys go from memory straight into the A operand
// (a lane's 16 bytes are consecutive dimensions of one token); values pass through the wave's own
// LDS, where bfloat16 is transposed by ds_read_b64_tr_b16 (16 lanes read a 4-token by 16-dimension
// tile and each gets one dimension's 4 tokens).  While a block is computed, the next one's
// keys and values are on their way into registers.
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

template <bool BF16, int DP, int RB>
constexpr int stream_lds() {
    using S = StreamShape<BF16, DP>;
    constexpr int values = kWaves * S::V_BYTES;
    constexpr int join = 2 * 16 * RB * DP * 4;
    return values > join ? values : join;
}

template <bool BF16, int DP, int RB>
__global__ __launch_bounds__(kThreads, (RB * DP >= 512 || DP == 256 ? 1 : 2)) void stream_kernel(AttentionArgs a, Plan p) {
    using S = StreamShape<BF16, DP>;
    using E = Elem<BF16>;
    constexpr int DB = DP / 16;
    __shared__ __align__(16) char s_mem[stream_lds<BF16, DP, RB>()];
    __shared__ int64_t s_off[kWaves][2][S::TOK];
    __shared__ float s_m[kWaves][16 * RB], s_l[kWaves][16 * RB];

    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = lane & 15, q = lane >> 4;
    int x = blockIdx.x;
    const int g = x % c.G;
    x /= c.G;
    const int tile = x % p.tiles;
    x /= p.tiles;
    const int b = x % c.B, part = x / c.B;

    const Seq s = load_seq(c, b);
    const int row0 = tile * p.tile_rows;
    const int rows = min(s.n * p.h - row0, p.tile_rows);
    if (rows <= 0) return;
    const int i_lo = row0 / p.h, i_hi = (row0 + rows - 1) / p.h;
    const Range range = tile_range(a, s, i_lo, i_hi);
    const int n_parts = max((range.hi - range.lo + p.chunk - 1) / p.chunk, 1);
    if (part >= n_parts) return;
    const int c0 = range.lo + part * p.chunk, c1 = min(c0 + p.chunk, range.hi);
    const int blocks = (c1 - c0 + S::TOK - 1) / S::TOK;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;

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
            qf[rb][kk] = on && d < c.D ? *(const u32x4*)(src + d * E::kBytes) : u32x4{0, 0, 0, 0};
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
    const float sc = a.scale * kLog2e;
    const int64_t head_at = (int64_t)g * c.stride_head;
    char* s_v = s_mem + wave * S::V_BYTES;

    // A block's tokens: lane t < TOK finds token t's place; -1: nothing there.
    auto locate = [&](int blk) -> int64_t {
        const int j = c0 + blk * S::TOK + lane;
        if (lane >= S::TOK || blk >= blocks || j >= c1) return -1;
        return token_offset(c, p, table, j);
    };
    // Loads are unconditional: a token that is not there reads the pool's first one instead, whose
    // scores are masked and whose values are zeroed, and a piece past the head's end reads its
    // last piece, which counts as zero in a key and goes to no output in a value.
    u32x4 kf[S::TT][S::KK], vf[S::NV];
    auto load_keys = [&](int slot) {
#pragma unroll
        for (int t = 0; t < S::TT; ++t) {
            const char* src = (const char*)c.k + (s_off[wave][slot][16 * t + r] + head_at) * E::kBytes;
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk)
                kf[t][kk] = *(const u32x4*)(src + min(kk * S::KSTEP + q * S::VEC, c.D - S::VEC) * E::kBytes);
        }
    };
    auto load_values = [&](int slot) {
        const int d = min((lane % S::LPR) * S::VEC, c.D - S::VEC);
        const char* src = (const char*)c.v + (head_at + d) * E::kBytes;
#pragma unroll
        for (int k = 0; k < S::NV; ++k)
            vf[k] = *(const u32x4*)(src + s_off[wave][slot][k * S::TPI + lane / S::LPR] * E::kBytes);
    };
    auto wave_sync = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    int64_t off = locate(wave), off_next = locate(wave + kWaves);
    if (lane < S::TOK) s_off[wave][0][lane] = max(off, (int64_t)0);
    wave_sync();
    if (wave < blocks) {
        load_keys(0);
        load_values(0);
    }
    int slot = 0;
    for (int blk = wave; blk < blocks; blk += kWaves, slot ^= 1) {
        const int j0 = c0 + blk * S::TOK;
        const uint32_t there = (uint32_t)__ballot(lane < S::TOK && off >= 0);
        const bool more = blk + kWaves < blocks;
        // every row sees the whole block, or bits say which tokens
        const uint32_t every = S::TOK == 32 ? ~0u : (1u << S::TOK) - 1u;
        const bool whole = there == every &&
                           (a.mask ? j0 + S::TOK <= s.first
                                   : j0 + S::TOK - 1 <= s.first + i_lo && (a.window == 0 || j0 > s.first + i_hi - a.window));
        if (c.D < DP) {
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk)
                if (kk * S::KSTEP + q * S::VEC >= c.D)
#pragma unroll
                    for (int t = 0; t < S::TT; ++t) kf[t][kk] = u32x4{0, 0, 0, 0};
        }
        Weights<BF16> w[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            f32x4 sv[S::TT];
#pragma unroll
            for (int t = 0; t < S::TT; ++t) {
                sv[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < S::KK; ++kk) sv[t] = multiply<BF16>(kf[t][kk], qf[rb][kk], sv[t]);
            }
            if (rb == RB - 1) {
                // the next block's keys set out
                off = off_next;
                if (lane < S::TOK) s_off[wave][slot ^ 1][lane] = max(off, (int64_t)0);
                wave_sync();
                if (more) load_keys(slot ^ 1);
                off_next = locate(blk + 2 * kWaves);
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

        // Values.  A row's weight 0 times an infinite or NaN value that the row does not see
        // would be NaN: where rows differ in what they see, such elements are taken out, and a second
        // product of the largest finite numbers puts infinity where a row does see one.
        bool odd = false;
        if (!whole) {
            bool mine = false;
#pragma unroll
            for (int k = 0; k < S::NV; ++k) {
                const bool gone = !((there >> (k * S::TPI + lane / S::LPR)) & 1u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (gone) vf[k][e] = 0;
                    mine |= odd_lo<BF16>(vf[k][e]) || odd_hi(vf[k][e]);
                }
            }
            odd = __any(mine);
        }
        auto put = [&]() {
#pragma unroll
            for (int k = 0; k < S::NV; ++k)
                *(u32x4*)(s_v + ((k * S::TPI + lane / S::LPR) * S::PITCH + (lane % S::LPR) * S::VEC) * E::kBytes) = vf[k];
            wave_sync();
        };
        // V^T of 16 dimensions as an A operand: this lane's dimension of the tokens of its weights
        auto get = [&](int db) -> u32x4 {
            if constexpr (BF16) {
                char* at = s_v + ((4 * q + r / 4) * S::PITCH + db * 16 + (r % 4) * 4) * 2;
                union {
                    s16x4 half[2];
                    u32x4 all;
                } v;
                v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
                v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(at + 16 * S::PITCH * 2));
                return v.all;
            } else {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = *(const uint32_t*)(s_v + ((4 * q + e) * S::PITCH + db * 16 + r) * 4);
                return v;
            }
        };
        if (odd) {
#pragma unroll
            for (int k = 0; k < S::NV; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (odd_lo<BF16>(vf[k][e])) vf[k][e] &= 0xFFFF0000u;
                    if (odd_hi(vf[k][e])) vf[k][e] &= BF16 ? 0xFFFFu : 0u;
                }
        }
        put();
        if (more && !odd) load_values(slot ^ 1);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const u32x4 v = get(db);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) o[rb][db] = multiply<BF16>(v, w[rb].all, o[rb][db]);
        }
        wave_sync();
        if (odd) {
            load_values(slot);
            constexpr uint32_t kLo = BF16 ? 0x7F7Fu : 0u, kHi = BF16 ? 0x7F7F0000u : 0x7F7FFFFFu;  // largest finite
#pragma unroll
            for (int k = 0; k < S::NV; ++k) {
                const bool gone = !((there >> (k * S::TPI + lane / S::LPR)) & 1u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t w = vf[k][e];
                    vf[k][e] = gone ? 0u : (odd_lo<BF16>(w) ? kLo : 0u) | (odd_hi(w) ? kHi : 0u);
                }
            }
            put();
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
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x4 v = get(db);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][db] = multiply<BF16>(v, w[rb].all, o[rb][db]);
            }
            wave_sync();
            if (more) load_values(slot ^ 1);
        }
    }

    // join the waves: a common maximum, then the outputs added pairwise through LDS
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        l[rb] += __shfl_xor(l[rb], 16);
        l[rb] += __shfl_xor(l[rb], 32);
        if (q == 0) {
            s_m[wave][rb * 16 + r] = m[rb];
            s_l[wave][rb * 16 + r] = l[rb];
        }
    }
    __syncthreads();
    float top[RB], total[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        top[rb] = kNoScore;
        total[rb] = 0.f;
        for (int w = 0; w < kWaves; ++w) top[rb] = fmaxf(top[rb], s_m[w][rb * 16 + r]);
        if (top[rb] != kNoScore)
            for (int w = 0; w < kWaves; ++w) total[rb] += s_l[w][rb * 16 + r] * exp2_hw(s_m[w][rb * 16 + r] - top[rb]);
        const float by = m[rb] == kNoScore ? 0.f : exp2_hw(m[rb] - top[rb]);
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] *= by;
    }
    float* s_o = (float*)s_mem;
#pragma unroll
    for (int step = kWaves / 2; step > 0; step /= 2) {
        if (wave >= step && wave < 2 * step) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    *(f32x4*)(s_o + ((((wave - step) * RB + rb) * DB + db) * 64 + lane) * 4) = o[rb][db];
        }
        __syncthreads();
        if (wave < step) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    o[rb][db] += *(const f32x4*)(s_o + (((wave * RB + rb) * DB + db) * 64 + lane) * 4);
        }
        __syncthreads();
    }
    if (wave != 0) return;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        if (rb * 16 + r >= rows) continue;
        const int rr = row0 + rb * 16 + r;
        const int head = g * p.h + rr - row_i[rb] * p.h;
        const int64_t t = s.row0 + row_i[rb];
        if (n_parts == 1) {
            const float by = top[rb] == kNoScore ? 0.f : 1.f / total[rb];
            char* dst = (char*)a.out.data + (t * a.out.stride_row + (int64_t)head * a.out.stride_head) * E::kBytes;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const int d = db * 16 + 4 * q;
                if (d >= c.D) continue;
                const f32x4 y = top[rb] == kNoScore ? f32x4{0.f, 0.f, 0.f, 0.f} : o[rb][db] * by;
                if constexpr (BF16)
                    *(uint2*)(dst + d * 2) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
                else
                    *(f32x4*)(dst + d * 4) = y;
            }
            if (q == 0 && a.lse) a.lse[t * a.H + head] = top[rb] == kNoScore ? kNoScore : (top[rb] + log2f(total[rb])) * kLn2;
        } else {
            const int64_t at = ((int64_t)part * c.rows + t) * a.H + head;
            float* dst = (float*)a.workspace + at * c.D;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const int d = db * 16 + 4 * q;
                if (d < c.D) *(f32x4*)(dst + d) = o[rb][db];
            }
            if (q == 0) {
                float2* ml = (float2*)((float*)a.workspace + (int64_t)p.parts * c.rows * a.H * c.D);
                ml[at] = make_float2(top[rb], total[rb]);
            }
        }
    }
}

// ---------------------------------------------------------------- many rows

// One workgroup: 128 rows of one (sequence, key/value head), 32 a wave, over one part of its cache.
// Blocks of 64 tokens go through LDS, which all four waves read: 32x32x16 products, 64 x 32
// scores a wave in 32 registers, the outputs in D/2 more.  Two buffers, one barrier a block: while
// block n is computed, block n + 1 is on its way into registers, and is stored behind the
// arithmetic.  Two workgroups a CU (two waves a SIMD), so one wave's exponentials overlap
// the other's products.
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int DP>
struct TileShape {
    static constexpr int TOK = 64;
    static constexpr int ROWS = 128;
    static constexpr int LPR = DP / 8;              // 16-byte pieces of a token
    static constexpr int TPP = kThreads / LPR;      // tokens of one load of the workgroup
    static constexpr int N = TOK / TPP;             // loads a block
    // Row pitches (elements): 8 lanes reading 16 bytes of 8 consecutive keys, and the 4-token by
    // 64-byte tiles of the transposing reads, fall on different banks.
    static constexpr int KP = DP + 8, VP = DP + 32;
    static constexpr int BYTES = TOK * (KP + VP) * 2;
};

template <int DP>
__global__ __launch_bounds__(kThreads, (DP == 256 ? 1 : 2)) void tile_kernel(AttentionArgs a, Plan p) {
    using S = TileShape<DP>;
    constexpr int KK = DP / 16, DB = DP / 32;
    __shared__ __align__(16) char s_mem[2 * S::BYTES];  // two buffers of keys and values
    __shared__ int64_t s_off[4][S::TOK];                // written two blocks ahead, read in two
    __shared__ uint64_t s_there[4];
    __shared__ int s_odd[2];

    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = lane & 31, hi = lane >> 5;
    int x = blockIdx.x;
    const int g = x % c.G;
    x /= c.G;
    const int tile = p.tiles - 1 - x % p.tiles;  // causal rows: the longest first
    x /= p.tiles;
    const int b = x % c.B, part = x / c.B;

    const Seq s = load_seq(c, b);
    const int row0 = tile * S::ROWS;
    const int rows = min(s.n * p.h - row0, S::ROWS);
    if (rows <= 0) return;
    const int i_lo = row0 / p.h, i_hi = (row0 + rows - 1) / p.h;
    const Range range = tile_range(a, s, i_lo, i_hi);
    const int n_parts = max((range.hi - range.lo + p.chunk - 1) / p.chunk, 1);
    if (part >= n_parts) return;
    const int c0 = range.lo + part * p.chunk, c1 = min(c0 + p.chunk, range.hi);
    const int blocks = (c1 - c0 + S::TOK - 1) / S::TOK;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;

    // this wave's rows: new tokens [w_lo, w_hi]; a wave without rows keeps company with zeros
    const int mine = min(max(rows - wave * 32, 0), 32);
    const int w_lo = (row0 + min(wave * 32, rows - 1)) / p.h, w_hi = (row0 + min(wave * 32 + 31, rows - 1)) / p.h;
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
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const int d = kk * 16 + hi * 8;
            qf[kk] = u32x4{0, 0, 0, 0};
            if (on && d < c.D) {
                qf[kk] = *(const u32x4*)(src + d * 2);
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[kk][e] ^= sign;
            }
        }
    }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
    float m = kNoScore, l = 0.f;

    const int64_t head_at = (int64_t)g * c.stride_head;
    const int piece = tid % S::LPR, token = tid / S::LPR;
    const int d_piece = min(piece * 8, c.D - 8);
    const bool past = piece * 8 >= c.D;  // keys past the head's end count as zero
    const char* k_src = (const char*)c.k + (head_at + d_piece) * 2;
    const char* v_src = (const char*)c.v + (head_at + d_piece) * 2;

    auto locate = [&](int blk) -> int64_t {  // threads of wave 0
        const int j = c0 + blk * S::TOK + tid;
        if (blk >= blocks || j >= c1) return -1;
        return token_offset(c, p, table, j);
    };
    auto publish = [&](int blk, int64_t off) {
        s_off[blk & 3][tid] = max(off, (int64_t)0);
        const uint64_t bits = __ballot(off >= 0);
        if (tid == 0) s_there[blk & 3] = bits;
    };
    u32x4 kf[S::N], vf[S::N];
    auto load = [&](int blk) {
#pragma unroll
        for (int k = 0; k < S::N; ++k) {
            const int64_t at = s_off[blk & 3][k * S::TPP + token] * 2;
            kf[k] = *(const u32x4*)(k_src + at);
            vf[k] = *(const u32x4*)(v_src + at);
        }
    };
    // Does every row of new tokens [lo, hi] see the whole block?
    auto whole = [&](int blk, int lo, int top) {
        const int j0 = c0 + blk * S::TOK;
        if (s_there[blk & 3] != ~0ull) return false;
        if (a.mask) return j0 + S::TOK <= s.first;
        return j0 + S::TOK - 1 <= s.first + lo && (a.window == 0 || j0 > s.first + top - a.window);
    };
    auto key_at = [&](int blk) { return s_mem + (blk & 1) * S::BYTES; };
    auto value_at = [&](int blk) { return s_mem + (blk & 1) * S::BYTES + S::TOK * S::KP * 2; };
    // Into LDS.  Where rows differ in what they see, values of tokens that are not there are zeroed
    // and infinite or NaN values taken out (a weight 0 times them is NaN for rows that do not see them).
    auto store = [&](int blk) {
        if (past)
#pragma unroll
            for (int k = 0; k < S::N; ++k) kf[k] = u32x4{0, 0, 0, 0};
        if (!whole(blk, i_lo, i_hi)) {
            const uint64_t there = s_there[blk & 3];
            bool odd = false;
#pragma unroll
            for (int k = 0; k < S::N; ++k) {
                const bool gone = !((there >> (k * S::TPP + token)) & 1u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t w = gone ? 0u : vf[k][e];
                    const bool lo_odd = odd_lo<true>(w), hi_odd = odd_hi(w);
                    odd |= lo_odd || hi_odd;
                    if (lo_odd) w &= 0xFFFF0000u;
                    if (hi_odd) w &= 0xFFFFu;
                    vf[k][e] = w;
                }
            }
            if (odd) s_odd[blk & 1] = blk + 1;
        }
        char* keys = key_at(blk);
        char* values = value_at(blk);
#pragma unroll
        for (int k = 0; k < S::N; ++k) {
            *(u32x4*)(keys + ((k * S::TPP + token) * S::KP + piece * 8) * 2) = kf[k];
            *(u32x4*)(values + ((k * S::TPP + token) * S::VP + piece * 8) * 2) = vf[k];
        }
    };
    // this lane's dimension of 32 db + .., tokens 16 ks + {4 hi .., 8 + 4 hi ..}, as an A operand
    auto value = [&](const char* values, int db, int ks) -> bf16x8 {
        const int i = lane & 15;
        const char* at = values + ((16 * ks + 4 * hi + i / 4) * S::VP + db * 32 + ((lane >> 4) & 1) * 16 + (i % 4) * 4) * 2;
        union {
            s16x4 half[2];
            bf16x8 all;
        } v;
        v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * S::VP * 2));
        return v.all;
    };

    int64_t off = -1;
    if (wave == 0) {
        publish(0, locate(0));
        off = locate(1);
    }
    if (tid < 2) s_odd[tid] = 0;
    __syncthreads();
    if (blocks > 0) load(0);
    if (wave == 0) {
        publish(1, off);
        off = locate(2);
    }
    if (blocks > 0) store(0);
    for (int blk = 0; blk < blocks; ++blk) {
        __syncthreads();
        const int j0 = c0 + blk * S::TOK;
        const bool more = blk + 1 < blocks;
        if (more) load(blk + 1);
        const bool seen_by_all = whole(blk, w_lo, w_hi);
        const uint64_t there = s_there[blk & 3];
        // nothing of the block lies before this wave's last row's end (or behind its window)
        const bool idle = mine == 0 || (!a.mask && (j0 > s.first + w_hi ||
                                                    (a.window > 0 && j0 + S::TOK - 1 <= s.first + w_lo - a.window)));
        uint32_t bits[2] = {~0u, ~0u};
        if (!idle) {
            const char* keys = key_at(blk);
            const char* values = value_at(blk);
            f32x16 sv[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sv[t][e] = 0.f;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const u32x4 kv = *(const u32x4*)(keys + ((32 * t + r) * S::KP + kk * 16 + hi * 8) * 2);
                    sv[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kv),
                                                                    __builtin_bit_cast(bf16x8, qf[kk]), sv[t], 0, 0, 0);
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
            }
            float top = sv[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, sv[t][e]);
            top *= sc;
            if (__any(top > m + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float next = fmaxf(m, top);
                const float by = next == kNoScore ? 1.f : exp2_hw(m - next);
                m = next;
                l *= by;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db] *= by;
            }
            const float from = m == kNoScore ? 0.f : m;
            u32x4 w[4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float w0 = exp2_hw(__builtin_fmaf(sv[t][e], sc, -from));
                    const float w1 = exp2_hw(__builtin_fmaf(sv[t][e + 1], sc, -from));
                    l += w0;
                    l += w1;
                    w[2 * t + e / 8][(e % 8) / 2] = pack_bf16(w0, w1);
                }
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(values, db, ks), __builtin_bit_cast(bf16x8, w[ks]), o[db],
                                                                    0, 0, 0);
        }
        if (s_odd[blk & 1] == blk + 1) {
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
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(values, db, ks), __builtin_bit_cast(bf16x8, w[ks]),
                                                                        o[db], 0, 0, 0);
            }
        }
        if (more) store(blk + 1);
        if (wave == 0) {
            publish(blk + 2, off);
            off = locate(blk + 3);
        }
    }

    l += __shfl_xor(l, 32);
    if (!on) return;
    if (n_parts == 1) {
        const float by = m == kNoScore ? 0.f : 1.f / l;
        char* dst = (char*)a.out.data + (t_row * a.out.stride_row + (int64_t)head * a.out.stride_head) * 2;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = db * 32 + 2 * e + 4 * hi;
                if (d >= c.D) continue;
                uint2 y = make_uint2(0, 0);
                if (m != kNoScore)
                    y = make_uint2(pack_bf16(o[db][e] * by, o[db][e + 1] * by), pack_bf16(o[db][e + 2] * by, o[db][e + 3] * by));
                *(uint2*)(dst + d * 2) = y;
            }
        if (hi == 0 && a.lse) a.lse[t_row * a.H + head] = m == kNoScore ? kNoScore : (m + log2f(l)) * kLn2;
    } else {
        const int64_t at = ((int64_t)part * c.rows + t_row) * a.H + head;
        float* dst = (float*)a.workspace + at * c.D;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = db * 32 + 2 * e + 4 * hi;
                if (d < c.D) *(f32x4*)(dst + d) = f32x4{o[db][e], o[db][e + 1], o[db][e + 2], o[db][e + 3]};
            }
        if (hi == 0) {
            float2* ml = (float2*)((float*)a.workspace + (int64_t)p.parts * c.rows * a.H * c.D);
            ml[at] = make_float2(m, l);
        }
    }
}

// Joins the parts of each (row, head): one wave each, the weights of up to 64 parts in its lanes.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void join_kernel(AttentionArgs a, Plan p) {
    using E = Elem<BF16>;
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
    const float2* ml = (const float2*)((const float*)a.workspace + (int64_t)p.parts * c.rows * a.H * c.D);
    const int64_t step = (int64_t)c.rows * a.H;
    float2 mine = make_float2(kNoScore, 0.f);
    if (lane < n_parts) mine = ml[lane * step + item];
    float top = mine.x;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float by = mine.x == kNoScore ? 0.f : exp2_hw(mine.x - top);
    float total = mine.y * by;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) total += __shfl_xor(total, k);
    if (mine.y != mine.y) total = mine.y;
    const int d = lane * 4;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < n_parts; ++k) {
        const float w = __shfl(by, k);
        if (d < c.D && w != 0.f) o += *(const f32x4*)((const float*)a.workspace + (k * step + item) * c.D + d) * w;
    }
    if (d < c.D) {
        const f32x4 y = top == kNoScore ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.f / total);
        char* dst = (char*)a.out.data + ((int64_t)t * a.out.stride_row + (int64_t)head * a.out.stride_head + d) * E::kBytes;
        if constexpr (BF16)
            *(uint2*)dst = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
        else
            *(f32x4*)dst = y;
    }
    if (lane == 0 && a.lse) a.lse[item] = top == kNoScore ? kNoScore : (top + log2f(total)) * kLn2;
}

constexpr int kMaxParts = 64;   // join_kernel holds a part's weight in a lane
constexpr int kMinChunk = 128;  // cached tokens of a part at least: a block per wave
constexpr long kFill = 1024;    // workgroups that fill the device: 4 for each of 256 CUs

Plan make_plan(const CacheArgs& c, int H, bool bf16, int span) {
    Plan p;
    p.h = H / c.G;
    const long most = (long)c.max_new * p.h;
    const int limit = c.D > 128 ? 32 : 64;
    p.tile_rows = most <= 16 ? 16 : most <= 32 ? 32 : bf16 && most > 64 ? 128 : limit;
    p.tiles = (int)((most + p.tile_rows - 1) / p.tile_rows);
    const long groups = (long)c.B * c.G * p.tiles;
    const long want = std::min<long>(std::min<long>((kFill + groups - 1) / groups, (span + kMinChunk - 1) / kMinChunk), kMaxParts);
    p.parts = (int)std::max<long>(want, 1);
    p.chunk = ((span + p.parts - 1) / p.parts + kMinChunk - 1) / kMinChunk * kMinChunk;
    p.parts = (span + p.chunk - 1) / p.chunk;
    p.page_shift = -1;
    for (int k = 0; k <= 16; ++k)
        if (c.P == 1 << k) p.page_shift = k;
    return p;
}

template <bool BF16, int DP>
void launch_stream(const AttentionArgs& a, const Plan& p, dim3 grid, hipStream_t stream) {
    if (p.tile_rows == 16)
        hipLaunchKernelGGL((stream_kernel<BF16, DP, 1>), grid, dim3(kThreads), 0, stream, a, p);
    else if (p.tile_rows == 32)
        hipLaunchKernelGGL((stream_kernel<BF16, DP, 2>), grid, dim3(kThreads), 0, stream, a, p);
    else if constexpr (DP <= 128)
        hipLaunchKernelGGL((stream_kernel<BF16, DP, 4>), grid, dim3(kThreads), 0, stream, a, p);
}

}  // namespace

size_t attention_workspace(const CacheArgs& c, int H, bool bf16) {
    const Plan p = make_plan(c, H, bf16, c.max_kv);
    if (p.parts == 1) return 0;
    return align256((size_t)p.parts * c.rows * H * (c.D + 2) * 4);
}

bool attention_fits(const CacheArgs& c, int H, bool bf16) {
    const Plan p = make_plan(c, H, bf16, c.max_kv);
    return (long)c.B * c.G * p.tiles * p.parts < 1L << 23;
}

hipError_t launch_attention(const AttentionArgs& a, bool bf16, hipStream_t stream) {
    const CacheArgs& c = a.c;
    // a windowed row sees at most `window` positions, a tile's rows together max_new - 1 more
    const int span = a.window > 0 ? (int)std::min<long>(c.max_kv, (long)a.window + c.max_new - 1) : c.max_kv;
    const Plan p = make_plan(c, a.H, bf16, span);
    const dim3 grid((unsigned)((long)c.B * c.G * p.tiles * p.parts));
    if (p.tile_rows == 128) {
        if (c.D <= 64)
            hipLaunchKernelGGL(tile_kernel<64>, grid, dim3(kThreads), 0, stream, a, p);
        else if (c.D <= 128)
            hipLaunchKernelGGL(tile_kernel<128>, grid, dim3(kThreads), 0, stream, a, p);
        else
            hipLaunchKernelGGL(tile_kernel<256>, grid, dim3(kThreads), 0, stream, a, p);
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
    if (e != hipSuccess || p.parts == 1) return e;
    const dim3 joins((unsigned)(((long)c.rows * a.H + kWaves - 1) / kWaves));
    if (bf16)
        hipLaunchKernelGGL(join_kernel<true>, joins, dim3(kThreads), 0, stream, a, p);
    else
        hipLaunchKernelGGL(join_kernel<false>, joins, dim3(kThreads), 0, stream, a, p);
    return hipGetLastError();
}

}  // namespace psd
