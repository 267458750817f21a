// psd_attention_device.hpp -- what the attention kernels over the paged caches share: which positions a row sees,
// matrix products, how a workgroup finds its stretch of the work, and how the outputs of waves and of parts
// are joined (device; internal to libpsd).
#pragma once

#include <hip/hip_runtime.h>

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

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

// LDS of a few-row kernel's workgroup beside its values.
template <int NT, int ROWS>
struct StreamShared {
    float m[NT / 64][ROWS], l[NT / 64][ROWS], top[ROWS], sum[ROWS];
    int units[NT + 1], wave[NT / 64], longest[NT / 64];
    int parts[3];  // aligned: workgroups before the item's, its own, and all
    Seq seq[NT];  // of the items, while there are no more than threads
    int chunk, last;
};

// A workgroup's stretch [u0, u1) of the units of all items in a row, which begins in item `item`, whose units
// begin at `before`.
struct Stretch {
    int items, each, u0, u1, item, before;
    bool whole_items;  // (or aligned: stretches end where items end)
    int first, parts;  // aligned: the item's first workgroup and its workgroups
    Division cut;
    template <class Shared>
    __device__ int start(const Shared& sh, int w) const {
        return whole_items ? sh.units[min(w, items)] : cut.start(w);
    }
};

// Workgroup wg's stretch, an empty one (u0 == u1) where there is none.  Lengths are known on the device alone, so each
// workgroup scans them.  SLACK > 0: stretches of one length that end where an item ends, where aligned_length says so.
template <int SLACK, int NT, int ROWS>
__device__ __forceinline__ Stretch find_stretch(const AttentionArgs& a, const Plan& p, StreamShared<NT, ROWS>& sh, int wg,
                                                int least_units) {
    constexpr int NW = NT / 64;
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    // units before each thread's items, by a scan over the workgroup
    const int items = c.B * p.tiles;
    const int each = (items + NT - 1) / NT;
    auto seq_at = [&](int i) { return load_seq(c, i / p.tiles); };
    auto units_at = [&](int i, const Seq& s) { return item_units(a.mask != nullptr, a.window, p, s, i % p.tiles); };
    int mine = 0, longest = 0;
    for (int i = tid * each; i < min((tid + 1) * each, items); ++i) {
        const Seq s = seq_at(i);
        const int n = units_at(i, s);
        sh.seq[tid] = s;
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
        sh.wave[wave] = upto;
        sh.longest[wave] = longest;
    }
    __syncthreads();
    for (int w = 0; w < NW; ++w) {
        if (w < wave) upto += sh.wave[w];
        longest = max(longest, sh.longest[w]);
    }
    sh.units[tid + 1] = upto;
    if (tid == 0) sh.units[0] = 0;
    __syncthreads();
    const int units = uniform(sh.units[NT]);
    // While no item is much longer than a stretch, each workgroup takes one item whole and none is joined.
    const Division cut = divide(units, p.wgs, SLACK > 0 ? least_units4(least_units, uniform(longest)) : least_units);
    const bool whole_items = SLACK == 0 && each == 1 && items <= p.wgs && uniform(longest) <= units / p.wgs + 1 + least_units;
    Stretch st;
    st.first = st.parts = 0;
    if constexpr (SLACK > 0) {
        const int most = uniform(longest);
        const int length = each == 1 ? aligned_length(units, items, most, p.wgs, least_units, SLACK) : 0;
        if (length > 0) {
            st.items = items;
            st.each = 1;
            st.whole_items = true;
            st.cut = cut;
            st.u0 = st.u1 = st.item = st.before = 0;
            if (most <= length) {  // an item each
                if (wg >= items) return st;
                st.item = wg;
                st.before = st.u0 = uniform(sh.units[wg]);
                st.u1 = uniform(sh.units[wg + 1]);
                return st;
            }
            // workgroups before each item, by a scan as above
            const int mine = tid < items ? aligned_parts(sh.units[tid + 1] - sh.units[tid], length) : 0;
            int upto = mine;
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) {
                const int below = __shfl_up(upto, k);
                if (lane >= k) upto += below;
            }
            if (lane == 63) sh.wave[wave] = upto;
            __syncthreads();
            for (int w = 0; w < wave; ++w) upto += sh.wave[w];
            if (upto - mine <= wg && wg < upto) {
                sh.chunk = tid;
                sh.parts[0] = upto - mine;
                sh.parts[1] = mine;
            }
            if (tid == NT - 1) sh.parts[2] = upto;
            __syncthreads();
            if (wg >= uniform(sh.parts[2])) return st;
            st.item = uniform(sh.chunk);
            st.first = uniform(sh.parts[0]);
            st.parts = uniform(sh.parts[1]);
            st.before = uniform(sh.units[st.item]);
            st.u0 = st.before + (wg - st.first) * length;
            st.u1 = min(st.u0 + length, uniform(sh.units[st.item + 1]));
            return st;
        }
    }
    st.items = items;
    st.each = each;
    st.whole_items = whole_items;
    st.cut = cut;
    st.u0 = st.u1 = st.item = st.before = 0;
    if (wg >= (whole_items ? items : cut.wgs)) return st;
    st.u0 = uniform(st.start(sh, wg));
    st.u1 = uniform(st.start(sh, wg + 1));
    if (st.u0 == st.u1) return st;
    if (sh.units[tid] <= st.u0 && st.u0 < sh.units[tid + 1]) sh.chunk = tid;
    __syncthreads();
    const int chunk = uniform(sh.chunk);
    st.item = chunk * each;
    st.before = uniform(sh.units[chunk]);
    return st;
}

// One item of a stretch: row tile [row0, row0 + rows) of a sequence, units [before, before + n_units), of which the
// workgroup computed [from, to).
struct Item {
    Seq s;
    int row0, rows, before, n_units, from, to;
};

// Joins the waves' outputs o, maxima m and sums l of an item, and the parts of one that is cut; writes the rows.  A part is
// left in the workspace, and the workgroup that leaves last joins them, in the order of the parts.
// AHEAD: parts whose outputs are in flight together.
template <bool BF16, int DP, int RB, int NT, int AHEAD = 2>
__device__ __forceinline__ void finish_item(const AttentionArgs& a, const Plan& p, StreamShared<NT, 16 * RB>& sh, char* s_mem,
                                            const Stretch& st, const Item& it, int wg, int g, f32x4 (&o)[RB][DP / 16], float (&m)[RB],
                                            float (&l)[RB]) {
    using E = Elem<BF16>;
    constexpr int DB = DP / 16, NW = NT / 64, ROWS = 16 * RB;
    const CacheArgs& c = a.c;
    const Seq& s = it.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    constexpr int kSlot = ROWS * DP + 2 * ROWS;  // floats of what a workgroup leaves of an item
    auto slot_of = [&](int w, int second) {
        return (float*)a.workspace + kCounterFloats + (((int64_t)w * c.G + g) * 2 + second) * kSlot;
    };
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
            sh.m[wave][rb * 16 + er] = m[rb];
            sh.l[wave][rb * 16 + er] = l[rb];
        }
    }
    __syncthreads();
    float* s_o = (float*)s_mem;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = rb * 16 + er;
        float top = kNoScore;
        for (int w = 0; w < NW; ++w) top = fmaxf(top, sh.m[w][row]);
        const float by = m[rb] == kNoScore ? 0.f : exp2_hw(m[rb] - top);
#pragma unroll
        for (int db = 0; db < DB; ++db) *(f32x4*)(s_o + (wave * ROWS + row) * OP + db * 16 + 4 * eq) = o[rb][db] * by;
        if (wave == 0 && eq == 0) {
            float sum = 0.f;
            for (int w = 0; w < NW; ++w) sum = add_sums(sum, top, sh.l[w][row], sh.m[w][row], top);
            sh.top[row] = top;
            sh.sum[row] = sum;
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
    if (it.from != it.before || it.to != it.before + it.n_units) {
        // A part of an item.  What a workgroup leaves of an item that its stretch begins with goes to
        // its first slot, of one that begins later to its second.
        const bool aligned = st.parts > 0;
        const int w_first = aligned ? st.first : st.cut.owner(it.before);
        const int n_parts = aligned ? st.parts : st.cut.owner(it.before + it.n_units - 1) - w_first + 1;
        float* dst = slot_of(wg, it.from == st.u0 ? 0 : 1);
#pragma unroll
        for (int i = 0; i < NP; ++i) leave2(dst + (i * NT + et) * 2, y[i].x, y[i].y);
        if (et < ROWS) leave2(dst + ROWS * DP + 2 * et, sh.top[et], sh.sum[et]);
        // all of it is written when the counter goes up: the workgroup that counts last finds every part
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (et == 0) {
            unsigned* counter = (unsigned*)a.workspace + w_first * c.G + g;
            const unsigned was = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh.last = was == (unsigned)(n_parts - 1);
            if (sh.last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!sh.last) return;  // sh.last is written again two barriers later at the earliest
        // The parts' common maximum and sum of each row, then their outputs, kBatch parts at a time.  The first AHEAD parts'
        // outputs set out before the maxima are known, each later one as one is added.
        constexpr int kSubs = NT / ROWS, kBatch = 2048 / ROWS;
        static_assert(kBatch % AHEAD == 0, "a part's registers follow from its place in a batch");
        float* s_red = (float*)s_mem;   // [kSubs][ROWS][2]
        float* s_fac = s_red + 2 * NT;  // [kBatch][ROWS]: the parts' maxima, then factors
        const int first_slot = aligned || it.before == st.start(sh, w_first) ? 0 : 1;
        auto part_slot = [&](int k) { return slot_of(w_first + k, k == 0 ? first_slot : 0); };
        float2 x[AHEAD][NP];
        auto fetch = [&](int k, float2 (&into)[NP]) {
            const float* src = part_slot(min(k, n_parts - 1)) + 2 * et;
#pragma unroll
            for (int i = 0; i < NP; ++i) into[i] = fetch2(src + 2 * i * NT);
        };
        const int row = et % ROWS;
        float mm = kNoScore, ll = 0.f;
        constexpr int kLoads = 4;
        for (int k0 = et / ROWS; k0 < n_parts; k0 += kLoads * kSubs) {
            float2 ml[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) ml[i] = fetch2(part_slot(min(k0 + i * kSubs, n_parts - 1)) + ROWS * DP + 2 * row);
            if (k0 == et / ROWS)
#pragma unroll
                for (int n = 0; n < AHEAD; ++n) fetch(n, x[n]);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int k = k0 + i * kSubs;
                if (k >= n_parts) break;
                const float up = fmaxf(mm, ml[i].x);
                ll = add_sums(ll, mm, ml[i].y, ml[i].x, up);
                mm = up;
                if (k < kBatch) s_fac[k * ROWS + row] = ml[i].x;
            }
        }
        if (et / ROWS >= n_parts)
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) fetch(n, x[n]);
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
            sh.top[et] = mm;
            sh.sum[et] = ll;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NP; ++i) y[i] = make_float2(0.f, 0.f);
        for (int k0 = 0; k0 < n_parts; k0 += kBatch) {
            const int nk = min(kBatch, n_parts - k0);
            for (int i = et; i < nk * ROWS; i += NT) {
                const float pm = k0 == 0 ? s_fac[i] : fetch2(part_slot(k0 + i / ROWS) + ROWS * DP + 2 * (i % ROWS)).x;
                s_fac[i] = pm == kNoScore ? 0.f : exp2_hw(pm - sh.top[i % ROWS]);
            }
            __syncthreads();
            for (int k = 0; k < nk; k += AHEAD)
#pragma unroll
                for (int n = 0; n < AHEAD; ++n) {
                    if (k + n >= nk) break;
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const float f = s_fac[(k + n) * ROWS + (i * NT + et) * 2 / DP];
                        y[i].x += x[n][i].x * f;
                        y[i].y += x[n][i].y * f;
                    }
                    fetch(k0 + k + n + AHEAD, x[n]);
                }
            __syncthreads();
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int e = (i * NT + et) * 2;
        const int row = e / DP, d = e % DP;
        if (row >= it.rows || d >= c.D) continue;
        const int rr = it.row0 + row, ri = rr / p.h;
        const int head = g * p.h + rr - ri * p.h;
        const int64_t t = s.row0 + ri;
        const bool none = sh.top[row] == kNoScore && sh.sum[row] == 0.f;
        const float by = none ? 0.f : 1.f / sh.sum[row];
        const float y0 = none ? 0.f : y[i].x * by, y1 = none ? 0.f : y[i].y * by;
        char* dst = (char*)a.out.data + (t * a.out.stride_row + (int64_t)head * a.out.stride_head + d) * E::kBytes;
        if constexpr (BF16)
            *(uint32_t*)dst = pack_bf16(y0, y1);
        else
            *(float2*)dst = make_float2(y0, y1);
        if (d == 0 && a.lse) a.lse[t * a.H + head] = none ? kNoScore : (sh.top[row] + log2f(sh.sum[row])) * kLn2;
    }
    __syncthreads();
}

}  // namespace psd
