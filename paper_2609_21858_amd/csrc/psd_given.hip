// psd_given.hip -- verification of drafted tokens from given random numbers (gfx950).
//
// With p_s, q_s the softmaxes of target and draft row s, draft x_s is accepted while
// u_s q_s(x_s) < p_s(x_s); the token after the accepted ones is argmin_v e_v / r(v) with
// r = max(p_n - q_n, 0) at a refusal and r = p_n after all drafts.  The residual's total is
// not needed: the race is invariant to scale.
//
// Two launches (one for few short rows, see kWhole).  given_stream_kernel reads every row once (memory bounds it: (2 gamma + 1) V
// elements a sequence) and leaves each segment's maximum and sum of exponentials.
// given_race_kernel merges them (every workgroup again: a few hundred values), finds the
// first refusal and races one segment of the one row that decides, whose logits the
// first launch has just brought into the caches; only e comes new from memory.  The last
// workgroup of a sequence writes its tokens.
//
// V=128256, gamma=4, 64 sequences, bfloat16: 26 us for the rows (5.7 TB/s), then 21 - 22 us for the race,
// which its chain bounds: segments' sums, acceptance, the row's and e's first pieces, the second round's pieces of
// the rows, which are asked for only when it begins, then the join (35 MB).  Float32, 32 sequences: 24 us (6.1 TB/s)
// and 17.  V=1024, gamma=4, one sequence: 8.9 us in one launch, two chains of load, exponentials and exchange.
//
// Rounding: maxima are exact; exponentials are of (l - max) / T, where the subtraction is
// exact near the top of a row, and sums are float32 sums of at most a few thousand values a
// thread, merged in trees.  Probabilities are good to a few 1e-7, and a race or an acceptance
// whose two sides are closer than that may go either way (about one in 10^6).
#include <hip/hip_runtime.h>

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNoLogit = -__builtin_inff();
constexpr unsigned long long kNone = ~0ull;

// 16 bytes at any element boundary (rows of an odd vocabulary start off the 16-byte grid;
// one global_load_dwordx4 serves them).
typedef uint32_t u32x4_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_b16 __attribute__((ext_vector_type(4), aligned(2)));
template <bool BF16>
__device__ __forceinline__ u32x4 load_any(const void* base, int64_t element) {
    if constexpr (BF16)
        return *(const u32x4_b16*)((const uint16_t*)base + element);
    else
        return *(const u32x4_f32*)((const float*)base + element);
}
template <bool BF16>
__device__ __forceinline__ float load_one(const void* base, int64_t element) {
    if constexpr (BF16)
        return __uint_as_float((uint32_t)((const uint16_t*)base)[element] << 16);
    else
        return ((const float*)base)[element];
}

// The last, incomplete 16 bytes of a row of floats or logits: n elements, `none` past them.
template <bool BF16>
__device__ __forceinline__ u32x4 load_tail(const void* base, int64_t element, int n, uint32_t none) {
    u32x4 w;
    if constexpr (BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = 2 * j < n ? ((const uint16_t*)base)[element + 2 * j] : none;
            const uint32_t hi = 2 * j + 1 < n ? ((const uint16_t*)base)[element + 2 * j + 1] : none;
            w[j] = lo | hi << 16;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = j < n ? ((const uint32_t*)base)[element + j] : none;
    }
    return w;
}

// Element j of 16 bytes.
template <bool BF16>
__device__ __forceinline__ float pick(const u32x4 w, int j) {
    const int i = BF16 ? j >> 1 : j;
    const uint32_t x = i < 2 ? (i == 0 ? w[0] : w[1]) : (i == 2 ? w[2] : w[3]);
    if constexpr (BF16) return j & 1 ? word_hi(x) : word_lo(x);
    return __uint_as_float(x);
}

struct Layout {
    size_t part, best, count, total;
    int rows, nseg, seg, rseg, rlen;  // stream segments per row and their length; race segments and theirs
    int lanes;                        // log2 of the lanes that join a row's segments
};

// Segments: enough workgroups to fill the device (2048 for the rows, 1024 for the races, which
// are resident together), but at least 16 bytes a thread.
inline Layout layout(int B, int gamma, int V, bool bf16) {
    Layout L;
    const int grain = kThreads * (bf16 ? 8 : 4);
    L.rows = B * (2 * gamma + 1);
    auto cut = [&](long rows, long fill, int* n, int* len) {
        long want = std::min<long>(std::max<long>((fill + rows - 1) / rows, 1), 64);
        long l = ((V + want - 1) / want + grain - 1) / grain * grain;
        *len = (int)l;
        *n = (int)((V + l - 1) / l);
    };
    cut(L.rows, 2048, &L.nseg, &L.seg);
    cut(B, 1024, &L.rseg, &L.rlen);
    L.lanes = 0;
    while (1 << L.lanes < L.nseg) ++L.lanes;
    L.part = 0;
    L.best = align256((size_t)L.rows * L.nseg * 8);
    L.count = align256(L.best + (size_t)B * 8);
    L.total = align256(L.count + (size_t)B * 4);
    return L;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// (maximum, sum of 2^((l - maximum) c)) of two parts as one; an empty part has maximum -inf.
__device__ __forceinline__ void merge(float& m, float& s, float m2, float s2, float c) {
    const float top = fmaxf(m, m2);
    if (top == kNoLogit) return;
    s = s * exp2_hw((m - top) * c) + s2 * exp2_hw((m2 - top) * c);
    m = top;
}

// Maximum and sum of 2^((l - maximum) c) over [lo, hi) of the row at `at`, by `threads` threads of which
// this is number `me`: this thread's share.
template <bool BF16>
__device__ __forceinline__ void row_share(const void* base, int64_t at, int lo, int hi, int me, int threads, float c, float& m,
                                          float& s) {
    constexpr int VEC = Elem<BF16>::kVec;
    constexpr int U = 4;  // loads in flight before the first is used
    m = kNoLogit;
    s = 0.f;
    for (int v0 = lo + me * VEC; v0 < hi; v0 += U * threads * VEC) {
        u32x4 w[U];
        float x[U][VEC];
        float top = kNoLogit;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int v = v0 + k * threads * VEC;
            if (v + VEC <= hi) w[k] = load_any<BF16>(base, at + v);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int v = v0 + k * threads * VEC;
            if (v + VEC <= hi) {
                Elem<BF16>::widen(w[k], x[k]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[k][j] = v + j < hi ? load_one<BF16>(base, at + v + j) : kNoLogit;
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) top = fmaxf(top, x[k][j]);
        }
        if (top > m) {
            s *= exp2_hw((m - top) * c);  // m = -inf: s is 0 and stays 0
            m = top;
        }
        if (m != kNoLogit) {
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s += exp2_hw((x[k][j] - m) * c);
        }
    }
}

// Rows [0, B (gamma + 1)) are the target's, the others the drafts'.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void given_stream_kernel(GivenArgs a, Layout L) {
    const int row = blockIdx.x / L.nseg, part = blockIdx.x - row * L.nseg;
    const int targets = a.B * (a.gamma + 1);
    const bool target = row < targets;
    const float c = kLog2e / (target ? a.T_target : a.T_draft);
    const int lo = part * L.seg, hi = min(lo + L.seg, a.V);
    const int tid = threadIdx.x;
    char* ws = (char*)a.workspace;
    if (part == 0 && tid == 0 && row < a.B) {
        // the race's slot and counter of sequence `row`: written before its launch begins
        ((unsigned long long*)(ws + L.best))[row] = kNone;
        ((unsigned*)(ws + L.count))[row] = 0;
    }
    float m, s;
    row_share<BF16>(target ? a.target : a.draft, (int64_t)(target ? row : row - targets) * a.V, lo, hi, tid, kThreads, c, m, s);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), c);
    __shared__ float s_m[kWaves], s_s[kWaves];
    if ((tid & 63) == 0) {
        s_m[tid >> 6] = m;
        s_s[tid >> 6] = s;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kWaves; ++w) merge(m, s, s_m[w], s_s[w], c);
        ((float2*)(ws + L.part))[(int64_t)row * L.nseg + part] = make_float2(m, s);
    }
}

constexpr int kMaxRows = 2 * 32 + 1;
constexpr int kRaceUnroll = 2;  // 16-byte pieces of a row that a thread scores between two exchanges
// Relative error assumed of a probability from the hardware's exponential: (l - max) / T is at most 149 in
// units of ln 2 (a float's range) and errs by 3 2^-24 of itself, 2e-5 in the probability at most.
constexpr float kErr = 4e-5f;
// Elements of a sequence's rows up to which one workgroup does all of it in one launch, while there is a CU
// for each sequence (V=1024, gamma=4, from Python: 15.5 us and 18.0 us in two launches up to 64 sequences,
// 27.0 and 20.9 us with 512).
constexpr long kWhole = 32768;
constexpr int kWholeBatch = 256;
constexpr int kWholeThreads = 1024;

// Full-precision scores of tokens of the row that decides, as (score bits, token): scores
// are positive, so their bits order them, and equal ones go to the lowest token.
template <bool BF16>
struct RaceRow {
    const GivenArgs* a;
    float top_p, sum_p, top_q, sum_q;
    int64_t at_p, at_q, at_e;
    __device__ float p(float l) const { return expf((l - top_p) / a->T_target) / sum_p; }
    __device__ float q(float l) const { return sum_q > 0.f ? expf((l - top_q) / a->T_draft) / sum_q : 0.f; }
    __device__ static unsigned long long key(float r, float e, int v) {
        return r > 0.f ? (unsigned long long)__float_as_uint(e / r) << 32 | (unsigned)v : kNone;
    }
};

// WHOLE: a workgroup a sequence, which also reads its rows.  Otherwise a workgroup a segment of the race.
template <bool BF16, bool WHOLE>
__global__ __launch_bounds__(WHOLE ? kWholeThreads : kThreads, WHOLE ? 1 : 4) void given_race_kernel(GivenArgs a, Layout L) {
    constexpr int VEC = Elem<BF16>::kVec;
    constexpr int NT = WHOLE ? kWholeThreads : kThreads, NW = NT / 64;
    __shared__ float s_top[kMaxRows], s_sum[kMaxRows];
    __shared__ int s_taken;
    __shared__ unsigned long long s_best[NW];
    const int b = blockIdx.x / L.rseg, part = blockIdx.x - b * L.rseg;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = a.gamma;
    const int targets = a.B * (g + 1);
    char* ws = (char*)a.workspace;
    const float2* parts = (const float2*)(ws + L.part);

    // lane s of the first wave: draft s, its logits and its number, on their way while sums are joined
    const int drafts = a.n_drafts ? min(max(a.n_drafts[b], 0), g) : g;
    int x = -1;
    float lt = 0.f, ld = 0.f, u = 0.f;
    if (wave == 0 && lane < drafts) {
        x = a.draft_tokens[(int64_t)b * g + lane];
        u = a.u[(int64_t)b * g + lane];
        if (x >= 0 && x < a.V) {
            lt = load_one<BF16>(a.target, ((int64_t)b * (g + 1) + lane) * a.V + x);
            ld = load_one<BF16>(a.draft, ((int64_t)b * g + lane) * a.V + x);
        }
    }

    // the first pieces of e, which need nothing else
    const int lo = part * L.rlen, hi = min(lo + L.rlen, a.V);
    u32x4 we[kRaceUnroll][VEC / 4];
    auto load_e = [&](int v0) {
#pragma unroll
        for (int k = 0; k < kRaceUnroll; ++k)
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                const int v = v0 + k * NT * VEC;
                if (v + VEC <= hi)
                    we[k][j / 4] = load_any<false>(a.e, (int64_t)b * a.V + v + j);
                else
                    we[k][j / 4] = load_tail<false>(a.e, (int64_t)b * a.V + v + j, hi - v - j, 0x3F800000u);
            }
    };
    load_e(lo + tid * VEC);

    // Every row of the sequence: rows [0, g] the target's, [g + 1, 2 g] the drafts'.  A row's segments
    // lie on neighbouring lanes, 2^L.lanes of them; a whole row on all of a wave's.
    const int row_lanes = WHOLE ? 64 : 1 << L.lanes;
    for (int r0 = 0; r0 < 2 * g + 1; r0 += NT / row_lanes) {
        const int r = r0 + tid / row_lanes, at = tid & (row_lanes - 1);
        const bool target = r <= g;
        const float T = target ? a.T_target : a.T_draft;
        const float c = kLog2e / T;
        const int64_t row = target ? (int64_t)b * (g + 1) + r : targets + (int64_t)b * g + (r - g - 1);
        const int64_t to = target ? row : row - targets;  // among the target's or the drafts' rows
        float m = kNoLogit, s = 0.f;
        if (r < 2 * g + 1) {
            if constexpr (WHOLE) {
                row_share<BF16>(target ? a.target : a.draft, to * a.V, 0, a.V, lane, 64, c, m, s);
            } else if (at < L.nseg) {
                const float2 v = parts[row * L.nseg + at];
                m = v.x;
                s = v.y;
            }
        }
        for (int o = row_lanes / 2; o > 0; o >>= 1) merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), c);
        if (at == 0 && r < 2 * g + 1) {
            s_top[r] = m == kNoLogit ? 0.f : m;
            s_sum[r] = m == kNoLogit ? 0.f : s;
            if (part == 0) {
                float* out = target ? a.target_lse : a.draft_lse;
                if (out) out[to] = m == kNoLogit ? kNoLogit : m / T + logf(s);
            }
        }
    }
    __syncthreads();

    // the first refusal
    if (wave == 0) {
        bool ok = false;
        if (x >= 0 && x < a.V) {
            const float sp = s_sum[lane], sq = s_sum[g + 1 + lane];
            const float p = sp > 0.f ? expf((lt - s_top[lane]) / a.T_target) / sp : 0.f;
            const float q = sq > 0.f ? expf((ld - s_top[g + 1 + lane]) / a.T_draft) / sq : 0.f;
            ok = u * q < p;
        }
        const unsigned long long refused = ~__ballot(ok);  // bit `drafts` is set: at most 32 drafts
        if (lane == 0) s_taken = __ffsll(refused) - 1;
    }
    __syncthreads();
    const int taken = s_taken;
    const bool residual = taken < drafts;

    // The race over one segment of row `taken`.  First every token's score from fast exponentials
    // and reciprocals, as an interval: with both probabilities good to kErr of themselves,
    // r is within kErr (p + q) of p - q.  Then only pieces with a lower bound that does not exceed
    // the wave's smallest upper bound (one or two) are scored with full precision.
    RaceRow<BF16> row;
    row.a = &a;
    row.top_p = s_top[taken];
    row.sum_p = s_sum[taken];
    row.top_q = residual ? s_top[g + 1 + taken] : 0.f;
    row.sum_q = residual ? s_sum[g + 1 + taken] : 0.f;
    row.at_p = ((int64_t)b * (g + 1) + taken) * a.V;
    row.at_q = ((int64_t)b * g + min(taken, g - 1)) * a.V;
    row.at_e = (int64_t)b * a.V;
    unsigned long long best = kNone;
    if (row.sum_p > 0.f) {
        const bool use_q = row.sum_q > 0.f;
        const float cp = kLog2e / a.T_target, cq = use_q ? kLog2e / a.T_draft : 0.f;
        const float inv_p = 1.f / row.sum_p, inv_q = use_q ? 1.f / row.sum_q : 0.f;
        // smallest lower and upper bounds so far; an upper bound needs r to be more than rounding
        auto bounds = [&](float lp, float lq, float e, float& low, float& high) {
            const float p = exp2_hw((lp - row.top_p) * cp) * inv_p;
            const float q = use_q ? exp2_hw((lq - row.top_q) * cq) * inv_q : 0.f;
            const float r = p - q, err = (p + q) * kErr;
            const float down = e * __builtin_amdgcn_rcpf(r + err) * (1.f - kErr);
            if (r + err > 0.f) low = fminf(low, down);
            const float up = e * __builtin_amdgcn_rcpf(r - err) * (1.f + kErr);
            if (r - err > 0.f) high = fminf(high, up);
        };
        for (int v0 = lo + tid * VEC; v0 - tid * VEC < hi; v0 += kRaceUnroll * NT * VEC) {
            float low[kRaceUnroll];  // of each piece: its smallest lower bound
            float high = __builtin_inff();
            u32x4 wp[kRaceUnroll], wq[kRaceUnroll];
#pragma unroll
            for (int k = 0; k < kRaceUnroll; ++k) {
                const int v = v0 + k * NT * VEC;
                wq[k] = u32x4{0, 0, 0, 0};
                if (v + VEC <= hi) {
                    wp[k] = load_any<BF16>(a.target, row.at_p + v);
                    if (use_q) wq[k] = load_any<BF16>(a.draft, row.at_q + v);
                } else {
                    wp[k] = load_tail<BF16>(a.target, row.at_p + v, hi - v, BF16 ? 0xFF80u : 0xFF800000u);  // -inf
                    if (use_q) wq[k] = load_tail<BF16>(a.draft, row.at_q + v, hi - v, 0);
                }
            }
#pragma unroll
            for (int k = 0; k < kRaceUnroll; ++k) {
                float lp[VEC], lq[VEC], e[VEC];
                Elem<BF16>::widen(wp[k], lp);
                Elem<BF16>::widen(wq[k], lq);
#pragma unroll
                for (int j = 0; j < VEC; j += 4) Elem<false>::widen(we[k][j / 4], e + j);
                low[k] = __builtin_inff();
#pragma unroll
                for (int j = 0; j < VEC; ++j) bounds(lp[j], lq[j], e[j], low[k], high);
                __builtin_amdgcn_sched_barrier(0);  // a piece's temporaries end here
            }
            // the wave's smallest upper bound: pieces whose tokens all lie above it have lost
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) high = fminf(high, __shfl_xor(high, o));
            if (best != kNone) high = fminf(high, __uint_as_float((unsigned)(best >> 32)));
#pragma unroll
            for (int k = 0; k < kRaceUnroll; ++k)
                if (low[k] <= high) {
                    const int v = v0 + k * NT * VEC;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float lp = pick<BF16>(wp[k], j), lq = pick<BF16>(wq[k], j);
                        const float e = pick<false>(VEC == 8 && j >= 4 ? we[k][VEC / 4 - 1] : we[k][0], j & 3);
                        float down = __builtin_inff(), up = high;
                        bounds(lp, lq, e, down, up);
                        if (down <= high && v + j < hi) best = min(best, row.key(row.p(lp) - row.q(lq), e, v + j));
                    }
                }
            load_e(v0 + kRaceUnroll * NT * VEC);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = min(best, (unsigned long long)__shfl_xor((long long)best, o));
    if (lane == 0) s_best[wave] = best;
    __syncthreads();
    unsigned long long won;
    if constexpr (WHOLE) {
        won = s_best[0];
        for (int w = 1; w < NW; ++w) won = min(won, s_best[w]);
    } else {
        __shared__ int s_last;
        unsigned long long* slot = (unsigned long long*)(ws + L.best) + b;
        if (tid == 0) {
            for (int w = 1; w < NW; ++w) best = min(best, s_best[w]);
            // A minimum does not depend on the order of the workgroups.  Its returned value is waited for,
            // so it has taken place when the count goes up: the workgroup that counts last reads
            // the minimum of all.  Nothing else passes between them, and no fence is needed, which
            // would empty the caches that the other workgroups stream through.
            const unsigned long long was = __hip_atomic_fetch_min(slot, best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("" ::"v"(was) : "memory");
            const unsigned before = __hip_atomic_fetch_add((unsigned*)(ws + L.count) + b, 1u, __ATOMIC_RELAXED,
                                                           __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (unsigned)(L.rseg - 1);
        }
        __syncthreads();
        if (!s_last) return;
        won = __hip_atomic_fetch_min(slot, kNone, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (won == kNone && residual && row.sum_p > 0.f) {
        // a refusal with p <= q everywhere (rounding: two rows nearly the same): the race over p
        for (int v = tid; v < a.V; v += NT) won = min(won, row.key(row.p(load_one<BF16>(a.target, row.at_p + v)), a.e[row.at_e + v], v));
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) won = min(won, (unsigned long long)__shfl_xor((long long)won, o));
        __syncthreads();
        if (lane == 0) s_best[wave] = won;
        __syncthreads();
        for (int w = 0; w < NW; ++w) won = min(won, s_best[w]);
    }
    if (tid <= g) {
        int token = -1;
        if (tid < taken)
            token = a.draft_tokens[(int64_t)b * g + tid];
        else if (tid == taken && won != kNone)
            token = (int)(unsigned)won;
        a.out_tokens[(int64_t)b * (g + 1) + tid] = token;
        if (tid == 0) a.out_len[b] = taken + 1;
    }
}

bool given_whole(int B, int gamma, int V) { return B <= kWholeBatch && (2L * gamma + 1) * V <= kWhole; }

}  // namespace

size_t given_workspace(int B, int gamma, int V, bool bf16) { return layout(B, gamma, V, bf16).total; }

hipError_t launch_given(const GivenArgs& a, bool bf16, hipStream_t stream) {
    Layout L = layout(a.B, a.gamma, a.V, bf16);
    if (given_whole(a.B, a.gamma, a.V)) {
        L.rseg = 1;
        L.rlen = a.V;
        if (bf16)
            hipLaunchKernelGGL((given_race_kernel<true, true>), dim3(a.B), dim3(kWholeThreads), 0, stream, a, L);
        else
            hipLaunchKernelGGL((given_race_kernel<false, true>), dim3(a.B), dim3(kWholeThreads), 0, stream, a, L);
        return hipGetLastError();
    }
    const dim3 stream_grid((unsigned)L.rows * L.nseg), race_grid((unsigned)a.B * L.rseg);
    if (bf16) {
        hipLaunchKernelGGL(given_stream_kernel<true>, stream_grid, dim3(kThreads), 0, stream, a, L);
        hipLaunchKernelGGL((given_race_kernel<true, false>), race_grid, dim3(kThreads), 0, stream, a, L);
    } else {
        hipLaunchKernelGGL(given_stream_kernel<false>, stream_grid, dim3(kThreads), 0, stream, a, L);
        hipLaunchKernelGGL((given_race_kernel<false, false>), race_grid, dim3(kThreads), 0, stream, a, L);
    }
    return hipGetLastError();
}

}  // namespace psd
