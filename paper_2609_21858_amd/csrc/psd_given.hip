// psd_given.hip -- verification of drafted tokens from given random numbers (gfx950).
//
// With p_s, q_s the softmaxes of target and draft row s, draft x_s is accepted while
// u_s q_s(x_s) < p_s(x_s); the token after the accepted ones is argmin_v e_v / r(v) with
// r = max(p_n - q_n, 0) at a refusal and r = p_n after all drafts.  The residual's total is
// not needed: the race is invariant to scale.
//
// Two launches.  given_stream_kernel reads every row once (memory bounds it: (2 gamma + 1) V
// elements a sequence) and leaves each segment's maximum and sum of exponentials.
// given_race_kernel merges them (every workgroup again: a few hundred values), finds the
// first refusal and races one segment of the one row that decides, whose logits the
// first launch has just brought into the caches; only e comes new from memory.  The last
// workgroup of a sequence writes its tokens.
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

struct Layout {
    size_t part, best, count, total;
    int rows, nseg, seg, rseg, rlen;  // stream segments per row and their length; race segments and theirs
};

// Segments: enough workgroups to fill the device several times over (2048), but at least
// 2048 elements each, in multiples of a workgroup's 16-byte loads.
inline Layout layout(int B, int gamma, int V, bool bf16) {
    Layout L;
    const int grain = kThreads * (bf16 ? 8 : 4);
    L.rows = B * (2 * gamma + 1);
    auto cut = [&](long rows, int* n, int* len) {
        long want = std::min<long>(std::max<long>((2048 + rows - 1) / rows, 1), 64);
        long l = ((V + want - 1) / want + grain - 1) / grain * grain;
        *len = (int)l;
        *n = (int)((V + l - 1) / l);
    };
    cut(L.rows, &L.nseg, &L.seg);
    cut(B, &L.rseg, &L.rlen);
    L.part = 0;
    L.best = align256((size_t)L.rows * L.nseg * 8);
    L.count = align256(L.best + (size_t)B * 16);
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

// Rows [0, B (gamma + 1)) are the target's, the others the drafts'.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void given_stream_kernel(GivenArgs a, Layout L) {
    constexpr int VEC = Elem<BF16>::kVec;
    constexpr int U = 4;  // loads in flight before the first is used
    const int row = blockIdx.x / L.nseg, part = blockIdx.x - row * L.nseg;
    const int targets = a.B * (a.gamma + 1);
    const bool target = row < targets;
    const void* base = target ? a.target : a.draft;
    const int64_t at = (int64_t)(target ? row : row - targets) * a.V;
    const float c = kLog2e / (target ? a.T_target : a.T_draft);
    const int lo = part * L.seg, hi = min(lo + L.seg, a.V);
    const int tid = threadIdx.x;
    char* ws = (char*)a.workspace;
    if (part == 0 && tid < 2 && row < a.B) {
        // the race's slots and counter of sequence `row`: written before its launch begins
        ((unsigned long long*)(ws + L.best))[2 * row + tid] = kNone;
        if (tid == 0) ((unsigned*)(ws + L.count))[row] = 0;
    }
    float m = kNoLogit, s = 0.f;
    for (int v0 = lo + tid * VEC; v0 < hi; v0 += U * kThreads * VEC) {
        u32x4 w[U];
        float x[U][VEC];
        float top = kNoLogit;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int v = v0 + k * kThreads * VEC;
            if (v + VEC <= hi) w[k] = load_any<BF16>(base, at + v);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int v = v0 + k * kThreads * VEC;
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

template <bool BF16>
__global__ __launch_bounds__(kThreads) void given_race_kernel(GivenArgs a, Layout L) {
    constexpr int VEC = Elem<BF16>::kVec;
    __shared__ float s_top[kMaxRows], s_sum[kMaxRows];
    __shared__ int s_taken;
    __shared__ unsigned long long s_best[kWaves][2];
    const int b = blockIdx.x / L.rseg, part = blockIdx.x - b * L.rseg;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = a.gamma;
    const int targets = a.B * (g + 1);
    char* ws = (char*)a.workspace;
    const float2* parts = (const float2*)(ws + L.part);

    // every row of the sequence: rows [0, g] the target's, [g + 1, 2 g] the drafts'
    for (int r = wave; r < 2 * g + 1; r += kWaves) {
        const bool target = r <= g;
        const float T = target ? a.T_target : a.T_draft;
        const float c = kLog2e / T;
        const int64_t row = target ? (int64_t)b * (g + 1) + r : targets + (int64_t)b * g + (r - g - 1);
        float m = kNoLogit, s = 0.f;
        if (lane < L.nseg) {
            const float2 v = parts[row * L.nseg + lane];
            m = v.x;
            s = v.y;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), c);
        if (lane == 0) {
            s_top[r] = m == kNoLogit ? 0.f : m;
            s_sum[r] = m == kNoLogit ? 0.f : s;
            if (part == 0) {
                float* out = target ? a.target_lse : a.draft_lse;
                const int64_t at = target ? row : row - targets;
                if (out) out[at] = m == kNoLogit ? kNoLogit : m / T + logf(s);
            }
        }
    }
    __syncthreads();

    // the first refusal
    const int drafts = a.n_drafts ? min(max(a.n_drafts[b], 0), g) : g;
    if (wave == 0) {
        bool ok = false;
        if (lane < drafts) {
            const int x = a.draft_tokens[(int64_t)b * g + lane];
            if (x >= 0 && x < a.V) {
                const float lt = load_one<BF16>(a.target, ((int64_t)b * (g + 1) + lane) * a.V + x);
                const float ld = load_one<BF16>(a.draft, ((int64_t)b * g + lane) * a.V + x);
                const float sp = s_sum[lane], sq = s_sum[g + 1 + lane];
                const float p = sp > 0.f ? expf((lt - s_top[lane]) / a.T_target) / sp : 0.f;
                const float q = sq > 0.f ? expf((ld - s_top[g + 1 + lane]) / a.T_draft) / sq : 0.f;
                ok = a.u[(int64_t)b * g + lane] * q < p;
            }
        }
        const unsigned long long refused = ~__ballot(ok);  // bit `drafts` is set: at most 32 drafts
        if (lane == 0) s_taken = __ffsll(refused) - 1;
    }
    __syncthreads();
    const int taken = s_taken;
    const bool residual = taken < drafts;

    // the race over row `taken`: the smallest e / max(p - q, 0), and the smallest e / p for a
    // residual that is zero everywhere
    const float top_p = s_top[taken], sum_p = s_sum[taken];
    const float top_q = residual ? s_top[g + 1 + taken] : 0.f, sum_q = residual ? s_sum[g + 1 + taken] : 0.f;
    const int64_t at_p = ((int64_t)b * (g + 1) + taken) * a.V;
    const int64_t at_q = residual ? ((int64_t)b * g + taken) * a.V : 0;
    const int64_t at_e = (int64_t)b * a.V;
    const int lo = part * L.rlen, hi = min(lo + L.rlen, a.V);
    unsigned long long best_r = kNone, best_p = kNone;
    if (sum_p > 0.f) {
        auto race = [&](int v, float lp, float lq, float e) {
            const float p = expf((lp - top_p) / a.T_target) / sum_p;
            const float q = sum_q > 0.f ? expf((lq - top_q) / a.T_draft) / sum_q : 0.f;
            if (p > 0.f) best_p = min(best_p, (unsigned long long)__float_as_uint(e / p) << 32 | (unsigned)v);
            const float r = p - q;
            if (r > 0.f) best_r = min(best_r, (unsigned long long)__float_as_uint(e / r) << 32 | (unsigned)v);
        };
        for (int v = lo + tid * VEC; v < hi; v += kThreads * VEC) {
            float lp[VEC], lq[VEC], e[VEC];
            if (v + VEC <= hi) {
                const u32x4 wp = load_any<BF16>(a.target, at_p + v);
                u32x4 wq = {0, 0, 0, 0};
                if (residual) wq = load_any<BF16>(a.draft, at_q + v);
#pragma unroll
                for (int j = 0; j < VEC; j += 4) {
                    const u32x4 we = load_any<false>(a.e, at_e + v + j);
                    Elem<false>::widen(we, e + j);
                }
                Elem<BF16>::widen(wp, lp);
                Elem<BF16>::widen(wq, lq);
#pragma unroll
                for (int j = 0; j < VEC; ++j) race(v + j, lp[j], lq[j], e[j]);
            } else {
                for (int j = 0; v + j < hi; ++j)
                    race(v + j, load_one<BF16>(a.target, at_p + v + j),
                         residual ? load_one<BF16>(a.draft, at_q + v + j) : 0.f, a.e[at_e + v + j]);
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        best_r = min(best_r, (unsigned long long)__shfl_xor((long long)best_r, o));
        best_p = min(best_p, (unsigned long long)__shfl_xor((long long)best_p, o));
    }
    if (lane == 0) {
        s_best[wave][0] = best_r;
        s_best[wave][1] = best_p;
    }
    __syncthreads();
    __shared__ int s_last;
    unsigned long long* slots = (unsigned long long*)(ws + L.best) + 2 * (int64_t)b;
    if (tid == 0) {
        for (int w = 1; w < kWaves; ++w) {
            best_r = min(best_r, s_best[w][0]);
            best_p = min(best_p, s_best[w][1]);
        }
        // minima do not depend on the order of the workgroups
        __hip_atomic_fetch_min(&slots[0], best_r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_fetch_min(&slots[1], best_p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned before = __hip_atomic_fetch_add((unsigned*)(ws + L.count) + b, 1u, __ATOMIC_ACQ_REL,
                                                       __HIP_MEMORY_SCOPE_AGENT);
        s_last = before == (unsigned)(L.rseg - 1);
    }
    __syncthreads();
    if (!s_last || wave != 0) return;
    if (lane <= g) {
        const unsigned long long r = __hip_atomic_load(&slots[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned long long p = __hip_atomic_load(&slots[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned long long won = r != kNone ? r : p;
        int token = -1;
        if (lane < taken)
            token = a.draft_tokens[(int64_t)b * g + lane];
        else if (lane == taken && won != kNone)
            token = (int)(unsigned)won;
        a.out_tokens[(int64_t)b * (g + 1) + lane] = token;
        if (lane == 0) a.out_len[b] = taken + 1;
    }
}

}  // namespace

size_t given_workspace(int B, int gamma, int V, bool bf16) { return layout(B, gamma, V, bf16).total; }

hipError_t launch_given(const GivenArgs& a, bool bf16, hipStream_t stream) {
    const Layout L = layout(a.B, a.gamma, a.V, bf16);
    const dim3 stream_grid((unsigned)L.rows * L.nseg), race_grid((unsigned)a.B * L.rseg);
    if (bf16) {
        hipLaunchKernelGGL(given_stream_kernel<true>, stream_grid, dim3(kThreads), 0, stream, a, L);
        hipLaunchKernelGGL(given_race_kernel<true>, race_grid, dim3(kThreads), 0, stream, a, L);
    } else {
        hipLaunchKernelGGL(given_stream_kernel<false>, stream_grid, dim3(kThreads), 0, stream, a, L);
        hipLaunchKernelGGL(given_race_kernel<false>, race_grid, dim3(kThreads), 0, stream, a, L);
    }
    return hipGetLastError();
}

}  // namespace psd
