// psd_adjust.hip -- penalties for repeated tokens, biases and masks on logits (gfx950).
//
//   c > 0:  z = (l > 0 ? l / rho : l rho) - (frequency c + presence),  else z = l
//   z + sum of the token's biases;  -inf where the mask's bit is 0
// with c the token's count in the sequence's text and among the row's own earlier drafts.  Memory
// bounds it: every logit is read and written once; the texts are counted by each workgroup for its own
// stretch of the vocabulary.  1280 rows of 128256 bfloat16 logits of 64 sequences, texts of 2048 tokens, 657 MB: 146 us,
// 4.5 TB/s (a device copy 4.9), with a mask a row 152; in place, where most pieces only pass, 108, with masks 160; 1152 float32
// rows of 151936 293; 5 rows of 1024 5.  Every workgroup of a sequence counts its whole text: with texts of up to 16384, 131072 and
// 1000000 tokens 148, 176 and 430 us, 5 rows of 1 sequence 7, 22 and 200 (none: 143 and 4.7).
#include <hip/hip_runtime.h>

#include "psd_adjust_plan.hpp"
#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxBias = 1024;
// A token's word: bit 31 where it has biases, their place in the list, and its count below.
constexpr uint32_t kBiased = 1u << 31, kCount = (1u << 20) - 1;
constexpr float kGone = -__builtin_inff();

// 16 bytes at any element boundary (rows of an odd vocabulary start off the 16-byte grid).
typedef uint32_t u32x4_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_b16 __attribute__((ext_vector_type(4), aligned(2)));
typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));
template <bool BF16>
struct Piece;
template <>
struct Piece<true> {
    typedef u32x4_b16 any;
    typedef uint16_t one;
    __device__ static float widen1(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    __device__ static uint16_t narrow1(float x) { return (uint16_t)pack_bf16(x, x); }
    // -inf where a bit of `may` is 0
    __device__ static u32x4 masked(u32x4 w, uint32_t may) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = __builtin_amdgcn_sbfe(may, 2 * i, 1), hi = __builtin_amdgcn_sbfe(may, 2 * i + 1, 1);
            const uint32_t keep = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
            w[i] = (w[i] & keep) | (0xFF80FF80u & ~keep);
        }
        return w;
    }
};
template <>
struct Piece<false> {
    typedef u32x4_f32 any;
    typedef float one;
    __device__ static float widen1(float x) { return x; }
    __device__ static float narrow1(float x) { return x; }
    __device__ static u32x4 masked(u32x4 w, uint32_t may) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t keep = __builtin_amdgcn_sbfe(may, i, 1);
            w[i] = (w[i] & keep) | (0xFF800000u & ~keep);
        }
        return w;
    }
};

// One workgroup: a stretch of SEG tokens of rows [r0, r1) of a sequence.  A row's next pieces are on their way while
// this one's are computed.  Pieces that nothing touches pass through as they are; in place they are not written, and without
// a mask not read.
template <bool BF16, int SEG>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a, int segments, int per) {
    using E = Elem<BF16>;
    using Pc = Piece<BF16>;
    constexpr int VEC = E::kVec;
    __shared__ __align__(16) uint32_t s_word[SEG];
    __shared__ float s_bias[kMaxBias];
    __shared__ uint16_t s_bias_token[kMaxBias];  // (less than 4 workgroups of 8192 tokens would fit a CU with 32 bits)
    __shared__ int s_wave[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seg = blockIdx.x % segments;
    const int rest = blockIdx.x / segments;
    const int R = a.K * a.S, groups = (R + per - 1) / per;
    const int b = rest / groups, r0 = (rest - b * groups) * per, r1 = min(r0 + per, R);
    const int v0 = seg * SEG, v1 = min(v0 + SEG, a.V);

    const bool same = a.out == a.logits;
    constexpr int N = SEG / (kThreads * VEC);  // pieces of a thread in a row
    const int64_t row0 = (int64_t)b * R * a.V;
    const typename Pc::one* src0 = (const typename Pc::one*)a.logits + row0;
    typename Pc::one* dst0 = (typename Pc::one*)a.out + row0;
    auto at = [&](int n) { return v0 + (n * kThreads + tid) * VEC; };
    u32x4 next[N];
    uint32_t allowed_next[N];  // (words as loaded: shifted here, they would be waited for before the row)
    bool here_next[N];  // in place: is the piece on its way?
    constexpr uint32_t kEvery = (1u << VEC) - 1;
    auto load = [&](int r) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int v = at(n);
            allowed_next[n] = ~0u;
            if (v >= v1) continue;
            if (a.allowed) allowed_next[n] = a.allowed[b * a.allowed_seq + r * a.allowed_row + v / 32];
            // in place without a mask: pieces that the text or a bias touches (those of a draft alone are read when they are due)
            bool wanted = !same || a.allowed != nullptr;
            if (same) {
#pragma unroll
                for (int i = 0; i < VEC; i += 4) {
                    const u32x4 w = *(const u32x4*)(s_word + v - v0 + i);
                    wanted |= (w[0] | w[1] | w[2] | w[3]) != 0;
                }
                here_next[n] = wanted;
            }
            if (wanted && v + VEC <= a.V) next[n] = *(const typename Pc::any*)(src0 + (int64_t)r * a.V + v);
        }
    };
    for (int i = tid; i < SEG / 4; i += kThreads) ((u32x4*)s_word)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    // the stretch's biases, in the order of the list
    int n_bias = 0;
    for (int i0 = 0; i0 < a.bias_width; i0 += kThreads) {
        const int i = i0 + tid;
        const int v = i < a.bias_width ? a.bias_tokens[(int64_t)b * a.bias_width + i] : -1;
        const bool in = v >= v0 && v < v1;
        const uint64_t who = __ballot(in);
        if (lane == 0) s_wave[wave] = __popcll(who);
        __syncthreads();
        int at = n_bias + __popcll(who & ((1ull << lane) - 1));
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) at += s_wave[w];
            n_bias += s_wave[w];
        }
        if (in) {
            s_bias_token[at] = (uint16_t)(v - v0);
            s_bias[at] = a.bias[(int64_t)b * a.bias_width + i];
            atomicMax(&s_word[v - v0], kBiased | (uint32_t)(kMaxBias - 1 - at) << 20);  // the first of a token's entries stands for it
        }
        __syncthreads();
    }
    // a token's entries are summed in their order
    float sums[kMaxBias / kThreads];
#pragma unroll
    for (int k = 0; k < kMaxBias / kThreads; ++k) {
        const int i = k * kThreads + tid;
        sums[k] = 0.f;
        if (i < n_bias) {
            const int v = s_bias_token[i];
            if ((s_word[v] >> 20 & 1023) == (uint32_t)(kMaxBias - 1 - i))
                for (int j = i; j < n_bias; ++j)
                    if (s_bias_token[j] == v) sums[k] += s_bias[j];
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kMaxBias / kThreads; ++k)
        if (k * kThreads + tid < n_bias) s_bias[k * kThreads + tid] = sums[k];
    // counts of the text's tokens in the stretch
    auto count = [&](int v, uint32_t by) {
        if ((unsigned)(v - v0) < (unsigned)(v1 - v0)) atomicAdd(&s_word[v - v0], by);
    };
    if (a.text) {
        const int32_t* text = a.text + (int64_t)b * a.text_stride;
        const int to = (int)min(max(a.length[b], (int64_t)0), (int64_t)a.text_max);
        const int from = a.from ? (int)min(max(a.from[b], (int64_t)0), (int64_t)a.text_max) : 0;
        // four tokens a load, four loads in flight
        int i = from + tid * 4;
        for (; i + 3 * kThreads * 4 + 4 <= to; i += 4 * kThreads * 4) {
            i32x4 v[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = *(const i32x4*)(text + i + n * kThreads * 4);
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) count(v[n][e], 1);
        }
        for (; i < to; i += kThreads * 4) {
            int v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = i + e < to ? text[i + e] : -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) count(v[e], 1);
        }
    }
    const int32_t* drafts = a.drafts ? a.drafts + (int64_t)b * a.K * a.gamma : nullptr;
    const float rho = a.repetition ? a.repetition[b] : 1.f;
    const float presence = a.presence ? a.presence[b] : 0.f, frequency = a.frequency ? a.frequency[b] : 0.f;
    // bfloat16: a product with 1 / rho where a quotient is meant, 2^-24 more of what is rounded to 2^-8 (148 us instead of 154,
    // in place 108 and 120).  A float32 quotient is the definition's, and costs nothing there (293 us).
    const float inverse = 1.f / rho;
    // Without a branch for the tokens that came: a wave's pieces mostly have one.
    auto penalized = [&](float l, uint32_t word) {
        const uint32_t c = word & kCount;
        const float scaled = BF16 ? l * (l > 0.f ? inverse : rho) : l > 0.f ? l / rho : l * rho;
        const float z = scaled - (frequency * (float)c + presence);
        return c > 0 ? z : l;
    };
    auto biased = [&](float z, uint32_t word) {
        if (word & kBiased) z += s_bias[kMaxBias - 1 - (word >> 20 & 1023)];
        return z;
    };
    int path = -1, depth = 0;  // the drafts that are counted: `path`'s before `depth`
    __syncthreads();
    load(r0);
    for (int r = r0; r < r1; ++r) {
        if (drafts) {
            const int k = r / a.S, d = a.depth0 + r - k * a.S;
            const int keep = k == path ? depth : 0;
            if (r > r0) __syncthreads();
            if (k != path && tid < depth) count(drafts[path * a.gamma + tid], ~0u);  // (minus one)
            if (tid >= keep && tid < d) count(drafts[k * a.gamma + tid], 1);
            path = k;
            depth = d;
            __syncthreads();
        }
        u32x4 now[N];
        uint32_t may[N];
        bool here[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            now[n] = next[n];
            may[n] = allowed_next[n] >> (at(n) % 32) & kEvery;
            here[n] = here_next[n];
        }
        if (r + 1 < r1) load(r + 1);
        const typename Pc::one* src = src0 + (int64_t)r * a.V;
        typename Pc::one* dst = dst0 + (int64_t)r * a.V;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int v = at(n);
            if (v >= v1) break;
            uint32_t words[VEC];
            uint32_t any = 0;
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const u32x4 w = *(const u32x4*)(s_word + v - v0 + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    words[i + e] = w[e];
                    any |= w[e];
                }
            }
            const bool touched = any != 0 || may[n] != kEvery;
            if (same && !touched) continue;
            if (v + VEC <= a.V) {
                if (same && !here[n]) now[n] = *(const typename Pc::any*)(src + v);
                u32x4 y = now[n];
                if (any != 0) {
                    float x[VEC];
                    E::widen(y, x);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) x[i] = penalized(x[i], words[i]);
                    if (any & kBiased)
#pragma unroll
                        for (int i = 0; i < VEC; ++i) x[i] = biased(x[i], words[i]);
                    y = E::narrow(x);
                }
                if (may[n] != kEvery) y = Pc::masked(y, may[n]);
                *(typename Pc::any*)(dst + v) = y;
            } else {
                for (int i = 0; v + i < a.V; ++i) {
                    const uint32_t word = s_word[v - v0 + i];
                    dst[v + i] = Pc::narrow1(may[n] >> i & 1 ? biased(penalized(Pc::widen1(src[v + i]), word), word) : kGone);
                }
            }
        }
    }
}

template <bool BF16>
void launch(const AdjustArgs& a, const AdjustCut& c, hipStream_t stream) {
    const dim3 grid((unsigned)c.wgs(a.B, a.K * a.S));
    constexpr int kLong = adjust_stretch(BF16), kShort = adjust_short_stretch(BF16);
    if (c.seg == kShort)
        hipLaunchKernelGGL((adjust_kernel<BF16, kShort>), grid, dim3(kThreads), 0, stream, a, c.segments, c.per);
    else
        hipLaunchKernelGGL((adjust_kernel<BF16, kLong>), grid, dim3(kThreads), 0, stream, a, c.segments, c.per);
}

}  // namespace

bool adjust_fits(const AdjustArgs& a, bool bf16) {
    const int R = a.K * a.S;
    return adjust_cut(a.B, R, a.V, bf16).wgs(a.B, R) < 1L << 23;
}

hipError_t launch_adjust(const AdjustArgs& a, bool bf16, hipStream_t stream) {
    const AdjustCut c = adjust_cut(a.B, a.K * a.S, a.V, bf16);
    if (bf16)
        launch<true>(a, c, stream);
    else
        launch<false>(a, c, stream);
    return hipGetLastError();
}

}  // namespace psd
