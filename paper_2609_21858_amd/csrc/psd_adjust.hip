// psd_adjust.hip -- penalties for repeated tokens, biases and masks on logits (gfx950).
//
//   c > 0:  z = (l > 0 ? l / rho : l rho) - (frequency c + presence),  else z = l
//   z + sum of the token's biases;  -inf where the mask's bit is 0
// with c the token's count in the sequence's text and among the row's own earlier drafts.  Memory
// bounds it: every logit is read and written once; the texts are counted by each workgroup for its own
// stretch of the vocabulary.
#include <hip/hip_runtime.h>

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kSeg = 8192;         // tokens of a workgroup's stretch
constexpr int kMaxBias = 1024;
// A token's word: bit 31 where it has biases, their place in the list, and its count below.
constexpr uint32_t kBiased = 1u << 31, kCount = (1u << 20) - 1;
constexpr float kGone = -__builtin_inff();

// 16 bytes at any element boundary (rows of an odd vocabulary start off the 16-byte grid).
typedef uint32_t u32x4_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_b16 __attribute__((ext_vector_type(4), aligned(2)));
template <bool BF16>
struct Piece;
template <>
struct Piece<true> {
    typedef u32x4_b16 any;
    typedef uint16_t one;
    __device__ static float widen1(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    __device__ static uint16_t narrow1(float x) { return (uint16_t)pack_bf16(x, x); }
};
template <>
struct Piece<false> {
    typedef u32x4_f32 any;
    typedef float one;
    __device__ static float widen1(float x) { return x; }
    __device__ static float narrow1(float x) { return x; }
};

// One workgroup: a stretch of kSeg tokens of rows [r0, r1) of a sequence.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a, int segments, int per) {
    using E = Elem<BF16>;
    using Pc = Piece<BF16>;
    constexpr int VEC = E::kVec;
    __shared__ __align__(16) uint32_t s_word[kSeg];
    __shared__ float s_bias[kMaxBias];
    __shared__ int s_bias_token[kMaxBias];
    __shared__ int s_wave[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seg = blockIdx.x % segments;
    const int rest = blockIdx.x / segments;
    const int R = a.K * a.S, groups = (R + per - 1) / per;
    const int b = rest / groups, r0 = (rest - b * groups) * per, r1 = min(r0 + per, R);
    const int v0 = seg * kSeg, v1 = min(v0 + kSeg, a.V);

    for (int i = tid; i < kSeg / 4; i += kThreads) ((u32x4*)s_word)[i] = u32x4{0, 0, 0, 0};
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
            s_bias_token[at] = v - v0;
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
        const int to = (int)min(a.length[b], (int64_t)a.text_max);
        const int from = a.from ? (int)min(max(a.from[b], (int64_t)0), (int64_t)a.text_max) : 0;
        for (int i = from + tid; i < to; i += kThreads) count(text[i], 1);
    }
    const int32_t* drafts = a.drafts ? a.drafts + (int64_t)b * a.K * a.gamma : nullptr;
    const float rho = a.repetition ? a.repetition[b] : 1.f;
    const float presence = a.presence ? a.presence[b] : 0.f, frequency = a.frequency ? a.frequency[b] : 0.f;
    const bool same = a.out == a.logits;
    auto value = [&](float l, uint32_t word, bool may) {
        const uint32_t c = word & kCount;
        float z = l;
        if (c > 0) z = (l > 0.f ? l / rho : l * rho) - (frequency * (float)c + presence);
        if (word & kBiased) z += s_bias[kMaxBias - 1 - (word >> 20 & 1023)];
        return may ? z : kGone;
    };
    int path = -1, depth = 0;  // the drafts that are counted: `path`'s before `depth`
    for (int r = r0; r < r1; ++r) {
        const int k = r / a.S, d = a.depth0 + r - k * a.S;
        __syncthreads();
        if (drafts) {
            const int keep = k == path ? depth : 0;
            if (k != path && tid < depth) count(drafts[path * a.gamma + tid], ~0u);  // (minus one)
            if (tid >= keep && tid < d) count(drafts[k * a.gamma + tid], 1);
            path = k;
            depth = d;
            __syncthreads();
        }
        const int64_t row = ((int64_t)b * R + r) * a.V;
        const typename Pc::one* src = (const typename Pc::one*)a.logits + row;
        typename Pc::one* dst = (typename Pc::one*)a.out + row;
        const uint32_t* allowed = a.allowed ? a.allowed + b * a.allowed_seq + r * a.allowed_row : nullptr;
        for (int v = v0 + tid * VEC; v < v1; v += kThreads * VEC) {
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
            const uint32_t every = (1u << VEC) - 1;
            const uint32_t may = allowed ? allowed[v / 32] >> (v % 32) & every : every;
            if (same && any == 0 && may == every) continue;
            if (v + VEC <= a.V) {
                float x[VEC];
                E::widen(*(const typename Pc::any*)(src + v), x);
#pragma unroll
                for (int i = 0; i < VEC; ++i) x[i] = value(x[i], words[i], may >> i & 1);
                *(typename Pc::any*)(dst + v) = E::narrow(x);
            } else {
                for (int i = 0; v + i < a.V; ++i) dst[v + i] = Pc::narrow1(value(Pc::widen1(src[v + i]), s_word[v - v0 + i], may >> i & 1));
            }
        }
    }
}

}  // namespace

bool adjust_fits(const AdjustArgs& a) { return (long)((a.V + kSeg - 1) / kSeg) * a.B * a.K * a.S < 1L << 23; }

hipError_t launch_adjust(const AdjustArgs& a, bool bf16, hipStream_t stream) {
    const int segments = (a.V + kSeg - 1) / kSeg;
    const int R = a.K * a.S;
    const int per = R;
    const dim3 grid((unsigned)((long)segments * a.B * ((R + per - 1) / per)));
    if (bf16)
        hipLaunchKernelGGL((adjust_kernel<true>), grid, dim3(kThreads), 0, stream, a, segments, per);
    else
        hipLaunchKernelGGL((adjust_kernel<false>), grid, dim3(kThreads), 0, stream, a, segments, per);
    return hipGetLastError();
}

}  // namespace psd
