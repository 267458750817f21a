// psd_serve_device.hpp -- device helpers of the paged cache's kernels (internal to libpsd).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "psd_serve.hpp"

namespace psd {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float word_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float word_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two floats as packed bf16, round to nearest even (one instruction; NaN stays NaN).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// Elements of one type in 16-byte pieces, as floats.
template <bool BF16>
struct Elem;
template <>
struct Elem<true> {
    static constexpr int kBytes = 2, kVec = 8;
    __device__ static void widen(const u32x4 w, float* x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = word_lo(w[i]);
            x[2 * i + 1] = word_hi(w[i]);
        }
    }
    __device__ static u32x4 narrow(const float* x) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        return w;
    }
};
template <>
struct Elem<false> {
    static constexpr int kBytes = 4, kVec = 4;
    __device__ static void widen(const u32x4 w, float* x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
    __device__ static u32x4 narrow(const float* x) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
        return w;
    }
};

// The sequence of packed row t: the number of b with new_start[b + 1] <= t.  Called by whole
// waves; 64 probes a step, so that up to 64 sequences cost one load's latency and 4096 two.
__device__ __forceinline__ int find_seq(const int32_t* new_start, int B, int t) {
    const int lane = __lane_id();
    int lo = 0, n = B;  // the answer is in [lo, lo + n]
    while (n > 0) {
        const int step = (n + 63) / 64;
        // lane i asks about the end of piece i
        const int at = min((lane + 1) * step, n);
        const bool below = lane * step < n && new_start[lo + at] <= t;
        const int pieces = __popcll(__ballot(below));
        if (step == 1) return lo + pieces;
        const int skip = min(pieces * step, n);
        lo += skip;
        n = min(step - 1, n - skip);
    }
    return lo;
}

}  // namespace psd
