// psd_quant4.hpp -- elements in 4 bits with a power-of-two scale to every 32 of them (device; internal to libpsd).
//
// Code c stands for the (c & 7)th of 0, 0.5, 1, 1.5, 2, 3, 4, 6, negative with c & 8, times 2^(s - 127); s = 255 is NaN.
// gfx950's conversions take the scale as a float whose exponent bits are s and convert two codes at once, rounding to
// the nearest with ties to the even code.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "psd_serve_device.hpp"

namespace psd {
namespace quant4 {

constexpr int kNan = 255;   // scale byte
constexpr int kMost = 252;  // the largest that is written, 6 2^125; the two above it stand for nothing that is defined

// The scale byte that elements z alone would have: k + 127 with the least k in [-126, 125] such that all are at most
// 7 2^k (1.75 2^(k+2): the exponent, and one more where the mantissa passes 0.75).  It grows with the largest
// magnitude, so a group's is the largest of its parts'.
template <int N>
__device__ __forceinline__ int scale_of(const float (&z)[N]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) top = max(top, __float_as_uint(z[j]) & 0x7FFFFFFFu);
    if (top >= 0x7F800000u) return kNan;
    const int k = (int)(top >> 23) - 129 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return min(max(k, -126) + 127, kMost);
}
template <int N>
__device__ __forceinline__ int scale_of(const double (&z)[N]) {
    // the upper words decide, with the lower ones' bits gathered in the last: only whether there are any matters
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const uint64_t w = (uint64_t)__double_as_longlong(z[j]);
        top = max(top, ((uint32_t)(w >> 32) & 0x7FFFFFFFu) | ((uint32_t)w != 0));
    }
    if (top >= (1023u + 128u) << 20) return kNan;  // past float32's range
    const int k = (int)(top >> 20) - 1025 + ((top & 0xFFFFFu) > 0xC0000u ? 1 : 0);
    return min(max(k, -126) + 127, kMost);
}

// Elements as floats that round to the codes that the elements round to.
template <int N>
__device__ __forceinline__ void narrowed(const float (&z)[N], float (&f)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = z[j];
}
// Rounding to float moves an element past no border between codes, but may move it onto one, where all bits of the
// mantissa but the upper two are 0.  Where a float of the wave looks like that, each is taken next to its element towards zero,
// with the last bit set where it is not the element itself: rounding it again gives what rounding the element gives.
template <int N>
__device__ __forceinline__ void narrowed(const double (&z)[N], float (&f)[N]) {
    uint32_t least = ~0u;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        f[j] = (float)z[j];
        least = min(least, __float_as_uint(f[j]) & 0x1FFFFFu);
    }
    if (__any(least == 0)) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const double back = f[j];
            uint32_t w = __float_as_uint(f[j]);
            if (back != z[j]) w = (fabs(back) > fabs(z[j]) ? w - 1 : w) | 1u;
            f[j] = __uint_as_float(w);
        }
    }
}

__device__ __forceinline__ float scale_value(int s) { return __uint_as_float((uint32_t)s << 23); }

// The codes of 8 elements, or of 4 in the lower half.
template <class T, int N>
__device__ __forceinline__ uint32_t encode(const T (&z)[N], int s) {
    static_assert(N == 8 || N == 4, "pieces of 16 bytes");
    const float by = scale_value(s);
    float f[N];
    narrowed(z, f);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], by, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], by, 1);
    if constexpr (N == 8) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], by, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], by, 3);
    }
    return s == kNan ? 0 : w;
}

// 8 codes as bfloat16 (exact).
__device__ __forceinline__ u32x4 decode8(uint32_t w, float by) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 3))};
}

// A group as bfloat16 into 64 bytes of LDS, 16 at a time, of which the (e ^ turn)th is the e-th to go: lanes whose groups begin
// on the same banks take different turns.
__device__ __forceinline__ void decode_group(char* to, u32x4 w, float by, int turn) {
    w = turn & 1 ? u32x4{w[1], w[0], w[3], w[2]} : w;
    w = turn & 2 ? u32x4{w[2], w[3], w[0], w[1]} : w;
#pragma unroll
    for (int e = 0; e < 4; ++e) *(u32x4*)(to + 16 * (e ^ turn)) = decode8(w[e], by);
}

// 16 bytes of elements: 8 bfloat16, or 4 float32 from the lower half.
template <bool BF16>
__device__ __forceinline__ u32x4 decode(uint32_t w, int s) {
    const u32x4 x = decode8(w, scale_value(s));
    if constexpr (BF16) return x;
    return u32x4{x[0] << 16, x[0] & 0xFFFF0000u, x[1] << 16, x[1] & 0xFFFF0000u};
}

}  // namespace quant4
}  // namespace psd
