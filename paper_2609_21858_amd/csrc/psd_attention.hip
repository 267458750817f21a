// psd_attention.hip -- attention of a block's new tokens over a paged cache (gfx950).
//
//   s_j = scale q . k_j over the cached tokens j that a row sees,
//   out = sum_j exp(s_j - lse) v_j,  lse = ln sum_j exp(s_j),
// in one pass over the cache with the running maximum m and sum l of the softmax: a new
// maximum m' rescales the sum and the output by exp(m - m').
#include <hip/hip_runtime.h>

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kThreads = 256;

// One wave per (packed row, query head); a lane holds the score of one of 64 tokens, then D/64
// elements of the output.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void attention_kernel(AttentionArgs a) {
    using E = Elem<BF16>;
    const CacheArgs& c = a.c;
    const int lane = threadIdx.x & 63;
    const long item = (long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (item >= (long)c.rows * a.H) return;
    const int t = (int)(item / a.H), h = (int)(item - (long)t * a.H);
    const int b = find_seq(c.new_start, c.B, t);
    if (b >= c.B) return;
    const Seq s = load_seq(c, b);
    const int i = t - s.row0;
    if (i < 0 || i >= s.n) return;
    const int g = h / (a.H / c.G);
    const int pos = s.first + i;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    const char* q = (const char*)a.q.data + ((int64_t)t * a.q.stride_row + (int64_t)h * a.q.stride_head) * E::kBytes;
    float m = -__builtin_inff(), l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    const int end = a.mask ? s.kv : min(s.kv, pos + 1);
    const int begin = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
    for (int j0 = begin; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        bool see = j < end;
        int64_t at = 0;
        if (see && a.mask && j >= s.first) {
            const int w = (j - s.first) / 32;
            see = w < a.mask_words && (a.mask[(int64_t)t * a.mask_words + w] >> ((j - s.first) % 32) & 1u);
        }
        if (see) {
            const int page = table[j / c.P];
            see = (unsigned)page < (unsigned)c.pages;
            at = (int64_t)page * c.stride_page + (int64_t)(j % c.P) * c.stride_token + (int64_t)g * c.stride_head;
        }
        float x = -__builtin_inff();
        if (see) {
            float sum = 0.f;
            for (int d = 0; d < c.D; d += E::kVec) {
                float kk[E::kVec], qq[E::kVec];
                E::widen(*(const u32x4*)((const char*)c.k + (at + d) * E::kBytes), kk);
                E::widen(*(const u32x4*)(q + d * E::kBytes), qq);
                for (int e = 0; e < E::kVec; ++e) sum += kk[e] * qq[e];
            }
            x = sum * a.scale;
        }
        float top = x;
        for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
        top = fmaxf(top, m);
        const float from = top == -__builtin_inff() ? 0.f : top;
        const float p = see ? expf(x - from) : 0.f;
        const float keep = expf(m - from);
        float sum = p;
        for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
        l = l * keep + sum;
        m = top;
        for (int e = 0; e < 4; ++e) o[e] *= keep;
        unsigned long long todo = __ballot(see);
        while (todo) {
            const int k = __ffsll(todo) - 1;
            todo &= todo - 1;
            const float w = __shfl(p, k);
            const int64_t from_at = __shfl((long long)at, k);
            for (int e = 0; e < 4; ++e) {
                const int d = e * 64 + lane;
                if (d < c.D) {
                    const char* v = (const char*)c.v + (from_at + d) * E::kBytes;
                    const float vv = BF16 ? __uint_as_float((uint32_t) * (const uint16_t*)v << 16) : *(const float*)v;
                    o[e] += w * vv;
                }
            }
        }
    }
    for (int e = 0; e < 4; ++e) {
        const int d = e * 64 + lane;
        if (d >= c.D) continue;
        const float y = m == -__builtin_inff() ? 0.f : o[e] / l;
        char* out = (char*)a.out.data + ((int64_t)t * a.out.stride_row + (int64_t)h * a.out.stride_head + d) * E::kBytes;
        if (BF16)
            *(uint16_t*)out = (uint16_t)pack_bf16(y, 0.f);
        else
            *(float*)out = y;
    }
    if (lane == 0 && a.lse) a.lse[(int64_t)t * a.H + h] = m + logf(l);
}

}  // namespace

size_t attention_workspace(const CacheArgs& c, int H, bool bf16) { return 0; }

hipError_t launch_attention(const AttentionArgs& a, bool bf16, hipStream_t stream) {
    const long items = (long)a.c.rows * a.H;
    const dim3 grid((unsigned)((items + 3) / 4));
    if (bf16)
        hipLaunchKernelGGL(attention_kernel<true>, grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL(attention_kernel<false>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace psd
