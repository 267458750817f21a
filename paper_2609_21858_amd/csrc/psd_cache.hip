// psd_cache.hip -- new keys and values into a paged cache, and keeping an accepted path (gfx950).
//
// Append, for each head x of a new token's query and key (values are copied):
//   y_d = x_d / sqrt(mean(x^2) + eps) * w_d            (optional)
//   (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin)  for the R/2 pairs (a, b) of the first
//   R dimensions, with the row's cosine and sine; one rounding to the output's type.
// It reads and writes each element once, so memory bounds it: (H + 2G) D elements a row both
// ways.
#include <hip/hip_runtime.h>

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kAppendThreads = 256;

// One workgroup per packed row.  A head's 16-byte pieces lie on neighbouring lanes (GS of
// them, a power of two at least D / VEC), and a thread takes the same piece of several heads,
// so the row's cosines and sines are loaded once into registers.  The pair partner of an
// element in the half-split order is in another lane: the normed head goes through LDS,
// transposed so that neighbouring lanes hit neighbouring banks (any R, no alignment rule).
template <bool BF16>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a, int GS) {
    using E = Elem<BF16>;
    constexpr int VEC = E::kVec;
    __shared__ float s_x[VEC][kAppendThreads];
    const CacheArgs& c = a.c;
    const int t = blockIdx.x;
    const int tid = threadIdx.x;
    const int b = find_seq(c.new_start, c.B, t);
    if (b >= c.B) return;
    const Seq s = load_seq(c, b);
    const int i = t - s.row0;
    if (i < 0 || i >= s.n) return;
    const int pos = s.first + i;
    const int half = a.R / 2;
    const int lane = tid & (GS - 1), group = tid / GS, groups = kAppendThreads / GS;
    const int d0 = lane * VEC;
    const bool in_head = d0 < c.D;

    // the place in the cache, if the token has one
    int64_t at = -1;
    if (pos >= 0 && pos < c.max_kv) {
        const int pi = pos / c.P;
        if (pi < c.table_width) {
            const int page = c.table[(int64_t)b * c.table_stride + pi];
            if ((unsigned)page < (unsigned)c.pages)
                at = (int64_t)page * c.stride_page + (int64_t)(pos - pi * c.P) * c.stride_token;
        }
    }

    // cosine and signed sine of this thread's elements: y_d = x_d * cs + partner * sn
    float cs[VEC], sn[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        cs[j] = 1.f;
        sn[j] = 0.f;
    }
    if (in_head && d0 < a.R) {
        const int p = a.positions ? a.positions[t] : pos;
        const bool known = p >= 0 && p < a.positions_max;
        const int64_t base = (int64_t)(known ? p : 0) * half;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int d = d0 + j;
            if (d < a.R) {
                const int r = a.interleaved ? d / 2 : (d < half ? d : d - half);
                const bool second = a.interleaved ? (d & 1) : d >= half;
                const float cc = known ? a.cos[base + r] : __builtin_nanf("");
                const float ss = known ? a.sin[base + r] : __builtin_nanf("");
                cs[j] = cc;
                sn[j] = second ? ss : -ss;
            }
        }
    }

    const int slots = a.H + 2 * c.G;
    // every group runs the same number of rounds: the shuffles and the LDS exchange stay
    // within a group's lanes, all of one wave
    for (int h0 = 0; h0 < slots; h0 += groups) {
        const int h = h0 + group;
        const bool on = h < slots && in_head;
        const int kind = h < a.H ? 0 : h < a.H + c.G ? 1 : 2;  // query, key, value
        const int head = kind == 0 ? h : kind == 1 ? h - a.H : h - a.H - c.G;
        u32x4 w = {0, 0, 0, 0};
        if (on) {
            const RowsArgs& r = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
            w = *(const u32x4*)((const char*)r.data + ((int64_t)t * r.stride_row + (int64_t)head * r.stride_head + d0) * E::kBytes);
        }
        float x[VEC];
        E::widen(w, x);
        const void* norm = kind == 0 ? a.q_norm : a.k_norm;
        if (a.q_norm || a.k_norm) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum += x[j] * x[j];
            for (int o = GS / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            if (on && kind != 2 && norm) {
                const float scale = 1.f / sqrtf(sum / (float)c.D + a.eps);
                float wt[VEC];
                E::widen(*(const u32x4*)((const char*)norm + (int64_t)d0 * E::kBytes), wt);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[j] = x[j] * scale * wt[j];
            }
        }
        if (a.R > 0) {
            float y[VEC];
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) y[j] = x[j ^ 1];
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) s_x[j][tid] = x[j];
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int d = d0 + j;
                    const int p = d < half ? d + half : d - half;
                    y[j] = d < a.R ? s_x[p % VEC][tid - lane + p / VEC] : 0.f;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
            if (kind != 2 && d0 < a.R) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (d0 + j < a.R) x[j] = x[j] * cs[j] + y[j] * sn[j];
            }
        }
        if (on) {
            if (kind == 0) {
                *(u32x4*)((char*)a.q_out.data +
                          ((int64_t)t * a.q_out.stride_row + (int64_t)head * a.q_out.stride_head + d0) * E::kBytes) =
                    E::narrow(x);
            } else if (at >= 0) {
                char* pool = (char*)(kind == 1 ? c.k : c.v);
                *(u32x4*)(pool + (at + (int64_t)head * c.stride_head + d0) * E::kBytes) = kind == 1 ? E::narrow(x) : w;
            }
        }
    }
}

constexpr int kKeepThreads = 256;
constexpr int kKeepBatch = 4;

// One thread moves one 16-byte column (keys or values, head, piece) of a sequence's kept
// tokens in one layer.  Indices ascend strictly, so keep[i] >= i and the places still to be
// read lie behind the places written so far: kKeepBatch tokens are read together, then written.
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KeepArgs a, int vec, int bytes) {
    const CacheArgs& c = a.c;
    const int pieces = c.D / vec;
    const int blocks = (2 * c.G * pieces + kKeepThreads - 1) / kKeepThreads;  // of one sequence and layer
    const int b = blockIdx.x / blocks, part = blockIdx.x - b * blocks;
    const int layer = blockIdx.y;
    const Seq s = load_seq(c, b);
    const int total = max(c.new_start[b + 1] - max(c.new_start[b], 0), 0);
    const int n = max(min(min(a.n_keep[b], a.keep_width), total), 0);
    if (layer == 0 && part == 0 && threadIdx.x == 0 && a.kv_out) a.kv_out[b] = s.first + n;
    const int col = part * kKeepThreads + threadIdx.x;
    if (col >= 2 * c.G * pieces) return;
    const bool value = col >= c.G * pieces;
    const int rest = value ? col - c.G * pieces : col;
    const int g = rest / pieces, d0 = (rest - g * pieces) * vec;
    char* pool = (char*)(value ? c.v : c.k) + ((int64_t)layer * c.stride_layer + (int64_t)g * c.stride_head + d0) * bytes;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    const int32_t* keep = a.keep + (int64_t)b * a.keep_stride;
    auto place = [&](int i) -> int64_t {
        const int pos = s.first + i;
        if (i < 0 || i >= total || pos < 0 || pos >= c.max_kv) return -1;
        const int pi = pos / c.P;
        if (pi >= c.table_width) return -1;
        const int page = table[pi];
        if ((unsigned)page >= (unsigned)c.pages) return -1;
        return ((int64_t)page * c.stride_page + (int64_t)(pos - pi * c.P) * c.stride_token) * bytes;
    };
    for (int i0 = 0; i0 < n; i0 += kKeepBatch) {
        u32x4 w[kKeepBatch];
        int64_t to[kKeepBatch];
#pragma unroll
        for (int j = 0; j < kKeepBatch; ++j) {
            const int i = i0 + j;
            const int from = i < n ? keep[i] : -1;
            const int64_t src = from >= 0 && from != i ? place(from) : -1;
            to[j] = src >= 0 ? place(i) : -1;
            if (to[j] >= 0) w[j] = *(const u32x4*)(pool + src);
        }
#pragma unroll
        for (int j = 0; j < kKeepBatch; ++j)
            if (to[j] >= 0) *(u32x4*)(pool + to[j]) = w[j];
    }
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, bool bf16, hipStream_t stream) {
    int gs = 1;
    while (gs * (bf16 ? 8 : 4) < a.c.D) gs *= 2;
    if (bf16)
        hipLaunchKernelGGL(append_kernel<true>, dim3(a.c.rows), dim3(kAppendThreads), 0, stream, a, gs);
    else
        hipLaunchKernelGGL(append_kernel<false>, dim3(a.c.rows), dim3(kAppendThreads), 0, stream, a, gs);
    return hipGetLastError();
}

hipError_t launch_kv_keep(const KeepArgs& a, bool bf16, hipStream_t stream) {
    const int vec = bf16 ? 8 : 4;
    const int cols = 2 * a.c.G * (a.c.D / vec);
    hipLaunchKernelGGL(keep_kernel, dim3((cols + kKeepThreads - 1) / kKeepThreads * a.c.B, a.c.layers), dim3(kKeepThreads), 0,
                       stream, a, vec, bf16 ? 2 : 4);
    return hipGetLastError();
}

}  // namespace psd
