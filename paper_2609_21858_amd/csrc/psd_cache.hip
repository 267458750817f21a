// psd_cache.hip -- new keys and values into a paged cache, and keeping an accepted path (gfx950).
//
// Append, for each head x of a new token's query and key (values are copied):
//   y_d = x_d / sqrt(mean(x^2) + eps) * w_d            (optional)
//   (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin)  for the R/2 pairs (a, b) of the first
//   R dimensions, with the row's cosine and sine; one rounding to the output's type.
// It reads and writes each element once, so memory bounds it: (H + 2G) D elements a row both
// ways.  8 prompts of up to 2048 tokens, H=32, G=8, D=128, bfloat16, normed: 53.4 us, 5.2 TB/s read
// and written (a device copy moves 4.9), float32 119.5 us, 4.7 TB/s; one token of 4 sequences, three dependent
// loads: 4.4 us, float32 6.5.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "psd_quant4.hpp"
#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kAppendThreads = 256;

// Where the pair partner of an element lies.
enum Turn {
    kNoTurn,       // R = 0
    kInterleaved,  // in the same 16 bytes
    kPieces,       // halves of whole 16-byte pieces: one other piece, read again (from the first-level cache)
    kAnywhere,     // halves that cut a piece: through LDS
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__host__ __device__ __forceinline__ const AppendArgs& rows_of(const AppendArgs& a) { return a; }
__host__ __device__ __forceinline__ const AppendArgs& rows_of(const Append4Args& a) { return a.a; }

// 1 / sqrt(x) within a few 2^-53: the hardware's estimate (about 2^-26) and two Newton steps, a fifth of the instructions of
// a square root and a division.  Of 0, infinity and NaN the estimate is the answer.
__device__ __forceinline__ double rsqrt64(double x) {
    const double r0 = __builtin_amdgcn_rsq(x);
    double r = r0;
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.), r);
    return x > 0. && x < (double)__builtin_inf() ? r : r0;
}

// One piece of N heads at once.
template <int N>
struct Heads {
    u32x4 own[N], other[N];  // this thread's piece, and its partners' (kPieces)
};

// A packed row per 64 or 256 threads.  A head's 16-byte pieces lie on neighbouring lanes (GS of
// them, a power of two at least D / VEC, all of one wave), and a thread takes the same piece of
// several heads.  What a row needs once per piece stays in registers: with A = weight cos and
// B = partner's weight sin,
//   y_d = (x_d A_d + x_partner B_d) / sqrt(mean(x^2) + eps).
// The row's data sets out before its place is known, which takes three dependent loads.  q_out may
// be q: a wave has read a head, partners included, before it writes it.
//
// Q4: keys and values go into 4 bits (psd_quant4.hpp), a group of 32 dimensions from 4 or 8 lanes.  Keys
// are computed in 64 bits, since an error of 2^-24 would put one code in a million on the other side of a border.
// The prompts above, 293 MB with the held keys and values: 71 us, 4.1 TB/s; one token of 4 sequences 5.4.
template <bool BF16, Turn TURN, bool Q4>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(std::conditional_t<Q4, Append4Args, AppendArgs> args, int GS,
                                                                int row_threads) {
    const AppendArgs& a = rows_of(args);
    using E = Elem<BF16>;
    constexpr int VEC = E::kVec;
    // heads of a thread whose loads are in flight together: queries; keys, values (Q4: registers for four waves a SIMD)
    constexpr int NQ = 4, NK = Q4 && TURN != kAnywhere ? 1 : 2;
    __shared__ float s_x[TURN == kAnywhere ? VEC : 1][kAppendThreads];
    const CacheArgs& c = a.c;
    const int tid = threadIdx.x;
    const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * (kAppendThreads / row_threads) + tid / row_threads);
    if (t >= c.rows) return;
    const int half = a.R / 2;
    const int lane = tid & (GS - 1), group = (tid & (row_threads - 1)) / GS, groups = row_threads / GS;
    const int d0 = lane * VEC;
    const bool in_head = d0 < c.D;
    const bool turns = TURN != kNoTurn && in_head && d0 < a.R;
    const int dp = TURN == kPieces && turns ? (d0 < half ? d0 + half : d0 - half) : d0;

    // heads h0, h0 + groups, ...: clamped, so that loads are unconditional
    auto load = [&](auto& w, const RowsArgs& r, int heads, int h0, bool pairs) {
        const char* src = (const char*)r.data + (int64_t)t * r.stride_row * E::kBytes;
        constexpr int N = sizeof(w.own) / sizeof(w.own[0]);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const char* at = src + (int64_t)min(h0 + k * groups, heads - 1) * r.stride_head * E::kBytes;
            w.own[k] = *(const u32x4*)(at + min(d0, c.D - VEC) * E::kBytes);
            if (TURN == kPieces && pairs) w.other[k] = *(const u32x4*)(at + min(dp, c.D - VEC) * E::kBytes);
        }
    };
    Heads<NQ> wq;
    Heads<NK> wk, wv;
    if (a.H > 0) load(wq, a.q, a.H, group, true);
    load(wk, a.k, c.G, group, true);
    load(wv, a.v, c.G, group, false);

    const int b = find_seq(c.new_start, c.B, t);
    if (b >= c.B) return;
    const Seq s = load_seq(c, b);
    const int i = t - s.row0;
    if (i < 0 || i >= s.n) return;
    const int pos = s.first + i;

    // the place in the cache, if the token has one (elements; Q4: bytes)
    int64_t at = -1, scale_at = 0;
    if (pos >= 0 && pos < c.max_kv) {
        const int pi = pos / c.P;
        if (pi < c.table_width) {
            const int page = c.table[(int64_t)b * c.table_stride + pi];
            if ((unsigned)page < (unsigned)c.pages) {
                at = (int64_t)page * c.stride_page + (int64_t)(pos - pi * c.P) * c.stride_token;
                if constexpr (Q4) scale_at = (int64_t)page * args.s.page + (int64_t)(pos - pi * c.P) * args.s.token;
            }
        }
    }

    // cosines and signed sines of this thread's elements
    float cs[VEC], sn[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        cs[j] = 1.f;
        sn[j] = 0.f;
    }
    if (turns) {
        const int p = a.positions ? a.positions[t] : pos;
        const bool known = p >= 0 && p < a.positions_max;
        const int64_t base = (int64_t)(known ? p : 0) * half;
        if constexpr (TURN == kPieces) {
            const int r0 = d0 < half ? d0 : d0 - half;
            const float sign = d0 < half ? -1.f : 1.f;
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                const f32x4_any cc = *(const f32x4_any*)(a.cos + base + r0 + j), ss = *(const f32x4_any*)(a.sin + base + r0 + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    cs[j + e] = cc[e];
                    sn[j + e] = ss[e] * sign;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int d = d0 + j;
                if (d < a.R) {
                    const int r = TURN == kInterleaved ? d / 2 : d < half ? d : d - half;
                    const bool second = TURN == kInterleaved ? (j & 1) : d >= half;
                    cs[j] = a.cos[base + r];
                    sn[j] = second ? a.sin[base + r] : -a.sin[base + r];
                }
            }
        }
        if (!known)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (d0 + j < a.R) cs[j] = __builtin_nanf("");
    }

    const float inv_d = 1.f / (float)c.D;
    const double inv_d64 = 1. / (double)c.D;
    // Queries or keys, in the arithmetic of `zero`'s type; each head's elements go to `emit`.
    auto turn = [&](auto zero, auto& w, const RowsArgs& r, int heads, const void* norm, auto emit) {
        using T = decltype(zero);
        constexpr int N = sizeof(w.own) / sizeof(w.own[0]);
        T A[VEC], B[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            A[j] = cs[j];
            B[j] = sn[j];
        }
        if (norm && in_head) {
            float wt[VEC];
            E::widen(*(const u32x4*)((const char*)norm + (int64_t)d0 * E::kBytes), wt);
#pragma unroll
            for (int j = 0; j < VEC; ++j) A[j] *= wt[j];
            if constexpr (TURN == kPieces) {
                float wp[VEC];
                E::widen(*(const u32x4*)((const char*)norm + (int64_t)dp * E::kBytes), wp);
#pragma unroll
                for (int j = 0; j < VEC; ++j) B[j] *= wp[j];
            } else if constexpr (TURN == kInterleaved) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) B[j] *= wt[j ^ 1];
            } else if constexpr (TURN == kAnywhere) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int d = d0 + j;
                    if (d < a.R) {
                        const int p = d < half ? d + half : d - half;
                        if constexpr (BF16)
                            B[j] *= __uint_as_float((uint32_t)((const uint16_t*)norm)[p] << 16);
                        else
                            B[j] *= ((const float*)norm)[p];
                    }
                }
            }
        }
        // every group runs the same rounds: exchanges stay within a group's lanes, all of one wave
        for (int h0 = 0; h0 < heads; h0 += N * groups) {
            if (h0 > 0) load(w, r, heads, h0 + group, true);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (h0 + k * groups >= heads) break;
                const int h = h0 + k * groups + group;
                float x[VEC], y[VEC];
                E::widen(w.own[k], x);
                T scale = 1;
                if (norm) {
                    T sum = 0;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sum += (T)x[j] * x[j];
                    if (!in_head) sum = 0;
                    for (int o = GS / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
                    if constexpr (sizeof(T) == 4)
                        scale = rsqrtf(sum * inv_d + a.eps);
                    else
                        scale = rsqrt64(sum * inv_d64 + a.eps);
                }
                if constexpr (TURN == kPieces) {
                    E::widen(w.other[k], y);
                } else if constexpr (TURN == kInterleaved) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) y[j] = x[j ^ 1];
                } else if constexpr (TURN == kAnywhere) {
                    // transposed, so that neighbouring lanes meet neighbouring banks
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s_x[j][tid] = x[j];
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const int d = d0 + j;
                        const int p = d < half ? d + half : d - half;
                        y[j] = d < a.R ? s_x[p % VEC][tid - lane + p / VEC] : 0.f;
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
                T z[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    T v = x[j] * A[j];
                    if (TURN != kNoTurn && turns && (TURN == kPieces || d0 + j < a.R)) v += y[j] * B[j];
                    z[j] = norm ? v * scale : v;
                }
                emit(h, z);
            }
        }
    };
    if (a.H > 0) {
        char* to = (char*)a.q_out.data + (int64_t)t * a.q_out.stride_row * E::kBytes;
        turn(0.f, wq, a.q, a.H, a.q_norm, [&](int h, const float (&z)[VEC]) {
            if (in_head && h < a.H) *(u32x4*)(to + ((int64_t)h * a.q_out.stride_head + d0) * E::kBytes) = E::narrow(z);
        });
    }
    if constexpr (Q4) {
        // VEC elements of a head in 4 bits: a group's lanes agree on its scale, its first lane writes it
        const int padded = (c.D + 31) / 32 * 32;
        auto put = [&](auto (&z)[VEC], int h, void* codes, void* scales, const RowsArgs& held) {
            if (!in_head)
#pragma unroll
                for (int j = 0; j < VEC; ++j) z[j] = 0;
            int s = quant4::scale_of(z);
#pragma unroll
            for (int o = 1; o < 32 / VEC; o <<= 1) s = max(s, __shfl_xor(s, o));
            const uint32_t w = quant4::encode(z, s);
            if (h >= c.G) return;
            if (at >= 0 && d0 < padded) {
                char* to = (char*)codes + at + (int64_t)h * c.stride_head + d0 / 2;
                if constexpr (VEC == 8)
                    *(uint32_t*)to = w;
                else
                    *(uint16_t*)to = (uint16_t)w;
                if (d0 % 32 == 0) ((uint8_t*)scales)[scale_at + (int64_t)h * args.s.head + d0 / 32] = (uint8_t)s;
            }
            if (held.data && in_head)
                *(u32x4*)((char*)held.data + ((int64_t)t * held.stride_row + (int64_t)h * held.stride_head + d0) * E::kBytes) =
                    quant4::decode<BF16>(w, s);
        };
        turn(0., wk, a.k, c.G, a.k_norm, [&](int h, double (&z)[VEC]) { put(z, h, c.k, args.s.k, args.k_held); });
        for (int h0 = 0; h0 < c.G; h0 += NK * groups) {
            if (h0 > 0) load(wv, a.v, c.G, h0 + group, false);
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                if (h0 + k * groups >= c.G) break;
                float z[VEC];
                E::widen(wv.own[k], z);
                put(z, h0 + k * groups + group, c.v, args.s.v, args.v_held);
            }
        }
        return;
    }
    turn(0.f, wk, a.k, c.G, a.k_norm, [&](int h, const float (&z)[VEC]) {
        if (in_head && h < c.G && at >= 0)
            *(u32x4*)((char*)c.k + (at + (int64_t)h * c.stride_head + d0) * E::kBytes) = E::narrow(z);
    });
    if (at < 0) return;
    for (int h0 = 0; h0 < c.G; h0 += NK * groups) {
        if (h0 > 0) load(wv, a.v, c.G, h0 + group, false);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const int h = h0 + k * groups + group;
            if (in_head && h < c.G) *(u32x4*)((char*)c.v + (at + (int64_t)h * c.stride_head + d0) * E::kBytes) = wv.own[k];
        }
    }
}

constexpr int kKeepThreads = 256;
constexpr int kKeepBatch = 4;
constexpr int kKeepPlaces = 64;

// Moves 2 G D elements a kept token and layer, both ways.  The chain of dependent loads bounds it: 32
// layers of 64 sequences, K=4, gamma=4, G=8, D=128: 7.9 us (25 MB, 5.1 us at a copy's rate), float32 12.4; 4
// layers of one sequence: 3.2 us.
//
// One thread moves one 16-byte column (keys or values, head, piece) of a sequence's kept
// tokens in one layer.  The places of 64 tokens at a time are found by 64 threads together: the
// chain of dependent loads is lengths and indices, page table, data.  Indices ascend strictly,
// so keep[i] >= i and the places still to be read lie behind those written so far: kKeepBatch
// tokens are read together, then written.
//
// Q4: a column is a group's 16 bytes of codes, and its scale byte.  The same calls: 7.8 us, 6.7 MB, and 3.0.
template <bool Q4>
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KeepArgs a, ScaleArgs scales, int vec, int bytes) {
    __shared__ int64_t s_from[kKeepPlaces], s_to[kKeepPlaces];
    __shared__ int64_t s_scale_from[Q4 ? kKeepPlaces : 1], s_scale_to[Q4 ? kKeepPlaces : 1];
    const CacheArgs& c = a.c;
    const int pieces = (c.D + vec - 1) / vec;
    const int blocks = (2 * c.G * pieces + kKeepThreads - 1) / kKeepThreads;  // of one sequence and layer
    const int b = blockIdx.x / blocks, part = blockIdx.x - b * blocks;
    const int layer = blockIdx.y;
    const int tid = threadIdx.x;
    const int32_t* keep = a.keep + (int64_t)b * a.keep_stride;
    int from = tid < min(kKeepPlaces, a.keep_width) ? keep[tid] : -1;
    const int kept = a.n_keep[b];
    const Seq s = load_seq(c, b);
    const int total = s.total;
    const int n = max(min(min(kept, a.keep_width), total), 0);
    if (layer == 0 && part == 0 && tid == 0 && a.kv_out) a.kv_out[b] = s.first + n;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    auto place = [&](int i, int64_t* scale) -> int64_t {
        const int pos = s.first + i;
        if (i < 0 || i >= total || pos < 0 || pos >= c.max_kv) return -1;
        const int pi = pos / c.P;
        if (pi >= c.table_width) return -1;
        const int page = table[pi];
        if ((unsigned)page >= (unsigned)c.pages) return -1;
        if constexpr (Q4) *scale = (int64_t)page * scales.page + (int64_t)(pos - pi * c.P) * scales.token;
        return ((int64_t)page * c.stride_page + (int64_t)(pos - pi * c.P) * c.stride_token) * bytes;
    };
    const int col = part * kKeepThreads + tid;
    const bool on = col < 2 * c.G * pieces;
    const bool value = col >= c.G * pieces;
    const int rest = value ? col - c.G * pieces : col;
    const int g = rest / pieces, d0 = (rest - g * pieces) * vec;
    char* pool = (char*)(value ? c.v : c.k);
    uint8_t* scale_pool = nullptr;
    if constexpr (Q4) {
        pool += (int64_t)layer * c.stride_layer + (int64_t)g * c.stride_head + d0 / 2;
        scale_pool = (uint8_t*)(value ? scales.v : scales.k) + (int64_t)layer * scales.layer + (int64_t)g * scales.head + d0 / 32;
    } else {
        pool += ((int64_t)layer * c.stride_layer + (int64_t)g * c.stride_head + d0) * bytes;
    }
    for (int i0 = 0; i0 < n; i0 += kKeepPlaces) {
        if (i0 > 0) {
            __syncthreads();
            from = tid < min(kKeepPlaces, n - i0) ? keep[i0 + tid] : -1;
        }
        if (tid < kKeepPlaces) {
            const int i = i0 + tid;
            int64_t scale_src = 0, scale_dst = 0;
            const int64_t src = i < n && from != i ? place(from, &scale_src) : -1, dst = i < n ? place(i, &scale_dst) : -1;
            s_from[tid] = src;
            s_to[tid] = src >= 0 ? dst : -1;
            if constexpr (Q4) {
                s_scale_from[tid] = scale_src;
                s_scale_to[tid] = scale_dst;
            }
        }
        __syncthreads();
        const int m = min(kKeepPlaces, n - i0);
        if (!on) continue;
        for (int j0 = 0; j0 < m; j0 += kKeepBatch) {
            u32x4 w[kKeepBatch];
            uint8_t scale[kKeepBatch];
            int64_t to[kKeepBatch];
#pragma unroll
            for (int j = 0; j < kKeepBatch; ++j) {
                to[j] = j0 + j < m ? s_to[j0 + j] : -1;
                if (to[j] >= 0) w[j] = *(const u32x4*)(pool + s_from[j0 + j]);
                if (Q4 && to[j] >= 0) scale[j] = scale_pool[s_scale_from[j0 + j]];
            }
#pragma unroll
            for (int j = 0; j < kKeepBatch; ++j) {
                if (to[j] >= 0) *(u32x4*)(pool + to[j]) = w[j];
                if (Q4 && to[j] >= 0) scale_pool[s_scale_to[j0 + j]] = scale[j];
            }
        }
    }
}

constexpr int kWaveRows = 1024;

template <bool BF16, bool Q4, class Args>
void append(const Args& args, hipStream_t stream) {
    const AppendArgs& a = rows_of(args);
    int gs = 1;
    while (gs * (BF16 ? 8 : 4) < (Q4 ? (a.c.D + 31) / 32 * 32 : a.c.D)) gs *= 2;
    // A wave a row has the less to set up, a workgroup a row the shorter chain: from 1024 rows on (a wave
    // for each SIMD) the first is ahead (H=32, G=8, D=128, 1300 rows: 9.6 us and 10.8, 5400: 24.5 and 27.8).
    const int row_threads = a.c.rows >= kWaveRows ? 64 : kAppendThreads;
    const int per = kAppendThreads / row_threads;
    const dim3 grid((a.c.rows + per - 1) / per), block(kAppendThreads);
    if (a.R == 0)
        hipLaunchKernelGGL((append_kernel<BF16, kNoTurn, Q4>), grid, block, 0, stream, args, gs, row_threads);
    else if (a.interleaved)
        hipLaunchKernelGGL((append_kernel<BF16, kInterleaved, Q4>), grid, block, 0, stream, args, gs, row_threads);
    else if (a.R / 2 % Elem<BF16>::kVec == 0)
        hipLaunchKernelGGL((append_kernel<BF16, kPieces, Q4>), grid, block, 0, stream, args, gs, row_threads);
    else
        hipLaunchKernelGGL((append_kernel<BF16, kAnywhere, Q4>), grid, block, 0, stream, args, gs, row_threads);
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, bool bf16, hipStream_t stream) {
    if (bf16)
        append<true, false>(a, stream);
    else
        append<false, false>(a, stream);
    return hipGetLastError();
}

hipError_t launch_kv_append4(const Append4Args& a, bool bf16, hipStream_t stream) {
    if (bf16)
        append<true, true>(a, stream);
    else
        append<false, true>(a, stream);
    return hipGetLastError();
}

hipError_t launch_kv_keep(const KeepArgs& a, bool bf16, hipStream_t stream) {
    const int vec = bf16 ? 8 : 4;
    const int cols = 2 * a.c.G * (a.c.D / vec);
    hipLaunchKernelGGL((keep_kernel<false>), dim3((cols + kKeepThreads - 1) / kKeepThreads * a.c.B, a.c.layers), dim3(kKeepThreads),
                       0, stream, a, ScaleArgs{}, vec, bf16 ? 2 : 4);
    return hipGetLastError();
}

hipError_t launch_kv_keep4(const KeepArgs& a, const ScaleArgs& s, hipStream_t stream) {
    const int cols = 2 * a.c.G * ((a.c.D + 31) / 32);
    hipLaunchKernelGGL((keep_kernel<true>), dim3((cols + kKeepThreads - 1) / kKeepThreads * a.c.B, a.c.layers), dim3(kKeepThreads),
                       0, stream, a, s, 32, 1);
    return hipGetLastError();
}

}  // namespace psd
