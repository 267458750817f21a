// psd_pages.hip -- places for a call's new tokens: page tables, row starts, lengths, positions and slots
// from request lengths, pages from a ring of free ones (gfx950).
//
// With W_b = pages of kv_have + n_new and need_b = max(W_b - held_b, 0), sequence b is granted where the sums
// of n_new and of need up to it stay inside the call's rows and the free pages; what is granted, taken
// and given back is summed again, and those sums are every row's and page's place.  All of it is
// prefix sums over the sequences, then one independent step for each row, taken page and given page.
//
// Chains of dependent loads bound it (lengths, sums, ring or table, stores): 17 tokens of 64 sequences 8 us, up to 2048
// tokens of 512 sequences, 10.8 MB, 13.4, and 15.4 to take back the pages that they leave (107 by one workgroup).
#include <hip/hip_runtime.h>

#include "psd_serve.hpp"
#include "psd_serve_device.hpp"

namespace psd {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kBatch = 4;

typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef int64_t i64x2 __attribute__((ext_vector_type(2), aligned(8)));

// Inclusive sums over the workgroup of N values a thread; the totals in `total`.
template <int N>
__device__ __forceinline__ void block_sums(int64_t (&x)[N], int64_t (&total)[N], int64_t (*s_wave)[kWaves]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t below = __shfl_up(x[i], k);
            if (lane >= k) x[i] += below;
        }
    __syncthreads();  // the last sums' readers are done
    if (lane == 63)
#pragma unroll
        for (int i = 0; i < N; ++i) s_wave[i][wave] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        total[i] = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) x[i] += total[i];
            total[i] += s_wave[i][w];
        }
    }
}

// One sequence's share of a chunk of kThreads.
struct Share {
    int have, held, n, keep;  // tokens that stay, pages held, tokens granted, pages of both
    int64_t take, give;
};

// Every workgroup takes the sums over all sequences, a chunk of kThreads at a time, and its part of each chunk's rows
// and pages.  What it reads of `held` and `state` it has read before it counts itself out; the one that counts last writes both.
__global__ __launch_bounds__(kThreads) void reserve_kernel(ReserveArgs a) {
    __shared__ int64_t s_wave[3][kWaves];
    __shared__ int s_start[kThreads + 1], s_have[kThreads], s_held[kThreads], s_keep[kThreads];
    __shared__ int64_t s_take[kThreads + 1], s_give[kThreads + 1];
    __shared__ int s_last;
    const int tid = threadIdx.x, wg = blockIdx.x, wgs = gridDim.x;
    // a state that no call leaves is cut, so that every place lies in the ring
    const int free = min(max(a.state[1], 0), a.pages);
    const int first = min(max(a.state[0], 0), a.pages - 1);
    auto pages_of = [&](int tokens) {
        return a.page_shift >= 0 ? (int)(((int64_t)tokens + a.P - 1) >> a.page_shift) : (int)(((int64_t)tokens + a.P - 1) / a.P);
    };
    auto page_at = [&](int pos) { return a.page_shift >= 0 ? pos >> a.page_shift : pos / a.P; };
    auto ring_at = [&](int64_t i) {  // free page i, or the i-th place behind it; i < pages
        const uint32_t at = (uint32_t)first + (uint32_t)i;
        return at >= (uint32_t)a.pages ? at - a.pages : at;
    };
    const int64_t width = (int64_t)a.table_width * a.P;
    const int most = (int)min((int64_t)a.max_kv, width);
    int64_t asked = 0, needed = 0;           // of the chunks before
    int64_t rows = 0, taken = 0, given = 0;  // granted there
    auto share = [&](int c0) {
        Share s;
        const int b = c0 + tid;
        const bool on = b < a.B;
        s.have = on ? min(max(a.kv_have[b], 0), most) : 0;
        s.held = on ? min(max(a.held[b], 0), a.table_width) : 0;
        int n = on ? max(a.n_new[b], 0) : 0;
        if (n > a.max_new || n > most - s.have) n = 0;
        const int64_t need = max(pages_of(s.have + n) - s.held, 0);
        int64_t x[2] = {n, need}, sum[2];
        block_sums<2>(x, sum, s_wave);
        const bool ok = asked + x[0] <= a.rows && (need == 0 || needed + x[1] <= free);
        asked += sum[0];
        needed += sum[1];
        s.n = ok ? n : 0;
        s.take = ok ? need : 0;
        s.keep = pages_of(s.have + s.n);
        s.give = max(s.held - s.keep, 0);
        return s;
    };
    Share s;
    for (int c0 = 0; c0 < a.B; c0 += kThreads) {
        s = share(c0);
        int64_t x[3] = {s.n, s.take, s.give}, sum[3];
        block_sums<3>(x, sum, s_wave);
        s_start[tid + 1] = (int)x[0];
        s_take[tid + 1] = x[1];
        s_give[tid + 1] = x[2];
        if (tid == 0) {
            s_start[0] = 0;
            s_take[0] = s_give[0] = 0;
        }
        s_have[tid] = s.have;
        s_held[tid] = s.held;
        s_keep[tid] = s.keep;
        const int b = c0 + tid;
        if (c0 / kThreads % wgs == wg && b < a.B) {
            if (b == 0) a.new_start[0] = 0;
            a.new_start[b + 1] = (int)(rows + x[0]);
            a.kv_len[b] = s.have + s.n;
            if (a.granted) a.granted[b] = s.n;
        }
        __syncthreads();
        // the sequence of entry i of a chunk's sums: the last whose sum before it is at most i
        auto find = [&](const auto* sums, int64_t i) {
            int lo = 0;
#pragma unroll
            for (int step = kThreads / 2; step > 0; step >>= 1)
                if (sums[lo + step] <= i) lo += step;
            return lo;
        };
        // Four consecutive rows a thread: one search, mostly one page, and stores of 16 bytes.
        if (a.row_seq || a.positions || a.slots)
            for (int64_t t0 = (rows / 4 + (int64_t)wg * kThreads + tid) * 4; t0 < rows + sum[0]; t0 += (int64_t)wgs * kThreads * 4) {
                int q = find(s_start, max(t0 - rows, (int64_t)0));
                int had = -1, page = 0;  // position of the page that was found last
                i32x4 seq, pos;
                i64x2 slot[2];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = (int)(t0 + e - rows);
                    if (i < 0 || i >= sum[0]) continue;
                    while (s_start[q + 1] <= i) {
                        ++q;
                        had = -1;
                    }
                    seq[e] = c0 + q;
                    pos[e] = s_have[q] + i - s_start[q];
                    if (!a.slots) continue;
                    const int pi = page_at(pos[e]);
                    if (pi != had)
                        page = pi < s_held[q] ? a.table[(int64_t)(c0 + q) * a.table_stride + pi]
                                              : a.ring[ring_at(taken + s_take[q] + pi - s_held[q])];
                    had = pi;
                    slot[e / 2][e % 2] = (unsigned)page < (unsigned)a.pages ? (int64_t)page * a.P + (pos[e] - pi * a.P) : -1;
                }
                if (t0 >= rows && t0 + 4 <= rows + sum[0]) {
                    if (a.row_seq) *(i32x4*)(a.row_seq + t0) = seq;
                    if (a.positions) *(i32x4*)(a.positions + t0) = pos;
                    if (a.slots) {
                        *(i64x2*)(a.slots + t0) = slot[0];
                        *(i64x2*)(a.slots + t0 + 2) = slot[1];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t t = t0 + e;
                        if (t < rows || t >= rows + sum[0]) continue;
                        if (a.row_seq) a.row_seq[t] = seq[e];
                        if (a.positions) a.positions[t] = pos[e];
                        if (a.slots) a.slots[t] = slot[e / 2][e % 2];
                    }
                }
            }
        // Pages, kBatch of a thread together, so that their loads are in flight together.
        for (int64_t i0 = (int64_t)wg * kThreads + tid; i0 < sum[1]; i0 += (int64_t)wgs * kThreads * kBatch) {
            int32_t* to[kBatch];
            int page[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int64_t i = min(i0 + (int64_t)k * wgs * kThreads, sum[1] - 1);
                const int q = find(s_take, i);
                to[k] = a.table + (int64_t)(c0 + q) * a.table_stride + s_held[q] + (i - s_take[q]);
                page[k] = a.ring[ring_at(taken + i)];
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (i0 + (int64_t)k * wgs * kThreads < sum[1]) *to[k] = page[k];
        }
        for (int64_t i0 = (int64_t)wg * kThreads + tid; i0 < sum[2]; i0 += (int64_t)wgs * kThreads * kBatch) {
            int32_t* from[kBatch];
            int page[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int64_t i = min(i0 + (int64_t)k * wgs * kThreads, sum[2] - 1);
                const int q = find(s_give, i);
                from[k] = a.table + (int64_t)(c0 + q) * a.table_stride + s_keep[q] + (i - s_give[q]);
                page[k] = *from[k];
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int64_t i = i0 + (int64_t)k * wgs * kThreads;
                if (i >= sum[2]) continue;
                // (more than the ring holds: the caller's error, dropped)
                if (free + given + i < a.pages) a.ring[ring_at(free + given + i)] = page[k];
                *from[k] = -1;
            }
        }
        rows += sum[0];
        taken += sum[1];
        given += sum[2];
        __syncthreads();
    }
    for (int64_t t = rows + (int64_t)wg * kThreads + tid; t < a.rows; t += (int64_t)wgs * kThreads) {
        if (a.row_seq) a.row_seq[t] = -1;
        if (a.positions) a.positions[t] = -1;
        if (a.slots) a.slots[t] = -1;
    }
    if (wgs > 1) {
        __syncthreads();
        if (tid == 0) s_last = atomicAdd((unsigned*)a.state + 2, 1u) == (unsigned)wgs - 1;
        __syncthreads();
        if (!s_last) return;
    }
    asked = needed = 0;
    for (int c0 = 0; c0 < a.B; c0 += kThreads) {
        if (a.B > kThreads) s = share(c0);  // (else it is at hand)
        if (c0 + tid < a.B) a.held[c0 + tid] = s.held - (int)s.give + (int)s.take;
    }
    if (tid == 0) {
        a.state[0] = (int)ring_at(taken < a.pages ? taken : 0);
        a.state[1] = (int)min((int64_t)free - taken + given, (int64_t)a.pages);
        a.state[2] = 0;
    }
}

}  // namespace

hipError_t launch_kv_reserve(const ReserveArgs& args, hipStream_t stream) {
    ReserveArgs a = args;
    a.page_shift = -1;
    for (int k = 0; k <= 16; ++k)
        if (a.P == 1 << k) a.page_shift = k;
    // Workgroups for four rows a thread, and for half of the tables' entries in turn (how many change only the device knows);
    // each more takes the sums again.
    const long rows = a.row_seq || a.positions || a.slots ? a.rows : 0;
    const long work = std::max<long>(rows, (long)a.B * a.table_width / 2);
    const int wgs = (int)std::min<long>(std::max<long>((work + 4 * kThreads - 1) / (4 * kThreads), 1), 512);
    hipLaunchKernelGGL(reserve_kernel, dim3(wgs), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace psd
