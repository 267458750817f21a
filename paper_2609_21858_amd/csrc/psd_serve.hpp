// psd_serve.hpp -- launch arguments of the paged cache, its attention and the verification
// from given random numbers (internal to libpsd).
#pragma once

#include <hip/hip_runtime.h>

#include "psd_attention_plan.hpp"
#include "psd_layout.hpp"

namespace psd {

struct RowsArgs {
    void* data;
    int64_t stride_row, stride_head;
};

struct AppendArgs {
    CacheArgs c;
    RowsArgs k, v, q, q_out;
    int H;  // 0: no queries
    int R, interleaved, positions_max;
    const float* cos;
    const float* sin;
    const int32_t* positions;
    const void* q_norm;
    const void* k_norm;
    float eps;
};
hipError_t launch_kv_append(const AppendArgs& a, bool bf16, hipStream_t stream);

struct KeepArgs {
    CacheArgs c;
    const int32_t* keep;
    int64_t keep_stride;
    int keep_width;
    const int32_t* n_keep;
    int32_t* kv_out;
};
hipError_t launch_kv_keep(const KeepArgs& a, bool bf16, hipStream_t stream);

struct AttentionArgs {
    CacheArgs c;
    RowsArgs q, out;
    int H;
    float scale;
    int window;
    const uint32_t* mask;
    int mask_words;
    float* lse;
    void* workspace;
    size_t workspace_bytes;
};
hipError_t launch_attention(const AttentionArgs& a, bool bf16, hipStream_t stream);

struct GivenArgs {
    const void* target;
    const void* draft;
    const int32_t* draft_tokens;
    const int32_t* n_drafts;
    const float* u;
    const float* e;
    int32_t* out_tokens;
    int32_t* out_len;
    float* target_lse;
    float* draft_lse;
    void* workspace;
    int B, gamma, V;
    float T_target, T_draft;
};
size_t given_workspace(int B, int gamma, int V, bool bf16);
hipError_t launch_given(const GivenArgs& a, bool bf16, hipStream_t stream);

}  // namespace psd
