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

// The scale bytes of a cache held in 4 bits, whose CacheArgs strides are the codes', in bytes.
struct ScaleArgs {
    void* k;
    void* v;
    int64_t layer, page, token, head;
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

struct Append4Args {
    AppendArgs a;
    ScaleArgs s;
    RowsArgs k_held, v_held;  // data NULL: not asked for
};
hipError_t launch_kv_append4(const Append4Args& a, bool bf16, hipStream_t stream);

struct KeepArgs {
    CacheArgs c;
    const int32_t* keep;
    int64_t keep_stride;
    int keep_width;
    const int32_t* n_keep;
    int32_t* kv_out;
};
hipError_t launch_kv_keep(const KeepArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_kv_keep4(const KeepArgs& a, const ScaleArgs& s, hipStream_t stream);

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

// Joins the parts of tile_kernel's rows.
hipError_t launch_attention_join(const AttentionArgs& a, const Plan& p, hipStream_t stream);

struct Attention4Args {
    AttentionArgs a;
    ScaleArgs s;
};
hipError_t launch_attention4(const Attention4Args& a, bool bf16, hipStream_t stream);

struct ReserveArgs {
    int P, pages, page_shift;
    int32_t* ring;
    int32_t* state;
    int B, rows, max_new, max_kv, table_width;
    int64_t table_stride;
    const int32_t* n_new;
    const int32_t* kv_have;
    int32_t* held;
    int32_t* table;
    int32_t* new_start;
    int32_t* kv_len;
    int32_t* granted;
    int32_t* row_seq;
    int32_t* positions;
    int64_t* slots;
};
hipError_t launch_kv_reserve(const ReserveArgs& a, hipStream_t stream);

struct AdjustArgs {
    const void* logits;
    void* out;
    int B, K, S, V, depth0;
    const int32_t* text;
    int64_t text_stride;
    int text_max;
    const int64_t* length;
    const int64_t* from;
    const int32_t* drafts;
    int gamma;
    const float* repetition;
    const float* presence;
    const float* frequency;
    const int32_t* bias_tokens;
    const float* bias;
    int bias_width;
    const uint32_t* allowed;
    int64_t allowed_seq, allowed_row;
};
bool adjust_fits(const AdjustArgs& a, bool bf16);  // the launch stays inside a grid's limits
hipError_t launch_adjust(const AdjustArgs& a, bool bf16, hipStream_t stream);

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
