// Internal launch interface between the C-ABI layer and the kernel translation units.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/vardrop.h"

namespace vardrop {

// Kernel identities for the launch counter and the optional per-kernel event timer (vardrop_profile_*).
enum KernelId {
    K_HASH = 0, K_SELECT_SMALL, K_SELECT_COUNT, K_SELECT_GROUP, K_SELECT_SAMPLE, K_ATTN_FWD, K_BWD_PREP, K_ATTN_BWD, K_BWD_CONVERT, K_PEARSON_NORM, K_PEARSON_MAX, K_GATHER_ROWS,
    K_SELECT_PLACE, K_SELECT_CLUSTER, K_PACKED_PLAN, K_PACKED_FWD, K_PACKED_TILE, K_PACKED_SHORT, K_PACKED_PREP, K_PACKED_BWD, K_PACKED_CONVERT, K_NORM_FWD, K_NORM_BWD, K_NORM_PARAMS, K_GRAD_NORM, K_GRAD_SCALE,
    K_EMBED_FWD, K_EMBED_COUNT, K_EMBED_SORT, K_EMBED_SUM, K_EMBED_JOIN, K_EMBED_SCAN, K_EMBED_PLACE, K_ACT_FWD, K_ACT_BWD,
    K_LOSS_COUNT, K_LOSS_ROWS, K_LOSS_STATS, K_LOSS_JOIN, K_LOSS_GRAD, K_LOSS_BACK, K_LOSS_REST,
    K_COUNT
};
// Wrap a kernel launch: counts it and, when the timer is armed, brackets it with a pair of CUDA events on `stream`.
struct LaunchScope {
    LaunchScope(int id, cudaStream_t stream);
    ~LaunchScope();
    int id_;
    cudaStream_t stream_;
    void* stop_;
};

// hash.cu
size_t hash_workspace_bytes(const vardrop_hash_cfg& cfg);
int hash_validate(const vardrop_hash_cfg& cfg, int* f_lo, int* f_hi);
int hash_launch(const float* x, const vardrop_hash_cfg& cfg, uint64_t* keys, int32_t* freqs, float* amp_dbg, int* status,
                cudaStream_t stream);

// how the transform in shared memory shares a call out: windows of a row per pass, rows to a CTA
struct HashSplit {
    int rows_total, win_per_row, rows_per_cta, chunk;
    bool few_rows;
};
HashSplit hash_split(const vardrop_hash_cfg& cfg);

// hash_rows.cu: register-blocked plans for selected lookback lengths; -1 = no plan for this configuration
int hash_rows_launch(const float* x, const vardrop_hash_cfg& cfg, int f_lo, int f_hi, uint64_t* keys, int32_t* freqs, float* amp_dbg,
                     int* status, cudaStream_t stream);
// hash_dft.cu: the candidate bins as a matrix product; -1 = the transform in shared memory is better
int hash_dft_launch(const float* x, const vardrop_hash_cfg& cfg, int f_lo, int f_hi, uint64_t* keys, int32_t* freqs, float* amp_dbg, int* status,
                    cudaStream_t stream);
int sm_count();       // multiprocessors of the current device

// select.cu
size_t select_workspace_bytes(const vardrop_select_cfg& cfg);
int select_validate(const vardrop_select_cfg& cfg);
int select_launch(const uint64_t* keys, const vardrop_select_cfg& cfg, int32_t* group_id, int32_t* group_offsets, int32_t* members,
                  int32_t* n_groups, int32_t* sel_idx, int32_t* n_sel, int32_t* inv_idx, void* ws, cudaStream_t stream, bool one_cta = false);

// allocation-free variant: scratch is a fixed array inside the module
constexpr int kStaticMaxRows = 16384;                 // largest S * N it accepts
constexpr int kStaticSelectBytes = 400 * 1024;        // size of that array
int select_static_launch(const uint64_t* keys, const vardrop_select_cfg& cfg, int32_t* group_id, int32_t* group_offsets,
                         int32_t* members, int32_t* n_groups, int32_t* sel_idx, int32_t* n_sel, int32_t* inv_idx, cudaStream_t stream);

// gather_rows.cu
int gather_rows_validate(const vardrop_gather_cfg& cfg);
int gather_rows_launch(const float* x, const int32_t* sel_idx, const int32_t* n_sel, const vardrop_gather_cfg& cfg, float* x_sel, cudaStream_t stream);

// pearson.cu
size_t pearson_workspace_bytes(const vardrop_pearson_cfg& cfg);
int pearson_validate(const vardrop_pearson_cfg& cfg);
int pearson_launch(const float* x, const vardrop_pearson_cfg& cfg, float* max_rho, int32_t* n_above, void* ws, cudaStream_t stream);

// attn_*.cu
size_t attn_workspace_bytes(const vardrop_attn_cfg& cfg);
int attn_validate(const vardrop_attn_cfg& cfg);
int attn_fwd_launch(const void* q, const void* k, const void* v, const int32_t* sel_idx, const int32_t* n_sel,
                    const vardrop_attn_cfg& cfg, void* o, float* lse, void* ws, cudaStream_t stream);
int attn_bwd_launch(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o,
                    const int32_t* sel_idx, const int32_t* n_sel, const int32_t* inv_idx, const vardrop_attn_cfg& cfg, void* dq,
                    void* dk, void* dv, void* ws, cudaStream_t stream);
int attn_bwd_many_launch(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o, const int32_t* sel_idx,
                         const int32_t* n_sel, const int32_t* inv_idx, const vardrop_attn_cfg& cfg, void* dq, void* dk, void* dv, void* ws, cudaStream_t stream);

// packed_plan.cu, attn_packed_fwd.cu, attn_packed_bwd.cu
int packed_validate(const vardrop_packed_cfg& cfg);
size_t packed_plan_bytes(const vardrop_packed_cfg& cfg);
int packed_plan_launch(const int32_t* cu_seqlens, const vardrop_packed_cfg& cfg, void* plan, cudaStream_t stream);
size_t attn_packed_workspace_bytes(const vardrop_packed_cfg& cfg);
int attn_packed_fwd_launch(const void* q, const void* k, const void* v, const void* plan, const vardrop_packed_cfg& cfg, void* o, float* lse, void* ws, cudaStream_t stream);
int attn_packed_bwd_launch(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o, const void* plan, const vardrop_packed_cfg& cfg, void* dq,
                           void* dk, void* dv, void* ws, cudaStream_t stream);

// norm.cu
int norm_validate(const vardrop_norm_cfg& cfg);
size_t norm_workspace_bytes(const vardrop_norm_cfg& cfg);
int norm_fwd_launch(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const float* b_pre, const int32_t* sel_idx,
                    const int32_t* n_sel, const vardrop_norm_cfg& cfg, void* h, void* u, float* stats, cudaStream_t stream);
int norm_bwd_launch(const void* x, const void* y, const float* gate, const float* w_post, const float* b_post, const float* w_pre, const int32_t* sel_idx, const int32_t* n_sel,
                    const int32_t* inv_idx, const float* stats, const void* d_h, const void* d_u, const vardrop_norm_cfg& cfg, void* dx, void* dy, float* d_gate, float* d_w_post,
                    float* d_b_post, float* d_w_pre, float* d_b_pre, void* ws, cudaStream_t stream);

// grad_clip.cu
size_t grad_clip_workspace_bytes();
int grad_clip_validate(const vardrop_tensor* tensors, int32_t count, const vardrop_clip_cfg& cfg);
int grad_clip_launch(const vardrop_tensor* tensors, int32_t count, const vardrop_clip_cfg& cfg, float* norm, void* ws, cudaStream_t stream);

// embed.cu
int embed_validate(const vardrop_embed_cfg& cfg);
size_t embed_workspace_bytes(const vardrop_embed_cfg& cfg);
int embed_fwd_launch(const void* table, const int32_t* idx, const vardrop_embed_cfg& cfg, void* out, void* ws, cudaStream_t stream);
int embed_bwd_launch(const void* d_out, const int32_t* idx, const vardrop_embed_cfg& cfg, void* d_table, void* ws, cudaStream_t stream);

// act.cu
int act_validate(const vardrop_act_cfg& cfg);
size_t act_ckpt_bytes(const vardrop_act_cfg& cfg);
int act_fwd_launch(const void* a, const void* b, const int32_t* n_sel, const vardrop_act_cfg& cfg, void* y, void* ckpt, cudaStream_t stream);
int act_bwd_launch(const void* d_y, const void* ckpt, const int32_t* n_sel, const vardrop_act_cfg& cfg, void* d_a, void* d_b, void* y, cudaStream_t stream);

// loss.cu
int loss_validate(const vardrop_loss_cfg& cfg);
size_t loss_workspace_bytes(const vardrop_loss_cfg& cfg);
int loss_fwd_launch(const void* h, const void* w, const int32_t* labels, const vardrop_loss_cfg& cfg, float* loss, float* lse, void* ws, cudaStream_t stream);
int loss_bwd_launch(const void* h, const void* w, const int32_t* labels, const float* lse, const float* d_loss, const vardrop_loss_cfg& cfg, void* d_h, void* d_w, void* ws, cudaStream_t stream);

}  // namespace vardrop
