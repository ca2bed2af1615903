// Host-side launchers of the paged-cache operators (rope.hip, pages.hip,
// paged_attention.hip); the entry points that check their arguments are in
// cache.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/dlm.h"

constexpr int kCacheMaxSeqs = 1024;      // the page kernels give a sequence a thread of one workgroup
constexpr int kCacheMaxKvHeads = 128;
constexpr int kCacheMaxPages = 1 << 20;

// The part of a dlm_cache that the kernels take.
struct CacheArgs {
    char* k;
    char* v;
    int32_t* ref;
    int32_t* len;
    int32_t* table;
    int n_layers, n_pages, page_len, page_log2, n_kv, head_dim, n_seqs, max_pages;
};
inline CacheArgs cache_args(const dlm_cache& c) {
    return {(char*)c.d_k, (char*)c.d_v, c.d_ref, c.d_len, c.d_table, c.n_layers, c.n_pages, c.page_len,
            __builtin_ctz((unsigned)c.page_len), c.n_kv_heads, c.head_dim, c.n_seqs, c.max_pages};
}

// ----------------------------------------------------------------- rope.hip
hipError_t launch_rope(const dlm_rope& rope, int dtype, int rows, int heads, const void* x, int64_t x_row,
                       int64_t x_head, void* y, int64_t y_row, int64_t y_head, const int32_t* pos, bool transpose,
                       hipStream_t st);
hipError_t launch_append(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                         int max_rows, int src_dtype, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                         const dlm_rope* rope, const int32_t* pos, int n_heads, const void* q, int64_t q_stride,
                         void* q_out, int64_t q_out_stride, hipStream_t st);

// ------------------------------------------------------------- head_norm.hip
hipError_t launch_rope_norm(const dlm_rope& rope, int dtype, int rows, const dlm_norm_heads* q, const dlm_norm_heads* k,
                            float eps, const int32_t* pos, hipStream_t st);
size_t norm_grad_workspace_bytes(int head_dim);
hipError_t launch_rope_norm_grad(const dlm_rope& rope, int dtype, int rows, const dlm_norm_heads* q,
                                 const dlm_norm_heads* k, const dlm_norm_grads* dq, const dlm_norm_grads* dk, float eps,
                                 const int32_t* pos, void* ws, hipStream_t st);
hipError_t launch_append_norm(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                              int max_rows, int src_dtype, const void* k, int64_t k_stride, const void* v,
                              int64_t v_stride, const dlm_rope* rope, const int32_t* pos, int n_heads, const void* q,
                              int64_t q_stride, void* q_out, int64_t q_out_stride, int gain_dtype, const void* q_gain,
                              const void* k_gain, float eps, hipStream_t st);

// ----------------------------------------------------------------- pages.hip
// Workspace of reserve and compact.
size_t pages_workspace_bytes(int n_seqs, int n_pages);
hipError_t launch_cache_reset(const CacheArgs& c, hipStream_t st);
hipError_t launch_reserve(const CacheArgs& c, const int32_t* row_start, int total_rows, int32_t* ok, void* ws,
                          hipStream_t st);
hipError_t launch_commit(const CacheArgs& c, const int32_t* row_start, int total_rows, const int32_t* keep,
                         const int32_t* keep_start, int total_keep, int32_t* ok, hipStream_t st);
hipError_t launch_fork(const CacheArgs& c, int n_pairs, const int32_t* src, const int32_t* dst, int32_t* ok,
                       hipStream_t st);
hipError_t launch_truncate(const CacheArgs& c, const int32_t* new_len, hipStream_t st);
hipError_t launch_compact(const CacheArgs& c, int32_t* n_used, void* ws, hipStream_t st);

// ------------------------------------------------------ paged_attention.hip
size_t attend_workspace_bytes(int n_seqs, int n_kv, int head_dim, int total_rows, int max_rows, int group);
hipError_t launch_attend(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                         int max_rows, int max_keys, int n_heads, const void* q, int64_t q_stride,
                         const uint32_t* mask, int mask_words, float scale, void* o, int64_t o_stride, float* lse,
                         void* ws, hipStream_t st);
// What the sequences of a group share (its words are paged_attention.hip's own), and
// attention that reads it once per group.
size_t share_bytes(int n_seqs, int total_rows);
hipError_t launch_share(const CacheArgs& c, const int32_t* row_start, int total_rows, int max_rows, const int32_t* group,
                        int max_group_rows, int32_t* share, hipStream_t st);
// Whether a call could share at all: windows of more packed rows fill their workgroups' tiles
// by themselves.
bool attend_may_share(int max_rows, int max_group_rows, int group);
size_t attend_shared_workspace_bytes(int n_seqs, int n_kv, int head_dim, int total_rows, int max_rows, int max_group_rows,
                                     int group);
hipError_t launch_attend_shared(const CacheArgs& c, int dtype, int layer, const int32_t* row_start, int total_rows,
                                int max_rows, int max_group_rows, int max_keys, const int32_t* share, int n_heads,
                                const void* q, int64_t q_stride, const uint32_t* mask, int mask_words, float scale, void* o,
                                int64_t o_stride, float* lse, void* ws, hipStream_t st);
