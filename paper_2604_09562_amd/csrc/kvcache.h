// Internal declarations of the cache's append, compaction and commit (not part of the C ABI).
#pragma once

#include "common.h"

namespace ss {

struct KvAppendArgs {
    void *k, *v;
    float *k_scale, *v_scale;
    int32_t num_kv_heads, head_dim, kv_dtype;
    int32_t batch, max_blocks;
    const int32_t *block_table, *kv_len, *q_indptr;
    const void *k_new, *v_new;
    int32_t new_dtype;
    int32_t max_q_len;   // bound of the new tokens per request (sizes the append grid)
    int32_t num_blocks;  // of the cache (compaction follows no id beyond)
};
int32_t kv_append_launch(const KvAppendArgs &a, hipStream_t stream);
int32_t kv_compact_launch(const KvAppendArgs &a, const int32_t *accepted_nodes, const int32_t *accepted_len,
                          hipStream_t stream);   // k_new/v_new/new_dtype of the arguments are not used
int32_t kv_commit_launch(int batch, const int32_t *q_indptr, const int32_t *accepted_len, int32_t *kv_len,
                         hipStream_t stream);

}  // namespace ss
