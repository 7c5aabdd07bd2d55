// Internal declarations of the verification of wide draft trees (not part of the C ABI).
#pragma once

#include "common.h"

namespace ss {

struct TreeVerifyArgs {
    int32_t batch, vocab, logit_dtype, total_rows, max_depth;
    int64_t row_stride;
    const int32_t *q_indptr, *parent, *tokens;
    const void *target;
    const float *uniforms, *temperature;   // temperature may be nullptr
    float temperature_scalar;
    int32_t *accepted_len, *out_tokens, *accepted_nodes;
    float *logprobs;                       // may be nullptr
    void *workspace;
    size_t workspace_bytes;
};
size_t tree_verify_least_bytes(int batch, int vocab);
size_t tree_verify_workspace_bytes(int batch, int total_rows, int vocab);
int32_t tree_verify_launch(const TreeVerifyArgs &a, hipStream_t stream);

}  // namespace ss
