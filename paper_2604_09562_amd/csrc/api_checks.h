// Checks of host-visible arguments that the calls on the paged cache share (not part of the C ABI).
#pragma once

#include "prefill.h"

namespace ss {

constexpr int32_t kMaxSlots = 0x7fffffff;   // slots are 32-bit

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int32_t check_cache(const ss_paged_kv *kv)
{
    if (!kv) return fail(SS_ERR_INVALID_ARG, "the cache descriptor must not be NULL");
    if (kv->block_size != SS_BLOCK_SIZE) return fail(SS_ERR_INVALID_ARG, "block_size must be %d, got %d", SS_BLOCK_SIZE, kv->block_size);
    if (kv->head_dim != 64 && kv->head_dim != 128) return fail(SS_ERR_INVALID_ARG, "head_dim must be 64 or 128, got %d", kv->head_dim);
    if (kv->num_kv_heads <= 0 || kv->num_blocks < 0) return fail(SS_ERR_INVALID_ARG, "bad num_kv_heads or num_blocks");
    if (kv->dtype < SS_F32 || kv->dtype > SS_FP8_E4M3) return fail(SS_ERR_INVALID_ARG, "unknown KV dtype %d", kv->dtype);
    if ((int64_t)kv->num_blocks * kv->num_kv_heads > 0x7fffffffll || (int64_t)kv->num_blocks * SS_BLOCK_SIZE > kMaxSlots)
        return fail(SS_ERR_UNSUPPORTED, "num_blocks * num_kv_heads and num_blocks * %d must fit 31 bits", SS_BLOCK_SIZE);
    return SS_OK;
}

inline int32_t check_cache_pointers(const ss_paged_kv *kv)
{
    if (!kv->k || !kv->v) return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if (!aligned16(kv->k) || !aligned16(kv->v)) return fail(SS_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    if ((kv->dtype == SS_FP8_E4M3) != (kv->k_scale != nullptr) || (kv->k_scale == nullptr) != (kv->v_scale == nullptr))
        return fail(SS_ERR_INVALID_ARG, "k_scale/v_scale must both be given for fp8 caches and be NULL otherwise");
    return SS_OK;
}

// Rows of `width` elements, `stride` elements apart, that are read 16 bytes at a time.
inline int32_t check_rows(const char *name, const void *p, int64_t stride, int64_t width, int dtype)
{
    if (!p) return fail(SS_ERR_INVALID_ARG, "%s is NULL", name);
    if (stride < width) return fail(SS_ERR_INVALID_ARG, "%s: rows of %lld elements are %lld apart", name, (long long)width, (long long)stride);
    if (!aligned16(p) || stride * (dtype == SS_F32 ? 4 : 2) % 16)
        return fail(SS_ERR_INVALID_ARG, "%s: rows must start 16-byte aligned (base and stride)", name);
    return SS_OK;
}

inline int32_t check_chunk(const ss_paged_kv *kv, const ss_batch *b, int32_t q_dtype, int32_t num_q_heads, int32_t total_rows)
{
    const int32_t rc = check_cache(kv);
    if (rc != SS_OK) return rc;
    if (!b) return fail(SS_ERR_INVALID_ARG, "the batch descriptor must not be NULL");
    if (q_dtype != SS_F32 && q_dtype != SS_BF16) return fail(SS_ERR_INVALID_ARG, "q_dtype must be SS_F32 or SS_BF16");
    if (num_q_heads <= 0 || num_q_heads % kv->num_kv_heads)
        return fail(SS_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)", num_q_heads, kv->num_kv_heads);
    if (num_q_heads / kv->num_kv_heads > 16) return fail(SS_ERR_UNSUPPORTED, "more than 16 query heads per KV head is not built");
    if (b->batch < 0 || total_rows < 0) return fail(SS_ERR_INVALID_ARG, "negative batch or total_rows");
    if (b->batch > 0 && b->max_blocks_per_seq <= 0) return fail(SS_ERR_INVALID_ARG, "max_blocks_per_seq must be positive");
    if (b->max_q_len < 0) return fail(SS_ERR_INVALID_ARG, "max_q_len must be 0 (unknown) or positive");
    if (b->flags & ~SS_BATCH_REUSE_PLAN) return fail(SS_ERR_INVALID_ARG, "unknown bits in ss_batch.flags (%d)", b->flags);
    if (b->tree_mask) return fail(SS_ERR_UNSUPPORTED, "draft trees are served by ss_spec_verify_attn only");
    if ((int64_t)b->batch * b->max_blocks_per_seq > 0x7fffffffll || (int64_t)b->max_blocks_per_seq * SS_BLOCK_SIZE > kMaxSlots ||
        (int64_t)total_rows * num_q_heads > 0x7fffffffll)
        return fail(SS_ERR_UNSUPPORTED, "batch * max_blocks, max_blocks * %d and total_rows * num_q_heads must fit 31 bits", SS_BLOCK_SIZE);
    return SS_OK;
}

}  // namespace ss
