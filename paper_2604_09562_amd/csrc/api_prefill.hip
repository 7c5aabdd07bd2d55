// C-ABI entry points of the calls that fill the paged cache: argument validation, workspace sizing, dispatch.  No arithmetic here.
#include "chunk_plan.h"

namespace ss {

namespace {

constexpr int32_t kMaxSlots = 0x7fffffff;   // slots are 32-bit

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int32_t check_cache(const ss_paged_kv *kv)
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

int32_t check_cache_pointers(const ss_paged_kv *kv)
{
    if (!kv->k || !kv->v) return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if (!aligned16(kv->k) || !aligned16(kv->v)) return fail(SS_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    if ((kv->dtype == SS_FP8_E4M3) != (kv->k_scale != nullptr) || (kv->k_scale == nullptr) != (kv->v_scale == nullptr))
        return fail(SS_ERR_INVALID_ARG, "k_scale/v_scale must both be given for fp8 caches and be NULL otherwise");
    return SS_OK;
}

// Rows of `width` elements, `stride` elements apart, that are read 16 bytes at a time.
int32_t check_rows(const char *name, const void *p, int64_t stride, int64_t width, int dtype)
{
    if (!p) return fail(SS_ERR_INVALID_ARG, "%s is NULL", name);
    if (stride < width) return fail(SS_ERR_INVALID_ARG, "%s: rows of %lld elements are %lld apart", name, (long long)width, (long long)stride);
    if (!aligned16(p) || stride * (dtype == SS_F32 ? 4 : 2) % 16)
        return fail(SS_ERR_INVALID_ARG, "%s: rows must start 16-byte aligned (base and stride)", name);
    return SS_OK;
}

int32_t check_chunk(const ss_paged_kv *kv, const ss_batch *b, int32_t q_dtype, int32_t num_q_heads, int32_t total_rows)
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

}  // namespace

ChunkShape chunk_shape(bool mfma, int batch, int max_blocks, int num_q_heads, int num_kv_heads, int total_rows)
{
    ChunkShape s;
    const int64_t G = num_q_heads / num_kv_heads;
    s.rows = mfma ? kChunkRows : kChunkRowsF32;
    // workgroups that run at a time: of the matrix-core kernel one to a compute unit, of the fp32 kernel two
    const int64_t wgs = attn_chip_waves() / (mfma ? 4 : 2), tiles = (int64_t)total_rows * G / s.rows + (batch < total_rows ? batch : total_rows);
    // as many spans as workgroups run at a time, if there can be work enough
    const int64_t keys = mfma ? kChunkKeys : kChunkKeysF32, steps = ((int64_t)max_blocks * SS_BLOCK_SIZE + keys - 1) / keys;
    const int64_t most = tiles * ((steps + kMinPiece - 1) / kMinPiece), each = wgs > num_kv_heads ? wgs / num_kv_heads : 1;
    s.spans = (int32_t)(most < each ? (most < 1 ? 1 : most) : each);
    s.cap = s.spans > 1 ? 2 * s.spans * num_kv_heads : 0;
    return s;
}

size_t chunk_workspace_bytes(const ChunkShape &s, int head_dim)
{
    return align_up(sizeof(int32_t) * kChunkRecInts * (size_t)s.spans, 256) + align_up((size_t)s.cap * s.rows * 2 * sizeof(float), 256) +
           (size_t)s.cap * s.rows * head_dim * sizeof(float);
}

void chunk_carve(ChunkArgs &a, const ChunkShape &s, void *workspace)
{
    char *w = static_cast<char *>(workspace);
    a.spans = s.spans;
    a.cap = s.cap;
    a.rec = reinterpret_cast<int32_t *>(w);
    w += align_up(sizeof(int32_t) * kChunkRecInts * (size_t)s.spans, 256);
    a.part_ml = reinterpret_cast<float *>(w);
    w += align_up((size_t)s.cap * s.rows * 2 * sizeof(float), 256);
    a.part_o = reinterpret_cast<float *>(w);
}

}  // namespace ss

using namespace ss;

extern "C" {

size_t ss_block_map_workspace(int32_t batch)
{
    if (batch < 0) {
        fail(SS_ERR_INVALID_ARG, "negative batch");
        return 0;
    }
    return align_up(block_map_scratch_ints(batch) * sizeof(int32_t), 256);
}

int32_t ss_block_map(const ss_batch *batch, const ss_block_pool *pool, int32_t *held, int32_t total_rows, int32_t *slot_map, int32_t *positions,
                     int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!batch || !pool) return fail(SS_ERR_INVALID_ARG, "batch and pool descriptors must not be NULL");
    if (batch->batch < 0 || total_rows < 0) return fail(SS_ERR_INVALID_ARG, "negative batch or total_rows");
    if (batch->batch > 0 && batch->max_blocks_per_seq <= 0) return fail(SS_ERR_INVALID_ARG, "max_blocks_per_seq must be positive");
    if (pool->num_blocks < 0) return fail(SS_ERR_INVALID_ARG, "negative num_blocks");
    if ((int64_t)batch->batch * batch->max_blocks_per_seq > 0x7fffffffll || (int64_t)pool->num_blocks * SS_BLOCK_SIZE > kMaxSlots ||
        (int64_t)batch->max_blocks_per_seq * SS_BLOCK_SIZE > kMaxSlots)
        return fail(SS_ERR_UNSUPPORTED, "batch * max_blocks, max_blocks * %d and num_blocks * %d must fit 31 bits", SS_BLOCK_SIZE, SS_BLOCK_SIZE);
    if (!status || !pool->free_count || (pool->num_blocks > 0 && !pool->free_ids) || (total_rows > 0 && !slot_map) ||
        (batch->batch > 0 && (!batch->block_table || !batch->kv_len || !batch->q_indptr || !held)))
        return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    const size_t need = ss_block_map_workspace(batch->batch);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(SS_ERR_INVALID_ARG, "workspace must be a 256-byte aligned device buffer");
    if (workspace_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    BlockMapArgs a{};
    a.batch = batch->batch; a.max_blocks = batch->max_blocks_per_seq; a.num_blocks = pool->num_blocks; a.total_rows = total_rows;
    a.block_table = const_cast<int32_t *>(batch->block_table); a.kv_len = batch->kv_len; a.q_indptr = batch->q_indptr;
    a.free_ids = pool->free_ids; a.free_count = pool->free_count; a.held = held;
    a.slot_map = slot_map; a.positions = positions; a.status = status; a.scratch = static_cast<int32_t *>(workspace);
    return block_map_launch(a, static_cast<hipStream_t>(stream));
}

int32_t ss_kv_write(const ss_paged_kv *kv, const int32_t *slot_map, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                    int32_t new_dtype, int32_t total_rows, void *stream)
{
    int32_t rc = check_cache(kv);
    if (rc != SS_OK) return rc;
    if (total_rows < 0) return fail(SS_ERR_INVALID_ARG, "negative total_rows");
    if (new_dtype != SS_F32 && new_dtype != SS_BF16) return fail(SS_ERR_INVALID_ARG, "new_dtype must be SS_F32 or SS_BF16");
    if (total_rows == 0 || kv->num_blocks == 0) return SS_OK;
    if ((rc = check_cache_pointers(kv)) != SS_OK) return rc;
    if (!slot_map) return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    const int64_t width = (int64_t)kv->num_kv_heads * kv->head_dim;
    if ((rc = check_rows("k_new", k_new, k_stride, width, new_dtype)) != SS_OK) return rc;
    if ((rc = check_rows("v_new", v_new, v_stride, width, new_dtype)) != SS_OK) return rc;
    if ((int64_t)total_rows * width > 0x7fffffffll * 8) return fail(SS_ERR_UNSUPPORTED, "total_rows * kv heads * head_dim too large for one launch");
    if (option_validate()) {
        rc = validate_slots(slot_map, total_rows, (int64_t)kv->num_blocks * SS_BLOCK_SIZE, kv->dtype == SS_FP8_E4M3, static_cast<hipStream_t>(stream),
                            "ss_kv_write");
        if (rc != SS_OK) return rc;
    }
    KvWriteArgs a{};
    a.k = const_cast<void *>(kv->k); a.v = const_cast<void *>(kv->v);
    a.k_scale = const_cast<float *>(kv->k_scale); a.v_scale = const_cast<float *>(kv->v_scale);
    a.num_kv_heads = kv->num_kv_heads; a.head_dim = kv->head_dim; a.kv_dtype = kv->dtype; a.num_blocks = kv->num_blocks;
    a.slot_map = slot_map; a.k_new = k_new; a.v_new = v_new; a.k_stride = k_stride; a.v_stride = v_stride;
    a.new_dtype = new_dtype; a.total_rows = total_rows;
    return kv_write_launch(a, static_cast<hipStream_t>(stream));
}

size_t ss_chunk_attn_workspace(const ss_paged_kv *kv, const ss_batch *batch, int32_t q_dtype, int32_t num_q_heads, int32_t total_rows)
{
    if (check_chunk(kv, batch, q_dtype, num_q_heads, total_rows) != SS_OK) return 0;
    const bool mfma = chunk_mfma_supported(kv->head_dim, kv->dtype, q_dtype);
    return chunk_workspace_bytes(chunk_shape(mfma, batch->batch, batch->max_blocks_per_seq, num_q_heads, kv->num_kv_heads, total_rows), kv->head_dim);
}

int32_t ss_chunk_attn(const ss_paged_kv *kv, const ss_batch *batch, const void *q, int64_t q_stride, int32_t q_dtype, int32_t num_q_heads,
                      int32_t total_rows, float sm_scale, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_chunk(kv, batch, q_dtype, num_q_heads, total_rows);
    if (rc != SS_OK) return rc;
    if (batch->batch == 0 || total_rows == 0) return SS_OK;
    if ((rc = check_cache_pointers(kv)) != SS_OK) return rc;
    if (!batch->block_table || !batch->kv_len || !batch->q_indptr || !out) return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if ((rc = check_rows("q", q, q_stride, (int64_t)num_q_heads * kv->head_dim, q_dtype)) != SS_OK) return rc;
    if (!aligned16(out)) return fail(SS_ERR_INVALID_ARG, "out must be 16-byte aligned");
    if (!(sm_scale > 0.0f) || sm_scale > 2.0e38f)   // (times log2(e) it has to be a float, too)
        return fail(SS_ERR_INVALID_ARG, "sm_scale must be positive and at most 2e38");
    const bool mfma = chunk_mfma_supported(kv->head_dim, kv->dtype, q_dtype);
    const ChunkShape s = chunk_shape(mfma, batch->batch, batch->max_blocks_per_seq, num_q_heads, kv->num_kv_heads, total_rows);
    const size_t need = chunk_workspace_bytes(s, kv->head_dim);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(SS_ERR_INVALID_ARG, "workspace must be a 256-byte aligned device buffer");
    if (workspace_bytes < need) return fail(SS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    if (option_validate()) {
        rc = validate_chunk(batch->block_table, batch->kv_len, batch->q_indptr, batch->batch, batch->max_blocks_per_seq, kv->num_blocks, total_rows,
                            batch->max_q_len ? batch->max_q_len : total_rows, static_cast<hipStream_t>(stream), "ss_chunk_attn");
        if (rc != SS_OK) return rc;
    }
    ChunkArgs a{};
    a.k = kv->k; a.v = kv->v; a.k_scale = kv->k_scale; a.v_scale = kv->v_scale;
    a.num_kv_heads = kv->num_kv_heads; a.head_dim = kv->head_dim; a.kv_dtype = kv->dtype;
    a.batch = batch->batch; a.max_blocks = batch->max_blocks_per_seq; a.num_blocks = kv->num_blocks; a.total_rows = total_rows;
    a.block_table = batch->block_table; a.kv_len = batch->kv_len; a.q_indptr = batch->q_indptr;
    a.q = q; a.q_stride = q_stride; a.out = out; a.lse = lse; a.q_dtype = q_dtype; a.num_q_heads = num_q_heads; a.sm_scale = sm_scale;
    chunk_carve(a, s, workspace);
    return mfma ? chunk_mfma_launch(a, static_cast<hipStream_t>(stream)) : chunk_f32_launch(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
