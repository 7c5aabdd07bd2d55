// C-ABI entry points of wide draft trees and of blocks that several requests hold: argument validation, workspace sizing, dispatch.  No arithmetic here.
#include "api_checks.h"
#include "block_share.h"
#include "tree_verify.h"

namespace ss {

namespace {

int32_t check_workspace(const void *workspace, size_t bytes, size_t need)
{
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return fail(SS_ERR_INVALID_ARG, "workspace must be a 256-byte aligned device buffer");
    if (bytes < need) return fail(SS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", bytes, need);
    return SS_OK;
}

int32_t check_tree_attn(const ss_paged_kv *kv, const ss_batch *b, int32_t q_dtype, int32_t num_q_heads, int32_t total_rows)
{
    if (b && b->tree_mask) return fail(SS_ERR_INVALID_ARG, "ss_batch.tree_mask must be NULL (ss_tree_attn takes masks of any width as an argument)");
    return check_chunk(kv, b, q_dtype, num_q_heads, total_rows);
}

int32_t check_books(const ss_batch *b, const ss_block_pool *pool)
{
    if (!b || !pool) return fail(SS_ERR_INVALID_ARG, "batch and pool descriptors must not be NULL");
    if (b->batch < 0) return fail(SS_ERR_INVALID_ARG, "negative batch");
    if (b->batch > 0 && b->max_blocks_per_seq <= 0) return fail(SS_ERR_INVALID_ARG, "max_blocks_per_seq must be positive");
    if (pool->num_blocks < 0) return fail(SS_ERR_INVALID_ARG, "negative num_blocks");
    if ((int64_t)b->batch * b->max_blocks_per_seq > kMaxReleased || (int64_t)pool->num_blocks * SS_BLOCK_SIZE > kMaxSlots ||
        (int64_t)b->max_blocks_per_seq * SS_BLOCK_SIZE > kMaxSlots)
        return fail(SS_ERR_UNSUPPORTED, "batch * max_blocks must not pass 2^30, max_blocks * %d and num_blocks * %d must fit 31 bits", SS_BLOCK_SIZE, SS_BLOCK_SIZE);
    return SS_OK;
}

// Partial results of the kernel of short calls: (reference, sum) of their rows, then their outputs.
size_t unit_slots(const TreeUnitChoice &u, int batch, int heads) { return u.splits > 1 ? (size_t)batch * u.tiles * u.splits * heads : 0; }
size_t unit_part_o(const TreeUnitChoice &u, int batch, int heads) { return align_up(unit_slots(u, batch, heads) * kTreeUnitRows * 2 * sizeof(float), 256); }

// Which kernel takes a call.
struct TreeForm {
    bool mfma;
    TreeUnitChoice unit;
    ChunkShape shape;
    size_t workspace;
};
TreeForm tree_form(const ss_paged_kv *kv, const ss_batch *b, int32_t q_dtype, int32_t num_q_heads, int32_t total_rows)
{
    TreeForm f;
    f.mfma = chunk_mfma_supported(kv->head_dim, kv->dtype, q_dtype);
    const int64_t nodes = b->max_q_len > 0 && b->max_q_len < total_rows ? b->max_q_len : b->max_q_len > 0 || b->batch == 1 ? total_rows : 0;   // of the widest tree
    const int64_t rows = nodes * (num_q_heads / kv->num_kv_heads), keys = (int64_t)b->max_blocks_per_seq * SS_BLOCK_SIZE;
    const int cus = attn_chip_waves() / 4;
    f.unit = f.mfma ? tree_unit_rule(b->batch, kv->num_kv_heads, rows, keys, kv->head_dim, kv->dtype == SS_FP8_E4M3, cus)
                    : TreeUnitChoice{tree_unit_f32_rule(b->batch, kv->num_kv_heads, rows, keys, kv->head_dim, cus), 1};
    f.shape = chunk_shape(f.mfma, b->batch, b->max_blocks_per_seq, num_q_heads, kv->num_kv_heads, total_rows);
    f.workspace = f.unit.tiles ? unit_part_o(f.unit, b->batch, kv->num_kv_heads) + unit_slots(f.unit, b->batch, kv->num_kv_heads) * kTreeUnitRows * kv->head_dim * sizeof(float) + 256
                               : chunk_workspace_bytes(f.shape, kv->head_dim);
    return f;
}

bool pool_pointers(const ss_block_pool *pool) { return pool->free_count && (pool->num_blocks == 0 || pool->free_ids); }

constexpr int32_t kMaxForks = 1 << 20;

}  // namespace

}  // namespace ss

using namespace ss;

extern "C" {

size_t ss_tree_attn_workspace(const ss_paged_kv *kv, const ss_batch *batch, int32_t q_dtype, int32_t num_q_heads, int32_t total_rows)
{
    if (check_tree_attn(kv, batch, q_dtype, num_q_heads, total_rows) != SS_OK) return 0;
    return tree_form(kv, batch, q_dtype, num_q_heads, total_rows).workspace;
}

int32_t ss_tree_attn(const ss_paged_kv *kv, const ss_batch *batch, const uint32_t *node_mask, int32_t mask_words, const void *q, int64_t q_stride,
                     int32_t q_dtype, int32_t num_q_heads, int32_t total_rows, float sm_scale, void *out, float *lse, void *workspace,
                     size_t workspace_bytes, void *stream)
{
    int32_t rc = check_tree_attn(kv, batch, q_dtype, num_q_heads, total_rows);
    if (rc != SS_OK) return rc;
    if (mask_words <= 0 || mask_words > kMaxSlots / 32) return fail(SS_ERR_INVALID_ARG, "mask_words must be positive (and 32 of them fit 31 bits), got %d", mask_words);
    if (batch->batch == 0 || total_rows == 0) return SS_OK;
    if ((rc = check_cache_pointers(kv)) != SS_OK) return rc;
    if (!batch->block_table || !batch->kv_len || !batch->q_indptr || !node_mask || !out) return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if ((rc = check_rows("q", q, q_stride, (int64_t)num_q_heads * kv->head_dim, q_dtype)) != SS_OK) return rc;
    if (!aligned16(out)) return fail(SS_ERR_INVALID_ARG, "out must be 16-byte aligned");
    if (!(sm_scale > 0.0f) || sm_scale > 2.0e38f)   // (times log2(e) it has to be a float, too)
        return fail(SS_ERR_INVALID_ARG, "sm_scale must be positive and at most 2e38");
    const TreeForm f = tree_form(kv, batch, q_dtype, num_q_heads, total_rows);
    if ((rc = check_workspace(workspace, workspace_bytes, f.workspace)) != SS_OK) return rc;
    if (option_validate()) {
        rc = validate_chunk(batch->block_table, batch->kv_len, batch->q_indptr, batch->batch, batch->max_blocks_per_seq, kv->num_blocks, total_rows,
                            batch->max_q_len ? batch->max_q_len : total_rows, false, static_cast<hipStream_t>(stream), "ss_tree_attn");
        if (rc != SS_OK) return rc;
    }
    ChunkArgs a{};
    a.k = kv->k; a.v = kv->v; a.k_scale = kv->k_scale; a.v_scale = kv->v_scale;
    a.num_kv_heads = kv->num_kv_heads; a.head_dim = kv->head_dim; a.kv_dtype = kv->dtype;
    a.batch = batch->batch; a.max_blocks = batch->max_blocks_per_seq; a.num_blocks = kv->num_blocks; a.total_rows = total_rows;
    a.block_table = batch->block_table; a.kv_len = batch->kv_len; a.q_indptr = batch->q_indptr;
    a.q = q; a.q_stride = q_stride; a.out = out; a.lse = lse; a.q_dtype = q_dtype; a.num_q_heads = num_q_heads; a.sm_scale = sm_scale;
    a.node_mask = node_mask; a.mask_words = mask_words;
    if (f.unit.tiles) {
        a.part_ml = static_cast<float *>(workspace);
        a.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace) + unit_part_o(f.unit, batch->batch, kv->num_kv_heads));
        return f.mfma ? tree_unit_launch(a, f.unit, static_cast<hipStream_t>(stream)) : tree_unit_f32_launch(a, f.unit.tiles, static_cast<hipStream_t>(stream));
    }
    chunk_carve(a, f.shape, workspace);
    return f.mfma ? tree_mfma_launch(a, static_cast<hipStream_t>(stream)) : tree_f32_launch(a, static_cast<hipStream_t>(stream));
}

size_t ss_tree_verify_workspace(int32_t batch, int32_t total_rows, int32_t vocab)
{
    if (batch < 0 || total_rows < 0 || vocab <= 0 || vocab > 1 << 30) {
        fail(SS_ERR_INVALID_ARG, "bad batch/total_rows/vocab (%d, %d, %d)", batch, total_rows, vocab);
        return 0;
    }
    return tree_verify_workspace_bytes(batch, total_rows, vocab);
}

int32_t ss_tree_verify(int32_t batch, int32_t vocab, int64_t row_stride, int32_t logit_dtype, int32_t total_rows, int32_t max_depth, const int32_t *q_indptr,
                       const int32_t *tree_parent, const int32_t *node_tokens, const void *target_logits, const float *uniforms, const float *temperature,
                       float temperature_scalar, int32_t *accepted_len, int32_t *out_tokens, int32_t *accepted_nodes, float *logprobs, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    if (batch < 0 || total_rows < 0 || vocab <= 0 || vocab > 1 << 30) return fail(SS_ERR_INVALID_ARG, "bad batch/total_rows/vocab (%d, %d, %d)", batch, total_rows, vocab);
    if (max_depth < 0 || max_depth > SS_MAX_DEPTH) return fail(SS_ERR_INVALID_ARG, "max_depth must be 0 (%d is meant) or in [1, %d]", SS_MAX_DEPTH, SS_MAX_DEPTH);
    if (row_stride < vocab) return fail(SS_ERR_INVALID_ARG, "row_stride (%lld) < vocab (%d)", (long long)row_stride, vocab);
    if (logit_dtype != SS_F32 && logit_dtype != SS_BF16) return fail(SS_ERR_INVALID_ARG, "logit_dtype must be SS_F32 or SS_BF16");
    if (!temperature && !(temperature_scalar >= 0.0f)) return fail(SS_ERR_INVALID_ARG, "temperature_scalar must not be negative");
    if (batch == 0) return SS_OK;
    if (!q_indptr || !accepted_len || !out_tokens || !accepted_nodes || (total_rows > 0 && (!tree_parent || !node_tokens || !target_logits)))
        return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if (total_rows > 0 && !uniforms && (temperature || temperature_scalar > 0.0f))
        return fail(SS_ERR_INVALID_ARG, "uniforms are required unless the temperature of all requests is 0");
    if (!aligned16(target_logits) || row_stride * (logit_dtype == SS_F32 ? 4 : 2) % 16)
        return fail(SS_ERR_INVALID_ARG, "logits rows must start 16-byte aligned (base and row_stride)");
    if (batch >= 1 << 24) return fail(SS_ERR_UNSUPPORTED, "batch too large for one launch");
    const int32_t rc = check_workspace(workspace, workspace_bytes, tree_verify_least_bytes(batch, vocab));
    if (rc != SS_OK) return rc;
    TreeVerifyArgs a{};
    a.batch = batch; a.vocab = vocab; a.logit_dtype = logit_dtype; a.total_rows = total_rows; a.max_depth = max_depth ? max_depth : SS_MAX_DEPTH;
    a.row_stride = row_stride; a.q_indptr = q_indptr; a.parent = tree_parent; a.tokens = node_tokens; a.target = target_logits;
    a.uniforms = uniforms; a.temperature = temperature; a.temperature_scalar = temperature_scalar;
    a.accepted_len = accepted_len; a.out_tokens = out_tokens; a.accepted_nodes = accepted_nodes; a.logprobs = logprobs;
    a.workspace = workspace; a.workspace_bytes = workspace_bytes;
    return tree_verify_launch(a, static_cast<hipStream_t>(stream));
}

size_t ss_block_fork_workspace(int32_t batch, int32_t num_forks)
{
    if (batch < 0 || num_forks < 0) {
        fail(SS_ERR_INVALID_ARG, "negative batch or num_forks");
        return 0;
    }
    return align_up((block_fork_scratch_ints(batch, num_forks) + 1) * sizeof(int32_t), 256);
}

int32_t ss_block_fork(const ss_batch *batch, const ss_block_pool *pool, int32_t *shares, int32_t *held, int32_t num_forks, const int32_t *parent,
                      const int32_t *child, const int32_t *length, int32_t *copy_src, int32_t *copy_dst, int32_t *status, void *workspace,
                      size_t workspace_bytes, void *stream)
{
    int32_t rc = check_books(batch, pool);
    if (rc != SS_OK) return rc;
    if (num_forks < 0) return fail(SS_ERR_INVALID_ARG, "negative num_forks");
    if (num_forks > kMaxForks || (int64_t)num_forks * batch->max_blocks_per_seq > kMaxSlots)
        return fail(SS_ERR_UNSUPPORTED, "num_forks must not pass %d, num_forks * max_blocks must fit 31 bits", kMaxForks);
    if (!status || !pool_pointers(pool) || (pool->num_blocks > 0 && !shares) || (num_forks > 0 && (!parent || !child || !copy_src || !copy_dst)) ||
        (batch->batch > 0 && (!batch->block_table || !batch->kv_len || !held)))
        return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if ((rc = check_workspace(workspace, workspace_bytes, ss_block_fork_workspace(batch->batch, num_forks))) != SS_OK) return rc;
    BlockForkArgs a{};
    a.batch = batch->batch; a.max_blocks = batch->max_blocks_per_seq; a.num_blocks = pool->num_blocks; a.num_forks = num_forks;
    a.block_table = const_cast<int32_t *>(batch->block_table); a.kv_len = const_cast<int32_t *>(batch->kv_len); a.held = held; a.shares = shares;
    a.free_ids = pool->free_ids; a.free_count = pool->free_count; a.parent = parent; a.child = child; a.length = length;
    a.copy_src = copy_src; a.copy_dst = copy_dst; a.status = status; a.scratch = static_cast<int32_t *>(workspace);
    return block_fork_launch(a, static_cast<hipStream_t>(stream));
}

size_t ss_block_release_workspace(int32_t batch, int32_t max_blocks_per_seq, int32_t num_blocks)
{
    if (batch < 0 || max_blocks_per_seq < 0 || num_blocks < 0) {
        fail(SS_ERR_INVALID_ARG, "negative batch, max_blocks_per_seq or num_blocks");
        return 0;
    }
    return align_up(block_release_scratch_ints(batch, max_blocks_per_seq, num_blocks) * sizeof(int32_t), 256);
}

int32_t ss_block_release(const ss_batch *batch, const ss_block_pool *pool, int32_t *shares, int32_t *held, int32_t *status, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    int32_t rc = check_books(batch, pool);
    if (rc != SS_OK) return rc;
    if (!status || !pool_pointers(pool) || (pool->num_blocks > 0 && !shares) || (batch->batch > 0 && (!batch->block_table || !batch->kv_len || !held)))
        return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if ((rc = check_workspace(workspace, workspace_bytes, ss_block_release_workspace(batch->batch, batch->max_blocks_per_seq, pool->num_blocks))) != SS_OK) return rc;
    BlockReleaseArgs a{};
    a.batch = batch->batch; a.max_blocks = batch->max_blocks_per_seq; a.num_blocks = pool->num_blocks;
    a.block_table = batch->block_table; a.kv_len = batch->kv_len; a.held = held; a.shares = shares;
    a.free_ids = pool->free_ids; a.free_count = pool->free_count; a.status = status; a.scratch = static_cast<int32_t *>(workspace);
    return block_release_launch(a, static_cast<hipStream_t>(stream));
}

size_t ss_block_compact_workspace(int32_t num_blocks)
{
    if (num_blocks < 0) {
        fail(SS_ERR_INVALID_ARG, "negative num_blocks");
        return 0;
    }
    return align_up(block_compact_scratch_ints(num_blocks) * sizeof(int32_t), 256);
}

int32_t ss_block_compact(const ss_batch *batch, const ss_block_pool *pool, int32_t *shares, const int32_t *held, int32_t *remap, int32_t *copy_src,
                         int32_t *copy_dst, int32_t *num_copies, int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    int32_t rc = check_books(batch, pool);
    if (rc != SS_OK) return rc;
    if (!status || !num_copies || !pool_pointers(pool) || (pool->num_blocks > 1 && (!copy_src || !copy_dst)) || (batch->batch > 0 && (!batch->block_table || !held)))
        return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    if ((rc = check_workspace(workspace, workspace_bytes, ss_block_compact_workspace(pool->num_blocks))) != SS_OK) return rc;
    BlockCompactArgs a{};
    a.batch = batch->batch; a.max_blocks = batch->max_blocks_per_seq; a.num_blocks = pool->num_blocks;
    a.block_table = const_cast<int32_t *>(batch->block_table); a.shares = shares; a.held = held; a.free_ids = pool->free_ids; a.free_count = pool->free_count;
    a.remap = remap; a.copy_src = copy_src; a.copy_dst = copy_dst; a.num_copies = num_copies; a.status = status; a.scratch = static_cast<int32_t *>(workspace);
    return block_compact_launch(a, static_cast<hipStream_t>(stream));
}

int32_t ss_block_copy(const ss_paged_kv *layers, int32_t num_layers, const int32_t *copy_src, const int32_t *copy_dst, int32_t max_copies,
                      const int32_t *num_copies, void *stream)
{
    if (num_layers < 0 || max_copies < 0) return fail(SS_ERR_INVALID_ARG, "negative num_layers or max_copies");
    if (num_layers == 0 || max_copies == 0) return SS_OK;
    if (!layers) return fail(SS_ERR_INVALID_ARG, "the cache descriptors must not be NULL");
    if (!copy_src || !copy_dst) return fail(SS_ERR_INVALID_ARG, "a required device pointer is NULL");
    for (int32_t i = 0; i < num_layers; ++i) {
        const int32_t rc = check_cache(layers + i);
        if (rc != SS_OK) return rc;
        if (layers[i].num_blocks != layers[0].num_blocks || layers[i].num_kv_heads != layers[0].num_kv_heads || layers[i].head_dim != layers[0].head_dim ||
            layers[i].dtype != layers[0].dtype)
            return fail(SS_ERR_INVALID_ARG, "layer %d differs from the first one in shape or type", i);
        if (layers[i].num_blocks > 0) {
            const int32_t rp = check_cache_pointers(layers + i);
            if (rp != SS_OK) return rp;
        }
    }
    if (layers[0].num_blocks == 0) return SS_OK;
    static const int64_t size[] = {4, 2, 1};
    for (int32_t lo = 0; lo < num_layers; lo += kCopyLayers) {
        BlockCopyArgs a{};
        a.layers = num_layers - lo < kCopyLayers ? num_layers - lo : kCopyLayers;
        for (int32_t i = 0; i < a.layers; ++i) {
            const ss_paged_kv &kv = layers[lo + i];
            a.layer[i] = {{static_cast<char *>(const_cast<void *>(kv.k)), static_cast<char *>(const_cast<void *>(kv.v))},
                          {const_cast<float *>(kv.k_scale), const_cast<float *>(kv.v_scale)}};
        }
        a.num_blocks = layers[0].num_blocks; a.max_copies = max_copies; a.heads = layers[0].num_kv_heads;
        a.block_bytes = (int64_t)layers[0].num_kv_heads * SS_BLOCK_SIZE * layers[0].head_dim * size[layers[0].dtype];
        a.src = copy_src; a.dst = copy_dst; a.num_copies = num_copies;
        const int32_t rc = block_copy_launch(a, static_cast<hipStream_t>(stream));
        if (rc != SS_OK) return rc;
    }
    return SS_OK;
}

}  // extern "C"
