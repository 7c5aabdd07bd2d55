// Internal declarations of the calls that fill the paged cache: block tables and slot maps, the write of a chunk's keys and values,
// and attention of a chunk of new tokens (not part of the C ABI).
#pragma once

#include "common.h"
#include "tree_rule.h"

namespace ss {

bool option_validate();   // option "validate"

// ---- block tables and slot maps ----------------------------------------------------------------
struct BlockMapArgs {
    int32_t batch, max_blocks, num_blocks, total_rows;
    int32_t *block_table;
    const int32_t *kv_len, *q_indptr;
    int32_t *free_ids, *free_count, *held;
    int32_t *slot_map, *positions, *status;   // positions may be nullptr
    int32_t *scratch;                         // block_map_scratch_ints(batch) ints
};
size_t block_map_scratch_ints(int batch);
int32_t block_map_launch(const BlockMapArgs &a, hipStream_t stream);

// ---- the write of keys and values by slot ------------------------------------------------------
struct KvWriteArgs {
    void *k, *v;
    float *k_scale, *v_scale;
    int32_t num_kv_heads, head_dim, kv_dtype, num_blocks;
    const int32_t *slot_map;
    const void *k_new, *v_new;
    int64_t k_stride, v_stride;   // elements from one row to the next
    int32_t new_dtype, total_rows;
};
int32_t kv_write_launch(const KvWriteArgs &a, hipStream_t stream);

// ---- attention of a chunk ----------------------------------------------------------------------
struct ChunkArgs {
    const void *k, *v;
    const float *k_scale, *v_scale;
    int32_t num_kv_heads, head_dim, kv_dtype;
    int32_t batch, max_blocks;
    int32_t num_blocks, total_rows;   // bounds of what the table and q_indptr say
    const int32_t *block_table, *kv_len, *q_indptr;
    const void *q;
    int64_t q_stride;             // elements from one row to the next
    void *out;
    float *lse;
    int32_t q_dtype, num_q_heads;
    float sm_scale;
    // how the work is cut (chunk_plan.h)
    int32_t spans;                // at most, for each KV head
    int32_t cap;                  // partial results the workspace has room for: two for each span and KV head, or none
    int32_t *rec;                 // [spans][kChunkRecInts] the tile that a span begins and does not end
    float *part_ml, *part_o;      // [cap] partial results
    // draft trees only
    const uint32_t *node_mask;    // [total_rows][mask_words] which nodes of its request a row attends
    int32_t mask_words;
};
// A block id of the table as it is followed: one that is no block's, as behind a block map that lacked blocks, as the last block's.
__device__ __forceinline__ int chunk_block(const ChunkArgs &a, int id)
{
    const uint32_t last = (uint32_t)a.num_blocks - 1u;   // (requests with keys have a cache)
    return (int)((uint32_t)id < last ? (uint32_t)id : last);
}
constexpr int kChunkRecInts = 4;
constexpr int kChunkKeys = 32, kChunkKeysF32 = 64;   // keys of a step
constexpr int kChunkRows = 256, kChunkRowsF32 = 64;   // query rows of a tile: bf16 matrix-core kernel, fp32 kernel
// What a tile costs beside its steps, in steps.  With 5 | 9 | 13, us: a prompt of 2048 74.5 | 63.2 | 65.1, 24 mixed requests 322 | 316 | 311, four over an e4m3 cache 321 | 309 | 309;
// fp32: 2, 3 and 6 are level (25.0).
constexpr int kChunkOpen = 9, kChunkOpenF32 = 3;

struct ChunkShape {               // host-visible sizes a launch and its workspace follow from
    int32_t rows;                 // query rows of a tile
    int32_t spans, cap;
};
bool chunk_mfma_supported(int head_dim, int kv_dtype, int q_dtype);
ChunkShape chunk_shape(bool mfma, int batch, int max_blocks, int num_q_heads, int num_kv_heads, int total_rows);
size_t chunk_workspace_bytes(const ChunkShape &s, int head_dim);
void chunk_carve(ChunkArgs &a, const ChunkShape &s, void *workspace);
int32_t chunk_mfma_launch(const ChunkArgs &a, hipStream_t stream);
int32_t chunk_f32_launch(const ChunkArgs &a, hipStream_t stream);
int32_t tree_f32_launch(const ChunkArgs &a, hipStream_t stream);
int32_t tree_mfma_launch(const ChunkArgs &a, hipStream_t stream);
int32_t tree_unit_f32_launch(const ChunkArgs &a, int tiles, hipStream_t stream);
int32_t tree_unit_launch(const ChunkArgs &a, const TreeUnitChoice &how, hipStream_t stream);

// ---- optional checks of device-resident metadata -----------------------------------------------
int32_t validate_chunk(const int32_t *block_table, const int32_t *kv_len, const int32_t *q_indptr, int batch, int max_blocks,
                       int num_blocks, int total_rows, int max_q_len, bool cached, hipStream_t stream, const char *what);
int32_t validate_slots(const int32_t *slot_map, int total_rows, int64_t slots, bool runs, hipStream_t stream, const char *what);

}  // namespace ss
