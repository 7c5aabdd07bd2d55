// Internal declarations of the calls for blocks that several requests hold (not part of the C ABI).
#pragma once

#include "prefill.h"

namespace ss {

struct BlockForkArgs {
    int32_t batch, max_blocks, num_blocks, num_forks;
    int32_t *block_table, *kv_len, *held, *shares;
    const int32_t *free_ids;
    int32_t *free_count;
    const int32_t *parent, *child, *length;   // length may be nullptr: all of the parent
    int32_t *copy_src, *copy_dst, *status;
    int32_t *scratch;                         // block_fork_scratch_ints()
};
size_t block_fork_scratch_ints(int batch, int num_forks);
int32_t block_fork_launch(const BlockForkArgs &a, hipStream_t stream);

constexpr int64_t kMaxReleased = 1 << 30;     // entries of a table that block_release can count
struct BlockReleaseArgs {
    int32_t batch, max_blocks, num_blocks;
    const int32_t *block_table, *kv_len;
    int32_t *held, *shares, *free_ids, *free_count, *status;
    int32_t *scratch;                         // block_release_scratch_ints()
};
size_t block_release_scratch_ints(int batch, int max_blocks, int num_blocks);
int32_t block_release_launch(const BlockReleaseArgs &a, hipStream_t stream);

struct BlockCompactArgs {
    int32_t batch, max_blocks, num_blocks;
    int32_t *block_table, *shares;            // shares may be nullptr
    const int32_t *held;
    int32_t *free_ids;
    const int32_t *free_count;
    int32_t *remap;                           // may be nullptr
    int32_t *copy_src, *copy_dst, *num_copies, *status;
    int32_t *scratch;                         // block_compact_scratch_ints()
};
size_t block_compact_scratch_ints(int num_blocks);
int32_t block_compact_launch(const BlockCompactArgs &a, hipStream_t stream);

constexpr int kCopyLayers = 64;               // layers whose addresses go with one launch
struct BlockCopyArgs {
    struct Layer {
        char *side[2];                        // keys, values
        float *scale[2];                      // nullptr unless e4m3
    } layer[kCopyLayers];
    int32_t layers, num_blocks, max_copies;
    int32_t heads;                            // scales of a block
    int64_t block_bytes;                      // of keys, and of values
    const int32_t *src, *dst, *num_copies;    // num_copies may be nullptr
};
int32_t block_copy_launch(const BlockCopyArgs &a, hipStream_t stream);

}  // namespace ss
