// Attention of the nodes of wide draft trees on the bf16 matrix cores: the kernel of a chunk's attention (attn_chunk.hip), in which a row sees the context and the nodes that its
// mask names.  Steps that lie in the context are those of a chunk; in the others the lanes select by 32 bits of their rows' masks.
//
// A tile's rows read the same keys, so what bounds it depends on how many of its 256 rows there are (a step of 32 keys and values, per compute unit, all of them busy; bf16, 128-wide
// heads): 256 rows 1.06 us, the issue of matrix and vector instructions by one wavefront to a SIMD (1.02 PFLOP/s, 4.0 TB/s); 128 rows or less, one block of 32 to a wavefront, 0.755 us,
// bound by how far ahead the loads of two tiles in LDS reach (5.5 TB/s; 5.9 with 16 nodes; two blocks to a wavefront all the same 0.87). e4m3 1.27 and 0.97 us, 64-wide heads 0.6.
// Cuts weigh steps accordingly (kNarrowStep). What a call costs beside its steps is about 25 us: openings of tiles, partial results (50 MB where 16 trees of 64 nodes are cut for 256
// workgroups) and their merge. 16 trees of 33 .. 64 nodes behind 512 .. 8192 tokens 97 to 106 us by card (bytes alone 55), 16 of 32 nodes 82, eight over an e4m3 cache with eight query
// heads to one, behind 4096 .. 16384, 174 (1.36 PFLOP/s would be 69).
// Not kept: one block of rows to a wavefront and two wavefronts to a SIMD (140 to 340 bytes spilled; 99 us for 16 trees of 32 nodes), workgroups of two wavefronts, two to a compute
// unit (5.9 TB/s in the steps, 88 us for the call, and the chunk's e4m3 form spills).
#include "attn_chunk_kernel.h"

namespace ss {

int32_t tree_mfma_launch(const ChunkArgs &a, hipStream_t stream) { return launch_all<true>(a, stream); }

}  // namespace ss
