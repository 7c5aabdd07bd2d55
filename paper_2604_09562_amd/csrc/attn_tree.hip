// Attention of the nodes of wide draft trees on the bf16 matrix cores: the kernel of a chunk's attention (attn_chunk.hip), in which a row sees the context and the nodes that its
// mask names.  Steps that lie in the context are those of a chunk; in the others the lanes select by 32 bits of their rows' masks.
#include "attn_chunk_kernel.h"

namespace ss {

int32_t tree_mfma_launch(const ChunkArgs &a, hipStream_t stream) { return launch_all<true>(a, stream); }

}  // namespace ss
