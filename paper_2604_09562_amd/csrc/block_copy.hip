// Copies of cache blocks, keys, values and scales as they are, for all layers of a cache in one launch: bound by memory, read once and written once.
// Calls that may pass more than the last cache level holds go past the caches: 1 GB read and written 201 us (5.1 TB/s, a large copy's rate; through them 212), but 46 MB 11.8 us against
// 8.1 through them, of blocks that were written or are read a moment before or after.  Two, four or eight loads of a lane under way and four to 32 workgroups a compute unit are within
// 1 % of each other, 64 and more 3 % faster, but calls whose pairs are counted on the device would start them all for nothing.
#include "block_share.h"

namespace ss {
namespace {

constexpr int kThreads = 256, kEach = 4;               // 16-byte loads of a lane that are under way together
constexpr int kPiece = kThreads * kEach * 16;          // bytes of a block's keys or values that a workgroup copies at a time
constexpr int kWgs = 2048;                             // eight workgroups to a compute unit
constexpr int64_t kLastCache = 256 << 20;              // bytes

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool PAST>   // past the caches
__global__ __launch_bounds__(kThreads) void block_copy_kernel(BlockCopyArgs a)
{
    const int tid = threadIdx.x;
    const int n = a.num_copies ? min(max(a.num_copies[0], 0), a.max_copies) : a.max_copies;
    const int pieces = (int)((a.block_bytes + kPiece - 1) / kPiece), per = a.layers * 2 * pieces;
    for (int64_t it = blockIdx.x; it < (int64_t)n * per; it += gridDim.x) {
        const int pair = (int)(it / per), k = (int)(it % per);
        const int piece = k % pieces, side = k / pieces % 2, layer = k / pieces / 2;
        const int src = a.src[pair], dst = a.dst[pair];
        if ((unsigned)src >= (unsigned)a.num_blocks || (unsigned)dst >= (unsigned)a.num_blocks || src == dst) continue;
        char *cache = a.layer[layer].side[side];
        const int64_t at = (int64_t)piece * kPiece + tid * 16;
        const char *from = cache + (int64_t)src * a.block_bytes + at;
        char *to = cache + (int64_t)dst * a.block_bytes + at;
        u32x4 w[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (at + i * kThreads * 16 < a.block_bytes) {
                const u32x4 *p = reinterpret_cast<const u32x4 *>(from + i * kThreads * 16);
                w[i] = PAST ? __builtin_nontemporal_load(p) : *p;
            }
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (at + i * kThreads * 16 < a.block_bytes) {
                u32x4 *p = reinterpret_cast<u32x4 *>(to + i * kThreads * 16);
                if constexpr (PAST) __builtin_nontemporal_store(w[i], p);
                else *p = w[i];
            }
        float *scale = a.layer[layer].scale[side];
        if (scale && piece == 0)
            for (int h = tid; h < a.heads; h += kThreads) scale[(int64_t)dst * a.heads + h] = scale[(int64_t)src * a.heads + h];
    }
}

}  // namespace

int32_t block_copy_launch(const BlockCopyArgs &a, hipStream_t stream)
{
    const int64_t items = (int64_t)a.max_copies * a.layers * 2 * ((a.block_bytes + kPiece - 1) / kPiece);
    const dim3 grid((unsigned)(items < kWgs ? items : kWgs));
    if ((double)a.max_copies * a.layers * 4.0 * (double)a.block_bytes > (double)kLastCache)   // (read and written)
        hipLaunchKernelGGL(block_copy_kernel<true>, grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL(block_copy_kernel<false>, grid, dim3(kThreads), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch block_copy_kernel");
    return SS_OK;
}

}  // namespace ss
