// The kernel of a chunk's attention and of wide draft trees' on the bf16 matrix cores; what it computes and what bounds it stands in attn_chunk.hip and attn_tree.hip, which hold its
// instances.
#pragma once

#include <type_traits>

#include "chunk_merge.h"
#include "mfma_tiles.h"

namespace ss {
namespace {

constexpr int kWaves = 4;
constexpr int ROWS = 32 * 2 * kWaves;                 // query rows of a tile, two blocks of 32 to a wavefront
static_assert(ROWS == kChunkRows, "what launches and workspaces are sized by");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// How far (in powers of two) a row's scores may rise above the reference of its exponentials before the sums are rescaled.
constexpr float kLag = 16.0f;
// References beyond this (in powers of two) are taken care of apart: from 2^31 on the rounded reference and the scale's product with the largest score
// may be further apart than an exponential's range.
constexpr float kFar = 0x1p28f;
constexpr int kOddValues = 1;   // values that are not finite were taken out
constexpr int kFarRows = 2;     // a row's reference was beyond kFar

// The largest of three, or NaN (the other kind of maximum costs an instruction more for each operand that may be a signalling NaN).
__device__ __forceinline__ float max3(float x, float y, float z) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z); }
// Waits for this wavefront's LDS accesses, with LOADS also for what it brings into LDS, then for the others.
template <bool LOADS>
__device__ __forceinline__ void team_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(LOADS ? 0x0070 : 0xc07f);   // vmcnt(0) lgkmcnt(0) | lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// f(LO), f(LO + 1), .. f(HI - 1), each with its number as a type
template <int LO, int HI, typename F>
__device__ __forceinline__ void each(F &&f)
{
    if constexpr (LO < HI) {
        f(std::integral_constant<int, LO>{});
        each<LO + 1, HI>(f);
    }
}

constexpr int kKeys = kChunkKeys;   // keys that are taken at a time, two cache blocks
constexpr int kPairKeys = 2 * kKeys;
constexpr int kInfinity = 0x7f800000;   // its bits, those of an exponent too

// 64 keys or values in LDS, rows of D bf16 in pieces of 16 bytes.  Piece c of row t stands at place c ^ turn(t): 16 rows' pieces
// of equal c fill all banks (scores), and so do four rows' pieces 4 n .. 4 n + 3 (transposing reads of values).
template <int D>
struct Tile {
    u32x4 w[kPairKeys][D / 8];
};
// TREE: rows are the nodes of draft trees, which see the context and the nodes that their masks name.
template <int D, bool FP8, bool LSE, bool TREE>
__global__ __launch_bounds__(64 * kWaves, 1) void chunk_kernel(ChunkArgs a, const int32_t *__restrict__ block_table, const float *__restrict__ k_scale,
                                                               const float *__restrict__ v_scale)
{
    // (table and scales come in as no-alias arguments of their own, so that they are scalar loads)
    constexpr int KS = D / 16, DB = D / 32, PIECES = D / 8;
    constexpr int BLOCK_BYTES = kTile * D * (FP8 ? 1 : 2), LOADS = BLOCK_BYTES / (64 * 16);   // 16-byte loads of a lane for a cache block
    // Variables of their own: a tile's reads then do not wait for what is on its way into another one.
    __shared__ Tile<D> k_even, k_odd, v_even, v_odd;   // steps 3, 4, 7, 8, ..; 1, 2, 5, 6, ..; 0, 1, 4, 5, ..; 2, 3, 6, 7, .. (from the first)
    __shared__ int odd_flags[2][kWaves];               // of two steps' values each: whether a wavefront's block of them had values that are not finite
    const int g = blockIdx.x % a.num_kv_heads, span = blockIdx.x / a.num_kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ChunkWalk<ROWS, kKeys, kChunkOpen, TREE> s;
    int begun = 0, begun_q0 = 0, begun_rows = 0, begun_row0 = 0;   // of the tile that the span begins and does not end
    for (bool any = s.begin(a, span); any; any = s.next(a)) {
        if (s.part == 2 * span + 1) {
            begun = s.pieces();
            begun_q0 = s.u.q0;
            begun_rows = s.u.q_len * s.u.G;
            begun_row0 = s.t * ROWS;
        }
        if constexpr (TREE) {
            if (s.u.narrow(s.t)) {
                constexpr int NB = 1;
#include "attn_chunk_tile.h"
            } else {
                constexpr int NB = 2;
#include "attn_chunk_tile.h"
            }
        } else {
            constexpr int NB = 2;
#include "attn_chunk_tile.h"
        }
        team_barrier<false>();   // (the next tile's keys come to where the others may still read)
    }
    chunk_record(a, span, g, begun, begun_q0, begun_rows, begun_row0);
}

template <int D, bool FP8, bool LSE, bool TREE>
int32_t launch(const ChunkArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((chunk_kernel<D, FP8, LSE, TREE>), dim3((unsigned)(a.spans * a.num_kv_heads)), dim3(64 * kWaves), 0, stream, a, a.block_table, a.k_scale, a.v_scale);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_kernel");
    return chunk_merge_launch<ROWS, 32, D, SS_BF16>(a, stream);
}

template <bool TREE>
int32_t launch_all(const ChunkArgs &a, hipStream_t stream)
{
    const bool fp8 = a.kv_dtype == SS_FP8_E4M3;
    if (a.lse) {
        if (a.head_dim == 128) return fp8 ? launch<128, true, true, TREE>(a, stream) : launch<128, false, true, TREE>(a, stream);
        return fp8 ? launch<64, true, true, TREE>(a, stream) : launch<64, false, true, TREE>(a, stream);
    }
    if (a.head_dim == 128) return fp8 ? launch<128, true, false, TREE>(a, stream) : launch<128, false, false, TREE>(a, stream);
    return fp8 ? launch<64, true, false, TREE>(a, stream) : launch<64, false, false, TREE>(a, stream);
}

}  // namespace
}  // namespace ss
