// The merge of a cut tile's partial results by their log-sum-exp, for both kernels of a chunk's attention.
//
// A partial result is what its workgroup's wavefronts had in their accumulators, four values of one row to a lane, one KB after the other; a thread
// of the merge takes the same four values of every piece.  m is the reference of a row's exponentials (in powers of two), l their sum.
#pragma once

#include "chunk_plan.h"

namespace ss {

constexpr float kChunkNoMax = -1.0e30f;   // reference of a row that has seen nothing

typedef float chunk_float4 __attribute__((ext_vector_type(4)));

// Where quad number j of a tile's accumulators stands: its row and its first d.
// RB: rows of a wavefront (16 or 32); a wavefront's quads are [RB * D / 256][64 lanes].
template <int RB, int D>
__device__ __forceinline__ void chunk_quad(int j, int &row, int &d)
{
    constexpr int PER_WAVE = RB * D / 4;
    const int wave = j / PER_WAVE, k = (j % PER_WAVE) / 64, lane = j & 63;
    row = wave * RB + lane % RB;
    d = k * (256 / RB) + lane / RB * 4;
}

template <int Q_DT>
__device__ __forceinline__ void chunk_store4(void *out, int64_t i, chunk_float4 v)
{
    if constexpr (Q_DT == SS_F32) {
        *reinterpret_cast<chunk_float4 *>(static_cast<float *>(out) + i) = v;
    } else {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<b4 *>(static_cast<uint16_t *>(out) + i) = __builtin_convertvector(v, b4);
    }
}

template <int ROWS, int RB, int D, int Q_DT>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a)
{
    constexpr int QUADS = ROWS * D / 4, PARTS = QUADS / 256;
    const int part = blockIdx.x % PARTS, unit = blockIdx.x / PARTS;
    const int g = unit % a.num_kv_heads, span = unit / a.num_kv_heads;
    const int32_t *rec = a.rec + (int64_t)span * kChunkRecInts;
    const int pieces = rec[0], q0 = rec[1], rows = rec[2], row0 = rec[3];
    if (pieces == 0) return;
    const int j = part * 256 + threadIdx.x;
    int row, d;
    chunk_quad<RB, D>(j, row, d);
    const int G = a.num_q_heads / a.num_kv_heads, n = row0 + row;
    if (n >= rows) return;
    // the first piece is the second partial result of its span, the others the first of theirs
    const int64_t first = (2ll * span + 1) * a.num_kv_heads + g, step = 2ll * a.num_kv_heads, back = a.num_kv_heads;
    float m = a.part_ml[(first * ROWS + row) * 2];
    for (int p = 1; p < pieces; ++p) m = fmaxf(m, a.part_ml[((first - back + p * step) * ROWS + row) * 2]);
    float l = 0.f;
    chunk_float4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pieces; ++p) {
        const int64_t at = first + p * step - (p ? back : 0);
        const float *ml = a.part_ml + (at * ROWS + row) * 2;
        const chunk_float4 x = reinterpret_cast<const chunk_float4 *>(a.part_o)[at * QUADS + j];
        const float w = __builtin_amdgcn_exp2f(ml[0] - m);
        l += w * ml[1];
        o += w * x;
    }
    const int64_t at = (int64_t)(q0 + n / G) * a.num_q_heads + g * G + n % G;
    const float r = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;   // (a row that sees nothing: zeros; NaN stays)
    chunk_store4<Q_DT>(a.out, at * D + d, o * r);
    if (a.lse && d == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// What the merge needs to know of the tile that a span begins and does not end; called once for each span and KV head, with 0 pieces if there is none.
__device__ __forceinline__ void chunk_record(const ChunkArgs &a, int span, int g, int pieces, int q0, int rows, int row0)
{
    if (a.cap > 0 && g == 0 && threadIdx.x == 0) {
        int32_t *rec = a.rec + (int64_t)span * kChunkRecInts;
        rec[0] = pieces;
        rec[1] = q0;
        rec[2] = rows;
        rec[3] = row0;
    }
}

// Launches the merge for what a call has cut.
template <int ROWS, int RB, int D, int Q_DT>
int32_t chunk_merge_launch(const ChunkArgs &a, hipStream_t stream)
{
    if (a.cap == 0 || a.spans < 2) return SS_OK;
    hipLaunchKernelGGL((chunk_merge_kernel<ROWS, RB, D, Q_DT>), dim3((unsigned)(a.spans - 1) * a.num_kv_heads * (ROWS * D / 1024)), dim3(256), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_merge_kernel");
    return SS_OK;
}

}  // namespace ss
