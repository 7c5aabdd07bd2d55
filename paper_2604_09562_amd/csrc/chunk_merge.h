// The merge of a cut tile's partial results by their log-sum-exp, for both kernels of a chunk's attention.
//
// A partial result is what its workgroup's wavefronts had in their accumulators, four values of one row to a lane, one KB after the other; a thread
// of the merge takes the same four values of every piece.  m is the reference of a row's exponentials (in powers of two), l their sum.
#pragma once

#include <type_traits>

#include "chunk_plan.h"

namespace ss {

constexpr float kChunkNoMax = -3.4028234663852886e38f;   // reference of a row that has seen nothing: no finite score lies below it

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

// Two pieces, which most cut tiles have, are a form of their own: 15 us instead of 17 for 65 MB of them; eight asked for at a time take 25.
// A workgroup merges 256 quads of few pieces, a wavefront 64 of them.  Of many pieces (a tile of a long cache in some dozens) it merges 64 quads, each wavefront a
// quarter of the pieces, and the workgroups of the next three spans, which are in the middle of the tile, the others: 9 us instead
// of 16 for 34 MB of eight tiles in 31 pieces.
constexpr int kMergeWays = 4;

template <int ROWS, int RB, int D, int Q_DT>
__global__ __launch_bounds__(64 * kMergeWays) void chunk_merge_kernel(ChunkArgs a)
{
    constexpr int QUADS = ROWS * D / 4, PARTS = QUADS / (64 * kMergeWays);
    __shared__ chunk_float4 so[kMergeWays - 1][64];
    __shared__ float sm[kMergeWays - 1][64], sl[kMergeWays - 1][64];
    const int part = blockIdx.x % PARTS, unit = blockIdx.x / PARTS;
    const int g = unit % a.num_kv_heads, last = unit / a.num_kv_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the nearest span in front, or this one, that begins a tile and does not end it
    const int32_t *rec = a.rec + (int64_t)last * kChunkRecInts;
    int back = 0, pieces = rec[0];
    if (pieces == 0) {
        for (back = 1; back < kMergeWays && back <= last; ++back)
            if ((pieces = rec[-back * kChunkRecInts]) != 0) break;
        if (pieces == 0) return;
    }
    rec -= back * kChunkRecInts;
    const int span = last - back, q0 = rec[1], rows = rec[2], row0 = rec[3];
    const bool many = pieces > 2 * kMergeWays;
    if (back > 0 && !many) return;
    const int way = many ? wave : 0, ways = many ? kMergeWays : 1;
    const int G = a.num_q_heads / a.num_kv_heads;
    // the first piece is the second partial result of its span, the others the first of theirs
    auto place = [&](int p) { return (2ll * (span + p) + (p == 0)) * a.num_kv_heads + g; };
    const int k = many ? back : wave;
    const int j = (part * kMergeWays + k) * 64 + lane;
    int row, d;
    chunk_quad<RB, D>(j, row, d);
    const int n = row0 + row;
    float m = kChunkNoMax, l = 0.f;
    chunk_float4 o = {0.f, 0.f, 0.f, 0.f};
    auto gather = [&](auto ahead) __attribute__((always_inline)) {
        constexpr int AHEAD = decltype(ahead)::value;   // pieces asked for at a time
        for (int p0 = way; p0 < pieces; p0 += ways * AHEAD) {
            float mi[AHEAD], li[AHEAD];
            chunk_float4 x[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int p = p0 + i * ways;
                mi[i] = kChunkNoMax;
                li[i] = 0.f;
                x[i] = chunk_float4{0.f, 0.f, 0.f, 0.f};
                if (AHEAD == 2 || p < pieces) {
                    const int64_t at = place(p);
                    const float *ml = a.part_ml + (at * ROWS + row) * 2;
                    mi[i] = ml[0];
                    li[i] = ml[1];
                    x[i] = reinterpret_cast<const chunk_float4 *>(a.part_o)[at * QUADS + j];
                }
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const float up = fmaxf(m, mi[i]), down = __builtin_amdgcn_exp2f(m - up), w = __builtin_amdgcn_exp2f(mi[i] - up);
                m = up;
                l = l * down + w * li[i];
                o = o * down + w * x[i];
            }
        }
    };
    if (n < rows) {
        if (pieces == 2) gather(std::integral_constant<int, 2>{});   // (there are two at least)
        else gather(std::integral_constant<int, 4>{});
    }
    if (many) {
        if (way > 0) {
            sm[way - 1][lane] = m;
            sl[way - 1][lane] = l;
            so[way - 1][lane] = o;
        }
        __syncthreads();
        if (way == 0)
#pragma unroll
            for (int i = 0; i < kMergeWays - 1; ++i) {
                const float up = fmaxf(m, sm[i][lane]), down = __builtin_amdgcn_exp2f(m - up), w = __builtin_amdgcn_exp2f(sm[i][lane] - up);
                m = up;
                l = l * down + w * sl[i][lane];
                o = o * down + w * so[i][lane];
            }
    }
    if (way > 0 || n >= rows) return;
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
    hipLaunchKernelGGL((chunk_merge_kernel<ROWS, RB, D, Q_DT>), dim3((unsigned)(a.spans - 1) * a.num_kv_heads * (ROWS * D / (256 * kMergeWays))),
                       dim3(64 * kMergeWays), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_merge_kernel");
    return SS_OK;
}

}  // namespace ss
