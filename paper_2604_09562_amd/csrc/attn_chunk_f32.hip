// Attention of a chunk of new tokens, or of the nodes of a draft tree, in fp32 throughout: the path for fp32 queries or caches (the bf16 matrix-core kernels take the
// others).
//
// A workgroup takes a share (chunk_plan.h) of 64 query rows of a KV head, 16 to a wavefront.  A step brings 64 keys and values into LDS as fp32; a
// wavefront computes
//   S^T[token][row] = K[token][:] . Q[row][:]    v_mfma_f32_16x16x4_f32, a lane holds a quarter of a row's d in pieces of four
//   O^T[d][row]    += V[token][d] * P[row][token] the same shape; step i contracts tokens {4 jq + i}, so that P is taken straight from the
//                                                accumulators of S^T
// so that a lane has one row: its maximum, sum and rescaling need no exchange but over the four lanes of the row.
// Bound by the fp32 matrix rate where it is large, by the chain of offsets, table, keys and the merge where it is small.
#include "chunk_merge.h"

namespace ss {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kRows = kChunkRowsF32, kWaves = 4, kStepKeys = kChunkKeysF32;

// four consecutive elements (from a multiple of four) as fp32
template <int DT>
__device__ __forceinline__ float4v load4(const void *base, int64_t i)
{
    if constexpr (DT == SS_F32) {
        return *reinterpret_cast<const float4v *>(static_cast<const float *>(base) + i);
    } else if constexpr (DT == SS_BF16) {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(static_cast<const uint16_t *>(base) + i);
        return float4v{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(base) + i);
        const float2v x = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), y = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        return float4v{x.x, x.y, y.x, y.y};
    }
}

template <int D, int KV, int QDT, bool TREE>
__global__ __launch_bounds__(64 * kWaves) void chunk_f32_kernel(ChunkArgs a)
{
    constexpr int PAD = D + 4, PIECES = kStepKeys * D / 4 / (64 * kWaves);   // fours of a step's keys to a thread
    __shared__ float ks[kStepKeys][PAD];
    __shared__ float vs[kStepKeys][PAD];
    const int g = blockIdx.x % a.num_kv_heads, span = blockIdx.x / a.num_kv_heads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    ChunkWalk<kRows, kStepKeys, kChunkOpenF32, TREE> s;
    int begun = 0, begun_q0 = 0, begun_rows = 0, begun_row0 = 0;
    for (bool any = s.begin(a, span); any; any = s.next(a)) {
        if (s.part == 2 * span + 1) {
            begun = s.pieces();
            begun_q0 = s.u.q0;
            begun_rows = s.u.q_len * s.u.G;
            begun_row0 = s.t * kRows;
        }
        const int n16 = lane & 15, jq = lane >> 4;
        const int G = a.num_q_heads / a.num_kv_heads;
        const int rows = s.u.q_len * G, n = s.t * kRows + wave * 16 + n16;
        const int qi = min(n, rows - 1) / G, hh = n % G;
        const int lim = s.u.kv_len - s.u.q_len + qi;                     // the last position this lane's row sees
        const int64_t at = (int64_t)(s.u.q0 + qi) * a.num_q_heads + g * G + hh;
        float4v q[D / 16];   // B operand: d = 16 c + 4 jq ..
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            q[c] = float4v{0.f, 0.f, 0.f, 0.f};
            if (n < rows) q[c] = load4<QDT>(a.q, (int64_t)(s.u.q0 + qi) * a.q_stride + (int64_t)(g * G + hh) * D + 16 * c + 4 * jq);
        }
        // Weights are powers of two of scores' differences to the largest, which is subtracted before the scale is applied: the largest score's weight is one
        // whatever its size.  The factor in two parts, for the reference in powers of two (fp32 holds it to 2^-24 of a score's size only).
        const double c64 = (double)a.sm_scale * 1.4426950408889634;
        const float c_hi = (float)c64, c_lo = (float)(c64 - (double)c_hi);
        const int32_t *table = a.block_table + (int64_t)s.b * a.max_blocks;
        float m = kChunkNoMax, l = 0.f;   // (m: in scores before the scale)
        float4v o[D / 16];
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[c] = float4v{0.f, 0.f, 0.f, 0.f};

        // Steps from `full` on hold keys that some row of the tile does not see.  There a value that is not finite is taken out of the product, in
        // which it would reach every row (0 * inf), and added to the rows that see it.
        const int ctx = s.u.kv_len - s.u.q_len;
        const int full = max((TREE ? ctx : ctx + s.t * kRows / G + 1) / kStepKeys, 0);
        const uint32_t *mask = nullptr;
        if constexpr (TREE) mask = a.node_mask + (int64_t)(s.u.q0 + qi) * a.mask_words;
        for (int step = s.s0; step < s.s1; ++step) {
            bool odd = false;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int e = i * 64 * kWaves + tid, t = e / (D / 4), d = e % (D / 4) * 4;
                const int pos = step * kStepKeys + t;
                float4v k = {0.f, 0.f, 0.f, 0.f}, v = k;
                if (pos < s.u.kv_len) {   // what stands behind the last token is of no one
                    const int64_t tile = (int64_t)chunk_block(a, table[pos / kTile]) * a.num_kv_heads + g, from = (tile * kTile + pos % kTile) * D + d;
                    k = load4<KV>(a.k, from);
                    v = load4<KV>(a.v, from);
                    if constexpr (KV == SS_FP8_E4M3) { k *= a.k_scale[tile]; v *= a.v_scale[tile]; }
                }
                if (step >= full) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (!__builtin_isfinite(v[c])) { v[c] = 0.f; odd = true; }
                }
                *reinterpret_cast<float4v *>(&ks[t][d]) = k;
                *reinterpret_cast<float4v *>(&vs[t][d]) = v;
            }
            const int any_odd = __syncthreads_or(odd);
            uint32_t window[2] = {~0u, ~0u};   // TREE: which of the step's keys this lane's row attends
            if constexpr (TREE)
                if (step >= full)
#pragma unroll
                    for (int h = 0; h < 2; ++h) window[h] = tree_window(mask, a.mask_words, s.u.q_len, step * kStepKeys + h * 32 - ctx);
            float4v x[4];
            float top = kChunkNoMax;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                float4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const float4v k = *reinterpret_cast<const float4v *>(&ks[tb * 16 + n16][16 * c + 4 * jq]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[c][i], acc, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (TREE ? !(window[tb / 2] >> (tb % 2 * 16 + jq * 4 + i) & 1) : step * kStepKeys + tb * 16 + jq * 4 + i > lim) acc[i] = -__builtin_inff();
                    top = fmaxf(top, acc[i]);
                }
                x[tb] = acc;
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top), down = __builtin_amdgcn_exp2f((m - m_new) * c_hi);
            m = m_new;
            l *= down;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) o[c] *= down;
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = x[tb][i];
                    const float p = y == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((y - m) * c_hi);
                    x[tb][i] = p;
                    l += p;
                }
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
                for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vs[tb * 16 + jq * 4 + i][16 * c + n16], x[tb][i], o[c], 0, 0, 0);
            if (any_odd) {
                for (int pos = step * kStepKeys; pos < min((step + 1) * kStepKeys, TREE ? s.u.kv_len : lim + 1); ++pos) {
                    if constexpr (TREE)
                        if (!((pos % kStepKeys < 32 ? window[0] : window[1]) >> (pos % 32) & 1)) continue;
                    const int64_t tile = (int64_t)chunk_block(a, table[pos / kTile]) * a.num_kv_heads + g, from = (tile * kTile + pos % kTile) * D + 4 * jq;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        float4v v = load4<KV>(a.v, from + 16 * c);
                        if constexpr (KV == SS_FP8_E4M3) v *= a.v_scale[tile];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!__builtin_isfinite(v[i])) o[c][i] += v[i];
                    }
                }
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        // the reference in powers of two, and what its rounding leaves (of references so large that this is no factor, nothing: it is within the scores' own rounding)
        const float ref = l == 0.f ? kChunkNoMax : fmaxf(m * c_hi, kChunkNoMax);
        const float rest = fabsf(ref) < 0x1p20f ? __builtin_amdgcn_exp2f(__builtin_fmaf(m, c_lo, __builtin_fmaf(m, c_hi, -ref))) : 1.0f;
        if (s.part >= 0) {
            const int64_t part = (int64_t)s.part * a.num_kv_heads + g;
            float4v *po = reinterpret_cast<float4v *>(a.part_o) + part * (kRows * D / 4) + wave * (16 * D / 4) + lane;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) po[c * 64] = o[c] * rest;
            if (jq == 0) {
                float *ml = a.part_ml + (part * kRows + wave * 16 + n16) * 2;
                ml[0] = ref;
                ml[1] = l * rest;
            }
            continue;
        }
        if (n < rows) {   // (the walk takes whole wavefronts)
            const float r = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) chunk_store4<QDT>(a.out, at * D + 16 * c + 4 * jq, o[c] * r);
            if (a.lse && jq == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(l * rest)) * 0.6931471805599453f;
        }
    }
    chunk_record(a, span, g, begun, begun_q0, begun_rows, begun_row0);
}

template <int D, int KV, int QDT, bool TREE>
int32_t launch(const ChunkArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((chunk_f32_kernel<D, KV, QDT, TREE>), dim3((unsigned)(a.spans * a.num_kv_heads)), dim3(64 * kWaves), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_f32_kernel");
    return chunk_merge_launch<kRows, 16, D, QDT>(a, stream);
}

template <int D, int QDT, bool TREE>
int32_t launch_kv(const ChunkArgs &a, hipStream_t stream)
{
    switch (a.kv_dtype) {
    case SS_F32: return launch<D, SS_F32, QDT, TREE>(a, stream);
    case SS_BF16: return launch<D, SS_BF16, QDT, TREE>(a, stream);
    default: return launch<D, SS_FP8_E4M3, QDT, TREE>(a, stream);
    }
}

template <bool TREE>
int32_t launch_all(const ChunkArgs &a, hipStream_t stream)
{
    if (a.head_dim == 128) return a.q_dtype == SS_F32 ? launch_kv<128, SS_F32, TREE>(a, stream) : launch_kv<128, SS_BF16, TREE>(a, stream);
    return a.q_dtype == SS_F32 ? launch_kv<64, SS_F32, TREE>(a, stream) : launch_kv<64, SS_BF16, TREE>(a, stream);
}

}  // namespace

int32_t chunk_f32_launch(const ChunkArgs &a, hipStream_t stream) { return launch_all<false>(a, stream); }
int32_t tree_f32_launch(const ChunkArgs &a, hipStream_t stream) { return launch_all<true>(a, stream); }

}  // namespace ss
