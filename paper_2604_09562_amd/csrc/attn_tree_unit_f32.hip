// Attention of the nodes of wide draft trees in fp32 throughout, short calls: one launch, no plan and no merge.  fp32 queries or caches; the others are attn_tree_unit.hip's.
//
// A workgroup takes 16 query rows of a KV head, its wavefronts the cache blocks of 16 keys in turn,
//   S^T[key][row]  = K[key][:] . Q[row][:]        v_mfma_f32_16x16x4_f32, a lane holds a quarter of a row's d in pieces of four
//   O^T[d][row]   += V[key][d] * P[row][key]      the same shape; step i contracts keys {4 jq + i}, so that P is taken straight from the accumulators of S^T
// and add up what they have at the end.  Operands come from memory as the matrix instructions take them: the rows of a tile are the only ones that read a block, there is
// nothing for LDS to share.  Rounding is fp32's alone.
//
// Bound by latency (lengths, block id, keys and values, the sum over the wavefronts), then by the fp32 matrix rate: a block costs a SIMD 1024 cycles (64-wide heads) or 2048.
// Four requests of 10 .. 40 nodes behind 64 .. 512 tokens, 8 heads over 2 of 64: 12.5 us (24.5 in the chunk's kernel with its merge).
#include "chunk_merge.h"

namespace ss {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kRows = kTreeUnitRowsF32;

// Elements as they stand in memory, and as fp32.
template <int DT> struct Stored;
template <> struct Stored<SS_F32> {
    typedef float4v four;
    typedef float one;
    static __device__ __forceinline__ float4v wide(four x) { return x; }
    static __device__ __forceinline__ float wide1(one x) { return x; }
};
template <> struct Stored<SS_BF16> {
    typedef u32x2 four;
    typedef uint16_t one;
    static __device__ __forceinline__ float4v wide(four w)
    {
        return float4v{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
    }
    static __device__ __forceinline__ float wide1(one x) { return __uint_as_float((uint32_t)x << 16); }
};
template <> struct Stored<SS_FP8_E4M3> {
    typedef uint32_t four;
    typedef uint8_t one;
    static __device__ __forceinline__ float4v wide(four w)
    {
        const float2v x = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), y = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        return float4v{x.x, x.y, y.x, y.y};
    }
    static __device__ __forceinline__ float wide1(one x) { return __builtin_amdgcn_cvt_f32_fp8((uint32_t)x, 0); }
};

template <int D> constexpr int waves_of() { return D == 64 ? 16 : 8; }   // (what registers there are for)

template <int D, int KV, int QDT>
__global__ __launch_bounds__(64 * waves_of<D>()) void tree_unit_f32_kernel(ChunkArgs a, int tiles)
{
    constexpr int WAVES = waves_of<D>(), PAD = D + 4;
    typedef Stored<KV> In;
    __shared__ float sh_o[WAVES][kRows][PAD];
    __shared__ float sh_m[WAVES][kRows], sh_l[WAVES][kRows];
    const int g = blockIdx.x % a.num_kv_heads, at_wg = blockIdx.x / a.num_kv_heads, b = at_wg / tiles;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n16 = lane & 15, jq = lane >> 4;
    ChunkUnit<kRows, kTile, true> u;
    u.set(a, uniform(a.q_indptr[b]), uniform(a.q_indptr[b + 1]), uniform(a.kv_len[b]), 0);
    const int G = u.G, rows = u.q_len * G, ctx = u.kv_len - u.q_len;
    const int blocks = (int)(((unsigned)u.kv_len + kTile - 1) / kTile), full = max(ctx / kTile, 0), parts = min(blocks, WAVES);
    const int32_t *table = a.block_table + (int64_t)b * a.max_blocks;
    // the scale with log2(e), in two parts (weights are powers of two of differences to the largest score, taken before the scale)
    const double c64 = (double)a.sm_scale * 1.4426950408889634;
    const float c_hi = (float)c64, c_lo = (float)(c64 - (double)c_hi);
    for (int t = at_wg % tiles; t < u.tiles; t += tiles) {
        const int n = t * kRows + n16, qi = min(n, rows - 1) / G, hh = n % G;
        const uint32_t *mask = a.node_mask + (int64_t)(u.q0 + qi) * a.mask_words;
        typename In::four k_in[D / 16];
        typename In::one v_in[D / 16][4];
        float ks_in = 1.f, vs_in = 1.f;
        auto place = [&](int block) __attribute__((always_inline)) { return (int64_t)chunk_block(a, uniform(table[block])) * a.num_kv_heads + g; };
        auto bring_k = [&](int64_t tile) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
                k_in[c] = *reinterpret_cast<const typename In::four *>(static_cast<const typename In::one *>(a.k) + (tile * kTile + n16) * D + 16 * c + 4 * jq);
            if constexpr (KV == SS_FP8_E4M3) ks_in = a.k_scale[tile];
        };
        auto bring_v = [&](int64_t tile) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < D / 16; ++c) v_in[c][i] = static_cast<const typename In::one *>(a.v)[(tile * kTile + 4 * jq + i) * D + 16 * c + n16];
            if constexpr (KV == SS_FP8_E4M3) vs_in = a.v_scale[tile];
        };
        if (wave < blocks) {
            const int64_t tile = place(wave);
            bring_k(tile);
            bring_v(tile);
        }
        float4v q[D / 16];
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            q[c] = float4v{0.f, 0.f, 0.f, 0.f};
            if (n < rows)
                q[c] = Stored<QDT>::wide(*reinterpret_cast<const typename Stored<QDT>::four *>(
                    static_cast<const typename Stored<QDT>::one *>(a.q) + (int64_t)(u.q0 + qi) * a.q_stride + (int64_t)(g * G + hh) * D + 16 * c + 4 * jq));
        }
        float m = kChunkNoMax, l = 0.f;   // (m: in scores before the scale)
        float4v o[D / 16];
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[c] = float4v{0.f, 0.f, 0.f, 0.f};
        for (int block = wave; block < blocks; block += WAVES) {
            const bool more = block + WAVES < blocks;
            const int64_t next = more ? place(block + WAVES) : 0;
            uint32_t window = ~0u;   // which of the block's keys the lane's row attends
            bool odd = false;
            float4v x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                float4v k = In::wide(k_in[c]);
                if constexpr (KV == SS_FP8_E4M3) k *= ks_in;
#pragma unroll
                for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[c][i], x, 0, 0, 0);
            }
            if (more) bring_k(next);
            if (block >= full) window = tree_window(mask, a.mask_words, u.q_len, block * kTile - ctx);
            float top = kChunkNoMax;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!(window >> (4 * jq + i) & 1u)) x[i] = -__builtin_inff();
                top = fmaxf(top, x[i]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float up = fmaxf(m, top), down = __builtin_amdgcn_exp2f((m - up) * c_hi);
            m = up;
            l *= down;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) o[c] *= down;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = x[i] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((x[i] - m) * c_hi);
                l += x[i];
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = In::wide1(v_in[c][i]);
                    if constexpr (KV == SS_FP8_E4M3) v *= vs_in;
                    // one that is not finite is taken out of the product, in which it would reach every row (0 * inf), and added to the rows that see it
                    if (block >= full && !__builtin_isfinite(v)) { v = 0.f; odd = true; }
                    o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[i], o[c], 0, 0, 0);
                }
            if (more) bring_v(next);
            if (__builtin_expect(__ballot(odd) != 0, 0)) {
                const int64_t tile = (int64_t)chunk_block(a, table[block]) * a.num_kv_heads + g;
                for (int j = 0; j < min(kTile, u.kv_len - block * kTile); ++j) {
                    if (!(window >> j & 1u)) continue;
                    const auto *at = static_cast<const typename In::one *>(a.v) + (tile * kTile + j) * D + 4 * jq;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        float4v w = In::wide(*reinterpret_cast<const typename In::four *>(at + 16 * c));
                        if constexpr (KV == SS_FP8_E4M3) w *= a.v_scale[tile];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!__builtin_isfinite(w[i])) o[c][i] += w[i];
                    }
                }
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        // ---- the wavefronts' sums joined ----
        if (wave < parts) {
#pragma unroll
            for (int c = 0; c < D / 16; ++c) *reinterpret_cast<float4v *>(&sh_o[wave][n16][16 * c + 4 * jq]) = o[c];
            if (jq == 0) {
                sh_m[wave][n16] = m;
                sh_l[wave][n16] = l;
            }
        }
        __syncthreads();
        const int row = tid / (D / 4), d = tid % (D / 4) * 4, no = t * kRows + row;
        if (row < kRows && no < rows) {
            float M = kChunkNoMax, L = 0.f;
            float4v sum = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < parts; ++w) M = fmaxf(M, sh_m[w][row]);
            for (int w = 0; w < parts; ++w) {
                const float f = __builtin_amdgcn_exp2f((sh_m[w][row] - M) * c_hi);
                L += f * sh_l[w][row];
                sum += f * *reinterpret_cast<const float4v *>(&sh_o[w][row][d]);
            }
            // the reference in powers of two, and what its rounding leaves (of references so large that this is no factor, nothing: it is within the scores' own rounding)
            const float ref = L == 0.f ? kChunkNoMax : fmaxf(M * c_hi, kChunkNoMax);
            const float rest = fabsf(ref) < 0x1p20f ? __builtin_amdgcn_exp2f(__builtin_fmaf(M, c_lo, __builtin_fmaf(M, c_hi, -ref))) : 1.0f;
            const float r = L > 0.f ? 1.0f / L : L == 0.f ? 0.f : L;   // (a row that sees nothing: zeros; NaN stays)
            const int64_t at = (int64_t)(u.q0 + no / G) * a.num_q_heads + g * G + no % G;
            chunk_store4<QDT>(a.out, at * D + d, sum * r);
            if (a.lse && d == 0) a.lse[at] = L == 0.f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(L * rest)) * 0.6931471805599453f;
        }
        __syncthreads();   // (the next tile's sums come to where these stood)
    }
}

template <int D, int QDT>
int32_t launch_kv(const ChunkArgs &a, int tiles, hipStream_t stream)
{
    const dim3 grid((unsigned)a.batch * tiles * a.num_kv_heads), wg(64 * waves_of<D>());
    switch (a.kv_dtype) {
    case SS_F32: hipLaunchKernelGGL((tree_unit_f32_kernel<D, SS_F32, QDT>), grid, wg, 0, stream, a, tiles); break;
    case SS_BF16: hipLaunchKernelGGL((tree_unit_f32_kernel<D, SS_BF16, QDT>), grid, wg, 0, stream, a, tiles); break;
    default: hipLaunchKernelGGL((tree_unit_f32_kernel<D, SS_FP8_E4M3, QDT>), grid, wg, 0, stream, a, tiles);
    }
    SS_HIP_CHECK(hipGetLastError(), "launch tree_unit_f32_kernel");
    return SS_OK;
}

}  // namespace

int32_t tree_unit_f32_launch(const ChunkArgs &a, int tiles, hipStream_t stream)
{
    if (a.head_dim == 128) return a.q_dtype == SS_F32 ? launch_kv<128, SS_F32>(a, tiles, stream) : launch_kv<128, SS_BF16>(a, tiles, stream);
    return a.q_dtype == SS_F32 ? launch_kv<64, SS_F32>(a, tiles, stream) : launch_kv<64, SS_BF16>(a, tiles, stream);
}

}  // namespace ss
