// Attention of the nodes of wide draft trees, short calls: one launch, no plan and no merge.  bf16 queries over bf16 or e4m3 caches, heads of 64 or 128, any grouping.
//
// A workgroup of eight wavefronts takes 32 query rows of a KV head; the wavefronts take its steps of 32 keys in turn,
//   S^T[key][row]  = K[key][:] . Q[row][:]       v_mfma_f32_32x32x16_bf16, queries in registers
//   O^T[d][row]   += V^T[d][key] P^T[key][row]    the same shape; P is taken straight from the accumulators of S^T, V^T by transposing LDS reads
// each with keys and values of its own in LDS, and add up what they have at the end.  A lane holds one row: its softmax needs no exchange but with the lane that has the row's
// other keys.  Weights are 2^((s - m) c), m being the row's largest score so far, subtracted before the scale c is applied: the largest score's weight is one whatever its
// size.  They are rounded to bf16 for the second product (2^-8 at most), and outputs are divided by the sum of what they were rounded to; the log-sum-exp takes the sum of the
// weights themselves.  The last rounding is the outputs'.
//
// Bound by latency: lengths, block ids, keys and values, a step or two of a wavefront, and the sum over the wavefronts stand in one chain.  Every block of 32 rows reads the keys again
// (from L2), which is what bounds the calls that are better off in the other kernels.
#include <type_traits>

#include "chunk_merge.h"
#include "mfma_tiles.h"

namespace ss {
namespace {

constexpr int kWaves = 8, kRows = kTreeUnitRows, kKeys = 32;
constexpr float kFar = 0x1p28f;   // references beyond this (in powers of two) are taken care of apart

// Steps of a split of a tile.
__device__ __forceinline__ int split_steps(int steps, int splits) { return (steps + splits - 1) / splits; }

template <int D, bool FP8>
__global__ __launch_bounds__(64 * kWaves, 2) void tree_unit_kernel(ChunkArgs a, TreeUnitChoice how, const int32_t *__restrict__ block_table, const float *__restrict__ k_scale,
                                                                   const float *__restrict__ v_scale)
{
    constexpr int KS = D / 16, DB = D / 32, PIECES = D / 8;
    constexpr int BLOCK_BYTES = kTile * D * (FP8 ? 1 : 2), LOADS = BLOCK_BYTES / (64 * 16);   // 16-byte loads of a lane for a cache block
    // A wavefront's keys and values, later its outputs.  (Variables of their own: reads of keys then do not wait for values that are on their way.)
    typedef u32x4 Tile[kKeys][PIECES];
    __shared__ Tile k_tiles[kWaves], v_tiles[kWaves];
    __shared__ float sh_m[kWaves][kRows], sh_l[kWaves][kRows], sh_used[kWaves][kRows];
    static_assert(2 * sizeof(Tile) == kRows * D * sizeof(float), "outputs stand where keys and values were");
    // (the KV head first: neighbours, which read the same keys, then stand in one XCD where the heads are a multiple of its number)
    int at_wg = blockIdx.x;
    const int g = at_wg % a.num_kv_heads;
    at_wg /= a.num_kv_heads;
    const int tile0 = at_wg % how.tiles;
    at_wg /= how.tiles;
    const int split = at_wg % how.splits, b = at_wg / how.splits;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r32 = lane & 31, half = lane >> 5, i16 = lane & 15, group = lane >> 4;
    ChunkUnit<kRows, kKeys, true> u;
    u.set(a, uniform(a.q_indptr[b]), uniform(a.q_indptr[b + 1]), uniform(a.kv_len[b]), 0);
    const int G = u.G, rows = u.q_len * G, ctx = u.kv_len - u.q_len;
    const int all_steps = (int)(((unsigned)u.kv_len + kKeys - 1) / kKeys), full = max(ctx / kKeys, 0), last_block = (int)(((unsigned)u.kv_len + kTile - 1) / kTile) - 1;
    const float c = fmaxf(a.sm_scale * 1.4426950408889634f, 0x1p-126f);
    typedef const __attribute__((address_space(4))) int32_t *scalar_ints;
    const scalar_ints table = (scalar_ints)(uintptr_t)(block_table + (int64_t)b * a.max_blocks);
    const uint32_t block_stride = (uint32_t)a.num_kv_heads * BLOCK_BYTES;
    const char *k_base = static_cast<const char *>(a.k) + (int64_t)g * BLOCK_BYTES, *v_base = static_cast<const char *>(a.v) + (int64_t)g * BLOCK_BYTES;
    Tile &k_tile = k_tiles[wave], &v_tile = v_tiles[wave];
    uint32_t piece_at[FP8 ? 1 : LOADS];
    if constexpr (!FP8)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = i * 64 + lane, t = p / PIECES;
            piece_at[i] = (uint32_t)(t * PIECES + ((p % PIECES) ^ turn<D>(t))) * 16;
        }
    // two cache blocks of a step on their way: bf16 straight into LDS, e4m3 into registers
    auto bring = [&](const char *cache, const int (&id)[2], Tile &tile, u32x4 (&in)[2][FP8 ? LOADS : 1]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const char *at = cache + (uint64_t)(uint32_t)id[j] * block_stride;
            const __amdgpu_buffer_rsrc_t block = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, BLOCK_BYTES, 0x00020000);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if constexpr (FP8) in[j][i] = __builtin_amdgcn_raw_buffer_load_b128(block, (i * 64 + lane) * 16, 0, 0);
#ifdef __HIP_DEVICE_COMPILE__   // (the host's pass does not know that this GPU brings 16 bytes at a time)
                else
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(block, (__attribute__((address_space(3))) void *)(&tile[j * kTile + i * 64 / PIECES][0]), 16, piece_at[i], 0, 0, 0);
#endif
            }
        }
    };
    // e4m3 codes as bf16 into LDS, with the sign and the power of two of their scale, NaN all of them if it is not finite
    auto put = [&](const u32x4 (&in)[2][FP8 ? LOADS : 1], Tile &tile, const int (&scale)[2]) __attribute__((always_inline)) {
        if constexpr (FP8)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t sign = (uint32_t)(scale[j] >> 31) & 0x80808080u, nan = (scale[j] & 0x7fffffff) >= 0x7f800000 ? 0x7f7f7f7fu : 0u;
                const float power = __int_as_float(scale[j] & 0x7f800000);
#pragma unroll
                for (int i = 0; i < 2 * LOADS; ++i) {
                    const int el = (i / 2 * 64 + lane) * 16, t = el / D, col = el % D / 8;
                    u32x4 w;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t four = (in[j][i / 2][2 * (i % 2) + q] ^ sign) | nan;
                        w[2 * q] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, power, false));
                        w[2 * q + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, power, true));
                    }
                    tile[j * kTile + t][(col + i % 2) ^ turn<D>(t)] = w;
                }
            }
    };
    auto ids_of = [&](int step, int (&id)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) id[j] = chunk_block(a, table[min(step * 2 + j, last_block)]);
    };
    auto scales_of = [&](const float *scales, const int (&id)[2], int (&scale)[2]) __attribute__((always_inline)) {
        if constexpr (FP8)
#pragma unroll
            for (int j = 0; j < 2; ++j) scale[j] = ((scalar_ints)(uintptr_t)scales)[(uint32_t)id[j] * (uint32_t)a.num_kv_heads + (uint32_t)g];
    };
    auto fraction = [&](int scale) __attribute__((always_inline)) { return FP8 ? __int_as_float((scale & 0x7fffff) | 0x3f800000) : 1.0f; };

    for (int t = tile0; t < u.tiles; t += how.tiles) {
        // the workgroup's steps; tiles beyond those that the call has room for partial results of are one workgroup's each
        const bool whole = how.splits == 1 || t >= how.tiles;
        if (whole && split > 0) break;
        const int each = whole ? all_steps : split_steps(all_steps, how.splits), first = split * each, steps = min(all_steps, first + each);
        if (!whole && first >= all_steps && (split > 0 || all_steps > 0)) break;   // (of a request without keys the first one leaves that)
        const int n = t * kRows + r32, i_row = min(n, rows - 1) / G;
        const uint32_t *mask = a.node_mask + (int64_t)(u.q0 + i_row) * a.mask_words;
        u32x4 in_k[2][FP8 ? LOADS : 1], in_v[2][FP8 ? LOADS : 1];
        int id[2], next[2] = {}, ks[2] = {}, vs[2] = {};   // next: blocks of the wavefront's next step
        if (first + wave < steps) {
            ids_of(first + wave, id);
            ids_of(first + wave + kWaves, next);
            bring(k_base, id, k_tile, in_k);
            bring(v_base, id, v_tile, in_v);
            scales_of(k_scale, id, ks);
            scales_of(v_scale, id, vs);
        }
        bf16x8 q[KS];
        {
            const char *src = static_cast<const char *>(a.q) + ((int64_t)(u.q0 + i_row) * a.q_stride + (int64_t)(g * G + n % G) * D + half * 8) * 2;
            const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                u32x4 w = zero;
                if (n < rows) w = *reinterpret_cast<const u32x4 *>(src + k * 32);
                q[k] = __builtin_bit_cast(bf16x8, w);
            }
        }
        float m = kChunkNoMax, l = 0.f, used = 0.f;
        float16v o[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        const int turn32 = turn<D>(r32 & 15);
        for (int step = first + wave; step < steps; step += kWaves) {
            // which of the step's keys the lane's row sees: key 8 (i / 4) + 4 half + i % 4 is accumulator i
            uint32_t window = ~0u;
            if (step >= full) window = tree_window(mask, a.mask_words, u.q_len, step * kKeys - ctx) >> (4 * half);
            const bool more = step + kWaves < steps;
            int after[2], ks_next[2] = {}, vs_next[2] = {};
            ids_of(step + 2 * kWaves, after);   // (scalar loads, in time for the loads that follow them)
            scales_of(k_scale, next, ks_next);
            scales_of(v_scale, next, vs_next);
            // Keys are on their way from this step's scores to the next one's, values from the end of one step to the middle of the next.
            put(in_k, k_tile, ks);
            if constexpr (FP8) {
                if (more) bring(k_base, next, k_tile, in_k);
            } else {
                wait_loads<2 * LOADS>();   // all but the values, which were asked for last
            }
            wave_lds_fence();
            float16v x;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k_tile[r32][(2 * k + half) ^ turn32]), q[k], x, 0, 0, 0);
            wave_lds_fence();
            if constexpr (!FP8) {
                if (more) bring(k_base, next, k_tile, in_k);
            }
            // values: what stands behind the last token is of no one, and one that is not finite is taken out of the product, in which it would reach every row (0 * inf), and
            // added to the rows that see it
            put(in_v, v_tile, vs);
            if constexpr (FP8) {
                if (more) bring(v_base, next, v_tile, in_v);
            }
            bool odd = false;
            if (step >= full) {
                const int left = u.kv_len - step * kKeys;
                if constexpr (!FP8) wait_loads<0>();
                wave_lds_fence();
#pragma unroll
                for (int i = 0; i < kKeys * PIECES / 64; ++i) {
                    const int key = (i * 64 + lane) / PIECES, p = (i * 64 + lane) % PIECES;
                    u32x4 w = v_tile[key][p];
                    bool change = key >= left;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (key >= left) w[j] = 0u;
                        if ((w[j] & 0x7f80u) == 0x7f80u) { w[j] &= 0xffff0000u; odd = change = true; }
                        if ((w[j] & 0x7f800000u) == 0x7f800000u) { w[j] &= 0xffffu; odd = change = true; }
                    }
                    if (change) v_tile[key][p] = w;
                }
            }
            // The largest score, and the weights.  Scales of e4m3 blocks count by their fractions here (the rest of them is in what LDS holds): those of keys with c, those of values as
            // part of the exponent, and out of the sums again.
            float kc[2], vl[2] = {}, vr[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                kc[j] = FP8 ? fraction(ks[j]) * c : c;
                if constexpr (FP8) {
                    vl[j] = __builtin_amdgcn_logf(fraction(vs[j]));
                    vr[j] = __builtin_amdgcn_rcpf(fraction(vs[j]));
                }
            }
            if (step >= full)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!(window >> (i / 4 * 8 + i % 4) & 1u)) x[i] = -__builtin_inff();
            float top[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[j] = x[8 * j];
#pragma unroll
                for (int i = 1; i < 8; ++i) top[j] = __builtin_elementwise_maximum(top[j], x[8 * j + i]);
                if constexpr (FP8) top[j] *= fraction(ks[j]);
            }
            const float up = __builtin_elementwise_maximum(m, max_of_halves(__builtin_elementwise_maximum(top[0], top[1])));
            // Of references so large that a rounded one and the scale's product with the largest score may be far apart, differences are taken before the scale is applied.
            const bool far = __ballot(!(fabsf(up * c) < kFar || up == kChunkNoMax)) != 0;
            const float down = up == m ? 1.0f : __builtin_amdgcn_exp2f(far ? (m - up) * c : m * c - up * c);
            if (__ballot(up != m)) {
                l *= down;
                used *= down;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= down;
            }
            m = up;
            if (__builtin_expect(far, 0)) {
#pragma clang fp contract(off)   // (a score is rounded before the reference, which is one of them, is taken off)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f((FP8 ? x[i] * fraction(ks[i / 8]) - m : x[i] - m) * c + vl[i / 8]);
            } else {
                const float mc = fmaxf(m * c, kChunkNoMax);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], kc[i / 8], FP8 ? vl[i / 8] - mc : -mc));
            }
            bf16x8 p[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float part = 0.f, part_used = 0.f;
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    part += x[j * 8 + i];
                    part += x[j * 8 + i + 1];
                    w[i / 2] = pack_bf16(x[j * 8 + i], x[j * 8 + i + 1]);
                    part_used = pair_sum(w[i / 2], part_used);
                }
                l = FP8 ? __builtin_fmaf(part, vr[j], l) : l + part;
                used = FP8 ? __builtin_fmaf(part_used, vr[j], used) : used + part_used;
                p[j] = __builtin_bit_cast(bf16x8, w);
            }
            if constexpr (!FP8) {   // all but the next keys
                if (more) wait_loads<2 * LOADS>();
                else wait_loads<0>();
            }
            wave_lds_fence();
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    s16x4 vv[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int key = j * 16 + r * 8 + half * 4 + i16 / 4, el = d * 32 + (group & 1) * 16 + i16 % 4 * 4;
                        const auto *at = reinterpret_cast<const char *>(&v_tile[key][(el / 8) ^ turn<D>(key & 15)]) + el % 8 * 2;
                        vv[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at));
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(vv[0], vv[1], 0, 1, 2, 3, 4, 5, 6, 7)), p[j], o[d], 0, 0, 0);
                }
            wave_lds_fence();
            if (__builtin_expect(__ballot(odd) != 0, 0)) {
                for (int pos = step * kKeys; pos < min((step + 1) * kKeys, u.kv_len); ++pos) {
                    if (!(tree_window(mask, a.mask_words, u.q_len, pos - ctx) & 1u)) continue;
                    const int64_t block = (int64_t)chunk_block(a, block_table[(int64_t)b * a.max_blocks + pos / kTile]) * a.num_kv_heads + g, at0 = (block * kTile + pos % kTile) * D + half * 4;
                    const float scale = FP8 ? v_scale[block] : 1.f;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float4v four = load4<FP8>(a.v, at0 + d * 32 + i / 4 * 8);
                            const float v = FP8 ? four[i % 4] * scale : four[i % 4];
                            if (!__builtin_isfinite(v)) o[d][i] += v;
                        }
                }
            }
            if (more) {
                if constexpr (!FP8) bring(v_base, next, v_tile, in_v);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ks[j] = ks_next[j];
                    vs[j] = vs_next[j];
                    next[j] = after[j];
                }
            }
        }
        // ---- the wavefronts' sums joined ----
        l = sum_of_halves(l);
        used = sum_of_halves(used);
        const int parts = min(steps - first, kWaves);
        if (half == 0) {
            sh_m[wave][r32] = m;
            sh_l[wave][r32] = l;
            sh_used[wave][r32] = used;
        }
        if (wave < parts) {
            // a row's fours of d stand at place four ^ row, so that the lanes' rows fill all banks
            float4v *out = reinterpret_cast<float4v *>(r32 < kRows / 2 ? &k_tile : &v_tile);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    out[r32 % (kRows / 2) * (D / 4) + ((d * 8 + j * 2 + half) ^ (r32 & (D / 4 - 1)))] = float4v{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
        }
        __syncthreads();
        constexpr int FOURS = kRows * D / 4 / (64 * kWaves);   // of a row's d to a lane
        const int row = tid / (D / 4 / FOURS), four0 = tid % (D / 4 / FOURS) * FOURS, no = t * kRows + row;
        float M = kChunkNoMax, L = 0.f, U = 0.f;
        float4v sum[FOURS] = {};
        for (int w = 0; w < parts; ++w) M = __builtin_elementwise_maximum(M, sh_m[w][row]);
        for (int w = 0; w < parts; ++w) {
            const float f = __builtin_amdgcn_exp2f((sh_m[w][row] - M) * c);
            L += f * sh_l[w][row];
            U += f * sh_used[w][row];
#pragma unroll
            for (int j = 0; j < FOURS; ++j)
                sum[j] += f * reinterpret_cast<const float4v *>(row < kRows / 2 ? &k_tiles[w] : &v_tiles[w])[row % (kRows / 2) * (D / 4) + ((four0 + j) ^ (row & (D / 4 - 1)))];
        }
        if (!whole && no < rows) {
            const int64_t slot = (((int64_t)b * how.splits + split) * how.tiles + t) * a.num_kv_heads + g;
            const float level = U > 0.f ? L / U : 1.0f;   // (the merge divides by the sum of the weights)
            float4v *po = reinterpret_cast<float4v *>(a.part_o) + (slot * kRows + row) * (D / 4) + four0;
#pragma unroll
            for (int j = 0; j < FOURS; ++j) po[j] = sum[j] * level;
            if (four0 == 0) {
                float *ml = a.part_ml + (slot * kRows + row) * 2;
                ml[0] = M;
                ml[1] = L;
            }
        } else if (no < rows) {
            const int64_t at = (int64_t)(u.q0 + no / G) * a.num_q_heads + g * G + no % G;
            const float r = U > 0.f ? 1.0f / U : U == 0.f ? 0.f : U;   // (a row that sees nothing: zeros; NaN stays)
#pragma unroll
            for (int j = 0; j < FOURS; ++j) chunk_store4<SS_BF16>(a.out, at * D + (four0 + j) * 4, sum[j] * r);
            if (a.lse && four0 == 0) a.lse[at] = L == 0.f ? -__builtin_inff() : (M * c + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
        }
        __syncthreads();   // (the next tile's keys come to where these stood)
    }
}

// The splits of a tile joined: a lane has four of a row's d.  grid: KV heads * tiles * batch
constexpr int kMergeThreads = 256;

template <int D>
__global__ __launch_bounds__(kMergeThreads) void tree_unit_merge_kernel(ChunkArgs a, TreeUnitChoice how)
{
    constexpr int PARTS = kRows * D / 4 / kMergeThreads;   // workgroups to a tile
    int at_wg = blockIdx.x;
    const int part = at_wg % PARTS;
    at_wg /= PARTS;
    const int g = at_wg % a.num_kv_heads;
    at_wg /= a.num_kv_heads;
    const int t = at_wg % how.tiles, b = at_wg / how.tiles;
    ChunkUnit<kRows, kKeys, true> u;
    u.set(a, uniform(a.q_indptr[b]), uniform(a.q_indptr[b + 1]), uniform(a.kv_len[b]), 0);
    const int e = part * kMergeThreads + threadIdx.x, row = e / (D / 4), four = e % (D / 4), n = t * kRows + row;
    if (n >= u.q_len * u.G) return;
    const int all_steps = (int)(((unsigned)u.kv_len + kKeys - 1) / kKeys), each = split_steps(all_steps, how.splits);
    const int parts = all_steps > 0 ? (all_steps + each - 1) / each : 1;
    const float c = fmaxf(a.sm_scale * 1.4426950408889634f, 0x1p-126f);
    float M = kChunkNoMax, L = 0.f;
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    auto slot_of = [&](int split) { return ((((int64_t)b * how.splits + split) * how.tiles + t) * a.num_kv_heads + g) * kRows + row; };
    constexpr int AHEAD = 4;   // pieces asked for at a time
    for (int s0 = 0; s0 < parts; s0 += AHEAD) {
        float m[AHEAD], l[AHEAD];
        float4v x[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t slot = slot_of(min(s0 + i, parts - 1));
            m[i] = a.part_ml[slot * 2];
            l[i] = a.part_ml[slot * 2 + 1];
            x[i] = reinterpret_cast<const float4v *>(a.part_o)[slot * (D / 4) + four];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (s0 + i >= parts) break;
            const float up = __builtin_elementwise_maximum(M, m[i]), down = M == up ? 1.0f : __builtin_amdgcn_exp2f((M - up) * c), f = m[i] == up ? 1.0f : __builtin_amdgcn_exp2f((m[i] - up) * c);
            M = up;
            L = L * down + l[i] * f;
            sum = sum * down + x[i] * f;
        }
    }
    const int64_t at = (int64_t)(u.q0 + n / u.G) * a.num_q_heads + g * u.G + n % u.G;
    const float r = L > 0.f ? 1.0f / L : L == 0.f ? 0.f : L;
    chunk_store4<SS_BF16>(a.out, at * D + four * 4, sum * r);
    if (a.lse && four == 0) a.lse[at] = L == 0.f ? -__builtin_inff() : (M * c + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

template <int D, bool FP8>
int32_t launch(const ChunkArgs &a, const TreeUnitChoice &how, hipStream_t stream)
{
    const unsigned tiles = (unsigned)a.batch * how.tiles * a.num_kv_heads;
    hipLaunchKernelGGL((tree_unit_kernel<D, FP8>), dim3(tiles * how.splits), dim3(64 * kWaves), 0, stream, a, how, a.block_table, a.k_scale, a.v_scale);
    SS_HIP_CHECK(hipGetLastError(), "launch tree_unit_kernel");
    if (how.splits == 1) return SS_OK;
    hipLaunchKernelGGL(tree_unit_merge_kernel<D>, dim3(tiles * (kRows * D / 4 / kMergeThreads)), dim3(kMergeThreads), 0, stream, a, how);
    SS_HIP_CHECK(hipGetLastError(), "launch tree_unit_merge_kernel");
    return SS_OK;
}

}  // namespace

int32_t tree_unit_launch(const ChunkArgs &a, const TreeUnitChoice &how, hipStream_t stream)
{
    const bool fp8 = a.kv_dtype == SS_FP8_E4M3;
    if (a.head_dim == 128) return fp8 ? launch<128, true>(a, how, stream) : launch<128, false>(a, how, stream);
    return fp8 ? launch<64, true>(a, how, stream) : launch<64, false>(a, how, stream);
}

}  // namespace ss
