// Attention of a chunk of new tokens on the bf16 matrix cores: bf16 queries over bf16 or e4m3 caches, heads of 64 or 128, any grouping.
//
// A workgroup of four wavefronts takes a share (chunk_plan.h) of 128 NB query rows of a KV head, NB blocks of 32 to a wavefront.  32 keys at a time,
//   S^T[key][row]  = K[key][:] . Q[row][:]       v_mfma_f32_32x32x16_bf16, queries in registers
//   O^T[d][row]   += V^T[d][key] P^T[key][row]    the same shape; P is taken straight from the accumulators of S^T, V^T by transposing LDS reads
// so that a lane holds one row: maximum, sum and rescaling of the softmax need no exchange but with the lane that has the row's other keys.
#include <type_traits>

#include "chunk_merge.h"

namespace ss {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// How far (in powers of two) a row's scores may rise above the reference of its exponentials before the sums are rescaled.
constexpr float kLag = 6.0f;

__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    const float2v v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <bool HI>
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t w)   // exact
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}
// The largest of three, or NaN (the other kind of maximum costs an instruction more for each operand that may be a signalling NaN).
__device__ __forceinline__ float max3(float x, float y, float z) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z); }
// What the lane of the row's other keys has, joined.
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}
// Waits for this wavefront's LDS accesses, with LOADS also for what it brings into LDS, then for the others.
template <bool LOADS>
__device__ __forceinline__ void team_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(LOADS ? 0x0070 : 0xc07f);   // vmcnt(0) lgkmcnt(0) | lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int kKeys = 32;    // keys that are taken at a time, two cache blocks
constexpr int kPairKeys = 2 * kKeys;

// 64 keys or values in LDS, rows of D bf16 in pieces of 16 bytes.  Piece c of row t stands at place c ^ turn(t): 16 rows' pieces
// of equal c fill all banks (scores), and so do four rows' pieces 4 n .. 4 n + 3 (transposing reads of values).
template <int D>
struct Tile {
    u32x4 w[kPairKeys][D / 8];
};
template <int D>
__device__ __forceinline__ int turn(int t)
{
    return D == 128 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3);
}

template <int D, bool FP8, int NB>
__global__ __launch_bounds__(64 * kWaves, NB == 2 ? 1 : 2) void chunk_kernel(ChunkArgs a, const int32_t *__restrict__ block_table,
                                                                             const float *__restrict__ k_scale, const float *__restrict__ v_scale)
{
    // (table and scales come in as no-alias arguments of their own, so that they are scalar loads)
    constexpr int ROWS = 128 * NB, KS = D / 16, DB = D / 32, PIECES = D / 8;
    constexpr int BLOCK_BYTES = kTile * D * (FP8 ? 1 : 2), LOADS = BLOCK_BYTES / (64 * 16);   // 16-byte loads of a lane for a cache block
    // Variables of their own: a tile's reads then do not wait for what is on its way into another one.
    __shared__ Tile<D> k_even, k_odd, v_even, v_odd;   // steps 3, 4, 7, 8, ..; 1, 2, 5, 6, ..; 0, 1, 4, 5, ..; 2, 3, 6, 7, .. (from the first)
    __shared__ int odd_flags[2][kWaves];
    const int g = blockIdx.x % a.num_kv_heads, item = blockIdx.x / a.num_kv_heads;
    ChunkShare s;
    const bool any = chunk_share<ROWS>(a, item, s);
    if (a.cap > 0 && blockIdx.x == 0 && threadIdx.x == 0) a.head[0] = s.cuts;
    if (!any) return;
    chunk_record<ROWS>(a, s, g);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, half = lane >> 5;
    const int G = a.num_q_heads / a.num_kv_heads;
    const int rows = s.q_len * G, ctx = s.kv_len - s.q_len;
    const int n_first = s.tile * ROWS + wave * 32 * NB;
    int lim[NB];                                                        // the last position this lane's rows see
#pragma unroll
    for (int e = 0; e < NB; ++e) lim[e] = ctx + min(n_first + e * 32 + r32, rows - 1) / G;
    // In steps of 32 keys: the share's, up to where all rows of the wavefront see everything, from where none sees anything; all rows of the tile
    const int first = s.s0 * (kStepKeys / kKeys);
    const int end = min(s.s1 * (kStepKeys / kKeys), (max(ctx + min((s.tile + 1) * ROWS - 1, rows - 1) / G + 1, 0) + kKeys - 1) / kKeys);
    const int all = max((ctx + min(n_first, rows - 1) / G + 1) / kKeys, 0);
    const int none = n_first < rows ? min((max(ctx + min(n_first + 32 * NB - 1, rows - 1) / G + 1, 0) + kKeys - 1) / kKeys, end) : 0;
    const int full = max((ctx + s.tile * ROWS / G + 1) / kKeys, 0);
    const float c = a.sm_scale * kLog2e;

    bf16x8 q[NB][KS];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
        const int n = n_first + e * 32 + r32;
        const char *src = static_cast<const char *>(a.q) + ((int64_t)(s.q0 + min(n, rows - 1) / G) * a.q_stride + (int64_t)(g * G + n % G) * D + half * 8) * 2;
        const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            u32x4 w = zero;
            if (n < rows) w = *reinterpret_cast<const u32x4 *>(src + k * 32);
            q[e][k] = __builtin_bit_cast(bf16x8, w);
        }
    }

    typedef const __attribute__((address_space(4))) int32_t *scalar_ints;       // (read with scalar loads, whatever else is written meanwhile)
    typedef const __attribute__((address_space(4))) float *scalar_floats;
    const scalar_ints table = (scalar_ints)(uintptr_t)(block_table + (int64_t)s.b * a.max_blocks);
    const scalar_floats k_scales = (scalar_floats)(uintptr_t)k_scale, v_scales = (scalar_floats)(uintptr_t)v_scale;
    const int last_block = (int)(((unsigned)s.kv_len + kTile - 1) / kTile) - 1;
    // block j of a step (the last block again where there is none: what stands there is masked)
    auto block_id = [&](int step, int j) __attribute__((always_inline)) { return table[min(step * 2 + j, last_block)]; };
    auto block_of = [&](const void *cache, int id) __attribute__((always_inline)) { return static_cast<const char *>(cache) + ((int64_t)id * a.num_kv_heads + g) * BLOCK_BYTES; };

    // ---- a cache block into a quarter of a tile ----
    // bf16: straight into LDS, where a lane's 16 bytes stand behind those of the lane in front of it: the lanes read the pieces in the order of their places.
    // e4m3: through registers, turned into bf16.
    int piece_at[FP8 ? 1 : LOADS];
    if constexpr (!FP8)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = i * 64 + lane, t = p / PIECES;
            piece_at[i] = (t * PIECES + ((p % PIECES) ^ turn<D>(t))) * 16;
        }
    u32x4 in_k[FP8 ? LOADS : 1], in_v[FP8 ? LOADS : 1];
    auto bring = [&](const void *cache, int id, Tile<D> &tile, int quarter, u32x4 (&in)[FP8 ? LOADS : 1]) __attribute__((always_inline)) {
        const char *p = block_of(cache, id);
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) in[i] = *reinterpret_cast<const u32x4 *>(p + (i * 64 + lane) * 16);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) const void *)(p + piece_at[i]),
                                                 (__attribute__((address_space(3))) void *)(&tile.w[quarter * kTile + i * 64 / PIECES][0]), 16, 0, 0);
        }
    };
    auto put = [&](const u32x4 (&in)[FP8 ? LOADS : 1], Tile<D> &tile, int quarter) __attribute__((always_inline)) {
        if constexpr (FP8)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int el = (i * 64 + lane) * 16, t = el / D, col = el % D / 8;   // first element: row, piece
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        w[2 * j] = fp8x2_to_bf16x2<false>(in[i][2 * p + j]);
                        w[2 * j + 1] = fp8x2_to_bf16x2<true>(in[i][2 * p + j]);
                    }
                    tile.w[quarter * kTile + t][(col + p) ^ turn<D>(t)] = w;
                }
            }
    };
    // A step that some row of the tile does not see all of, once this wavefront's block of its values is in LDS.  What stands behind the last token is of no
    // one; a value that is not finite is taken out of the product, in which it would reach every row (0 * inf), and added to the rows that see it.
    auto clean = [&](int step, Tile<D> &tile, int pair) __attribute__((always_inline)) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < kTile * PIECES / 64; ++i) {
            const int p = i * 64 + lane, t = p / PIECES;
            u32x4 &at = tile.w[wave * kTile + t][p % PIECES];
            u32x4 w = at;
            const bool dead = step * kKeys + (wave & 1) * kTile + t >= s.kv_len;
            bool changed = dead;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t x = dead ? 0u : w[j];
                if ((x & 0x7f80u) == 0x7f80u) { x &= 0xffff0000u; changed = odd = true; }
                if ((x & 0x7f800000u) == 0x7f800000u) { x &= 0xffffu; changed = odd = true; }
                w[j] = x;
            }
            if (changed) at = w;
        }
        odd_flags[pair][wave] = __ballot(odd) != 0;
    };

    float m[NB], l[NB];
    float16v o[NB][DB];
#pragma unroll
    for (int e = 0; e < NB; ++e) {
        m[e] = kChunkNoMax;
        l[e] = 0.f;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[e][b][i] = 0.f;
    }

    const int turn32 = turn<D>(r32 & 15), group = lane >> 4, i16 = lane & 15;
    auto read_keys = [&](const Tile<D> &tile, int part, bf16x8 (&kf)[KS]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < KS; ++k) kf[k] = __builtin_bit_cast(bf16x8, tile.w[part * kKeys + r32][(2 * k + half) ^ turn32]);
    };
    // values as the other operand: a contraction takes 16 keys, the lane's eight of them in the order of its scores
    auto read_values = [&](const Tile<D> &tile, int part, bf16x8 (&vf)[2][DB]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int b = 0; b < DB; ++b) {
                s16x4 vv[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int t = k * 16 + r * 8 + half * 4 + i16 / 4, d = b * 32 + (group & 1) * 16 + i16 % 4 * 4;
                    const auto *p = reinterpret_cast<const char *>(&tile.w[part * kKeys + t][(d / 8) ^ turn<D>(t & 15)]) + d % 8 * 2;
                    vv[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p));
                }
                vf[k][b] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vv[0], vv[1], 0, 1, 2, 3, 4, 5, 6, 7));
            }
    };
    // scores of 32 keys: the lane has row r32 of each block of rows and keys 8 (i / 4) + 4 half + i % 4
    auto scores = [&](const bf16x8 (&kf)[KS], float16v (&x)[NB]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < NB; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[e][i] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < NB; ++e) x[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], q[e][k], x[e], 0, 0, 0);
    };
    // What scores need before their exponentials: scales, mask, and a reference that follows the largest score when that has risen by kLag.
    float vs[2] = {1.f, 1.f};
    auto settle = [&](auto fast, int step, float16v (&x)[NB]) __attribute__((always_inline)) {
        if constexpr (FP8) {   // one scale to 16 keys: they are in eight accumulators
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t tile = (int64_t)block_id(step, j) * a.num_kv_heads + g;
                const float ks = k_scales[tile] * c;
                vs[j] = v_scales[tile];
#pragma unroll
                for (int e = 0; e < NB; ++e)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[e][j * 8 + i] *= ks;
            }
        }
        if (!decltype(fast)::value && step >= all) {
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const int seen = lim[e] - step * kKeys - 4 * half;    // keys up to this one, counted from the lane's first
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i / 4 * 8 + i % 4 > seen) x[e][i] = -__builtin_inff();
            }
        }
        float top[NB];
        bool rise = false;
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            float t = max3(x[e][0], x[e][1], x[e][2]);
#pragma unroll
            for (int i = 3; i < 15; i += 2) t = max3(t, x[e][i], x[e][i + 1]);
            t = max_of_halves(__builtin_elementwise_maximum(t, x[e][15]));
            top[e] = FP8 ? t : t * c;
            rise = rise || top[e] > m[e] + kLag;
        }
        if (__ballot(rise)) {
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const float up = fmaxf(m[e], top[e]), down = __builtin_amdgcn_exp2f(m[e] - up);
                m[e] = up;
                l[e] *= down;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[e][b][i] *= down;
            }
        }
    };
    auto weights = [&](float16v &x, int e, bf16x8 (&pk)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float p = __builtin_amdgcn_exp2f(FP8 ? x[i] - m[e] : __builtin_fmaf(x[i], c, -m[e]));
            l[e] += p;
            x[i] = FP8 ? p * vs[i / 8] : p;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_bf16(x[k * 8 + 2 * j], x[k * 8 + 2 * j + 1]);
            pk[k] = __builtin_bit_cast(bf16x8, w);
        }
    };
    auto output = [&](const bf16x8 (&vf)[2][DB], const bf16x8 (&pk)[2], int e) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int b = 0; b < DB; ++b) o[e][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k][b], pk[k], o[e][b], 0, 0, 0);
    };
    auto add_odd = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < NB; ++e)
            for (int pos = t * kKeys; pos < min((t + 1) * kKeys, lim[e] + 1); ++pos) {
                const int64_t at0 = (((int64_t)table[pos / kTile] * a.num_kv_heads + g) * kTile + pos % kTile) * D + half * 4;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int64_t at = at0 + b * 32 + i / 4 * 8 + i % 4;
                        float v;
                        if constexpr (FP8) v = __builtin_amdgcn_cvt_f32_fp8((int)static_cast<const uint8_t *>(a.v)[at], 0);
                        else v = __uint_as_float((uint32_t) static_cast<const uint16_t *>(a.v)[at] << 16);
                        if (!__builtin_isfinite(v)) o[e][b][i] += v;
                    }
            }
    };

    // Step t: the next step's scores y between the exponentials of this one's, x, then the output, between what y needs before its exponentials.
    // Operands come from LDS half a step ahead of their use, keys a step ahead of values.  Every second step (ODD, counted from the first) the wavefronts meet
    // once; from there on 64 keys (of steps t + 4 and t + 5) and 64 values (t + 3, t + 4), one block each to a wavefront, are on their way that are needed
    // after the next meeting.
    // FAST: every row of the tile sees all that is in LDS (what would be read behind the share's last step is read as well, from the last block).
    // k_read: the tile of step t + 2's keys, v_read: of step t's values; k_next, v_next: those that are free after the meeting.
    bf16x8 kf[KS];
    auto step_of = [&](auto fast, auto parity, int t, float16v (&x)[NB], float16v (&y)[NB], Tile<D> &k_read, Tile<D> &v_read, Tile<D> &k_next, Tile<D> &v_next,
                       int pair) __attribute__((always_inline)) {
        constexpr bool FAST = decltype(fast)::value, ODD = decltype(parity)::value;
        const bool live = FAST || t < none, next = FAST || t + 1 < none, next2 = FAST || t + 2 < none;
        bf16x8 vf[2][DB], pk[2];
        if (live) read_values(v_read, ODD, vf);
        if (next) scores(kf, y);
        if (live) weights(x[0], 0, pk);
        if constexpr (ODD) {
            if constexpr (FP8) put(in_v, pair ? v_even : v_odd, wave);
            const int vstep = t + 1 + (wave >> 1);   // of the values that this wavefront has brought
            if (!FAST && vstep >= full) {
                if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
                clean(vstep, pair ? v_even : v_odd, pair ^ 1);
            }
            team_barrier<!FP8>();
            bring(a.k, block_id(t + 4, wave), k_next, wave, in_k);
            bring(a.v, block_id(t + 3, wave), v_next, wave, in_v);
        } else {
            put(in_k, pair ? k_odd : k_even, wave);
        }
        if (next2) read_keys(k_read, !ODD, kf);
        if (live) {
            output(vf, pk, 0);
            if constexpr (NB == 2) {
                bf16x8 pk1[2];
                weights(x[1], 1, pk1);
                output(vf, pk1, 1);
            }
            if (!FAST && t >= full && (odd_flags[pair][2 * ODD] | odd_flags[pair][2 * ODD + 1])) add_odd(t);
        }
        if (next) settle(fast, t + 1, y);
    };
    auto four_steps = [&](auto fast, int t, float16v (&x)[NB], float16v (&y)[NB]) __attribute__((always_inline)) {
        constexpr bool FAST = decltype(fast)::value;
        step_of(fast, std::false_type{}, t, x, y, k_odd, v_even, k_even, v_even, 0);
        if (FAST || t + 1 < end) step_of(fast, std::true_type{}, t + 1, y, x, k_even, v_even, k_odd, v_even, 0);
        if (FAST || t + 2 < end) step_of(fast, std::false_type{}, t + 2, x, y, k_even, v_odd, k_odd, v_odd, 1);
        if (FAST || t + 3 < end) step_of(fast, std::true_type{}, t + 3, y, x, k_odd, v_odd, k_even, v_odd, 1);
    };

    if (first < end) {
        // keys of the first three steps, values of the first two
        u32x4 in_0[FP8 ? LOADS : 1];
        if (wave < 2) bring(a.k, block_id(first, wave), k_even, 2 + wave, in_0);
        bring(a.k, block_id(first + 1, wave), k_odd, wave, in_k);
        bring(a.v, block_id(first, wave), v_even, wave, in_v);
        if (wave < 2) put(in_0, k_even, 2 + wave);
        put(in_k, k_odd, wave);
        put(in_v, v_even, wave);
        if (first + (wave >> 1) >= full) {
            if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
            clean(first + (wave >> 1), v_even, 0);
        }
        team_barrier<!FP8>();
        float16v x[NB], y[NB];
        if (first < none) {
            read_keys(k_even, 1, kf);
            scores(kf, x);
            settle(std::false_type{}, first, x);
        }
        if (first + 1 < none) read_keys(k_odd, 0, kf);
        team_barrier<false>();   // (new keys come to where these were)
        bring(a.k, block_id(first + 3, wave), k_even, wave, in_k);
        bring(a.v, block_id(first + 2, wave), v_odd, wave, in_v);
        int t = first;
        if (none > 0)   // (a wavefront without rows only brings keys and values)
            for (const int fast_end = min(full, end) - 5; t < fast_end; t += 4) four_steps(std::true_type{}, t, x, y);
        for (; t < end; t += 4) four_steps(std::false_type{}, t, x, y);
        if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): nothing is on its way into LDS when the workgroup ends
    }

#pragma unroll
    for (int e = 0; e < NB; ++e) {
        const int n = n_first + e * 32 + r32;
        const float sum = sum_of_halves(l[e]);
        if (s.pieces > 1) {
            const int64_t part = (int64_t)s.slot * a.num_kv_heads + g;
            float4v *po = reinterpret_cast<float4v *>(a.part_o) + part * (ROWS * D / 4) + (wave * NB + e) * (32 * D / 4) + lane;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) po[(b * 4 + j) * 64] = float4v{o[e][b][4 * j], o[e][b][4 * j + 1], o[e][b][4 * j + 2], o[e][b][4 * j + 3]};
            if (half == 0) {
                float *ml = a.part_ml + (part * ROWS + (wave * NB + e) * 32 + r32) * 2;
                ml[0] = m[e];
                ml[1] = sum;
            }
        } else if (n < rows) {
            const int64_t at = (int64_t)(s.q0 + n / G) * a.num_q_heads + g * G + n % G;
            const float r = sum > 0.f ? 1.0f / sum : sum == 0.f ? 0.f : sum;   // (a row that sees nothing: zeros; NaN stays)
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    chunk_store4<SS_BF16>(a.out, at * D + b * 32 + j * 8 + half * 4,
                                          float4v{o[e][b][4 * j], o[e][b][4 * j + 1], o[e][b][4 * j + 2], o[e][b][4 * j + 3]} * r);
            if (a.lse && half == 0) a.lse[at] = sum == 0.f ? -__builtin_inff() : (m[e] + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
}

template <int D, bool FP8, int NB>
int32_t launch(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream)
{
    constexpr int ROWS = 128 * NB;
    const int64_t shares = s.tiles + s.cap / a.num_kv_heads;
    hipLaunchKernelGGL((chunk_kernel<D, FP8, NB>), dim3((unsigned)(shares * a.num_kv_heads)), dim3(64 * kWaves), 0, stream, a, a.block_table, a.k_scale, a.v_scale);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_kernel");
    if (s.cap >= 2 * a.num_kv_heads) {
        const int64_t fit = s.cap / (2 * a.num_kv_heads), cuts = s.tiles < fit ? s.tiles : fit;
        hipLaunchKernelGGL((chunk_merge_kernel<ROWS, 32, D, SS_BF16>), dim3((unsigned)(cuts * a.num_kv_heads * (ROWS * D / 1024))), dim3(256), 0, stream, a);
        SS_HIP_CHECK(hipGetLastError(), "launch chunk_merge_kernel");
    }
    return SS_OK;
}

template <int D, bool FP8>
int32_t launch_rows(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream)
{
    return s.rows == 256 ? launch<D, FP8, 2>(a, s, stream) : launch<D, FP8, 1>(a, s, stream);
}

}  // namespace

bool chunk_mfma_supported(int head_dim, int kv_dtype, int q_dtype)
{
    return (head_dim == 64 || head_dim == 128) && q_dtype == SS_BF16 && (kv_dtype == SS_BF16 || kv_dtype == SS_FP8_E4M3);
}

int32_t chunk_mfma_launch(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream)
{
    const bool fp8 = a.kv_dtype == SS_FP8_E4M3;
    if (a.head_dim == 128) return fp8 ? launch_rows<128, true>(a, s, stream) : launch_rows<128, false>(a, s, stream);
    return fp8 ? launch_rows<64, true>(a, s, stream) : launch_rows<64, false>(a, s, stream);
}

}  // namespace ss
