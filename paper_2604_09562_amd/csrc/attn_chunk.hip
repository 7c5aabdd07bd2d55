// Attention of a chunk of new tokens on the bf16 matrix cores: bf16 queries over bf16 or e4m3 caches, heads of 64 or 128, any grouping.
//
// A workgroup of four wavefronts takes tiles of 256 query rows of a KV head, piece by piece (chunk_plan.h), two blocks of 32 rows to a wavefront.
// 32 keys at a time,
//   S^T[key][row]  = K[key][:] . Q[row][:]       v_mfma_f32_32x32x16_bf16, queries in registers
//   O^T[d][row]   += V^T[d][key] P^T[key][row]    the same shape; P is taken straight from the accumulators of S^T, V^T by transposing LDS reads
// so that a lane holds one row: maximum, sum and rescaling of the softmax need no exchange but with the lane that has the row's other keys.  Weights are rounded
// to bf16 for the second product, by half a step (2^-8) at most, about as much as the outputs are; scores, sums and outputs are fp32.
//
// What bounds it: one wavefront to a SIMD, so every instruction beside the matrix instructions (1024 of a step's cycles) takes issue slots of its own.  A step of
// a wavefront is 32 matrix instructions, 32 exponentials (two slots each), as many multiply-adds and additions, and half as many roundings and sums of them:
// about 1750 cycles.  Therefore
// - the next step's scores are made between this step's exponentials (913 -> 1020 TFLOP/s on 4096 tokens behind 12288), all in a fixed order (1100 -> 1140);
// - two blocks of rows to a wavefront, so that keys and values are read from LDS once for 64 rows, bf16 ones brought there without registers, and one meeting of
//   the wavefronts for 64 keys (1020 -> 1100);
// - sums follow a rising maximum only when it has risen by 2^kLag: weights up to 2^16 are exact enough in bf16 and far from fp32's end.
// Outputs are divided by the sum of the weights as rounded, a sum of its own (5 %): where a few weights are most of it their roundings cancel, and the error
// against 64 bits is 1.2 of what rounding the outputs costs instead of 1.4 (scores that spread by 1 to 4).  The log-sum-exp takes the sum of the weights
// themselves; calls that do not ask for it have a form without that sum (3 % faster).
// 900 .. 940 us there by card, 1.02 .. 1.07 PFLOP/s, where a large bf16 product of the library reaches 1.27 .. 1.36; 63 us for a prompt of 2048 tokens (32 heads over 8); e4m3 caches:
// 309 us, 768 TFLOP/s, for four requests of 200 .. 1000 tokens behind 1000 .. 6000 (64 heads over 8), their codes turned to bf16 on the way into LDS.
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
constexpr int NB = 2;                                  // blocks of 32 query rows to a wavefront
constexpr int ROWS = 32 * NB * kWaves;                // query rows of a tile
static_assert(ROWS == kChunkRows, "what launches and workspaces are sized by");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// How far (in powers of two) a row's scores may rise above the reference of its exponentials before the sums are rescaled.
constexpr float kLag = 16.0f;
// References beyond this (in powers of two) are taken care of apart: from 2^31 on the rounded reference and the scale's product with the largest score
// may be further apart than an exponential's range.
constexpr float kFar = 0x1p28f;
constexpr int kOddValues = 1;   // values that are not finite were taken out
constexpr int kFarRows = 2;     // a row's reference was beyond kFar

__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    const float2v v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// four consecutive elements of bf16 or e4m3, from a multiple of four
template <bool FP8>
__device__ __forceinline__ float4v load4(const void *base, int64_t i)
{
    if constexpr (FP8) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(base) + i);
        const float2v x = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), y = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        return float4v{x.x, x.y, y.x, y.y};
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(base) + i);
        return float4v{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
    }
}
// x and the two of a pair of bf16, added
__device__ __forceinline__ float pair_sum(uint32_t pair, float x)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), x, false);
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
template <int D>
__device__ __forceinline__ int turn(int t)
{
    return D == 128 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3);
}

template <int D, bool FP8, bool LSE>
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
    ChunkWalk<ROWS, kKeys, kChunkOpen> s;
    int begun = 0, begun_q0 = 0, begun_rows = 0, begun_row0 = 0;   // of the tile that the span begins and does not end
    for (bool any = s.begin(a, span); any; any = s.next(a)) {
        if (s.part == 2 * span + 1) {
            begun = s.pieces();
            begun_q0 = s.u.q0;
            begun_rows = s.u.q_len * s.u.G;
            begun_row0 = s.t * ROWS;
        }
        const int r32 = lane & 31, half = lane >> 5;
        const int G = a.num_q_heads / a.num_kv_heads;
        const int rows = s.u.q_len * G, ctx = s.u.kv_len - s.u.q_len;
        const int n_first = s.t * ROWS + wave * 32 * NB;
        int lim[NB];                                                        // the last position this lane's rows see
#pragma unroll
        for (int e = 0; e < NB; ++e) lim[e] = ctx + min(n_first + e * 32 + r32, rows - 1) / G;
        // In steps of 32 keys: the share's, and up to where all rows of the tile see everything
        const int first = s.s0, end = s.s1;
        const int full = max((ctx + s.t * ROWS / G + 1) / kKeys, 0);
        const float c = fmaxf(a.sm_scale * kLog2e, 0x1p-126f);
#pragma unroll
        for (int e = 0; e < NB; ++e) lim[e] = min(lim[e], end * kKeys - 1);   // (what a step reads behind the share is another one's)

        bf16x8 q[NB][KS];
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            const int n = n_first + e * 32 + r32;
            const char *src = static_cast<const char *>(a.q) + ((int64_t)(s.u.q0 + min(n, rows - 1) / G) * a.q_stride + (int64_t)(g * G + n % G) * D + half * 8) * 2;
            const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                u32x4 w = zero;
                if (n < rows) w = *reinterpret_cast<const u32x4 *>(src + k * 32);
                q[e][k] = __builtin_bit_cast(bf16x8, w);
            }
        }

        typedef const __attribute__((address_space(4))) int32_t *scalar_ints;       // (read with scalar loads, whatever else is written meanwhile)
        const scalar_ints table = (scalar_ints)(uintptr_t)(block_table + (int64_t)s.b * a.max_blocks);
        const scalar_ints k_scales = (scalar_ints)(uintptr_t)k_scale, v_scales = (scalar_ints)(uintptr_t)v_scale;
        const int last_block = (int)(((unsigned)s.u.kv_len + kTile - 1) / kTile) - 1;
        // block j of a step (the last block again where there is none: what stands there is masked).  Bounded where it is followed, not here, where that would wait for it.
        auto block_id = [&](int step, int j) __attribute__((always_inline)) { return table[min(step * 2 + j, last_block)]; };
        const uint32_t block_stride = (uint32_t)a.num_kv_heads * BLOCK_BYTES;
        const char *k_base = static_cast<const char *>(a.k) + (int64_t)g * BLOCK_BYTES, *v_base = static_cast<const char *>(a.v) + (int64_t)g * BLOCK_BYTES;

        // ---- a cache block into a quarter of a tile ----
        // bf16: straight into LDS, where a lane's 16 bytes stand behind those of the lane in front of it: the lanes read the pieces in the order of their places.
        // e4m3: through registers, turned into bf16, with the sign and the power of two of their scale, which bf16 holds exactly; NaN
        // all of them if it is not finite.
        uint32_t piece_at[FP8 ? 1 : LOADS];
        if constexpr (!FP8)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int p = i * 64 + lane, t = p / PIECES;
                piece_at[i] = (uint32_t)(t * PIECES + ((p % PIECES) ^ turn<D>(t))) * 16;
            }
        u32x4 in_k[FP8 ? LOADS : 1], in_v[FP8 ? LOADS : 1];
        // (a descriptor of its own for each block, so that a lane's place in it is all that the vector unit has to keep)
        auto block_at = [&](const char *cache, int id) __attribute__((always_inline)) {
            return cache + (uint64_t)(uint32_t)chunk_block(a, id) * block_stride;
        };
        auto bring_part = [&](const char *at, int i, Tile<D> &tile, int quarter, u32x4 (&in)[FP8 ? LOADS : 1]) __attribute__((always_inline)) {
            const __amdgpu_buffer_rsrc_t block = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, BLOCK_BYTES, 0x00020000);
            if constexpr (FP8)
                in[i] = __builtin_amdgcn_raw_buffer_load_b128(block, (i * 64 + lane) * 16, 0, 0);
#ifdef __HIP_DEVICE_COMPILE__   // (the host's pass does not know that this GPU brings 16 bytes at a time)
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(block, (__attribute__((address_space(3))) void *)(&tile.w[quarter * kTile + i * 64 / PIECES][0]), 16,
                                                         piece_at[i], 0, 0, 0);
#endif
        };
        auto bring = [&](const char *cache, int id, Tile<D> &tile, int quarter, u32x4 (&in)[FP8 ? LOADS : 1]) __attribute__((always_inline)) {
            const char *block = block_at(cache, id);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) bring_part(block, i, tile, quarter, in);
        };
        // part i of 2 LOADS
        auto put_part = [&](const u32x4 (&in)[FP8 ? LOADS : 1], int i, Tile<D> &tile, int quarter, int scale) __attribute__((always_inline)) {
            const uint32_t sign = (uint32_t)(scale >> 31) & 0x80808080u, nan = (scale & 0x7fffffff) >= kInfinity ? 0x7f7f7f7fu : 0u;
            const float power = __int_as_float(scale & kInfinity);
            const int el = (i / 2 * 64 + lane) * 16, t = el / D, col = el % D / 8;   // first element: row, piece
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t four = (in[i / 2][2 * (i % 2) + j] ^ sign) | nan;
                w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, power, false));
                w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, power, true));
            }
            tile.w[quarter * kTile + t][(col + i % 2) ^ turn<D>(t)] = w;
        };
        auto put = [&](const u32x4 (&in)[FP8 ? LOADS : 1], Tile<D> &tile, int quarter, int scale) __attribute__((always_inline)) {
            if constexpr (FP8)
#pragma unroll
                for (int i = 0; i < 2 * LOADS; ++i) put_part(in, i, tile, quarter, scale);
        };
        // A step that some row of the tile does not see all of, once this wavefront's block of its values is in LDS.  What stands behind the last token is of no
        // one; a value that is not finite is taken out of the product, in which it would reach every row (0 * inf), and added to the rows that see it.
        auto clean = [&](int step, Tile<D> &tile, int pair) __attribute__((always_inline)) {
            constexpr int N = kTile * PIECES / 64;
            const int left = s.u.kv_len - (step * kKeys + (wave & 1) * kTile);   // tokens of the block that there are
            u32x4 w[N];
            uint32_t carry = 0;                                                  // the sign bits of halves whose exponent is all ones
#pragma unroll
            for (int i = 0; i < N; ++i) {
                w[i] = tile.w[wave * kTile + (i * 64 + lane) / PIECES][(i * 64 + lane) % PIECES];
#pragma unroll
                for (int j = 0; j < 4; ++j) carry |= (w[i][j] & 0x7f807f80u) + 0x00800080u;
            }
            const bool found = __ballot((carry & 0x80008000u) != 0) != 0;
            bool odd = false;
            if (found || left < kTile) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = (i * 64 + lane) / PIECES;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t x = t >= left ? 0u : w[i][j];
                        if ((x & 0x7f80u) == 0x7f80u) { x &= 0xffff0000u; odd = true; }
                        if ((x & 0x7f800000u) == 0x7f800000u) { x &= 0xffffu; odd = true; }
                        w[i][j] = x;
                    }
                    tile.w[wave * kTile + t][(i * 64 + lane) % PIECES] = w[i];
                }
            }
            odd_flags[pair][wave] = __ballot(odd) ? kOddValues : 0;
        };

        int special = 0;                  // what the steps leave for their end: kOddValues, kFarRows
        float m[NB], l[NB], l_used[NB];   // reference, sum of the weights, sum of the weights as rounded
        float16v o[NB][DB];
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            m[e] = kChunkNoMax;
            l[e] = l_used[e] = 0.f;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[e][b][i] = 0.f;
        }

        const int turn32 = turn<D>(r32 & 15), group = lane >> 4, i16 = lane & 15;
        auto read_keys = [&](const Tile<D> &tile, int part, int k) __attribute__((always_inline)) {
            return __builtin_bit_cast(bf16x8, tile.w[part * kKeys + r32][(2 * k + half) ^ turn32]);
        };
        // values as the other operand: a contraction takes 16 keys, the lane's eight of them in the order of its scores
        auto read_values = [&](const Tile<D> &tile, int part, int k, int b) __attribute__((always_inline)) {
            s16x4 vv[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = k * 16 + r * 8 + half * 4 + i16 / 4, d = b * 32 + (group & 1) * 16 + i16 % 4 * 4;
                const auto *p = reinterpret_cast<const char *>(&tile.w[part * kKeys + t][(d / 8) ^ turn<D>(t & 15)]) + d % 8 * 2;
                vv[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p));
            }
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(vv[0], vv[1], 0, 1, 2, 3, 4, 5, 6, 7));
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
        // What scores need before their exponentials: scales (one to 16 keys: they are in eight accumulators), mask, the largest of each row, and a reference that
        // follows it when it has risen by kLag.  Scales count by their fractions here, from one to two: a masked score stays minus infinity, a weight of zero zero, and
        // no weight leaves the range of floats.  The rest of a scale is in what LDS holds.
        // The scale of values goes into the exponent: 2^(x - m) vs = 2^(x - (m - log2 vs)), and the sum over the values' block is divided by vs again.  That is two
        // instructions for eight weights instead of eight (336 -> 298 us for four requests of 200 .. 1000 tokens with the rest in LDS and scales asked for two steps ahead).
        float ks[2] = {c, c}, ks_next[2] = {c, c};                       // this step's, the next step's
        float vl[2] = {}, vl_next[2] = {}, vr[2] = {}, vr_next[2] = {};   // the scale of values: its logarithm, its inverse
        int k_raw[2] = {}, v_raw[2] = {};                                // and, as bits, those of the step behind it
        int sid[2] = {0, 0};                                             // and the blocks of the one behind that
        auto scale_of = [&](scalar_ints scales, int id) __attribute__((always_inline)) { return scales[(uint32_t)chunk_block(a, id) * (uint32_t)a.num_kv_heads + (uint32_t)g]; };
        auto fraction = [&](int scale) __attribute__((always_inline)) { return __int_as_float((scale & 0x7fffff) | 0x3f800000); };
        auto ask_scales = [&]() __attribute__((always_inline)) {
            if constexpr (FP8)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    k_raw[j] = scale_of(k_scales, sid[j]);
                    v_raw[j] = scale_of(v_scales, sid[j]);
                }
        };
        auto ask_blocks = [&](int step) __attribute__((always_inline)) {
            if constexpr (FP8) {
                sid[0] = block_id(step, 0);
                sid[1] = block_id(step, 1);
            }
        };
        auto take_key_scales = [&]() __attribute__((always_inline)) {
            if constexpr (FP8)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    ks_next[j] = __int_as_float(uniform(__float_as_int(fraction(k_raw[j]) * c)));
        };
        auto take_value_scales = [&]() __attribute__((always_inline)) {
            if constexpr (FP8)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    vl_next[j] = __int_as_float(uniform(__float_as_int(__builtin_amdgcn_logf(fraction(v_raw[j])))));
                    vr_next[j] = __int_as_float(uniform(__float_as_int(__builtin_amdgcn_rcpf(fraction(v_raw[j])))));
                }
        };
        auto step_scales = [&]() __attribute__((always_inline)) {
            if constexpr (FP8)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ks[j] = ks_next[j];
                    vl[j] = vl_next[j];
                    vr[j] = vr_next[j];
                }
        };
        // The largest of a row's 16 scores in the lane, in four parts for either eight; the scores are masked on the way.
        auto largest = [&](auto masked, int step, int e, float16v &x, int part, float (&top)[2]) __attribute__((always_inline)) {
            const int group = part / 4, lo = group * 8 + (part % 4 ? 2 * (part % 4) + 1 : 0), hi = group * 8 + (part % 4 < 3 ? 2 * (part % 4) + 3 : 8);
            if constexpr (decltype(masked)::value) {
                const int seen = lim[e] - step * kKeys - 4 * half;    // keys up to this one, counted from the lane's first
#pragma unroll
                for (int i = lo; i < hi; ++i)
                    if (i / 4 * 8 + i % 4 > seen) x[i] = -__builtin_inff();
            }
            if (part % 4 == 0) top[group] = max3(x[lo], x[lo + 1], x[lo + 2]);
            else top[group] = part % 4 < 3 ? max3(top[group], x[lo], x[lo + 1]) : __builtin_elementwise_maximum(top[group], x[lo]);
        };
        auto whole_row = [&](const float (&top)[2]) __attribute__((always_inline)) {
            if constexpr (FP8) return max_of_halves(__builtin_elementwise_maximum(top[0] * ks_next[0], top[1] * ks_next[1]));
            else return max_of_halves(__builtin_elementwise_maximum(top[0], top[1])) * c;
        };
        auto follow = [&](const float (&top)[NB]) __attribute__((always_inline)) {
            bool rise = false;
#pragma unroll
            for (int e = 0; e < NB; ++e) rise = rise || top[e] > m[e] + kLag;
            if (__builtin_expect(__ballot(rise) != 0, 0)) {
                bool beyond = false;
#pragma unroll
                for (int e = 0; e < NB; ++e) {
                    const float up = fmaxf(m[e], top[e]), down = __builtin_amdgcn_exp2f(m[e] - up);
                    beyond = beyond || (up > m[e] && fabsf(up) > kFar && fabsf(up) < __builtin_inff());
                    m[e] = up;
                    l[e] *= down;
                    l_used[e] *= down;
#pragma unroll
                    for (int b = 0; b < DB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[e][b][i] *= down;
                }
                if (__ballot(beyond)) special |= kFarRows;
            }
        };
        // Score j of the lane's 16 NB on its way to a weight: the exponents of the next one, its exponential, the sum and the rounding of those in front of it.
        float ref = 0.f, part_sum = 0.f, part_used = 0.f;
        auto advance = [&](float16v (&x)[NB], int j, bf16x8 (&pk)[NB][2]) __attribute__((always_inline)) {
            auto exponent = [&](int i) __attribute__((always_inline)) {
                if constexpr (FP8) {
                    if (i % 8 == 0) ref = m[i / 16] - vl[i % 16 / 8];
                    x[i / 16][i % 16] = __builtin_fmaf(x[i / 16][i % 16], ks[i % 16 / 8], -ref);
                } else {
                    x[i / 16][i % 16] = __builtin_fmaf(x[i / 16][i % 16], c, -m[i / 16]);
                }
            };
            if (j == 0) exponent(0);
            if (j + 1 < 16 * NB) exponent(j + 1);
            if (j < 16 * NB) x[j / 16][j % 16] = __builtin_amdgcn_exp2f(x[j / 16][j % 16]);
            if (j > 0) {
                const int i = j - 1;
                if constexpr (!LSE) {
                } else if constexpr (FP8) {
                    part_sum = i % 8 ? part_sum + x[i / 16][i % 16] : x[i / 16][i % 16];
                    if (i % 8 == 7) l[i / 16] = __builtin_fmaf(part_sum, vr[i % 16 / 8], l[i / 16]);
                } else {
                    l[i / 16] += x[i / 16][i % 16];
                }
                if (i % 2) {
                    u32x4 w = __builtin_bit_cast(u32x4, pk[i / 16][i % 16 / 8]);
                    w[i % 8 / 2] = pack_bf16(x[i / 16][i % 16 - 1], x[i / 16][i % 16]);
                    if constexpr (FP8) {
                        part_used = pair_sum(w[i % 8 / 2], i % 8 == 1 ? 0.f : part_used);
                        if (i % 8 == 7) l_used[i / 16] = __builtin_fmaf(part_used, vr[i % 16 / 8], l_used[i / 16]);
                    } else {
                        l_used[i / 16] = pair_sum(w[i % 8 / 2], l_used[i / 16]);
                    }
                    pk[i / 16][i % 16 / 8] = __builtin_bit_cast(bf16x8, w);
                }
            }
        };
        auto add_odd = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < NB; ++e)
                for (int pos = max(first, full) * kKeys; pos <= lim[e]; ++pos) {
                    const int64_t block = (int64_t)chunk_block(a, block_table[(int64_t)s.b * a.max_blocks + pos / kTile]) * a.num_kv_heads + g, at0 = (block * kTile + pos % kTile) * D + half * 4;
                    const float scale = FP8 ? v_scale[block] : 1.f;
#pragma unroll
                    for (int b = 0; b < DB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int64_t at = at0 + b * 32 + i / 4 * 8 + i % 4;
                            float v;
                            if constexpr (FP8) v = __builtin_amdgcn_cvt_f32_fp8((int)static_cast<const uint8_t *>(a.v)[at], 0);
                            else v = __uint_as_float((uint32_t) static_cast<const uint16_t *>(a.v)[at] << 16);
                            if constexpr (FP8) v *= scale;
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
        int kid = 0, vid = 0;   // this wavefront's blocks to bring next
        int k_put = 0, v_put = 0, v_put_next = 0;   // the scales of the blocks that are on their way
        // the meeting of the wavefronts; dirty: values of theirs have to be cleaned in front of it
        auto meet = [&](bool dirty, int t, Tile<D> &v_new, int pair) __attribute__((always_inline)) {
            const int vstep = t + 1 + (wave >> 1);   // of the values that this wavefront has brought
            if (dirty && vstep >= full) {
                if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
                clean(vstep, v_new, pair);
            }
            team_barrier<!FP8>();
        };
        auto step_of = [&](auto masked, auto parity, int t, float16v (&x)[NB], float16v (&y)[NB], Tile<D> &k_read, Tile<D> &v_read, Tile<D> &k_new, Tile<D> &v_new,
                           Tile<D> &k_next, Tile<D> &v_next, int pair) __attribute__((always_inline)) {
            // Both parts are as many matrix instructions and between them, in this order, what the vector unit and LDS have to do: the first EXPS of the 16 NB
            // exponentials and the values' operands (in its first half), the others, the next keys' operands (in its first half) and the largest scores.
            constexpr bool ODD = decltype(parity)::value, MASKED = decltype(masked)::value;
            constexpr int M1 = NB * KS, M2 = NB * 2 * DB, ELS = 16 * NB, EXPS = 20, LAST = M2 * 3 / 4, FRAGS = 2 * DB;
            constexpr auto least = [](int u, int v) { return u < v ? u : v; };
            constexpr auto exps_by = [](int i) { return i == 0 ? EXPS : i >= LAST ? ELS + 1 : EXPS + i * (ELS - EXPS) / LAST; };
            constexpr auto values_by = [least](int i) { return least(FRAGS, 2 * i * FRAGS / M1); };
            constexpr auto keys_by = [least](int i) { return least(KS, 2 * i * KS / M2); };
            constexpr auto parts_by = [](int i) { return i <= 2 ? 0 : (i - 2) * 8 * NB / (M2 - 2); };
            bf16x8 vf[2][DB], pk[NB][2];
            __builtin_amdgcn_sched_barrier(0);
            each<0, M1>([&](auto number) __attribute__((always_inline)) {
                constexpr int I = decltype(number)::value, E = I % NB, K = I / NB;
                if constexpr (K == 0)
#pragma unroll
                    for (int z = 0; z < 16; ++z) y[E][z] = 0.f;
                y[E] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[K], q[E][K], y[E], 0, 0, 0);
                each<values_by(I), values_by(I + 1)>([&](auto f) __attribute__((always_inline)) { vf[f / DB][f % DB] = read_values(v_read, ODD, f / DB, f % DB); });
                each<I * EXPS / M1, (I + 1) * EXPS / M1>([&](auto j) __attribute__((always_inline)) { advance(x, j, pk); });
                // (scalar loads, which whoever waits for LDS waits for: where nothing is waited for until the second part)
                constexpr int J = I - M1 / 2;
                if constexpr (J == 0 && !ODD) {
                    kid = block_id(t + 5, wave);
                    vid = block_id(t + 4, wave);
                }
                if constexpr (J == 0 && ODD && FP8) {
                    k_put = scale_of(k_scales, kid);
                    v_put_next = scale_of(v_scales, vid);
                }
                if constexpr (J == 1) take_key_scales();
                if constexpr (J == 2) take_value_scales();
                if constexpr (J == 3) {
                    ask_scales();
                    ask_blocks(t + 3);
                }
                if constexpr (FP8 && I >= M1 - 2 * LOADS) put_part(ODD ? in_v : in_k, I - (M1 - 2 * LOADS), ODD ? v_new : k_new, wave, ODD ? v_put : k_put);
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (ODD) meet(MASKED, t, v_new, pair ^ 1);
            const char *k_block = block_at(k_base, kid), *v_block = block_at(v_base, vid);
            if constexpr (ODD) v_put = v_put_next;
            float top[NB][2];
            __builtin_amdgcn_sched_barrier(0);
            each<0, M2>([&](auto number) __attribute__((always_inline)) {
                constexpr int I = decltype(number)::value, E = I / FRAGS, F = I % FRAGS;
                each<exps_by(I), exps_by(I + 1)>([&](auto j) __attribute__((always_inline)) { advance(x, j, pk); });
                o[E][F % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[F / DB][F % DB], pk[E][F / DB], o[E][F % DB], 0, 0, 0);
                each<keys_by(I), keys_by(I + 1)>([&](auto f) __attribute__((always_inline)) { kf[f] = read_keys(k_read, !ODD, f); });
                if constexpr (ODD)
                    each<least(2 * LOADS, 2 * I * 2 * LOADS / M2), least(2 * LOADS, 2 * (I + 1) * 2 * LOADS / M2)>([&](auto i) __attribute__((always_inline)) {
                        if constexpr (i < LOADS) bring_part(k_block, i, k_next, wave, in_k);
                        else bring_part(v_block, i - LOADS, v_next, wave, in_v);
                    });
                each<parts_by(I), parts_by(I + 1)>([&](auto part) __attribute__((always_inline)) {
                    largest(masked, t + 1, part / 8, y[part / 8], part % 8, top[part / 8]);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
            // (This step's flags and the next one's, which the same meeting has made known.  Behind the meeting in the next step the others may write them again.)
            if (MASKED && !ODD) {
                if (t >= full) special |= odd_flags[pair][0] | odd_flags[pair][1];
                if (t + 1 >= full) special |= odd_flags[pair][2] | odd_flags[pair][3];
            }
            float row_top[NB];
#pragma unroll
            for (int e = 0; e < NB; ++e) row_top[e] = whole_row(top[e]);
            follow(row_top);
            step_scales();
        };
        // a wavefront without rows
        auto idle_step = [&](auto parity, int t, Tile<D> &k_new, Tile<D> &v_new, Tile<D> &k_next, Tile<D> &v_next, int pair) __attribute__((always_inline)) {
            if constexpr (decltype(parity)::value) {
                put(in_v, v_new, wave, v_put);
                meet(true, t, v_new, pair ^ 1);
                bring(k_base, kid, k_next, wave, in_k);
                if constexpr (FP8) {
                    k_put = scale_of(k_scales, kid);
                    v_put = scale_of(v_scales, vid);
                }
                bring(v_base, vid, v_next, wave, in_v);
            } else {
                put(in_k, k_new, wave, k_put);
                kid = block_id(t + 5, wave);
                vid = block_id(t + 4, wave);
            }
        };
        auto four_steps = [&](auto masked, int t, float16v (&x)[NB], float16v (&y)[NB]) __attribute__((always_inline)) {
            constexpr bool MASKED = decltype(masked)::value;   // (the others are not near the share's end)
            step_of(masked, std::false_type{}, t, x, y, k_odd, v_even, k_even, v_odd, k_odd, v_even, 0);
            if (!MASKED || t + 1 < end) step_of(masked, std::true_type{}, t + 1, y, x, k_even, v_even, k_even, v_odd, k_odd, v_even, 0);
            if (!MASKED || t + 2 < end) step_of(masked, std::false_type{}, t + 2, x, y, k_even, v_odd, k_odd, v_even, k_even, v_odd, 1);
            if (!MASKED || t + 3 < end) step_of(masked, std::true_type{}, t + 3, y, x, k_odd, v_odd, k_odd, v_even, k_even, v_odd, 1);
        };

        if (first < end) {
            // keys of the first three steps, values of the first two
            u32x4 in_0[FP8 ? LOADS : 1];
            const int id_0 = block_id(first, wave), id_1 = block_id(first + 1, wave), id_2 = block_id(first + 2, wave), id_3 = block_id(first + 3, wave);
            if (wave < 2) bring(k_base, id_0, k_even, 2 + wave, in_0);
            bring(k_base, id_1, k_odd, wave, in_k);
            bring(v_base, id_0, v_even, wave, in_v);
            if constexpr (FP8) {
                if (wave < 2) put(in_0, k_even, 2 + wave, scale_of(k_scales, id_0));
                put(in_k, k_odd, wave, scale_of(k_scales, id_1));
                put(in_v, v_even, wave, scale_of(v_scales, id_0));
                k_put = scale_of(k_scales, id_3);
                v_put = scale_of(v_scales, id_2);
            }
            if (first + (wave >> 1) >= full) {
                if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
                clean(first + (wave >> 1), v_even, 0);
            }
            team_barrier<!FP8>();
            if (n_first < rows) {
                float16v x[NB], y[NB];
#pragma unroll
                for (int k = 0; k < KS; ++k) kf[k] = read_keys(k_even, 1, k);
                ask_blocks(first);
                ask_scales();
                take_key_scales();
                take_value_scales();
                ask_blocks(first + 1);
                ask_scales();
                ask_blocks(first + 2);
                scores(kf, x);
                float top[NB][2], row_top[NB];
#pragma unroll
                for (int e = 0; e < NB; ++e) {
                    each<0, 8>([&](auto part) __attribute__((always_inline)) { largest(std::true_type{}, first, e, x[e], part, top[e]); });
                    row_top[e] = whole_row(top[e]);
                }
                follow(row_top);
                step_scales();
#pragma unroll
                for (int k = 0; k < KS; ++k) kf[k] = read_keys(k_odd, 0, k);
                team_barrier<false>();   // (new keys come to where these were)
                bring(k_base, id_3, k_even, wave, in_k);
                bring(v_base, id_2, v_odd, wave, in_v);
                int t = first;
                for (const int fast_end = min(full, end) - 5; t < fast_end; t += 4) four_steps(std::false_type{}, t, x, y);
                for (; t < end; t += 4) four_steps(std::true_type{}, t, x, y);
                if (__builtin_expect((special & kOddValues) != 0, 0)) add_odd();
            } else {
                team_barrier<false>();
                bring(k_base, id_3, k_even, wave, in_k);
                bring(v_base, id_2, v_odd, wave, in_v);
                for (int t = first; t < end; t += 4) {
                    idle_step(std::false_type{}, t, k_even, v_odd, k_odd, v_even, 0);
                    if (t + 1 < end) idle_step(std::true_type{}, t + 1, k_even, v_odd, k_odd, v_even, 0);
                    if (t + 2 < end) idle_step(std::false_type{}, t + 2, k_odd, v_even, k_even, v_odd, 1);
                    if (t + 3 < end) idle_step(std::true_type{}, t + 3, k_odd, v_even, k_even, v_odd, 1);
                }
            }
            if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): nothing is on its way into LDS when the workgroup ends
        }

        // A block of rows: the weighted values, the reference, the sums of the weights (as rounded, and themselves)
        auto store = [&](int e, const float16v (&x)[DB], float ref, float used, float sum) __attribute__((always_inline)) {
            const int n = n_first + e * 32 + r32;
            if (s.part >= 0) {
                const int64_t part = (int64_t)s.part * a.num_kv_heads + g;
                const float level = used > 0.f ? sum / used : 1.0f;   // (the merge divides by the sum of the weights)
                float4v *po = reinterpret_cast<float4v *>(a.part_o) + part * (ROWS * D / 4) + (wave * NB + e) * (32 * D / 4) + lane;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int j = 0; j < 4; ++j) po[(b * 4 + j) * 64] = float4v{x[b][4 * j], x[b][4 * j + 1], x[b][4 * j + 2], x[b][4 * j + 3]} * level;
                if (half == 0) {
                    float *ml = a.part_ml + (part * ROWS + (wave * NB + e) * 32 + r32) * 2;
                    ml[0] = ref;
                    ml[1] = sum;
                }
            } else if (n < rows) {
                const int64_t at = (int64_t)(s.u.q0 + n / G) * a.num_q_heads + g * G + n % G;
                const float r = used > 0.f ? 1.0f / used : used == 0.f ? 0.f : used;   // (a row that sees nothing: zeros; NaN stays)
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        chunk_store4<SS_BF16>(a.out, at * D + b * 32 + j * 8 + half * 4, float4v{x[b][4 * j], x[b][4 * j + 1], x[b][4 * j + 2], x[b][4 * j + 3]} * r);
                if (LSE && half == 0) a.lse[at] = sum == 0.f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
            }
        };
#pragma unroll
        for (int e = 0; e < NB; ++e) {
            const float used = sum_of_halves(l_used[e]);
            store(e, o[e], m[e], used, LSE ? sum_of_halves(l[e]) : used);
        }
        // The wavefront's rows again, a key at a time in fp32, the scale applied before the reference is taken off: the largest score's weight is one whatever
        // its size.  (By itself, so that the steps need no register for it: 0.45 ms for 64 tokens behind 1936, 1.4 for a prompt of 2048, with 8 heads over 2.)
        if (__builtin_expect((uniform(special) & kFarRows) != 0, 0)) {
#pragma unroll 1
            for (int e = 0; e < NB; ++e) {
                const int n = min(n_first + e * 32 + r32, rows - 1), last = min(ctx + n / G, end * kKeys - 1);
                const int64_t q_at = (int64_t)(s.u.q0 + n / G) * a.q_stride + (int64_t)(g * G + n % G) * D + half * (D / 2);
                float ref = kChunkNoMax, sum = 0.f;
                float16v x[DB] = {};
#pragma unroll 1
                for (int pos = first * kKeys; pos < min(end * kKeys, s.u.kv_len); ++pos) {
#pragma clang fp contract(off)   // (a score is rounded before the reference, which is one of them, is taken off)
                    const int64_t block = (int64_t)chunk_block(a, block_table[(int64_t)s.b * a.max_blocks + pos / kTile]) * a.num_kv_heads + g, at = (block * kTile + pos % kTile) * D;
                    float y = 0.f;
#pragma unroll
                    for (int j = 0; j < D / 2; j += 4) {
                        const float4v key = load4<FP8>(a.k, at + half * (D / 2) + j), query = load4<false>(a.q, q_at + j);
#pragma unroll
                        for (int i = 0; i < 4; ++i) y = __builtin_fmaf(key[i], query[i], y);
                    }
                    y = (FP8 ? sum_of_halves(y) * k_scale[block] : sum_of_halves(y)) * c;
                    if (pos > last) continue;
                    const float up = fmaxf(ref, y), down = __builtin_amdgcn_exp2f(ref - up), w = __builtin_amdgcn_exp2f(y - up);
                    ref = up;
                    sum = sum * down + w;
#pragma unroll
                    for (int b = 0; b < DB; ++b)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float4v v = load4<FP8>(a.v, at + half * 4 + b * 32 + j * 8);
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[b][4 * j + i] = x[b][4 * j + i] * down + w * (FP8 ? v[i] * v_scale[block] : v[i]);
                        }
                }
                store(e, x, ref, sum, sum);
            }
        }
        team_barrier<false>();   // (the next tile's keys come to where the others may still read)
    }
    chunk_record(a, span, g, begun, begun_q0, begun_rows, begun_row0);
}

template <int D, bool FP8, bool LSE>
int32_t launch(const ChunkArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((chunk_kernel<D, FP8, LSE>), dim3((unsigned)(a.spans * a.num_kv_heads)), dim3(64 * kWaves), 0, stream, a, a.block_table, a.k_scale, a.v_scale);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_kernel");
    return chunk_merge_launch<ROWS, 32, D, SS_BF16>(a, stream);
}

}  // namespace

bool chunk_mfma_supported(int head_dim, int kv_dtype, int q_dtype)
{
    return (head_dim == 64 || head_dim == 128) && q_dtype == SS_BF16 && (kv_dtype == SS_BF16 || kv_dtype == SS_FP8_E4M3);
}

int32_t chunk_mfma_launch(const ChunkArgs &a, hipStream_t stream)
{
    const bool fp8 = a.kv_dtype == SS_FP8_E4M3;
    if (a.lse) {
        if (a.head_dim == 128) return fp8 ? launch<128, true, true>(a, stream) : launch<128, false, true>(a, stream);
        return fp8 ? launch<64, true, true>(a, stream) : launch<64, false, true>(a, stream);
    }
    if (a.head_dim == 128) return fp8 ? launch<128, true, false>(a, stream) : launch<128, false, false>(a, stream);
    return fp8 ? launch<64, true, false>(a, stream) : launch<64, false, false>(a, stream);
}

}  // namespace ss
