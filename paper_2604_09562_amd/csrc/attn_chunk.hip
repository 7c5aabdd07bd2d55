// Attention of a chunk of new tokens on the bf16 matrix cores: bf16 queries over bf16 or e4m3 caches, heads of 64 or 128, any grouping.
//
// A workgroup of four wavefronts takes a share (chunk_plan.h) of 128 query rows of a KV head, 32 to a wavefront, two workgroups to a compute unit.
// A step brings 64 keys and values into LDS (as bf16, exact for e4m3 codes; each wavefront reads one cache block); a wavefront computes
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
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kRows = kChunkRows, kWaves = 4;
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
// What the lane of the row's other keys has, joined.
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}
// Waits for this wavefront's LDS accesses only (not for the loads in flight), then for the others.
__device__ __forceinline__ void team_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A tile of 64 keys or values in LDS, rows of D bf16 in pieces of 16 bytes.  Piece c of row t stands at place c ^ turn(t): 16 rows' pieces
// of equal c fill all banks (scores), and so do four rows' pieces 4 n .. 4 n + 3 (transposing reads of values).
template <int D>
struct Tile {
    static constexpr int PIECES = D / 8;
    u32x4 w[kStepKeys][PIECES];
    static __device__ __forceinline__ int turn(int t) { return D == 128 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3); }
};

template <int D>
struct ChunkLds {
    Tile<D> k[2], v[2];
    int odd[2][kWaves];
};

// The largest of three, or NaN (the other kind of maximum costs an instruction more for each operand that may be a signalling NaN).
__device__ __forceinline__ float max3(float x, float y, float z) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z); }

template <int D, bool FP8>
__global__ __launch_bounds__(64 * kWaves, 2) void chunk_kernel(ChunkArgs a, const int32_t *__restrict__ block_table, const float *__restrict__ k_scale,
                                                               const float *__restrict__ v_scale)
{
    // (table and scales come in as no-alias arguments of their own, so that they are scalar loads)
    constexpr int KS = D / 16, DB = D / 32;
    constexpr int BLOCK_BYTES = kTile * D * (FP8 ? 1 : 2), LOADS = BLOCK_BYTES / (64 * 16);   // 16-byte loads of a lane for a cache block
    constexpr int STEP_BLOCKS = kStepKeys / kTile;
    __shared__ ChunkLds<D> lds;
    const int g = blockIdx.x % a.num_kv_heads, item = blockIdx.x / a.num_kv_heads;
    ChunkShare s;
    const bool any = chunk_share<kRows>(a, item, s);
    if (a.cap > 0 && blockIdx.x == 0 && threadIdx.x == 0) a.head[0] = s.cuts;
    if (!any) return;
    chunk_record<kRows>(a, s, g);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, half = lane >> 5;
    const int G = a.num_q_heads / a.num_kv_heads;
    const int rows = s.q_len * G, ctx = s.kv_len - s.q_len;
    const int n_first = s.tile * kRows + wave * 32, n = n_first + r32;
    const int qi = min(n, rows - 1) / G, hh = n % G;
    const int lim = ctx + qi;                                           // the last position this lane's row sees
    // steps up to which all rows of the wavefront see everything, from which none sees anything; the same of the tile
    const int all = max((ctx + min(n_first, rows - 1) / G + 1) / kStepKeys, 0);
    const int none = min((max(ctx + min(n_first + 31, rows - 1) / G + 1, 0) + kStepKeys - 1) / kStepKeys, s.s1);
    const int full = max((ctx + s.tile * kRows / G + 1) / kStepKeys, 0);
    const float c = a.sm_scale * kLog2e;

    bf16x8 q[KS];
    {
        const char *src = static_cast<const char *>(a.q) + ((int64_t)(s.q0 + qi) * a.q_stride + (int64_t)(g * G + hh) * D + half * 8) * 2;
        u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            u32x4 w = zero;
            if (n < rows) w = *reinterpret_cast<const u32x4 *>(src + k * 32);
            q[k] = __builtin_bit_cast(bf16x8, w);
        }
    }

    const int32_t *table = block_table + (int64_t)s.b * a.max_blocks;
    const int last_block = (int)(((unsigned)s.kv_len + kTile - 1) / kTile) - 1;
    // block j of a step (the last block again where there is none: what stands there is masked)
    auto block_id = [&](int step, int j) { return table[min(step * STEP_BLOCKS + j, last_block)]; };
    u32x4 in[LOADS];   // this wavefront's block of a step's keys, or of its values
    auto load = [&](const void *cache, int id) {
        const char *p = static_cast<const char *>(cache) + ((int64_t)id * a.num_kv_heads + g) * BLOCK_BYTES + lane * 16;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) in[i] = *reinterpret_cast<const u32x4 *>(p + i * 1024);
    };
    auto as_bf16 = [&](int i, u32x4 (&w)[FP8 ? 2 : 1]) {
        if constexpr (FP8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j / 2][j % 2 * 2] = fp8x2_to_bf16x2<false>(in[i][j]);
                w[j / 2][j % 2 * 2 + 1] = fp8x2_to_bf16x2<true>(in[i][j]);
            }
        } else {
            w[0] = in[i];
        }
    };
    auto put = [&](Tile<D> &tile, int i, const u32x4 (&w)[FP8 ? 2 : 1]) {
        const int e = (i * 64 + lane) * (FP8 ? 16 : 8), t = wave * kTile + e / D, col = e % D / 8;   // first element: row, piece
#pragma unroll
        for (int p = 0; p < (FP8 ? 2 : 1); ++p) tile.w[t][(col + p) ^ Tile<D>::turn(t & 15)] = w[p];
    };
    auto store_keys = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            u32x4 w[FP8 ? 2 : 1];
            as_bf16(i, w);
            put(lds.k[buf], i, w);
        }
    };
    auto store_values = [&](auto fast, int step, int buf) {
        if (decltype(fast)::value || step < full) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                u32x4 w[FP8 ? 2 : 1];
                as_bf16(i, w);
                put(lds.v[buf], i, w);
            }
            return;
        }
        // Some row does not see all of the step.  What stands behind the last token is of no one; a value that is not finite is taken out
        // of the product, in which it would reach every row (0 * inf), and added to the rows that see it.
        bool odd = false;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            u32x4 w[FP8 ? 2 : 1];
            as_bf16(i, w);
            const bool dead = step * kStepKeys + wave * kTile + (i * 64 + lane) * (FP8 ? 16 : 8) / D >= s.kv_len;
#pragma unroll
            for (int p = 0; p < (FP8 ? 2 : 1); ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t x = dead ? 0u : w[p][j];
                    if ((x & 0x7f80u) == 0x7f80u) { x &= 0xffff0000u; odd = true; }
                    if ((x & 0x7f800000u) == 0x7f800000u) { x &= 0xffffu; odd = true; }
                    w[p][j] = x;
                }
            put(lds.v[buf], i, w);
        }
        lds.odd[buf][wave] = __ballot(odd) != 0;
    };

    float m = kChunkNoMax, l = 0.f;
    float16v o[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;

    // scores of 32 keys: the lane has row r32 and keys 8 (i / 4) + 4 half + i % 4
    auto scores = [&](int buf, int b, float16v &x) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
        const int t = b * 32 + r32, turn = Tile<D>::turn(t & 15);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const bf16x8 kk = __builtin_bit_cast(bf16x8, lds.k[buf].w[t][(2 * k + half) ^ turn]);
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, q[k], x, 0, 0, 0);
        }
    };

    struct Scales {
        float k[FP8 ? STEP_BLOCKS : 1], v[FP8 ? STEP_BLOCKS : 1];
    };
    auto scales_of = [&](int step) {
        Scales r;
        if constexpr (FP8)
#pragma unroll
            for (int j = 0; j < STEP_BLOCKS; ++j) {
                const int64_t tile = (int64_t)block_id(step, j) * a.num_kv_heads + g;
                r.k[j] = k_scale[tile] * c;
                r.v[j] = v_scale[tile];
            }
        return r;
    };

    // One step: the scores of the next one are computed between the exponentials of this one.  buf: of this step's keys and values.
    // At its beginning LDS holds the step's values and the next step's keys, id1 and id2 are this wavefront's blocks of the next two steps.
    int id1 = 0, id2 = 0;
    // FAST: every row of the tile sees all of this step and the next (what would be read behind the share's last step is read as well, from the last block).
    auto step_of = [&](auto fast, int step, int buf, float16v (&x)[2], float16v (&y)[2]) {
        constexpr bool FAST = decltype(fast)::value;
        const bool more = FAST || step + 1 < s.s1, more2 = FAST || step + 2 < s.s1;
        if (more2) load(a.k, id2);
        const int id3 = block_id(step + 3, wave);
        const bool live = FAST || step < none, next = FAST || step + 1 < none;
        if (next) scores(buf ^ 1, 0, y[0]);
        Scales sc;
        if (live) {
            sc = scales_of(step);
            if constexpr (FP8)   // one scale to 16 keys: they are in eight accumulators
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[b][i] *= sc.k[b * 2 + i / 8];
            if (!FAST && step >= all) {
                const int seen = lim - step * kStepKeys - 4 * half;    // keys up to this one, counted from the lane's first
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (b * 32 + i / 4 * 8 + i % 4 > seen) x[b][i] = -__builtin_inff();
            }
            // the reference follows the largest score when that has risen by kLag
            float top = max3(x[0][0], x[0][1], x[0][2]);
#pragma unroll
            for (int i = 3; i < 31; i += 2) top = max3(top, x[i / 16][i % 16], x[(i + 1) / 16][(i + 1) % 16]);
            top = max3(top, x[1][15], x[1][15]);
            top = max_of_halves(top);
            if constexpr (!FP8) top *= c;
            if (__ballot(top > m + kLag || m == kChunkNoMax)) {
                const float up = fmaxf(m, top), down = __builtin_amdgcn_exp2f(m - up);
                m = up;
                l *= down;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[b][i] *= down;
            }
        }
        if (next) scores(buf ^ 1, 1, y[1]);
        u32x4 pw[4];
        if (live) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = __builtin_amdgcn_exp2f(FP8 ? x[b][i] - m : __builtin_fmaf(x[b][i], c, -m));
                    l += p;
                    x[b][i] = FP8 ? p * sc.v[b * 2 + i / 8] : p;
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) pw[k][j] = pack_bf16(x[k / 2][k % 2 * 8 + 2 * j], x[k / 2][k % 2 * 8 + 2 * j + 1]);
        }
        if (more2) store_keys(buf);
        if (more) load(a.v, id1);
        if (live) {
            // a contraction takes 16 keys, the lane's eight of them in the order of its accumulators
            const int group = lane >> 4, i16 = lane & 15;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bf16x8 pk = __builtin_bit_cast(bf16x8, pw[k]);
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    s16x4 vv[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int t = k * 16 + r * 8 + half * 4 + i16 / 4;
                        const int d = b * 32 + (group & 1) * 16 + i16 % 4 * 4;
                        const auto *p = reinterpret_cast<const char *>(&lds.v[buf].w[t][(d / 8) ^ Tile<D>::turn(t & 15)]) + d % 8 * 2;
                        vv[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p));
                    }
                    const bf16x8 vk = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vv[0], vv[1], 0, 1, 2, 3, 4, 5, 6, 7));
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vk, pk, o[b], 0, 0, 0);
                }
            }
            if (!FAST && step >= full && (lds.odd[buf][0] | lds.odd[buf][1] | lds.odd[buf][2] | lds.odd[buf][3])) {
                for (int pos = step * kStepKeys; pos < min((step + 1) * kStepKeys, lim + 1); ++pos) {
                    const int64_t tile = (int64_t)table[pos / kTile] * a.num_kv_heads + g;
                    const int64_t from = (tile * kTile + pos % kTile) * D + half * 4;
#pragma unroll
                    for (int b = 0; b < DB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int64_t at = from + b * 32 + i / 4 * 8 + i % 4;
                            float v;
                            if constexpr (FP8) v = __builtin_amdgcn_cvt_f32_fp8((int)static_cast<const uint8_t *>(a.v)[at], 0);
                            else v = __uint_as_float((uint32_t) static_cast<const uint16_t *>(a.v)[at] << 16);
                            if (!__builtin_isfinite(v)) o[b][i] += v;
                        }
                }
            }
        }
        if (more) store_values(fast, step + 1, buf ^ 1);
        id1 = id2;
        id2 = id3;
        team_barrier();
    };

    if (s.s0 < s.s1) {
        const int id0 = block_id(s.s0, wave);
        id1 = block_id(s.s0 + 1, wave);
        id2 = block_id(s.s0 + 2, wave);
        load(a.k, id0);
        store_keys(0);
        load(a.v, id0);
        store_values(std::false_type{}, s.s0, 0);
        if (s.s0 + 1 < s.s1) {
            load(a.k, id1);
            store_keys(1);
        }
        team_barrier();
        float16v x[2], y[2];
        if (s.s0 < none) {
            scores(0, 0, x[0]);
            scores(0, 1, x[1]);
        }
        team_barrier();   // (the first step brings new keys into the buffer that these scores came from)
        int step = s.s0;
        for (const int end = min(full, s.s1) - 2; step < end; step += 2) {
            step_of(std::true_type{}, step, 0, x, y);
            step_of(std::true_type{}, step + 1, 1, y, x);
        }
        for (; step < s.s1; step += 2) {
            step_of(std::false_type{}, step, 0, x, y);
            if (step + 1 < s.s1) step_of(std::false_type{}, step + 1, 1, y, x);
        }
    }

    l = sum_of_halves(l);
    if (s.pieces > 1) {
        const int64_t part = (int64_t)s.slot * a.num_kv_heads + g;
        float4v *po = reinterpret_cast<float4v *>(a.part_o) + part * (kRows * D / 4) + wave * (32 * D / 4) + lane;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) po[(b * 4 + j) * 64] = float4v{o[b][4 * j], o[b][4 * j + 1], o[b][4 * j + 2], o[b][4 * j + 3]};
        if (half == 0) {
            float *ml = a.part_ml + (part * kRows + wave * 32 + r32) * 2;
            ml[0] = m;
            ml[1] = l;
        }
        return;
    }
    if (n >= rows) return;
    const int64_t at = (int64_t)(s.q0 + qi) * a.num_q_heads + g * G + hh;
    const float r = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;   // (a row that sees nothing: zeros; NaN stays)
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            chunk_store4<SS_BF16>(a.out, at * D + b * 32 + j * 8 + half * 4, float4v{o[b][4 * j], o[b][4 * j + 1], o[b][4 * j + 2], o[b][4 * j + 3]} * r);
    if (a.lse && half == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D, bool FP8>
int32_t launch(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream)
{
    const int64_t shares = s.tiles + s.cap / a.num_kv_heads;
    hipLaunchKernelGGL((chunk_kernel<D, FP8>), dim3((unsigned)(shares * a.num_kv_heads)), dim3(64 * kWaves), 0, stream, a,
                       a.block_table, a.k_scale, a.v_scale);
    SS_HIP_CHECK(hipGetLastError(), "launch chunk_kernel");
    if (s.cap >= 2 * a.num_kv_heads) {
        const int64_t fit = s.cap / (2 * a.num_kv_heads), cuts = s.tiles < fit ? s.tiles : fit;
        hipLaunchKernelGGL((chunk_merge_kernel<kRows, 32, D, SS_BF16>), dim3((unsigned)(cuts * a.num_kv_heads * (kRows * D / 1024))), dim3(256), 0, stream, a);
        SS_HIP_CHECK(hipGetLastError(), "launch chunk_merge_kernel");
    }
    return SS_OK;
}

}  // namespace

bool chunk_mfma_supported(int head_dim, int kv_dtype, int q_dtype)
{
    return (head_dim == 64 || head_dim == 128) && q_dtype == SS_BF16 && (kv_dtype == SS_BF16 || kv_dtype == SS_FP8_E4M3);
}

int32_t chunk_mfma_launch(const ChunkArgs &a, const ChunkShape &s, hipStream_t stream)
{
    const bool fp8 = a.kv_dtype == SS_FP8_E4M3;
    if (a.head_dim == 128) return fp8 ? launch<128, true>(a, s, stream) : launch<128, false>(a, s, stream);
    return fp8 ? launch<64, true>(a, s, stream) : launch<64, false>(a, s, stream);
}

}  // namespace ss
