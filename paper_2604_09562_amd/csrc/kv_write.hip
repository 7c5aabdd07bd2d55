// The write of new keys and values into the paged cache by slot: row r goes to block slot[r] / 16, place slot[r] % 16, for every KV head.
//
// f32 and bf16 caches: eight elements of a key and of a value to a lane, consecutive lanes along a row, so that reads take whole rows and writes
// the 256 bytes (bf16, 128-wide heads) that a token has in a block.  Bound by memory.
//
// e4m3 caches: the rows of a block stand as far apart in the call as their slots (a run); a wavefront takes a run's keys or values of one
// head, has the largest magnitude of all of them in registers before it rounds the first, and writes each row's codes.  One read of the values
// instead of the two that a row by itself needs.
#include <type_traits>

#include "prefill.h"

namespace ss {
namespace {

typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kFp8Max = 448.0f;   // largest finite e4m3fn value
constexpr int kEl = 8;              // elements to a lane

__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    const float2v v = {x, y};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));   // nearest, ties to even
}

// eight values in storage format, from a 16-byte aligned place
template <int DT>
struct Eight {
    u32x4 w[DT == SS_F32 ? 2 : 1];
    __device__ void load(const void *base, int64_t i)
    {
        const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const char *>(base) + i * (DT == SS_F32 ? 4 : 2));
        w[0] = p[0];
        if constexpr (DT == SS_F32) w[1] = p[1];
    }
    __device__ float value(int e) const
    {
        if constexpr (DT == SS_F32) return __uint_as_float(w[e / 4][e % 4]);
        else return __uint_as_float(e & 1 ? w[0][e / 2] & 0xffff0000u : w[0][e / 2] << 16);
    }
};

template <int KV_DT, int NEW_DT>
__device__ __forceinline__ void store_eight(void *cache, int64_t i, const Eight<NEW_DT> &x)
{
    if constexpr (KV_DT == SS_F32) {
        u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<float *>(cache) + i);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            u32x4 w;
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = __float_as_uint(x.value(4 * j + c));
            p[j] = w;
        }
    } else {
        u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(cache) + i);
        if constexpr (NEW_DT == SS_BF16) {
            p[0] = x.w[0];
        } else {
            u32x4 w;
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = pack_bf16(x.value(2 * c), x.value(2 * c + 1));
            p[0] = w;
        }
    }
}

template <int KV_DT, int NEW_DT>
__global__ __launch_bounds__(256) void kv_write_kernel(KvWriteArgs a, uint32_t pieces, uint32_t total)
{
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = i / pieces, piece = i % pieces, per_head = (uint32_t)a.head_dim / kEl;
    const int slot = a.slot_map[row];
    Eight<NEW_DT> k, v;   // (asked for with the slot, not behind it)
    k.load(a.k_new, (int64_t)row * a.k_stride + piece * kEl);
    v.load(a.v_new, (int64_t)row * a.v_stride + piece * kEl);
    if (slot < 0 || slot >= a.num_blocks * kTile) return;
    const uint32_t h = piece / per_head, d = piece % per_head;
    const int64_t to = (((int64_t)(slot / kTile) * a.num_kv_heads + h) * kTile + slot % kTile) * a.head_dim + d * kEl;
    store_eight<KV_DT, NEW_DT>(a.k, to, k);
    store_eight<KV_DT, NEW_DT>(a.v, to, v);
}

// The code of x / scale, the quotient rounded once to fp32 (as one IEEE division gives it) and cut at the largest code.
//
// Within 2^-60 .. 2^60 a quotient is the product with the rounded inverse, corrected twice by what it leaves of x: the product is at most two steps off and the
// first correction leaves less than one, from where the second one, with an inverse that is off by at most half a step, gives the nearest number (Markstein's
// theorem).  Remainders are exact but for x so small that the code is zero anyway, and x is cut first, so that nothing overflows: 448 scale may be rounded up,
// by less than the 16 that a quotient may be above 448 and still round to it.  Seven instructions instead of a division's 15: 15.8 us instead of 21.6 where
// 43 MB of bf16 become 21 MB of codes.  The cut does not keep NaN: runs with one take the division and a cut that does (16.4 us if the quotients above had it).
struct Divisor {
    float scale, inverse, limit;
    bool near_one;
    __device__ explicit Divisor(float s) : scale(s), inverse(1.0f / s), limit(kFp8Max * fabsf(s)), near_one(fabsf(s) >= 0x1p-60f && fabsf(s) <= 0x1p60f) {}
    template <bool NEAR_ONE>
    __device__ float operator()(float x) const
    {
        // (saturated: finite values over a finite scale never give the NaN byte; values so small that their scale has become zero are zeros)
        if constexpr (!NEAR_ONE)
            return x == 0.f && scale == 0.f ? x : __builtin_elementwise_minimum(__builtin_elementwise_maximum(x / scale, -kFp8Max), kFp8Max);
        x = __builtin_amdgcn_fmed3f(x, -limit, limit);
        const float product = x * inverse;
        float q = product;
        q = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
        q = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
        return __builtin_copysignf(q, product);   // (corrections of minus zero are plus zero)
    }
};
template <bool NEAR_ONE, typename EIGHT>
__device__ __forceinline__ uint32_t four_codes(const EIGHT &x, int e, const Divisor &by)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(by.operator()<NEAR_ONE>(x.value(e)), by.operator()<NEAR_ONE>(x.value(e + 1)), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(by.operator()<NEAR_ONE>(x.value(e + 2)), by.operator()<NEAR_ONE>(x.value(e + 3)), w, true);
    return (uint32_t)w;
}

// A wavefront per (window of rows, KV head, keys or values); it takes the runs that begin in its window.
template <int NEW_DT, int D>
__global__ __launch_bounds__(256) void kv_write_e4m3_kernel(KvWriteArgs a, int window, uint32_t waves)
{
    constexpr int LANES = D / kEl, ROWS = 64 / LANES, N = kTile / ROWS;   // lanes to a row, rows to a pass, passes to a block
    const uint32_t wave = blockIdx.x * 4u + (threadIdx.x >> 6);
    if (wave >= waves) return;
    const int lane = threadIdx.x & 63;
    const int side = wave & 1, h = (wave >> 1) % a.num_kv_heads, r0 = (int)((wave >> 1) / a.num_kv_heads) * window;
    // slots of the window's rows, of the 15 in front of it and of the 15 behind it; outside the call or the cache: none
    constexpr int BACK = kTile - 1;
    int slot = -1;
    const int r = r0 - BACK + lane;
    if (lane < window + 2 * BACK && r >= 0 && r < a.total_rows) slot = a.slot_map[r];
    if (slot < 0 || slot >= a.num_blocks * kTile) slot = -1;
    // a row goes on a run if the nearest one in front of it that is not left out is as far away as its slot, in the same block
    const uint64_t valid = __ballot(slot >= 0), before = valid & ((1ull << lane) - 1);
    const int last = before ? 63 - __builtin_clzll(before) : lane;
    const int near = __shfl(slot, last);
    const bool goes_on = before && near / kTile == slot / kTile && slot - near == lane - last;
    uint64_t begins = valid & ~__ballot(goes_on) & (((1ull << window) - 1) << BACK);
    const void *src = side ? a.v_new : a.k_new;
    uint8_t *cache = static_cast<uint8_t *>(side ? a.v : a.k);
    float *scales = side ? a.v_scale : a.k_scale;
    const int64_t stride = side ? a.v_stride : a.k_stride;
    const int col = (lane % LANES) * kEl, sub = lane / LANES;
    while (begins) {
        const int p = __builtin_ctzll(begins);
        begins &= begins - 1;
        const int first = __builtin_amdgcn_readlane(slot, p);
        const int place = first % kTile, row0 = r0 - BACK + p;
        // bit j: the row j behind the first one is the run's (at most 16; rows that are left out or another block's may stand between)
        const uint64_t rows = __ballot(slot >= 0 && slot / kTile == first / kTile && slot - first == lane - p);
        if (rows & ((1ull << p) - 1)) continue;   // (the run began in front of this row, with another block's row between)
        const uint32_t run = (uint32_t)(rows >> p);
        const int64_t tile = (int64_t)(first / kTile) * a.num_kv_heads + h;
        Eight<NEW_DT> x[N];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (run >> (i * ROWS + sub) & 1) x[i].load(src, (int64_t)(row0 + i * ROWS + sub) * stride + (int64_t)h * D + col);
        float scale = 0.f;
        if (place != 0) scale = scales[tile];
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (run >> (i * ROWS + sub) & 1)
#pragma unroll
                for (int e = 0; e < kEl; ++e) top = __builtin_elementwise_maximum(top, fabsf(x[i].value(e)));   // (NaN if there is one)
        const bool odd = __ballot(top != top) != 0;
        if (__builtin_expect(odd, 0)) {
            top = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (run >> (i * ROWS + sub) & 1)
#pragma unroll
                    for (int e = 0; e < kEl; ++e) top = fmaxf(top, fabsf(x[i].value(e)));
        }
        if (place == 0) {   // the block begins with this call: its scale, for all of its rows that the call brings
#pragma unroll
            for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
            scale = top > 0.f ? top / kFp8Max : 1.0f;
            if (lane == 0) scales[tile] = scale;
        }
        const Divisor by(scale);
        auto write = [&](auto near_one) __attribute__((always_inline)) {
            constexpr bool NEAR_ONE = decltype(near_one)::value;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (run >> (i * ROWS + sub) & 1)
                    *reinterpret_cast<u32x2 *>(cache + (tile * kTile + place + i * ROWS + sub) * D + col) =
                        u32x2{four_codes<NEAR_ONE>(x[i], 0, by), four_codes<NEAR_ONE>(x[i], 4, by)};
        };
        if (by.near_one && !odd) write(std::true_type{});   // (one scale to the wavefront, and one answer)
        else write(std::false_type{});
    }
}

template <int NEW_DT>
int32_t launch(const KvWriteArgs &a, hipStream_t stream)
{
    if (a.kv_dtype == SS_FP8_E4M3) {
        // Windows of 16 rows have about a run each where chunks are long; few rows take smaller ones, so that runs of single rows are not taken one after the other.
        // With 4 | 16 rows, us, 8 heads of 128: 320 requests of a token 6.9 | 18.7, 2048 of them 13.3 | 21.7, 4096 of them 21.8 | 27.2; one chunk of 2048 tokens 9.2 | 7.0,
        // of 4096 15.1 | 7.6, of 16 384 46.6 | 22.1.  (Windows of a single row are level with 4 up to 320 tokens and slower from there.)
        const int64_t per_row = 2ll * a.num_kv_heads;
        const int window = a.total_rows * per_row <= 65536 ? 4 : 16;
        const int64_t waves = ((int64_t)a.total_rows + window - 1) / window * per_row;
        const dim3 grid((unsigned)((waves + 3) / 4));
        if (a.head_dim == 128)
            hipLaunchKernelGGL((kv_write_e4m3_kernel<NEW_DT, 128>), grid, dim3(256), 0, stream, a, window, (uint32_t)waves);
        else
            hipLaunchKernelGGL((kv_write_e4m3_kernel<NEW_DT, 64>), grid, dim3(256), 0, stream, a, window, (uint32_t)waves);
        SS_HIP_CHECK(hipGetLastError(), "launch kv_write_e4m3_kernel");
        return SS_OK;
    }
    const uint32_t pieces = (uint32_t)(a.num_kv_heads * a.head_dim / kEl), total = pieces * (uint32_t)a.total_rows;
    const dim3 grid((total + 255) / 256);
    if (a.kv_dtype == SS_F32) hipLaunchKernelGGL((kv_write_kernel<SS_F32, NEW_DT>), grid, dim3(256), 0, stream, a, pieces, total);
    else hipLaunchKernelGGL((kv_write_kernel<SS_BF16, NEW_DT>), grid, dim3(256), 0, stream, a, pieces, total);
    SS_HIP_CHECK(hipGetLastError(), "launch kv_write_kernel");
    return SS_OK;
}

}  // namespace

int32_t kv_write_launch(const KvWriteArgs &a, hipStream_t stream)
{
    return a.new_dtype == SS_F32 ? launch<SS_F32>(a, stream) : launch<SS_BF16>(a, stream);
}

}  // namespace ss
