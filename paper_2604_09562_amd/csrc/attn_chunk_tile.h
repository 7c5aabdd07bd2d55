// A workgroup's piece of a tile, as text inside chunk_kernel (attn_chunk_kernel.h): with NB blocks of 32 query rows to a wavefront, two, or one where the tile has no more than one
// for each.  (Text, because as a function of its own, inlined, the compiler spills what it keeps in registers here.)
const int r32 = lane & 31, half = lane >> 5;
const int G = a.num_q_heads / a.num_kv_heads;
const int rows = s.u.q_len * G, ctx = s.u.kv_len - s.u.q_len;
const int n_first = s.t * ROWS + wave * 32 * NB;
int lim[NB];                                                        // the last position this lane's rows see
int node[TREE ? NB : 1];                                            // TREE: their places in the call
#pragma unroll
for (int e = 0; e < NB; ++e) {
    const int i = min(n_first + e * 32 + r32, rows - 1) / G;
    lim[e] = TREE ? s.u.kv_len - 1 : ctx + i;
    if constexpr (TREE) node[e] = s.u.q0 + i;
}
// In steps of 32 keys: the share's, and up to where all rows of the tile see everything
const int first = s.s0, end = s.s1;
const int full = max((TREE ? ctx : ctx + s.t * ROWS / G + 1) / kKeys, 0);
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
// TREE: which of a step's keys the lane's rows see (of what is behind the share, none)
uint32_t window[TREE ? NB : 1];
auto see = [&](int step) __attribute__((always_inline)) {
    if constexpr (TREE)
#pragma unroll
        for (int e = 0; e < NB; ++e)
            window[e] = step < end ? tree_window(a.node_mask + (int64_t)node[e] * a.mask_words, a.mask_words, s.u.q_len, step * kKeys - ctx) >> (4 * half) : 0u;
};
auto sees = [&](int row, int pos) __attribute__((always_inline)) {
    return (tree_window(a.node_mask + (int64_t)row * a.mask_words, a.mask_words, s.u.q_len, pos - ctx) & 1u) != 0;
};
// The largest of a row's 16 scores in the lane, in four parts for either eight; the scores are masked on the way.
auto largest = [&](auto masked, int step, int e, float16v &x, int part, float (&top)[2]) __attribute__((always_inline)) {
    const int group = part / 4, lo = group * 8 + (part % 4 ? 2 * (part % 4) + 1 : 0), hi = group * 8 + (part % 4 < 3 ? 2 * (part % 4) + 3 : 8);
    if constexpr (decltype(masked)::value && TREE) {
#pragma unroll
        for (int i = lo; i < hi; ++i)
            if (!(window[e] >> (i / 4 * 8 + i % 4) & 1u)) x[i] = -__builtin_inff();
    } else if constexpr (decltype(masked)::value) {
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
            if constexpr (TREE)
                if (!sees(node[e], pos)) continue;
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
    // (weights of a contraction's first half have to be there when the second part begins, those of its second half when their products do)
    constexpr int M1 = NB * KS, M2 = NB * 2 * DB, ELS = 16 * NB, EXPS = NB == 2 ? 20 : 10, LAST = NB == 2 ? M2 * 3 / 4 : DB + 1, FRAGS = 2 * DB;
    constexpr auto least = [](int u, int v) { return u < v ? u : v; };
    constexpr auto exps_by = [](int i) { return i == 0 ? EXPS : i >= LAST ? ELS + 1 : EXPS + i * (ELS - EXPS) / LAST; };
    constexpr auto values_by = [least](int i) { return least(FRAGS, 2 * i * FRAGS / M1); };
    constexpr auto keys_by = [least](int i) { return least(KS, 2 * i * KS / M2); };
    constexpr auto parts_by = [](int i) { return i <= 2 ? 0 : (i - 2) * 8 * NB / (M2 - 2); };
    bf16x8 vf[2][DB], pk[NB][2];
    if constexpr (MASKED) see(t + 1);
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
        constexpr int J = I - M1 / 2, J1 = M1 / 2 >= 4 ? J : 2 * J, J2 = M1 / 2 >= 4 ? J : 2 * J + 1;   // (of few matrix instructions, two of these to each)
        if constexpr (J == 0 && !ODD) {
            kid = block_id(t + 5, wave);
            vid = block_id(t + 4, wave);
        }
        if constexpr (J == 0 && ODD && FP8) {
            k_put = scale_of(k_scales, kid);
            v_put_next = scale_of(v_scales, vid);
        }
        if constexpr (J1 == 1 || J2 == 1) take_key_scales();
        if constexpr (J1 == 2 || J2 == 2) take_value_scales();
        if constexpr (J1 == 3 || J2 == 3) {
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
        see(first);
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
        if (!TREE || n < rows)   // (the merge takes no others)
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
        const int n = min(n_first + e * 32 + r32, rows - 1), last = min(TREE ? s.u.kv_len - 1 : ctx + n / G, end * kKeys - 1);
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
            if constexpr (TREE)
                if (!sees(s.u.q0 + n / G, pos)) continue;
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
