// Which calls of wide trees' attention the kernels of short calls (attn_tree_unit.hip, attn_tree_unit_f32.hip) take, and how it cuts them.  Plain host code, with a test of its own.
//
// Both kernels' times, in us, from the sizes that the host knows: batch, heads, the widest tree, and the width of the table as the bound of the lengths.
//
// Short calls: a workgroup's beginning and end, its rounds of eight steps, workgroups one after the other where there are more than the chip runs at a time (one to a compute unit),
// and the second launch where keys are split.  Measured with equal lengths, bf16, 8 KV heads of 128 with 4 query heads each (the formula in brackets): one request of 25 nodes
// behind 300 | 1000 | 4000 | 10000 tokens 10.2 | 14.4 | 30 | 59 (10 | 14 | 30 | 62); 16 requests behind 300 | 4000 20 | 76 (21 | 77); 16 of 64 nodes behind 4000 151 (153); e4m3 with 8
// query heads, one of 25 nodes behind 10000 87 (88), 16 behind 4000 163 (174); 64-wide heads, 16 of 64 nodes behind 10000 94 (95).
//
// The other kernel: what a call costs it without keys, as soon as tiles are cut 6 more (openings, partial results and their merge), and steps of 32 keys for 256 rows: of bf16 1.0, of
// e4m3 1.25 (measured where all compute units are busy: 1.06 and 1.27), of 64-wide heads 0.6 to each compute unit, three quarters of that where a tile has 128 rows or less; of those
// that the bound of the lengths gives, six tenths.
//
// Of 282 calls of 1 .. 64 requests with 6 .. 150 nodes behind up to 30000 tokens (lengths from half of the bound on; 32 heads over 8 of 128 in bf16, 64 over 8 in e4m3, 16 over 2 of
// 64 in bf16) the rule takes the fastest form, or one within 15 %, in 274, and 1.8 % more time than the fastest in the mean (profiles/tree_attention_forms.txt has them all).
//
// A table wider than the lengths makes calls look longer than they are.  25 nodes behind 300 tokens with 21 | 64 | 256 | 2048 columns: 10.1 | 12.8 | 13.9 | 18.5 us, 16 requests of
// them 19 | 19 | 25 | 25; the fp32 call of four, 64 | 256 columns, 12.6 | 24.4; long calls are level.
#pragma once

#include <stdint.h>

namespace ss {

constexpr int kTreeUnitRows = 32, kTreeUnitRowsF32 = 16;   // query rows of a tile
struct TreeUnitChoice {
    int32_t tiles;    // of a request and KV head, that are taken side by side; 0: the call is another kernel's
    int32_t splits;   // workgroups that share a tile's keys
};

inline double tree_unit_time(double tiles, double steps, int splits, int head_dim, bool kv8, int cus)
{
    const double wgs = tiles * splits, at_once = cus;
    const double full = wgs < at_once ? wgs / at_once : 1.0;
    const double turns = (double)(int64_t)((wgs + at_once - 1) / at_once), rounds = (double)(int64_t)((steps + 8 * splits - 1) / (8 * splits));
    // a round's time where the chip is empty, and how much longer it takes where it is full
    const double round = head_dim == 64 ? 1.0 : kv8 ? 2.0 + 0.1 * full : 1.3 + 0.6 * full;
    return 1.5 + turns * (5.7 + round * rounds) + (splits > 1 ? 3.5 : 0.0);
}
inline double tree_tile_time(double units, int64_t rows, double steps, int head_dim, bool kv8, int cus)
{
    // (a last tile of half the rows or less takes three quarters)
    const double tiles = (double)(rows / 256) + (rows % 256 == 0 ? 0.0 : rows % 256 <= 128 ? 0.75 : 1.0), each = units * tiles * steps / cus;
    const double step = head_dim == 64 ? 0.6 : kv8 ? 1.25 : 1.0;
    return 20.0 + 6.0 * (each < 5.0 ? each / 5.0 : 1.0) + step * 0.6 * each;   // (lengths taken to be 0.6 of the bound in the mean)
}

// rows: of the widest tree and a KV head, 0 if no bound of them is known
inline TreeUnitChoice tree_unit_rule(int batch, int num_kv_heads, int64_t rows, int64_t max_keys, int head_dim, bool kv8, int cus)
{
    const int64_t each = (rows + kTreeUnitRows - 1) / kTreeUnitRows, tiles = each * batch * num_kv_heads;
    if (rows <= 0 || tiles > 65536) return {0, 1};
    const double steps = (double)((max_keys + 31) / 32);
    double best = tree_tile_time((double)batch * num_kv_heads, rows, steps, head_dim, kv8, cus);
    TreeUnitChoice c = {0, 1};
    for (int splits = 1; splits <= 16 && (splits == 1 || steps >= 8.0 * splits); splits *= 2) {
        const double t = tree_unit_time((double)tiles, steps, splits, head_dim, kv8, cus);
        if (t < best) {
            best = t;
            c = {(int32_t)each, splits};
        }
    }
    return c;
}

// The same choice for calls in fp32 (attn_tree_unit_f32.hip): tiles that are taken side by side, 0 for the other kernel, whose tiles have 64 rows that share its steps of 64 keys.
// Both are bound by the fp32 matrix rate where they are large.  Short calls: 7 us, and 3.15 us a round of 256 keys (64-wide heads: two requests of 25 nodes behind 0 | 300 | 1000 |
// 4000 | 10000 tokens 8.6 | 11.0 | 20 | 57 | 134) or 3.4 of 128 (128-wide: 7.8 | 17.4 | 36 | 114 | 271), once for every workgroup to a compute unit; the other kernel on the same 17 |
// 24.5 | 23 | 28 | 39 and 23.5 | 38 | 35 | 67 | 142, sixteen of 64 nodes behind 300 36 | 90 (here 22.5 | 128).  Of 373 calls of 1 .. 64 requests with 6 .. 150 nodes behind up to 10000
// tokens of one length (three types, both widths) the choice is within 15 % of the faster in 358, and 1.9 % above it in the mean.
inline int32_t tree_unit_f32_rule(int batch, int num_kv_heads, int64_t rows, int64_t max_keys, int head_dim, int cus)
{
    const int64_t each = (rows + kTreeUnitRowsF32 - 1) / kTreeUnitRowsF32, wgs = each * batch * num_kv_heads;
    if (rows <= 0 || wgs > 65536) return 0;
    const bool narrow = head_dim == 64;
    const int keys_of_round = narrow ? 256 : 128;   // (one block to each of 16 or 8 wavefronts)
    const double turns = (double)((wgs + cus - 1) / cus), rounds = (double)((max_keys + keys_of_round - 1) / keys_of_round);
    const double unit = 7.0 + turns * (1.0 + (narrow ? 3.15 : 3.4) * rounds);
    const double steps = (double)((max_keys + 63) / 64), tiles = (double)((rows + 63) / 64) * batch * num_kv_heads;
    const double few = steps < 3.0 ? steps : 3.0, spread = 0.75 * tiles * steps / cus;   // (lengths taken to be 0.75 of the bound in the mean)
    const double other = 15.0 + (narrow ? 3.3 : 7.5) * (spread > few ? spread : few);
    return unit < other ? (int32_t)each : 0;
}

}  // namespace ss
