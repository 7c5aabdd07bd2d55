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
#include "attn_chunk_kernel.h"

namespace ss {

bool chunk_mfma_supported(int head_dim, int kv_dtype, int q_dtype)
{
    return (head_dim == 64 || head_dim == 128) && q_dtype == SS_BF16 && (kv_dtype == SS_BF16 || kv_dtype == SS_FP8_E4M3);
}

int32_t chunk_mfma_launch(const ChunkArgs &a, hipStream_t stream) { return launch_all<false>(a, stream); }

}  // namespace ss
