// How attention of a chunk is cut into workgroups' shares, worked out by every workgroup for itself from the requests' lengths (there is no kernel in
// front).
//
// A unit is a request's query rows of one KV head (row n = head n % G of the group at new token n / G); a tile is ROWS of them, a step kStepKeys
// keys, and steps(t) what the last row of tile t sees.  A tile's time is its steps.  With W = the steps of the whole call over the workgroups that run
// at a time, tiles of more than W steps are cut into equal pieces of at most W (all the cut tiles of a request into as many as its last tile); their
// results are partial and merged by their log-sum-exp.  steps(t) grows with t, so the tiles that are cut are the last ones of each request.  Pieces
// come first, then whole tiles, the longest of a request first: workgroups are started in this order, and a long share that starts last is what
// leaves compute units without work.
#pragma once

#include "prefill.h"

namespace ss {

constexpr int kStepKeys = 64;        // keys of a step
constexpr int kMinPiece = 4;         // steps below which a piece costs more than it brings

struct ChunkUnit {                   // a request, as one lane sees it
    int q0, q_len, kv_len, tiles, last;   // last: steps of its last tile
};

template <int ROWS>
struct ChunkCut {
    int G;
    __device__ int steps(const ChunkUnit &u, int t) const
    {
        const int tok = min((int)((((int64_t)t + 1) * ROWS - 1) / G), u.q_len - 1);
        const int seen = u.kv_len - u.q_len + tok + 1;
        return seen > 0 ? (int)(((unsigned)seen + kStepKeys - 1) / kStepKeys) : 0;
    }
    __device__ ChunkUnit unit(const ChunkArgs &a, int b) const
    {
        ChunkUnit u = {0, 0, 0, 0, 0};
        if (b < a.batch) {
            u.q0 = a.q_indptr[b];
            u.q_len = a.q_indptr[b + 1] - u.q0;
            u.kv_len = a.kv_len[b];
            u.tiles = u.q_len > 0 ? (int)(((int64_t)u.q_len * G + ROWS - 1) / ROWS) : 0;
            u.last = u.tiles ? steps(u, u.tiles - 1) : 0;
        }
        return u;
    }
    // Pieces of the tiles that are cut, and the first of these (`tiles` if there is none), for shares of at most w steps.
    __device__ int pieces(const ChunkUnit &u, int w, int &t0) const
    {
        t0 = u.tiles;
        if (u.last <= w) return 1;
        // the first tile with steps > w: its last token sees more than w * kStepKeys keys
        const int64_t tok = (int64_t)w * kStepKeys - (u.kv_len - u.q_len);   // at least this token
        t0 = tok <= 0 ? 0 : (int)((tok * G + ROWS) / ROWS) - 1;
        t0 = min(t0, u.tiles - 1);
        return (u.last + w - 1) / w;
    }
};

template <typename T>
__device__ __forceinline__ T wave_incl_sum(T x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

struct ChunkShare {
    int b, q0, q_len, kv_len;   // the request
    int tile, s0, s1;           // its tile, the steps of this share
    int piece, pieces;          // pieces > 1: a partial result
    int slot;                   // of the partial result, without the KV head
    int cut;                    // the tile's place among those that are cut
    int cuts;                   // tiles that are cut, over all requests
};

template <int ROWS>
__device__ __forceinline__ bool chunk_find(const ChunkArgs &a, int item, ChunkShare &out)
{
    const ChunkCut<ROWS> c = {a.num_q_heads / a.num_kv_heads};
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    if (a.cap > 0) {   // (steps grow evenly over a request's tiles)
        for (int lo = 0; lo < a.batch; lo += 64) {
            const ChunkUnit u = c.unit(a, lo + lane);
            if (u.tiles) total += (int64_t)u.tiles * (u.last + c.steps(u, 0) + 1) / 2;
        }
#pragma unroll
        for (int off = 32; off; off >>= 1) total += __shfl_xor(total, off);
    }
    int64_t w64 = total * a.num_kv_heads / a.target + 1;
    int w = a.cap > 0 ? (int)(w64 < kMinPiece ? kMinPiece : w64 > 0x3fffffff ? 0x3fffffff : w64) : 0x3fffffff;
    // the partial results have to fit: seldom more than one round
    int split = 0, cuts = 0;
    for (;;) {
        int64_t n = 0;
        cuts = 0;
        for (int lo = 0; lo < a.batch; lo += 64) {
            const ChunkUnit u = c.unit(a, lo + lane);
            int t0;
            const int p = c.pieces(u, w, t0);
            n += (int64_t)(u.tiles - t0) * p;
            cuts += u.tiles - t0;
        }
#pragma unroll
        for (int off = 32; off; off >>= 1) {
            n += __shfl_xor(n, off);
            cuts += __shfl_xor(cuts, off);
        }
        if (n * a.num_kv_heads <= a.cap) { split = (int)n; break; }
        w = w > 0x1fffffff ? 0x3fffffff : 2 * w;
    }
    split = __builtin_amdgcn_readfirstlane(split);
    const bool whole = item >= split;
    int rest = whole ? item - split : item, cut_before = 0;
    for (int lo = 0; lo < a.batch; lo += 64) {
        const ChunkUnit u = c.unit(a, lo + lane);
        int t0;
        const int p = c.pieces(u, w, t0);
        const int mine = whole ? t0 : (u.tiles - t0) * p;
        const int incl = wave_incl_sum(mine), cut_incl = wave_incl_sum(u.tiles - t0);
        const uint64_t here = __ballot(incl > rest);
        if (here) {
            const int at = __builtin_ctzll(here);
            out.b = lo + at;
            out.q0 = __builtin_amdgcn_readlane(u.q0, at);
            out.q_len = __builtin_amdgcn_readlane(u.q_len, at);
            out.kv_len = __builtin_amdgcn_readlane(u.kv_len, at);
            const int idx = rest - __builtin_amdgcn_readlane(incl - mine, at);
            const int n = __builtin_amdgcn_readlane(p, at), tiles = __builtin_amdgcn_readlane(u.tiles, at);
            const int first = __builtin_amdgcn_readlane(t0, at);
            const ChunkUnit v = {out.q0, out.q_len, out.kv_len, tiles, 0};
            out.pieces = whole ? 1 : n;
            out.piece = whole ? 0 : idx % n;
            out.tile = whole ? first - 1 - idx : tiles - 1 - idx / n;
            const int s = c.steps(v, out.tile);
            out.s0 = (int)((int64_t)s * out.piece / out.pieces);
            out.s1 = (int)((int64_t)s * (out.piece + 1) / out.pieces);
            out.slot = item;
            out.cut = cut_before + __builtin_amdgcn_readlane(cut_incl - (u.tiles - t0), at) + idx / n;
            out.cuts = __builtin_amdgcn_readfirstlane(cuts);
            return true;
        }
        rest -= last_lane(incl);
        cut_before += last_lane(cut_incl);
    }
    out.cuts = __builtin_amdgcn_readfirstlane(cuts);
    return false;
}

// The share number `item`, for a whole wavefront, in scalar registers; false if there are not so many.
template <int ROWS>
__device__ __forceinline__ bool chunk_share(const ChunkArgs &a, int item, ChunkShare &out)
{
    ChunkShare s = {};
    const bool any = chunk_find<ROWS>(a, item, s);
    out.b = __builtin_amdgcn_readfirstlane(s.b);
    out.q0 = __builtin_amdgcn_readfirstlane(s.q0);
    out.q_len = __builtin_amdgcn_readfirstlane(s.q_len);
    out.kv_len = __builtin_amdgcn_readfirstlane(s.kv_len);
    out.tile = __builtin_amdgcn_readfirstlane(s.tile);
    out.s0 = __builtin_amdgcn_readfirstlane(s.s0);
    out.s1 = __builtin_amdgcn_readfirstlane(s.s1);
    out.piece = __builtin_amdgcn_readfirstlane(s.piece);
    out.pieces = __builtin_amdgcn_readfirstlane(s.pieces);
    out.slot = __builtin_amdgcn_readfirstlane(s.slot);
    out.cut = __builtin_amdgcn_readfirstlane(s.cut);
    out.cuts = __builtin_amdgcn_readfirstlane(s.cuts);
    return __builtin_amdgcn_readfirstlane(any);
}

}  // namespace ss
