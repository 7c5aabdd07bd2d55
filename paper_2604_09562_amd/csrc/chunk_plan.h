// How attention of a chunk is cut into workgroups' shares, worked out by every workgroup for itself from the requests' lengths (there is no kernel in
// front).
//
// A unit is a request's query rows of one KV head (row n = head n % G of the group at new token n / G), a tile `rows` of them, and steps(t) are the steps of
// `keys` keys up to what the last row of tile t sees.  The tiles of all requests, end to end, are cut into spans of equal cost, a tile costing its steps and
// OPEN more (its queries, the first keys, its results); every KV head has the same spans.  What a span's ends cut off a tile is a partial result, merged by its
// log-sum-exp; a workgroup has at most two.  The cost in front of tile t of a request is taken as if steps(t) grew evenly from its first to its
// last tile: workgroups need the same cuts, and cuts of nearly equal cost.
#pragma once

#include "prefill.h"

namespace ss {

// Steps below which a piece costs more than it brings, where there are not spans enough for all workgroups.  With 2 | 3 | 5, us: one token behind 64 14.1 | 11.6 |
// 12.3, 33 behind 700 18.7 | 21.0 | 21.4, a prompt of 500 28.7 | 26.7 | 28.4, 200 behind 1000 35.2 | 35.2 | 32.7 (32 heads over 8, bf16); over an e4m3 cache a prompt of 500
// 31.2 | 28.7 | 31.8, 64 behind 2000 27.7 | 27.0 | 30.7; fp32, two requests of 100 behind 400, 25.3 | 25.3 | 38.7.
constexpr int kMinPiece = 3;
constexpr int kOpenFew = 1;          // a tile's cost beside its steps where there are not spans enough for all workgroups: their openings run side by side
// Steps of a tile that no cut is made for.  With 0 | 1 | 2, us: 33 tokens behind 700 21.0 | 21.0 | 22.1, a prompt of 2048 64.2 | 63.2 | 63.2; fp32, four requests
// of 20 .. 150 tokens, 24.6 | 24.9 | 33.9.
constexpr int kSnap = 1;

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
__device__ __forceinline__ double lane_value(double x, int lane)
{
    const uint64_t w = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)w, lane), hi = __builtin_amdgcn_readlane((uint32_t)(w >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int ROWS, int KEYS>
struct ChunkUnit {                   // a request
    int q0, q_len, kv_len, G, open;  // open: what a tile costs beside its steps
    int tiles, first, last;          // steps of its first and last tile
    double slope;

    __device__ __forceinline__ int steps(int t) const
    {
        const int tok = min((int)(((uint32_t)(t + 1) * ROWS - 1) / (uint32_t)G), q_len - 1), seen = kv_len - q_len + tok + 1;
        return seen > 0 ? (int)(((unsigned)seen + KEYS - 1) / KEYS) : 0;
    }
    // A request.  One whose rows are outside of the call's or whose cache is longer than its row of the table has no tiles: nothing of it is read or written.
    __device__ __forceinline__ void set(const ChunkArgs &a, int q0_, int q1, int len, int open_)
    {
        open = open_;
        q0 = q0_;
        const bool fits = q0_ >= 0 && q1 >= q0_ && q1 <= a.total_rows && len <= (a.num_blocks > 0 ? a.max_blocks * kTile : 0);
        q_len = fits ? q1 - q0_ : 0;
        kv_len = max(len, 0);
        G = a.num_q_heads / a.num_kv_heads;
        tiles = q_len > 0 ? (int)(((uint32_t)q_len * (uint32_t)G + ROWS - 1) / ROWS) : 0;
        first = tiles ? steps(0) : 0;
        last = tiles ? steps(tiles - 1) : 0;
        slope = tiles > 1 ? (last - first) / (2.0 * (tiles - 1)) : 0.0;
    }
    // cost of the tiles in front of tile t
    __device__ __forceinline__ double before(int t) const { return (double)t * (open + first) + __builtin_floor(slope * t * (t - 1.0)); }
    // the step of tile t at which a cut of this cost (counted from the request's first tile) falls: 0 and steps(t) are no cuts
    __device__ __forceinline__ int cut(double x, int t, int n) const
    {
        const double off = x - before(t) - open;
        return off <= kSnap ? 0 : off >= n - kSnap ? n : (int)off;
    }
};

struct ChunkPos {
    int b, t, off;   // a request's tile, the steps of it that are done
    double base;     // cost in front of the request
};

// A workgroup's span, piece by piece; all of it uniform over a wavefront.
template <int ROWS, int KEYS, int OPEN>
struct ChunkWalk {
    typedef ChunkUnit<ROWS, KEYS> Unit;
    static_assert(OPEN > kOpenFew, "begin() takes the cost of few spans once, where the other one does not do");
    // the current piece: steps s0 to before s1 of tile t of request b.  part: place of its partial result, -1 if it is the whole tile.
    int b, t, s0, s1, part;
    Unit u;
    int spans;       // in use

    __device__ __forceinline__ bool begin(const ChunkArgs &a, int span)
    {
        me = span;
        const int lane = threadIdx.x & 63, G = a.num_q_heads / a.num_kv_heads;
        double total = 0.0, incl = 0.0;
        Unit mine = {};
        open = OPEN;
        for (;;) {   // the cost of everything
            total = 0.0;
            for (int lo = 0; lo < a.batch; lo += 64) {
                mine = unit(a, lo + lane, G);
                incl = wave_incl_sum(mine.before(mine.tiles));
                total += lane_value(incl, 63);
            }
            if (open < OPEN || total >= (double)a.spans * (OPEN + kMinPiece)) break;
            open = kOpenFew;
        }
        const double most = open == OPEN ? a.spans : total / kMinPiece;
        spans = uniform(most < 1.0 ? 1 : most < a.spans ? (int)most : a.spans);
        if (span >= spans || total == 0.0) return false;
        share = total / spans;
        Unit unused;
        const ChunkPos from = locate(a, __builtin_floor(share * span), mine, incl, G, u);
        to.b = a.batch;
        to.t = to.off = 0;
        if (span + 1 < spans) to = locate(a, __builtin_floor(share * (span + 1)), mine, incl, G, unused);
        base = from.base;
        b = from.b;
        t = from.t;
        s0 = from.off;
        if (s0 > 0 && s0 == u.steps(t)) {   // the span in front has all of this tile
            s0 = 0;
            ++t;
        }
        return settle(a);
    }
    __device__ __forceinline__ bool next(const ChunkArgs &a)
    {
        s0 = 0;
        ++t;
        return settle(a);
    }
    // pieces of the current tile, which this span begins and does not end: one more than the cuts that fall into it, as locate() assigns them (a cut is
    // the last tile's that begins at or in front of it, whatever is left of the tile's steps there: costs are interpolated, steps are not)
    __device__ __forceinline__ int pieces() const
    {
        const int lane = threadIdx.x & 63, n = u.steps(t);
        const double behind = u.before(t + 1);
        int count = 1;
        for (int j = me + 1;; j += 64) {
            const double x = __builtin_floor(share * (j + lane)) - base;
            const bool inside = j + lane < spans && x < behind && u.cut(x, t, n) < n;
            const uint64_t m = __ballot(inside);   // (the cuts ascend)
            count += __popcll(m);
            if (m != ~0ull) return uniform(count);
        }
    }

private:
    int me, open;
    double share, base;
    ChunkPos to;

    __device__ __forceinline__ Unit unit(const ChunkArgs &a, int i, int G) const
    {
        Unit r = {};
        r.G = G;
        r.open = open;
        if (i < a.batch) r.set(a, a.q_indptr[i], a.q_indptr[i + 1], a.kv_len[i], open);
        return r;
    }
    __device__ __forceinline__ Unit request(const ChunkArgs &a, int i) const
    {
        Unit r;
        r.set(a, uniform(a.q_indptr[i]), uniform(a.q_indptr[i + 1]), uniform(a.kv_len[i]), open);
        return r;
    }
    // Moves on to the next tile that there is and sets the piece's end; false behind the span's end.
    __device__ __forceinline__ bool settle(const ChunkArgs &a)
    {
        while (t >= u.tiles) {
            base += u.before(u.tiles);
            t = 0;
            if (++b >= a.batch) return false;
            u = request(a, b);
        }
        const int n = uniform(u.steps(t));
        s1 = n;
        if (b > to.b || (b == to.b && (t > to.t || (t == to.t && to.off == 0)))) return false;
        if (b == to.b && t == to.t) s1 = to.off;
        part = s0 > 0 ? 2 * me : s1 < n ? 2 * me + 1 : -1;
        return true;
    }
    // Where a cost falls, and in which request.  mine, incl: the units and sums of the last 64 requests.
    __device__ __forceinline__ ChunkPos locate(const ChunkArgs &a, double x, Unit mine, double incl, int G, Unit &v) const
    {
        const int lane = threadIdx.x & 63;
        ChunkPos p = {a.batch, 0, 0, 0.0};
        double front = 0.0;
        for (int lo = 0; lo < a.batch; lo += 64) {
            if (a.batch > 64) {
                mine = unit(a, lo + lane, G);
                incl = wave_incl_sum(mine.before(mine.tiles));
            }
            const uint64_t here = __ballot(front + incl > x);
            if (here) {
                const int at = __builtin_ctzll(here);
                v.G = G;
                v.open = open;
                v.q0 = __builtin_amdgcn_readlane(mine.q0, at);
                v.q_len = __builtin_amdgcn_readlane(mine.q_len, at);
                v.kv_len = __builtin_amdgcn_readlane(mine.kv_len, at);
                v.tiles = __builtin_amdgcn_readlane(mine.tiles, at);
                v.first = __builtin_amdgcn_readlane(mine.first, at);
                v.slope = lane_value(mine.slope, at);
                p.b = uniform(lo + at);
                p.base = at ? front + lane_value(incl, at - 1) : front;
                const double y = x - p.base;
                int t = 0, n = v.tiles;      // the last tile that begins at or in front of y
                while (n > 1) {
                    const int step = (n + 63) / 64, i = lane * step;
                    const int k = __popcll(__ballot(i < n && v.before(t + i) <= y)) - 1;
                    t += k * step;
                    n = min(step, n - k * step);
                }
                p.t = uniform(t);
                p.off = uniform(v.cut(y, p.t, v.steps(p.t)));
                return p;
            }
            front += lane_value(incl, 63);
        }
        return p;
    }
};

}  // namespace ss
