// Blocks that several requests hold: forks, releases, and the move of all blocks in use to the front of a cache.
//
// shares[x] counts a block's holders beyond the first.  All three calls are whole numbers in orders that their definitions fix, so the result does not
// depend on which thread comes first: additions to shares commute, and where an order counts (which block is taken, where one comes to
// stand in the free list) it is a prefix sum.  Bound by latency: chains of lengths, sums, ids and counts, about 1 us each: 96 forks of requests of 256 .. 4096 tokens 4.6 + 3.4 us, a small
// cache's compaction 5.4, one of 3910 blocks 4.8 + 6.4.
#include "block_share.h"

namespace ss {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kNone = 0x7fffffff;

__device__ __forceinline__ int blocks_of(int len) { return (int)(((unsigned)len + kTile - 1) / kTile); }

// Inclusive sum over the workgroup of `threads` threads; total: of all of them.
template <int THREADS>
__device__ __forceinline__ int group_scan(int x, int *part, int &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int add = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        add += w < wave ? part[w] : 0;
        total += part[w];
    }
    __syncthreads();
    return x + add;
}
// What other threads of this kernel have changed by atomics (a plain load may find it in the first cache as it was).
__device__ __forceinline__ int current(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// ---- forks -------------------------------------------------------------------------------------------------------------
struct ForkLds {
    int part[kWaves];
    int bad;
};

// One workgroup: whether all forks can be, and what of each is one number; 0 if it was done.
__device__ int fork_books(const BlockForkArgs &a, ForkLds &lds)
{
    const int tid = threadIdx.x;
    int32_t *rank = a.scratch, *named = rank + a.num_forks;   // blocks taken by the forks in front; the first fork that names a row as its child
    for (int b = tid; b < a.batch; b += kThreads) named[b] = kNone;
    if (tid == 0) lds.bad = kNone;
    const int count = a.free_count[0];
    __threadfence_block();
    __syncthreads();
    for (int i = tid; i < a.num_forks; i += kThreads) {
        const int c = a.child[i];
        if (a.parent[i] >= 0 && (unsigned)c < (unsigned)a.batch) atomicMin(&named[c], i);
    }
    __threadfence_block();
    __syncthreads();
    int taken = 0;
    for (int lo = 0; lo < a.num_forks; lo += kThreads) {
        const int i = lo + tid;
        int part = 0;
        if (i < a.num_forks && a.parent[i] >= 0) {
            const int p = a.parent[i], c = a.child[i];
            bool ok = p < a.batch && (unsigned)c < (unsigned)a.batch;
            if (ok) {
                const int n = a.kv_len[p], h = a.held[p], len = a.length ? a.length[i] : n;
                ok = current(&named[c]) == i && current(&named[p]) == kNone && a.held[c] == 0 && n >= 0 && len >= 0 && len <= n && h >= 0 &&
                     blocks_of(len) <= min(h, a.max_blocks);
                part = ok && len % kTile != 0;
            }
            if (!ok) atomicMin(&lds.bad, i);
        }
        int total;
        const int incl = group_scan<kThreads>(part, lds.part, total);
        if (i < a.num_forks) rank[i] = taken + incl - part;
        taken += total;
    }
    __syncthreads();
    int status = 0;
    if (lds.bad != kNone) status = -1 - lds.bad;
    else if (count < 0 || count > a.num_blocks) status = -1 - a.num_forks;
    else if (taken > count) status = taken - count;
    // (every thread has read what it needs of the parents; the rows written here are children, which no fork has as its parent)
    for (int i = tid; i < a.num_forks; i += kThreads) {
        int src = -1, dst = -1;
        const int p = a.parent[i];
        if (status == 0 && p >= 0) {
            const int c = a.child[i], len = a.length ? a.length[i] : a.kv_len[p], whole = len / kTile;
            if (len % kTile) {
                src = a.block_table[(int64_t)p * a.max_blocks + whole];
                dst = a.free_ids[count - 1 - rank[i]];
                a.block_table[(int64_t)c * a.max_blocks + whole] = dst;
            }
            a.held[c] = blocks_of(len);
            a.kv_len[c] = len;
        }
        a.copy_src[i] = src;
        a.copy_dst[i] = dst;
    }
    if (tid == 0) {
        a.status[0] = status;
        if (status == 0) a.free_count[0] = count - taken;
    }
    return status;
}

__device__ __forceinline__ void share_entry(const BlockForkArgs &a, int p, int c, int j)
{
    const int x = a.block_table[(int64_t)p * a.max_blocks + j];
    a.block_table[(int64_t)c * a.max_blocks + j] = x;
    if ((unsigned)x < (unsigned)a.num_blocks) atomicAdd(&a.shares[x], 1);
}

__global__ __launch_bounds__(kThreads) void block_fork_kernel(BlockForkArgs a, int whole_call)
{
    __shared__ ForkLds lds;
    if (fork_books(a, lds) != 0 || !whole_call) return;
    __threadfence_block();
    __syncthreads();
    for (int e = threadIdx.x; e < a.num_forks * a.max_blocks; e += kThreads) {
        const int i = e / a.max_blocks, j = e % a.max_blocks, p = a.parent[i];
        if (p < 0) continue;
        const int len = a.length ? a.length[i] : a.kv_len[p];
        if (j < len / kTile) share_entry(a, p, a.child[i], j);
    }
}

constexpr int kForkThreads = 256, kForkEach = 4;   // entries of a table's row to a thread

__global__ __launch_bounds__(kForkThreads) void block_fork_rows_kernel(BlockForkArgs a)
{
    const int i = blockIdx.x, p = a.parent[i];
    if (a.status[0] != 0 || p < 0) return;
    const int whole = (a.length ? a.length[i] : a.kv_len[p]) / kTile, c = a.child[i];
    for (int lo = blockIdx.y * kForkThreads * kForkEach + threadIdx.x; lo < whole; lo += gridDim.y * kForkThreads * kForkEach)
#pragma unroll
        for (int k = 0; k < kForkEach; ++k)
            if (lo + k * kForkThreads < whole) share_entry(a, p, c, lo + k * kForkThreads);
}

// ---- releases ----------------------------------------------------------------------------------------------------------
// Releases are counted in the order of request, logical block.  Release r takes one from its block's shares and leaves its number in the block's entry of `last`, if no later one
// does; what is below zero then has no holder left, and goes to the list at its last release's place, behind those of lower number.
// One workgroup does a table of up to 2^14 entries; else the sums are one workgroup's, while others clear `last`, and the releases many workgroups', in three launches: taken and named,
// those that free a block counted by pieces, put on the list (2.5 + 5.7 + 6.5 + 5 us for 240 000 entries; with names in a launch of their own 26 us in all). A workgroup by itself is
// bound by six scattered accesses a release: with 64 requests of 256 entries, by number of releases, 0 | 256 | 1024 | 2048 | 4096 | 16384, 6 | 6 | 10 | 18 | 32 | 118 us, and 14.5 to 16.5
// in four launches. A step gives back some blocks of drafts and those of a request or two that have ended.
constexpr int kReleaseHead = 4;       // scratch: length of the free list, releases
constexpr int kReleasePiece = 1024;   // releases whose freed blocks are counted together
constexpr int kReleaseLds = 1024;     // requests whose sums a workgroup keeps in LDS
constexpr int kReleaseThreads = 256;
constexpr int64_t kReleaseKept = 1 << 24;   // entries of a table up to which releases' blocks are kept in the workspace (64 MB)

struct ReleaseScratch {
    int32_t *head, *given, *freed_in, *last, *ids;   // ids: nullptr in large tables
};
__host__ __device__ inline ReleaseScratch release_scratch(int32_t *p, int batch, int max_blocks, int num_blocks)
{
    ReleaseScratch s;
    const int64_t entries = (int64_t)batch * max_blocks;
    s.head = p;
    s.given = p + kReleaseHead;                       // [batch + 1] releases in front of each request
    s.freed_in = s.given + batch + 1;                 // [pieces]
    s.last = s.freed_in + (entries + kReleasePiece - 1) / kReleasePiece;   // [num_blocks]
    s.ids = entries <= kReleaseKept ? s.last + num_blocks : nullptr;       // [entries]
    return s;
}

struct Releases {
    const BlockReleaseArgs &a;
    const ReleaseScratch &s;
    const int32_t *given;
    // the block of release r, -1 if it is none
    __device__ int find(int r) const
    {
        int lo = 0, hi = a.batch;     // the last request with given[lo] <= r
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (given[mid] <= r) lo = mid; else hi = mid;
        }
        const int x = a.block_table[(int64_t)lo * a.max_blocks + blocks_of(a.kv_len[lo]) + r - given[lo]];
        return (unsigned)x < (unsigned)a.num_blocks ? x : -1;
    }
    __device__ void take(int r) const
    {
        const int x = find(r);
        if (s.ids) s.ids[r] = x;
        if (x >= 0) {
            atomicSub(&a.shares[x], 1);
            atomicMax(&s.last[x], r);
        }
    }
    // the block that release r puts on the list, or -1
    __device__ int freed(int r) const
    {
        const int x = s.ids ? s.ids[r] : find(r);
        return x >= 0 && current(&s.last[x]) == r && current(&a.shares[x]) < 0 ? x : -1;
    }
};

struct ReleaseLds {
    int part[kWaves];
    int bad;
};

// One workgroup: the sums of all requests, and what they hold; false if something does not fit.
__device__ bool release_sums(const BlockReleaseArgs &a, ReleaseLds &lds, int32_t *given, int &count, int &releases)
{
    const int tid = threadIdx.x;
    if (tid == 0) lds.bad = kNone;
    count = a.free_count[0];
    __syncthreads();
    releases = 0;
    for (int lo = 0; lo < a.batch; lo += kThreads) {
        const int b = lo + tid;
        int g = 0;
        if (b < a.batch) {
            const int n = a.kv_len[b], h = a.held[b];
            if (n < 0 || h < 0 || h > a.max_blocks) atomicMin(&lds.bad, b);
            else g = max(h - blocks_of(n), 0);
        }
        int total;
        const int incl = group_scan<kThreads>(g, lds.part, total);
        if (b < a.batch) given[b] = releases + incl - g;
        releases += total;
    }
    __syncthreads();
    int status = 0;
    if (lds.bad != kNone) status = -1 - lds.bad;
    else if (count < 0 || count > a.num_blocks) status = -1 - a.batch;
    if (tid == 0) {
        given[a.batch] = releases;
        a.status[0] = status;
    }
    if (status == 0)
        for (int b = tid; b < a.batch; b += kThreads) a.held[b] = min(a.held[b], blocks_of(a.kv_len[b]));
    return status == 0;
}

__global__ __launch_bounds__(kThreads) void block_release_kernel(BlockReleaseArgs a)
{
    constexpr int EACH = 4;   // releases of a thread that are under way together
    __shared__ ReleaseLds lds;
    __shared__ int32_t sums[kReleaseLds + 1];
    const ReleaseScratch w = release_scratch(a.scratch, a.batch, a.max_blocks, a.num_blocks);
    int32_t *given = a.batch <= kReleaseLds ? sums : w.given;
    int count, releases;
    if (!release_sums(a, lds, given, count, releases)) return;
    __threadfence_block();
    __syncthreads();
    const Releases s = {a, w, given};
    for (int lo = threadIdx.x; lo < releases; lo += EACH * kThreads) {
        int x[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) x[k] = lo + k * kThreads < releases ? s.find(lo + k * kThreads) : -1;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (lo + k * kThreads < releases) w.ids[lo + k * kThreads] = x[k];
            if (x[k] >= 0) __hip_atomic_store(&w.last[x[k]], -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __threadfence_block();
    __syncthreads();
    for (int lo = threadIdx.x; lo < releases; lo += EACH * kThreads)
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int r = lo + k * kThreads, x = r < releases ? w.ids[r] : -1;
            if (x >= 0) {
                atomicSub(&a.shares[x], 1);
                atomicMax(&w.last[x], r);
            }
        }
    __threadfence_block();
    __syncthreads();
    int at = count;
    for (int lo = 0; lo < releases; lo += EACH * kThreads) {
        const int first = lo + threadIdx.x * EACH;
        int x[EACH], mine = 0, total;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            x[k] = first + k < releases ? s.freed(first + k) : -1;
            mine += x[k] >= 0;
        }
        int place = at + group_scan<kThreads>(mine, lds.part, total) - mine;
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (x[k] >= 0) {
                if (place < a.num_blocks) a.free_ids[place] = x[k];
                a.shares[x[k]] = 0;    // (this release alone has found it below zero)
                ++place;
            }
        at += total;
    }
    if (threadIdx.x == 0) a.free_count[0] = min(at, a.num_blocks);
}

// The first workgroup sums, the others clear.
__global__ __launch_bounds__(kThreads) void block_release_sum_kernel(BlockReleaseArgs a)
{
    __shared__ ReleaseLds lds;
    const ReleaseScratch w = release_scratch(a.scratch, a.batch, a.max_blocks, a.num_blocks);
    if (blockIdx.x > 0) {
        for (int64_t x = (int64_t)(blockIdx.x - 1) * kThreads + threadIdx.x; x < a.num_blocks; x += (int64_t)(gridDim.x - 1) * kThreads) w.last[x] = -1;
        return;
    }
    int count, releases;
    const bool ok = release_sums(a, lds, w.given, count, releases);
    if (threadIdx.x == 0) {
        w.head[0] = count;
        w.head[1] = ok ? releases : 0;
    }
}

enum { kTake, kCount, kPlace };

template <int PHASE>
__global__ __launch_bounds__(kReleaseThreads) void block_release_phase_kernel(BlockReleaseArgs a)
{
    constexpr int EACH = kReleasePiece / kReleaseThreads;
    __shared__ int32_t sums[kReleaseLds + 1];
    __shared__ int part[kReleaseThreads / 64];
    const ReleaseScratch w = release_scratch(a.scratch, a.batch, a.max_blocks, a.num_blocks);
    const int tid = threadIdx.x, count = w.head[0], releases = w.head[1];
    const bool search = PHASE == kTake || !w.ids, lds = search && a.batch <= kReleaseLds;
    if (blockIdx.x * (PHASE == kTake ? kReleaseThreads : kReleasePiece) >= (unsigned)releases) return;
    if (lds) {
        for (int b = tid; b <= a.batch; b += kReleaseThreads) sums[b] = w.given[b];
        __syncthreads();
    }
    const Releases s = {a, w, lds ? sums : w.given};
    if constexpr (PHASE == kTake) {
        for (int64_t r = (int64_t)blockIdx.x * kReleaseThreads + tid; r < releases; r += (int64_t)gridDim.x * kReleaseThreads) s.take((int)r);
    } else {
        const int pieces = (releases + kReleasePiece - 1) / kReleasePiece;
        for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
            const int first = piece * kReleasePiece + tid * EACH;
            int x[EACH], mine = 0, total;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                x[k] = first + k < releases ? s.freed(first + k) : -1;
                mine += x[k] >= 0;
            }
            const int incl = group_scan<kReleaseThreads>(mine, part, total);
            if constexpr (PHASE == kCount) {
                if (tid == 0) w.freed_in[piece] = total;
            } else {
                int front = 0, before;
                for (int i = tid; i < piece; i += kReleaseThreads) front += w.freed_in[i];
                group_scan<kReleaseThreads>(front, part, before);
                int place = count + before + incl - mine;
#pragma unroll
                for (int k = 0; k < EACH; ++k)
                    if (x[k] >= 0) {
                        if (place < a.num_blocks) a.free_ids[place] = x[k];
                        a.shares[x[k]] = 0;   // (this release alone has found it below zero)
                        ++place;
                    }
                if (piece == pieces - 1 && tid == 0) a.free_count[0] = min(count + before + total, a.num_blocks);
            }
        }
    }
}

// ---- all blocks in use to the front ------------------------------------------------------------------------------------
constexpr int kCompactHead = 4;          // scratch: status, length of the free list, moves
constexpr int kCompactThreads = 256;
constexpr int kBitmapWords = 15360;      // of the free blocks, up to which they are put together in LDS (491 520 blocks)

struct Compact {
    int32_t *head;
    uint32_t *bits;                      // bit per block: free
    int32_t *front;                      // free blocks in front of each word; one more
    __device__ bool free(int i) const { return bits[i >> 5] >> (i & 31) & 1; }
    __device__ int free_before(int i) const { return front[i >> 5] + __popc(bits[i >> 5] & ((1u << (i & 31)) - 1u)); }
    // the r-th free block
    __device__ int nth_free(int r, int words) const
    {
        int lo = 0, hi = words;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (front[mid] <= r) lo = mid; else hi = mid;
        }
        uint32_t w = bits[lo];
        for (int k = r - front[lo]; k > 0; --k) w &= w - 1;
        return lo * 32 + __ffs((int)w) - 1;
    }
};

__device__ __forceinline__ int words_of(int num_blocks) { return (num_blocks + 31) / 32; }

struct CompactLds {
    int part[kWaves];
    int bad, list;
};

// One workgroup: which blocks are free, and how many in front of each word of them.  build: where the bits are put together.
__device__ void compact_bits(const BlockCompactArgs &a, CompactLds &lds, uint32_t *build, const Compact &s)
{
    const int tid = threadIdx.x, words = words_of(a.num_blocks);
    if (tid == 0) { lds.bad = kNone; lds.list = 0; }
    for (int w = tid; w < words; w += kThreads) build[w] = 0;
    __threadfence_block();
    __syncthreads();
    const int count = a.free_count[0];
    if (count < 0 || count > a.num_blocks) {
        if (tid == 0) lds.list = 1;
    } else {
        for (int i = tid; i < count; i += kThreads) {
            const int x = a.free_ids[i];
            if ((unsigned)x >= (unsigned)a.num_blocks || atomicOr(&build[x >> 5], 1u << (x & 31)) >> (x & 31) & 1) lds.list = 1;
        }
    }
    for (int b = tid; b < a.batch; b += kThreads)
        if (a.held[b] < 0 || a.held[b] > a.max_blocks) atomicMin(&lds.bad, b);
    __threadfence_block();
    __syncthreads();
    const int status = lds.bad != kNone ? -1 - lds.bad : lds.list ? -1 - a.batch : 0;
    int before = 0;
    for (int lo = 0; lo < words; lo += kThreads) {
        const int w = lo + tid;
        uint32_t v = 0;
        if (w < words) v = __hip_atomic_load(&build[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int n = __popc(v);
        int total;
        const int incl = group_scan<kThreads>(n, lds.part, total);
        if (w < words) {
            s.bits[w] = v;
            s.front[w] = before + incl - n;
        }
        before += total;
    }
    if (tid == 0) {
        s.front[words] = before;
        s.head[0] = status;
        s.head[1] = count;
        a.status[0] = status;
    }
}

// Everything else, shared out over `threads` threads.
__device__ void compact_rest(const BlockCompactArgs &a, const Compact &s, int64_t first, int64_t threads)
{
    const int N = a.num_blocks, words = words_of(N), half = N / 2;
    const bool ok = s.head[0] == 0;
    const int count = s.head[1], used = ok ? N - count : N;
    const int moves = ok && used < N ? s.free_before(used) : 0;   // free ids below `used`, as many as blocks in use from there on
    if (first == 0) a.num_copies[0] = moves;
    for (int64_t k = moves + first; k < half; k += threads) a.copy_src[k] = a.copy_dst[k] = -1;
    for (int64_t i64 = first; i64 < N; i64 += threads) {
        const int i = (int)i64;
        int to = i;
        if (ok) {
            const bool is_free = s.free(i);
            const int f = s.free_before(i);
            if (is_free && i < used) {
                a.copy_dst[f] = i;
            } else if (!is_free && i >= used) {
                const int r = i - used - (f - moves);
                to = s.nth_free(r, words);
                a.copy_src[r] = i;
                if (a.shares) {
                    a.shares[to] = a.shares[i];
                    a.shares[i] = 0;
                }
            }
            if (i < count) a.free_ids[i] = N - 1 - i;
        }
        if (a.remap) a.remap[i] = to;
    }
    if (!ok) return;
    const int64_t entries = (int64_t)a.batch * a.max_blocks;
    for (int64_t e = first; e < entries; e += threads) {
        const int b = (int)(e / a.max_blocks), j = (int)(e % a.max_blocks);
        if (j >= a.held[b]) continue;
        const int x = a.block_table[e];
        if (x < used || x >= N || s.free(x)) continue;
        a.block_table[e] = s.nth_free(x - used - (s.free_before(x) - moves), words);
    }
}

template <bool LDS, bool WHOLE>
__global__ __launch_bounds__(kThreads) void block_compact_kernel(BlockCompactArgs a, Compact s)
{
    extern __shared__ uint32_t bitmap[];   // LDS: words of the bitmap
    __shared__ CompactLds lds;
    compact_bits(a, lds, LDS ? bitmap : s.bits, s);
    if constexpr (WHOLE) {
        __threadfence_block();
        __syncthreads();
        compact_rest(a, s, threadIdx.x, kThreads);
    }
}

__global__ __launch_bounds__(kCompactThreads) void block_compact_rest_kernel(BlockCompactArgs a, Compact s)
{
    compact_rest(a, s, (int64_t)blockIdx.x * kCompactThreads + threadIdx.x, (int64_t)gridDim.x * kCompactThreads);
}

// Entries of the table up to which one workgroup does a whole call.
constexpr int kFewEntries = 4096;
constexpr int kFewReleases = 1 << 14;   // of a release

}  // namespace

size_t block_fork_scratch_ints(int batch, int num_forks) { return (size_t)batch + num_forks; }

int32_t block_fork_launch(const BlockForkArgs &a, hipStream_t stream)
{
    const bool few = (int64_t)a.num_forks * a.max_blocks <= kFewEntries;
    hipLaunchKernelGGL(block_fork_kernel, dim3(1), dim3(kThreads), 0, stream, a, few ? 1 : 0);
    SS_HIP_CHECK(hipGetLastError(), "launch block_fork_kernel");
    if (few) return SS_OK;
    constexpr int per = kForkThreads * kForkEach;
    const int parts = (a.max_blocks + per - 1) / per;
    hipLaunchKernelGGL(block_fork_rows_kernel, dim3((unsigned)a.num_forks, (unsigned)(parts < 64 ? parts : 64)), dim3(kForkThreads), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch block_fork_rows_kernel");
    return SS_OK;
}

size_t block_release_scratch_ints(int batch, int max_blocks, int num_blocks)
{
    const int64_t entries = (int64_t)batch * max_blocks;
    return kReleaseHead + (size_t)batch + 1 + (entries + kReleasePiece - 1) / kReleasePiece + num_blocks + (entries <= kReleaseKept ? entries : 0);
}

int32_t block_release_launch(const BlockReleaseArgs &a, hipStream_t stream)
{
    const int64_t entries = (int64_t)a.batch * a.max_blocks;
    if (entries <= kFewReleases) {
        hipLaunchKernelGGL(block_release_kernel, dim3(1), dim3(kThreads), 0, stream, a);
        SS_HIP_CHECK(hipGetLastError(), "launch block_release_kernel");
        return SS_OK;
    }
    const int64_t pieces = (entries + kReleasePiece - 1) / kReleasePiece, clear = ((int64_t)a.num_blocks + kThreads - 1) / kThreads;
    const int64_t each = (entries + kReleaseThreads - 1) / kReleaseThreads;
    const dim3 grid((unsigned)(pieces < 1024 ? pieces : 1024)), wg(kReleaseThreads);
    hipLaunchKernelGGL(block_release_sum_kernel, dim3(1 + (unsigned)(clear < 255 ? clear : 255)), dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL(block_release_phase_kernel<kTake>, dim3((unsigned)(each < 1024 ? each : 1024)), wg, 0, stream, a);
    hipLaunchKernelGGL(block_release_phase_kernel<kCount>, grid, wg, 0, stream, a);
    hipLaunchKernelGGL(block_release_phase_kernel<kPlace>, grid, wg, 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch block_release kernels");
    return SS_OK;
}

size_t block_compact_scratch_ints(int num_blocks) { return kCompactHead + 2 * (((size_t)num_blocks + 31) / 32) + 1; }

int32_t block_compact_launch(const BlockCompactArgs &a, hipStream_t stream)
{
    const int words = (a.num_blocks + 31) / 32;
    const Compact s = {a.scratch, reinterpret_cast<uint32_t *>(a.scratch) + kCompactHead, a.scratch + kCompactHead + words};
    const int64_t entries = (int64_t)a.batch * a.max_blocks, most = entries > a.num_blocks ? entries : a.num_blocks;
    const size_t lds = words <= kBitmapWords ? words * sizeof(uint32_t) : 0;
    if (most <= kFewEntries) {
        hipLaunchKernelGGL((block_compact_kernel<true, true>), dim3(1), dim3(kThreads), lds, stream, a, s);
        SS_HIP_CHECK(hipGetLastError(), "launch block_compact_kernel");
        return SS_OK;
    }
    if (lds) hipLaunchKernelGGL((block_compact_kernel<true, false>), dim3(1), dim3(kThreads), lds, stream, a, s);
    else hipLaunchKernelGGL((block_compact_kernel<false, false>), dim3(1), dim3(kThreads), 0, stream, a, s);
    const int64_t wgs = (most + kCompactThreads - 1) / kCompactThreads;
    hipLaunchKernelGGL(block_compact_rest_kernel, dim3((unsigned)(wgs < 2048 ? wgs : 2048)), dim3(kCompactThreads), 0, stream, a, s);
    SS_HIP_CHECK(hipGetLastError(), "launch block_compact kernels");
    return SS_OK;
}

}  // namespace ss
