// Block tables and slot maps from the lengths of a step's requests.
//
// need_b = ceil(kv_len_b / 16).  A request that holds fewer blocks takes need - held ids from the free list, one that holds more gives the
// rest back.  What is given back lies on top of the list, in the order (request, logical block), before anything is taken:
//     S = ids[0 .. count) ++ returned[0 .. F),     the k-th block that is taken (same order) is S[count + F - 1 - k],     ids' = S[0 .. count + F - A)
// so both orders are prefix sums over the requests, and every row, taken block and returned block is found by a search in them.  Of the list only
// what changes is written: if more is taken than given back (A >= F) nothing is, and else nothing of it is read.
//
// Bound by latency: a chain of lengths, sums, ids and slots, about 1 us each.  A step's rows take one workgroup and one launch; from kFewRows rows on
// the sums are one workgroup's and the rows many's, in a second launch.
#include "prefill.h"

namespace ss {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kLdsRequests = 1024;   // requests whose sums a workgroup keeps in LDS
constexpr int kFewRows = 4096;
constexpr int kHeadInts = 8;         // scratch: free ids before the step, taken, given back, status; then held, taken before, given back before

struct Head {
    int count, taken, given, status;
};
struct Sums {
    const int32_t *start, *len;                   // q_indptr, kv_len
    const int32_t *held, *taken, *given;          // per request: held before the step; blocks taken / given back by the requests in front of it
};

__device__ __forceinline__ int blocks_of(int len) { return (int)(((unsigned)len + kTile - 1) / kTile); }

// The last i in [0, n) with sum[i] <= x (sum is ascending, sum[0] <= x).
__device__ __forceinline__ int owner(const int32_t *sum, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Inclusive sums over the workgroup of two values at a time.
__device__ __forceinline__ void scan2(int &x, int &y, int2 *part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(x, d), v = __shfl_up(y, d);
        if (lane >= d) { x += u; y += v; }
    }
    if (lane == 63) part[wave] = make_int2(x, y);
    __syncthreads();
    int2 add = make_int2(0, 0);
    for (int w = 0; w < wave; ++w) { add.x += part[w].x; add.y += part[w].y; }
    x += add.x;
    y += add.y;
    __syncthreads();
}

struct SumLds {
    int2 part[kWaves];
    int bad;
    int total[2];
};

// One workgroup: the sums of all requests into held/taken/given (of batch, batch + 1, batch + 1 entries), and the new state of the requests and
// of the list's length, unless something does not fit.
__device__ Head sum_requests(const BlockMapArgs &a, SumLds &lds, int32_t *held, int32_t *taken, int32_t *given, int32_t *start, int32_t *len)
{
    const int tid = threadIdx.x;
    if (tid == 0) lds.bad = 0x7fffffff;
    const int count = a.free_count[0];
    __syncthreads();
    int before_t = 0, before_g = 0;
    for (int lo = 0; lo < a.batch; lo += kThreads) {
        const int b = lo + tid;
        int t = 0, g = 0, h = 0;
        if (b < a.batch) {
            const int q0 = a.q_indptr[b], q1 = a.q_indptr[b + 1], L = a.kv_len[b];
            h = a.held[b];
            const int need = blocks_of(L);
            const bool bad = q0 < 0 || q1 < q0 || q1 > a.total_rows || (b == 0 && q0 != 0) || L < q1 - q0 || need > a.max_blocks || h < 0 ||
                             h > a.max_blocks;
            if (bad) {
                atomicMin(&lds.bad, b);
            } else {
                t = max(need - h, 0);
                g = max(h - need, 0);
            }
            if (start) { start[b] = q0; len[b] = L; }
            if (start && b == a.batch - 1) start[a.batch] = q1;
        }
        int st = t, sg = g;
        scan2(st, sg, lds.part);
        if (b < a.batch) {
            held[b] = h;
            taken[b] = before_t + st - t;
            given[b] = before_g + sg - g;
        }
        if (tid == kThreads - 1) { lds.total[0] = before_t + st; lds.total[1] = before_g + sg; }
        __syncthreads();
        before_t = lds.total[0];
        before_g = lds.total[1];
    }
    __syncthreads();
    Head head = {count, before_t, before_g, 0};
    if (lds.bad != 0x7fffffff) head.status = -1 - lds.bad;
    else if (count < 0 || count > a.num_blocks || (int64_t)count + before_g - before_t > a.num_blocks) head.status = -1 - a.batch;
    else if ((int64_t)count + before_g < before_t) head.status = before_t - before_g - count;
    if (tid == 0) {
        taken[a.batch] = before_t;
        given[a.batch] = before_g;
        a.status[0] = head.status;
        if (head.status == 0) a.free_count[0] = count + before_g - before_t;
    }
    if (head.status == 0)
        for (int b = tid; b < a.batch; b += kThreads) a.held[b] = blocks_of(a.kv_len[b]);
    return head;
}

struct Ids {
    const BlockMapArgs &a;
    const Head &head;
    const Sums &s;
    // the r-th block that is given back
    __device__ int returned(int r) const
    {
        const int b = owner(s.given, a.batch, r);
        return a.block_table[(int64_t)b * a.max_blocks + blocks_of(s.len[b]) + r - s.given[b]];
    }
    // the k-th block that is taken
    __device__ int next(int k) const
    {
        const int i = head.given - 1 - k;
        return i >= 0 ? returned(i) : a.free_ids[head.count + i];
    }
};

// Everything but the sums, shared out over `threads` threads.
__device__ void fill(const BlockMapArgs &a, const Head &head, const Sums &s, int first, int threads)
{
    const Ids ids = {a, head, s};
    const bool ok = head.status == 0;
    const int rows = ok && a.batch > 0 ? s.start[a.batch] : 0;
    for (int r = first; r < a.total_rows; r += threads) {
        int slot = -1, pos = -1;
        if (r < rows) {
            const int b = owner(s.start, a.batch, r);
            pos = s.len[b] - (s.start[b + 1] - r);
            const int j = pos / kTile, over = j - s.held[b];
            const int id = over < 0 ? a.block_table[(int64_t)b * a.max_blocks + j] : ids.next(s.taken[b] + over);
            slot = id * kTile + pos % kTile;
        }
        a.slot_map[r] = slot;
        if (a.positions) a.positions[r] = pos;
    }
    if (!ok) return;
    for (int k = first; k < head.taken; k += threads) {
        const int b = owner(s.taken, a.batch, k);
        a.block_table[(int64_t)b * a.max_blocks + s.held[b] + k - s.taken[b]] = ids.next(k);
    }
    for (int r = first; r < head.given - head.taken; r += threads) a.free_ids[head.count + r] = ids.returned(r);
}

template <bool LDS>
__global__ __launch_bounds__(kThreads) void block_map_kernel(BlockMapArgs a)
{
    __shared__ SumLds sl;
    __shared__ int32_t buf[LDS ? 5 * (kLdsRequests + 1) : 1];
    constexpr int N = kLdsRequests + 1;
    if constexpr (LDS) {
        const Head head = sum_requests(a, sl, buf, buf + N, buf + 2 * N, buf + 3 * N, buf + 4 * N);
        __syncthreads();
        const Sums s = {buf + 3 * N, buf + 4 * N, buf, buf + N, buf + 2 * N};
        fill(a, head, s, threadIdx.x, kThreads);
    } else {
        int32_t *held = a.scratch + kHeadInts, *taken = held + a.batch, *given = taken + a.batch + 1;
        const Head head = sum_requests(a, sl, held, taken, given, nullptr, nullptr);
        __threadfence_block();
        __syncthreads();
        const Sums s = {a.q_indptr, a.kv_len, held, taken, given};
        fill(a, head, s, threadIdx.x, kThreads);
    }
}

__global__ __launch_bounds__(kThreads) void block_sum_kernel(BlockMapArgs a)
{
    __shared__ SumLds sl;
    int32_t *held = a.scratch + kHeadInts, *taken = held + a.batch, *given = taken + a.batch + 1;
    const Head head = sum_requests(a, sl, held, taken, given, nullptr, nullptr);
    if (threadIdx.x == 0) {
        a.scratch[0] = head.count;
        a.scratch[1] = head.taken;
        a.scratch[2] = head.given;
        a.scratch[3] = head.status;
    }
}

constexpr int kFillThreads = 256;

template <bool LDS>
__global__ __launch_bounds__(kFillThreads) void block_fill_kernel(BlockMapArgs a)
{
    __shared__ int32_t buf[LDS ? 5 * (kLdsRequests + 1) : 1];
    const int32_t *held = a.scratch + kHeadInts, *taken = held + a.batch, *given = taken + a.batch + 1;
    const Head head = {a.scratch[0], a.scratch[1], a.scratch[2], a.scratch[3]};
    const int first = blockIdx.x * kFillThreads + threadIdx.x, threads = gridDim.x * kFillThreads;
    if constexpr (LDS) {
        constexpr int N = kLdsRequests + 1;
        for (int b = threadIdx.x; b <= a.batch && a.batch > 0; b += kFillThreads) {   // (no requests: there may be no arrays)
            buf[N + b] = taken[b];
            buf[2 * N + b] = given[b];
            buf[3 * N + b] = a.q_indptr[b];
            if (b < a.batch) {
                buf[b] = held[b];
                buf[4 * N + b] = a.kv_len[b];
            }
        }
        __syncthreads();
        const Sums s = {buf + 3 * N, buf + 4 * N, buf, buf + N, buf + 2 * N};
        fill(a, head, s, first, threads);
    } else {
        const Sums s = {a.q_indptr, a.kv_len, held, taken, given};
        fill(a, head, s, first, threads);
    }
}

}  // namespace

size_t block_map_scratch_ints(int batch) { return kHeadInts + 3 * (size_t)batch + 2; }

int32_t block_map_launch(const BlockMapArgs &a, hipStream_t stream)
{
    const bool lds = a.batch <= kLdsRequests;
    if (a.total_rows <= kFewRows) {
        if (lds) hipLaunchKernelGGL(block_map_kernel<true>, dim3(1), dim3(kThreads), 0, stream, a);
        else hipLaunchKernelGGL(block_map_kernel<false>, dim3(1), dim3(kThreads), 0, stream, a);
        SS_HIP_CHECK(hipGetLastError(), "launch block_map_kernel");
        return SS_OK;
    }
    hipLaunchKernelGGL(block_sum_kernel, dim3(1), dim3(kThreads), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch block_sum_kernel");
    const int64_t wgs = ((int64_t)a.total_rows + kFillThreads - 1) / kFillThreads;
    const dim3 grid((unsigned)(wgs < 2048 ? wgs : 2048));
    if (lds) hipLaunchKernelGGL(block_fill_kernel<true>, grid, dim3(kFillThreads), 0, stream, a);
    else hipLaunchKernelGGL(block_fill_kernel<false>, grid, dim3(kFillThreads), 0, stream, a);
    SS_HIP_CHECK(hipGetLastError(), "launch block_fill_kernel");
    return SS_OK;
}

}  // namespace ss
