// Verification of draft trees by the target's own draws: at a node the token is y ~ softmax(logits / T) by inverse CDF from a given uniform, and the walk goes
// on while a child of the node carries y.
//
// A row's blocks of 2048 entries leave their largest logit m_c and s_c = sum exp((x - m_c) / T); with M the row's largest, block c has mass s_c exp((m_c - M) / T), and the
// token is found by a scan of the masses and a search inside one block.  All of it in fp64, in fixed orders: tokens are whole numbers, and have to be those of
// the formula.  An exponential's argument is formed from the difference of two logits, which is exact to 2^-53, so that blocks with different
// references agree to 1e-15.
//
// Two forms.  Few rows: one pass over all of them, a workgroup a row for the draws, and the walk through the drawn tokens, three launches.  Many rows: only those on the paths are
// read, a round after the other; in a round every workgroup of a request first finds, each for itself, what was drawn at the node before and the child that the walk goes on with, and
// then takes its blocks of that child's row.  Bound by latency: a round is a chain of state, masses, one block, the tree and the new row (9 us, 13 where 64 rows of 128 256 entries are
// summed; the exponentials of those are half of that).
#include "accept_common.h"
#include "tree_verify.h"
#include "tree_verify_rule.h"

namespace ss {
namespace {

struct Draw {           // of a row
    int32_t token;
    float logprob;
};
struct Walk {           // where a request's walk is
    int32_t cur, n;     // node, -1 at its end; accepted nodes
    float u;            // the node's uniform
};

struct VerifyWorkspace {
    double *sum;        // [rows][nsub], in rounds [2][batch][nsub]
    float *top;         // the same: the blocks' largest logits
    Draw *draw;         // [rows]
    Walk *walk;         // in rounds [2][batch]
    int nsub;
};

// Arguments of exponentials, (x - max) / T in steps of the table.
struct DiffArg {
    double inv_t, m;
    __device__ __forceinline__ DiffArg(double inv_t_, float m_) : inv_t(inv_t_ * kExpSteps), m((double)m_) {}
    __device__ __forceinline__ double operator()(float x) const { return ((double)x - m) * inv_t; }
};

// Whether every lane's eight logits have exponentials that are normal numbers is one test.
__device__ __forceinline__ void exp8(const ExpTable &ex, const DiffArg &arg, const float (&x)[8], double (&e)[8])
{
    float low = x[0];
#pragma unroll
    for (int s = 1; s < 8; ++s) low = min_or_nan(low, x[s]);
    if (!__any(!(arg(low) >= kExpNormal))) {
#pragma unroll
        for (int s = 0; s < 8; ++s) e[s] = ex.normal(arg(x[s]));
    } else {
#pragma unroll
        for (int s = 0; s < 8; ++s) e[s] = ex(arg(x[s]));
    }
}

// 1 / T, or 0 for the largest logit's token.  Of an infinite T something so small that the difference of any two floats, 2^129 at most, times it leaves every exponential at one, and
// above zero, so that minus infinity is masked as ever.
__device__ __forceinline__ double inverse_temperature(const TreeVerifyArgs &a, int b)
{
    const float t = a.temperature ? a.temperature[b] : a.temperature_scalar;
    return t > 0.f ? t < INFINITY ? 1.0 / (double)t : 0x1p-1000 : 0.0;
}

__device__ __forceinline__ bool rows_of(const TreeVerifyArgs &a, int b, int &r0, int &rows)
{
    const int r1 = a.q_indptr[b + 1];
    r0 = a.q_indptr[b];
    rows = r1 - r0;
    return r0 >= 0 && r1 > r0 && r1 <= a.total_rows;
}

// Sums and maxima over a wavefront, in every lane.
__device__ __forceinline__ float wave_max(float x)
{
    for (int off = 32; off; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    return x;
}
__device__ __forceinline__ int wave_min(int x)
{
    for (int off = 32; off; off >>= 1) x = min(x, __shfl_xor(x, off));
    return x;
}
__device__ __forceinline__ double lane_of(double x, int lane)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane), __builtin_amdgcn_readlane(__double2loint(x), lane));
}

// The sums of block c of a row: a wavefront's, by itself.
template <int DT>
__device__ __forceinline__ void block_sums(const TreeVerifyArgs &a, int64_t row, int c, double inv_t, const ExpTable &ex, float *top, double *sum)
{
    constexpr int EACH = kSub / (64 * 8);
    const int lane = threadIdx.x & 63;
    const void *p = row_ptr(a.target, row, a.row_stride, DT);
    Raw8<DT> raw[EACH];
    if (c * kSub + kSub <= a.vocab) {   // (plain loads, all under way together)
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint4 *from = reinterpret_cast<const uint4 *>(static_cast<const char *>(p) + (int64_t)(c * kSub + i * 512 + lane * 8) * (DT == SS_BF16 ? 2 : 4));
#pragma unroll
            for (int j = 0; j < (DT == SS_BF16 ? 1 : 2); ++j) raw[i].w[j] = from[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) load8<DT>(p, a.vocab, c * kSub + i * 512 + lane * 8, raw[i]);
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        float x[8];
        unpack8<DT>(raw[i], x);
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, x[k]);   // (a NaN is masked)
    }
    m = wave_max(m);
    double s = 0.0;
    if (inv_t > 0.0) {
        const DiffArg arg(inv_t, m);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            float x[8];
            double e[8];
            unpack8<DT>(raw[i], x);
            exp8(ex, arg, x, e);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += e[k];
        }
        s = wave_scan(s);
    }
    if (lane == 63) {
        top[c] = m;
        sum[c] = s;
    }
}

struct DrawLds {
    double entry[4];
    int last[4], first[4], tok, child[4];
    float x;
};
// A drawn token, and what its log-probability is made of.
struct Drawn {
    int token;
    float x, m;     // its logit, the row's largest
    double all;     // the sum of the exponentials, 0 if the token was not drawn from a distribution
    __device__ Draw result(double inv_t) const { return {token, all > 0.0 ? (float)(((double)x - (double)m) * inv_t - log(all)) : 0.f}; }
};

// A row's blocks as the draw takes them: a lane's first one is asked for before the row is known to be needed.
struct Blocks {
    const float *top;
    const double *sum;
    int nsub, c0, c1;   // this lane's run of blocks
    float top0;
    double sum0;
    __device__ __forceinline__ Blocks(const VerifyWorkspace &w, int64_t at) : top(w.top + at), sum(w.sum + at), nsub(w.nsub)
    {
        const int lane = threadIdx.x & 63, per = (nsub + 63) / 64;
        c0 = lane * per;
        c1 = min(c0 + per, nsub);
        top0 = top[min(c0, nsub - 1)];
        sum0 = sum[min(c0, nsub - 1)];
    }
    __device__ __forceinline__ float largest(int c) const { return c == c0 ? top0 : top[c]; }
    __device__ __forceinline__ double mass(int c) const { return c == c0 ? sum0 : sum[c]; }
};

// The token of a row, in every lane of a workgroup.  Every wavefront scans the blocks for itself, a lane a run of them; the entries of the block are the workgroup's.
template <int DT>
__device__ __forceinline__ Drawn draw_of(const TreeVerifyArgs &a, const Blocks &blocks, int row, float u, double inv_t, const ExpTable &ex, DrawLds &sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c0 = blocks.c0, c1 = blocks.c1;
    const void *p = row_ptr(a.target, row, a.row_stride, DT);
    float own_top = -INFINITY;
    for (int c = c0; c < c1; ++c) own_top = fmaxf(own_top, blocks.largest(c));
    const float m = wave_max(own_top);
    auto entries = [&](int c, float (&x)[8]) {
        Raw8<DT> raw;
        load8<DT>(p, a.vocab, c * kSub + tid * 8, raw);
        unpack8<DT>(raw, x);
    };
    Drawn d = {0, 0.f, m, 0.0};
    if (inv_t > 0.0 && m < INFINITY && m > -INFINITY) {
        const DiffArg arg(inv_t, m);
        auto mass_of = [&](int c) {
            const float top = blocks.largest(c);
            return top == -INFINITY ? 0.0 : blocks.mass(c) * ex(arg(top));
        };
        double own = 0.0;
        int own_last = -1;   // last block of this lane with mass
        for (int c = c0; c < c1; ++c) {
            const double v = mass_of(c);
            own += v;
            if (v > 0.0) own_last = c;
        }
        const double cum = wave_scan(own), all = lane_of(cum, 63), thr = (double)u * all;
        const uint64_t over = __ballot(own > 0.0 && cum > thr), some = __ballot(own > 0.0);   // (there is mass: the block of the largest logit has)
        const bool take_last = over == 0;   // rounding left u times the sum at or past it: the last entry with mass
        const int owner = take_last ? 63 - __builtin_clzll(some) : __builtin_ctzll(over);
        double pre = cum - own;
        int cs = own_last;
        if (c1 - c0 > 1 && lane == owner) {   // inside the lane's run: the first with mass whose running sum crosses (rounding may leave none: then the last with mass)
            double run = pre;
            bool found = false;
            for (int c = c0; c < c1; ++c) {
                const double v = mass_of(c);
                if (v > 0.0 && !found) {
                    cs = c;
                    pre = run;
                    found = !take_last && run + v > thr;
                }
                run += v;
            }
        }
        const int block = __builtin_amdgcn_readlane(cs, owner);
        const double prefix = lane_of(pre, owner);
        float x[8];
        double r[8];
        entries(block, x);
        const float top = blocks.top[block];
        exp8(ex, DiffArg(inv_t, top), x, r);
        const double level = ex(arg(top));
        double local = 0.0;
        int my_last = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            r[i] *= level;
            local += r[i];
            if (r[i] > 0.0) my_last = i;
        }
        const double incl = wave_scan(local);
        const uint64_t mass = __ballot(my_last >= 0);
        if (lane == 63) sh.entry[wave] = incl;
        if (lane == 0) sh.last[wave] = mass ? wave * 64 + 63 - __builtin_clzll(mass) : -1;
        __syncthreads();
        double before = prefix;
        for (int w = 0; w < wave; ++w) before += sh.entry[w];
        const double excl = before + (incl - local);
        // (the scan groups its additions differently for every lane, so the sum at a lane without mass may lie an ulp above that of the lane in front of it)
        const uint64_t bal = __ballot(!take_last && local > 0.0 && excl + local > thr);
        if (lane == 0) sh.first[wave] = bal ? wave * 64 + __builtin_ctzll(bal) : 0x7fffffff;
        __syncthreads();
        const int first = min(min(sh.first[0], sh.first[1]), min(sh.first[2], sh.first[3]));
        const int at = first != 0x7fffffff ? first : max(max(sh.last[0], sh.last[1]), max(sh.last[2], sh.last[3]));
        if (tid == at) {
            double c = excl;
            int y = -1;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r[i] > 0.0) {
                    c += r[i];
                    if (first != 0x7fffffff && y < 0 && c > thr) y = i;
                }
            y = y >= 0 ? y : my_last;   // (the lane's total crossed but the sum entry by entry may round differently: its last entry with mass)
            sh.tok = block * kSub + tid * 8 + y;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i == y) sh.x = x[i];
        }
        __syncthreads();
        d.token = sh.tok;
        d.x = sh.x;
        d.all = all;
        return d;
    }
    if (m > -INFINITY) {   // the lowest token whose logit is the largest
        int c = 0x7fffffff;
        for (int i = c0; i < c1; ++i)
            if (blocks.largest(i) == m) { c = i; break; }
        c = wave_min(c);
        float x[8];
        entries(c, x);
        int y = 0x7fffffff;
#pragma unroll
        for (int i = 7; i >= 0; --i)
            if (x[i] == m) y = c * kSub + tid * 8 + i;
        y = wave_min(y);
        if (lane == 0) sh.first[wave] = y;
        __syncthreads();
        d.token = min(min(sh.first[0], sh.first[1]), min(sh.first[2], sh.first[3]));
    }
    return d;
}

// The lowest child of node cur that carries token y, INT_MAX if there is none; in every lane of a workgroup.  A lane's first node behind cur has been asked for before the draw.
struct Candidate {
    int parent, token;
};
__device__ __forceinline__ Candidate candidate(const TreeVerifyArgs &a, int r0, int rows, int cur)
{
    const int i = cur + 1 + threadIdx.x;
    return i < rows ? Candidate{a.parent[r0 + i], a.tokens[r0 + i]} : Candidate{-1, -1};
}
__device__ __forceinline__ int child_with(const TreeVerifyArgs &a, const Candidate &mine, int r0, int rows, int cur, int y, DrawLds &sh)
{
    int c = 0x7fffffff, i = cur + 1 + threadIdx.x;
    if (mine.parent == cur && mine.token == y) c = i;
    else
        for (i += kThreads; i < rows; i += kThreads)
            if (a.parent[r0 + i] == cur && a.tokens[r0 + i] == y) { c = i; break; }
    c = wave_min(c);
    __syncthreads();   // (a step in front may still read)
    if ((threadIdx.x & 63) == 0) sh.child[threadIdx.x >> 6] = c;
    __syncthreads();
    return min(min(sh.child[0], sh.child[1]), min(sh.child[2], sh.child[3]));
}

// What a request has before anything is drawn; whether it has rows.
__device__ __forceinline__ void clear_outputs(const TreeVerifyArgs &a, int b)
{
    const int tid = threadIdx.x;
    if (tid == 0) a.accepted_len[b] = 0;
    if (tid < SS_OUT_WIDTH) {
        a.out_tokens[(int64_t)b * SS_OUT_WIDTH + tid] = -1;
        if (a.logprobs) a.logprobs[(int64_t)b * SS_OUT_WIDTH + tid] = 0.f;
        if (tid < SS_MAX_DEPTH) a.accepted_nodes[(int64_t)b * SS_MAX_DEPTH + tid] = -1;
    }
}
__device__ __forceinline__ void emit(const TreeVerifyArgs &a, int b, int n, const Draw &d)
{
    a.out_tokens[(int64_t)b * SS_OUT_WIDTH + n] = d.token;
    if (a.logprobs) a.logprobs[(int64_t)b * SS_OUT_WIDTH + n] = d.logprob;
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// The request that a row belongs to, -1 if none does; in every lane of a workgroup.
__device__ __forceinline__ int request_of(const TreeVerifyArgs &a, int row, int *sh)
{
    int at = 0x7fffffff;
    for (int b = threadIdx.x; b < a.batch; b += kThreads) {
        int r0, rows;
        if (rows_of(a, b, r0, rows) && row >= r0 && row < r0 + rows) at = min(at, b);
    }
    for (int off = 32; off; off >>= 1) at = min(at, __shfl_xor(at, off));
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = at;
    __syncthreads();
    at = min(min(sh[0], sh[1]), min(sh[2], sh[3]));
    __syncthreads();
    return at == 0x7fffffff ? -1 : at;
}

// grid: rows * fours of blocks
template <int DT>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    __shared__ ExpTable ex;
    __shared__ int sh_b[4];
    const int fours = (w.nsub + 3) / 4, row = blockIdx.x / fours, c = blockIdx.x % fours * 4 + (threadIdx.x >> 6), b = request_of(a, row, sh_b);
    if (b < 0) return;
    ex.init();
    if (c < w.nsub) block_sums<DT>(a, row, c, inverse_temperature(a, b), ex, w.top + (int64_t)row * w.nsub, w.sum + (int64_t)row * w.nsub);
}

// grid: rows
template <int DT>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    __shared__ ExpTable ex;
    __shared__ DrawLds sh;
    __shared__ int sh_b[4];
    const int row = blockIdx.x;
    const Blocks blocks(w, (int64_t)row * w.nsub);
    const int b = request_of(a, row, sh_b);
    if (b < 0) return;
    ex.init();
    const double inv_t = inverse_temperature(a, b);
    const Drawn d = draw_of<DT>(a, blocks, row, inv_t > 0.0 ? a.uniforms[row] : 0.f, inv_t, ex, sh);
    if (threadIdx.x == 0) w.draw[row] = d.result(inv_t);
}

// grid: batch
__global__ __launch_bounds__(kThreads) void verify_walk_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    __shared__ DrawLds sh;
    const int b = blockIdx.x, tid = threadIdx.x;
    int r0, rows, n = 0, cur = 0;
    clear_outputs(a, b);
    if (!rows_of(a, b, r0, rows)) return;
    __syncthreads();   // (outputs are one lane's from here on)
    for (;;) {
        const Draw d = w.draw[r0 + cur];
        if (tid == 0) emit(a, b, n, d);
        if (n == a.max_depth) break;
        const int c = child_with(a, candidate(a, r0, rows, cur), r0, rows, cur, d.token, sh);
        if (c == 0x7fffffff) break;
        if (tid == 0) a.accepted_nodes[(int64_t)b * SS_MAX_DEPTH + n] = c;
        ++n;
        cur = c;
    }
    if (tid == 0) a.accepted_len[b] = n;
}

// ---- many rows ---------------------------------------------------------------------------------------------------------
// Round r: the draw at the node that round r - 1 has summed, the child, the sums of its row.  grid: batch * groups of 4 `each` blocks
template <int DT>
__global__ __launch_bounds__(kThreads) void verify_round_kernel(TreeVerifyArgs a, VerifyWorkspace w, int r, int each)
{
    __shared__ ExpTable ex;
    __shared__ DrawLds sh;
    const int groups = (w.nsub + 4 * each - 1) / (4 * each), b = blockIdx.x / groups, group = blockIdx.x % groups;
    const bool first = group == 0 && threadIdx.x == 0;   // whose the outputs are
    Walk *walk = w.walk + (int64_t)(r & 1) * a.batch + b;
    const Blocks blocks(w, ((int64_t)((r - 1) & 1) * a.batch + b) * w.nsub);   // (in round 0 of nothing)
    int r0, rows;
    const bool has = rows_of(a, b, r0, rows);
    const double inv_t = inverse_temperature(a, b);
    auto uniform_of = [&](int node) { return inv_t > 0.0 ? a.uniforms[r0 + node] : 0.f; };
    Walk at = {has ? 0 : -1, 0, has && r == 0 ? uniform_of(0) : 0.f};
    if (r == 0) {
        if (group == 0) clear_outputs(a, b);
    } else {
        at = w.walk[(int64_t)((r - 1) & 1) * a.batch + b];
    }
    ex.init();
    if (at.cur < 0) {
        if (first) *walk = at;
        return;
    }
    Drawn d = {};
    int n = -1;   // whose draw that is
    if (r > 0) {
        const Candidate mine = candidate(a, r0, rows, at.cur);
        n = at.n;
        d = draw_of<DT>(a, blocks, r0 + at.cur, at.u, inv_t, ex, sh);
        const int c = n < a.max_depth ? child_with(a, mine, r0, rows, at.cur, d.token, sh) : 0x7fffffff;
        if (c == 0x7fffffff) {
            if (first) {
                emit(a, b, n, d.result(inv_t));
                a.accepted_len[b] = n;
                *walk = {-1, n, 0.f};
            }
            return;
        }
        if (first) a.accepted_nodes[(int64_t)b * SS_MAX_DEPTH + n] = c;
        at = {c, n + 1, first ? uniform_of(c) : 0.f};
    }
    if (first) *walk = at;
    const int64_t back = ((int64_t)(r & 1) * a.batch + b) * w.nsub;
    for (int i = 0; i < each; ++i) {
        const int c = (group * each + i) * 4 + (threadIdx.x >> 6);
        if (c < w.nsub) block_sums<DT>(a, r0 + at.cur, c, inv_t, ex, w.top + back, w.sum + back);
    }
    if (first && n >= 0) emit(a, b, n, d.result(inv_t));
}

// Room for the sums and draws of so many rows.
__host__ VerifyWorkspace carve_verify(void *ws, int batch, int64_t rows, int vocab, size_t *bytes)
{
    VerifyWorkspace w;
    w.nsub = num_sub(vocab);
    const size_t n = (size_t)rows * w.nsub;
    char *p = static_cast<char *>(ws);
    w.sum = reinterpret_cast<double *>(p); p += align_up(sizeof(double) * n, 256);
    w.top = reinterpret_cast<float *>(p); p += align_up(sizeof(float) * n, 256);
    w.draw = reinterpret_cast<Draw *>(p); p += align_up(sizeof(Draw) * (size_t)rows, 256);
    w.walk = reinterpret_cast<Walk *>(p); p += align_up(2 * sizeof(Walk) * (size_t)batch, 256);
    *bytes = (size_t)(p - static_cast<char *>(ws)) + 256;
    return w;
}
size_t verify_bytes(int batch, int64_t rows, int vocab)
{
    size_t bytes;
    carve_verify(nullptr, batch, rows, vocab, &bytes);
    return bytes;
}
// Rounds have two rows a request, which is the least room that either form is given.
int64_t round_rows(int batch) { return 2 * (int64_t)batch; }

// Workgroups of a round, about: a few more than the 1024 that the chip runs at a time, of which those of ended requests are gone at once.  With 1024 | 1280 | 2560, us: 160 requests with
// 128 256 entries 135 | 122 | 128, 80 of them 96 | 90 | 90, 300 with 32 000 102 | 96 | 96; 64 and 100 requests are level.
constexpr int kRoundWgs = 1280;

template <int DT>
int32_t launch(const TreeVerifyArgs &a, hipStream_t stream)
{
    const int64_t rows = a.total_rows > round_rows(a.batch) ? a.total_rows : round_rows(a.batch);
    const bool at_once = verify_all_rows(a.batch, a.total_rows, a.vocab, a.max_depth) && verify_bytes(a.batch, rows, a.vocab) <= a.workspace_bytes;
    size_t unused;
    const VerifyWorkspace w = carve_verify(a.workspace, a.batch, at_once ? rows : round_rows(a.batch), a.vocab, &unused);
    const dim3 wg(kThreads);
    if (at_once) {
        if (a.total_rows > 0) {
            hipLaunchKernelGGL(verify_sums_kernel<DT>, dim3((unsigned)a.total_rows * (unsigned)((w.nsub + 3) / 4)), wg, 0, stream, a, w);
            hipLaunchKernelGGL(verify_draw_kernel<DT>, dim3((unsigned)a.total_rows), wg, 0, stream, a, w);
        }
        hipLaunchKernelGGL(verify_walk_kernel, dim3((unsigned)a.batch), wg, 0, stream, a, w);
        SS_HIP_CHECK(hipGetLastError(), "launch tree_verify kernels");
        return SS_OK;
    }
    const int fours = (w.nsub + 3) / 4;
    const int64_t all = (int64_t)a.batch * fours;
    int each = (int)((all + kRoundWgs - 1) / kRoundWgs);
    each = each < fours ? each : fours;
    const unsigned groups = (unsigned)((fours + each - 1) / each);
    for (int r = 0; r <= a.max_depth; ++r) hipLaunchKernelGGL(verify_round_kernel<DT>, dim3(groups * (unsigned)a.batch), wg, 0, stream, a, w, r, each);
    hipLaunchKernelGGL(verify_round_kernel<DT>, dim3((unsigned)a.batch), wg, 0, stream, a, w, a.max_depth + 1, fours);   // (the draws at the deepest nodes)
    SS_HIP_CHECK(hipGetLastError(), "launch verify_round_kernel");
    return SS_OK;
}

}  // namespace

size_t tree_verify_least_bytes(int batch, int vocab) { return verify_bytes(batch, round_rows(batch), vocab); }

// What any max_depth takes, of this call and of those with fewer rows or requests: a program has one workspace for its largest step.  (Calls of more rows than a launch takes are no
// bound that a program would have: they get what they need.)
size_t tree_verify_workspace_bytes(int batch, int total_rows, int vocab)
{
    int64_t rows = 0;
    if (total_rows * verify_fours(vocab) < kVerifyGroups) {
        const int64_t most = verify_most_rows(batch, vocab, SS_MAX_DEPTH);
        rows = total_rows < most ? total_rows : most;
    }
    return verify_bytes(batch, rows > round_rows(batch) ? rows : round_rows(batch), vocab);
}

int32_t tree_verify_launch(const TreeVerifyArgs &a, hipStream_t stream)
{
    return a.logit_dtype == SS_BF16 ? launch<SS_BF16>(a, stream) : launch<SS_F32>(a, stream);
}

}  // namespace ss
