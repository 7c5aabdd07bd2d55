// Verification of draft trees by the target's own draws: at a node the token is y ~ softmax(logits / T) by inverse CDF from a given uniform, and the walk goes
// on while a child of the node carries y.
//
// A row's blocks of 2048 entries leave their largest logit m_c and s_c = sum exp((x - m_c) / T); with M the row's largest, block c has mass s_c exp((m_c - M) / T), and the
// token is found by a scan of the masses and a search inside one block.  All of it in fp64, in fixed orders: tokens are whole numbers, and have to be those of
// the formula.  An exponential's argument is formed from the difference of two logits, which is exact to 2^-53, so that blocks with different
// references agree to 1e-15.
//
// One pass over all rows, one workgroup a row for the draw, and the walk through the drawn tokens.
#include "accept_common.h"
#include "tree_verify.h"

namespace ss {
namespace {

struct Draw {           // of a row
    int32_t token;
    float logprob;
};

struct VerifyWorkspace {
    float *top;         // [rows][nsub] the blocks' largest logits
    double *sum;        // [rows][nsub]
    Draw *draw;         // [rows]
    int32_t *request;   // [rows] whose row it is, -1: no one's
    int nsub;
};

__host__ VerifyWorkspace carve_verify(void *ws, int total_rows, int vocab)
{
    VerifyWorkspace w;
    w.nsub = num_sub(vocab);
    char *p = static_cast<char *>(ws);
    const size_t n = (size_t)total_rows * w.nsub;
    w.sum = reinterpret_cast<double *>(p); p += align_up(sizeof(double) * n, 256);
    w.top = reinterpret_cast<float *>(p); p += align_up(sizeof(float) * n, 256);
    w.draw = reinterpret_cast<Draw *>(p); p += align_up(sizeof(Draw) * (size_t)total_rows, 256);
    w.request = reinterpret_cast<int32_t *>(p);
    return w;
}

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

// 1 / T, or 0 for the largest logit's token
__device__ __forceinline__ double inverse_temperature(const TreeVerifyArgs &a, int b)
{
    const float t = a.temperature ? a.temperature[b] : a.temperature_scalar;
    return t > 0.f ? 1.0 / (double)t : 0.0;
}

__device__ __forceinline__ bool rows_of(const TreeVerifyArgs &a, int b, int &r0, int &rows)
{
    const int r1 = a.q_indptr[b + 1];
    r0 = a.q_indptr[b];
    rows = r1 - r0;
    return r0 >= 0 && r1 > r0 && r1 <= a.total_rows;
}

__global__ __launch_bounds__(kThreads) void verify_rows_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    const int row = blockIdx.x * kThreads + threadIdx.x;
    if (row < a.total_rows) w.request[row] = -1;
}
__global__ __launch_bounds__(kThreads) void verify_requests_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    int r0, rows;
    if (!rows_of(a, blockIdx.x, r0, rows)) return;
    for (int i = threadIdx.x; i < rows; i += kThreads) w.request[r0 + i] = blockIdx.x;
}

// grid: rows * blocks
template <int DT>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    __shared__ ExpTable ex;
    __shared__ float sh_m[4];
    __shared__ double sh_s[4];
    const int row = blockIdx.x / w.nsub, c = blockIdx.x % w.nsub, b = w.request[row];
    if (b < 0) return;
    const double inv_t = inverse_temperature(a, b);
    ex.init();
    Raw8<DT> raw;
    float x[8];
    load8<DT>(row_ptr(a.target, row, a.row_stride, DT), a.vocab, c * kSub + threadIdx.x * 8, raw);
    unpack8<DT>(raw, x);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, x[i]);   // (a NaN is masked)
    m = block_max(m, sh_m);
    double s = 0.0;
    if (inv_t > 0.0) {
        double e[8];
        exp8(ex, DiffArg(inv_t, m), x, e);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += e[i];
        s = block_sum(s, sh_s);
    }
    if (threadIdx.x == 0) {
        w.top[(int64_t)row * w.nsub + c] = m;
        w.sum[(int64_t)row * w.nsub + c] = s;
    }
}

// The token of a row, in every lane of a workgroup.
template <int DT>
__device__ Draw draw_of(const TreeVerifyArgs &a, const VerifyWorkspace &w, int row, double inv_t, const ExpTable &ex, DrawShared &sh, float *sh_m, double *sh_s)
{
    const float *top = w.top + (int64_t)row * w.nsub;
    const double *sum = w.sum + (int64_t)row * w.nsub;
    float m = -INFINITY;
    for (int c = threadIdx.x; c < w.nsub; c += kThreads) m = fmaxf(m, top[c]);
    m = block_max(m, sh_m);
    Draw d = {-1, 0.f};
    if (inv_t > 0.0 && m < INFINITY && m > -INFINITY) {
        const DiffArg arg(inv_t, m);
        auto mass_of = [&](int c) { return top[c] == -INFINITY ? 0.0 : sum[c] * ex(arg(top[c])); };
        double part = 0.0;
        for (int c = threadIdx.x; c < w.nsub; c += kThreads) part += mass_of(c);
        const double all = block_sum(part, sh_s);
        __syncthreads();
        const void *p = row_ptr(a.target, row, a.row_stride, DT);
        d.token = draw_token(w.nsub, a.uniforms[row], sh, mass_of, [&](int c, double (&r)[kSubPer]) {
            Raw8<DT> raw;
            float x[8];
            load8<DT>(p, a.vocab, c * kSub + threadIdx.x * 8, raw);
            unpack8<DT>(raw, x);
            exp8(ex, DiffArg(inv_t, top[c]), x, r);
            const double level = ex(arg(top[c]));
#pragma unroll
            for (int i = 0; i < kSubPer; ++i) r[i] *= level;
        });
        if (d.token >= 0) d.logprob = (float)(((double)load_logit(a.target, row, a.row_stride, DT, d.token) - (double)m) * inv_t - log(all));
    }
    if (d.token < 0) d.token = m > -INFINITY ? lowest_index_of(a.target, row, a.row_stride, DT, a.vocab, m, sh) : 0;
    return d;
}

// grid: rows
template <int DT>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    __shared__ ExpTable ex;
    __shared__ DrawShared sh;
    __shared__ float sh_m[4];
    __shared__ double sh_s[4];
    const int row = blockIdx.x, b = w.request[row];
    if (b < 0) return;
    ex.init();
    const Draw d = draw_of<DT>(a, w, row, inverse_temperature(a, b), ex, sh, sh_m, sh_s);
    if (threadIdx.x == 0) w.draw[row] = d;
}

// The lowest child of node cur that carries token y, INT_MAX if there is none; in every lane of a workgroup.
__device__ __forceinline__ int child_with(const TreeVerifyArgs &a, int r0, int rows, int cur, int y, int *sh)
{
    int c = 0x7fffffff;
    for (int i = cur + 1 + threadIdx.x; i < rows; i += kThreads)
        if (a.parent[r0 + i] == cur && a.tokens[r0 + i] == y) { c = i; break; }
    for (int off = 32; off; off >>= 1) c = min(c, __shfl_xor(c, off));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = c;
    __syncthreads();
    return min(min(sh[0], sh[1]), min(sh[2], sh[3]));
}

// grid: batch
__global__ __launch_bounds__(kThreads) void verify_walk_kernel(TreeVerifyArgs a, VerifyWorkspace w)
{
    __shared__ int sh[4];
    const int b = blockIdx.x, tid = threadIdx.x;
    int r0, rows, n = 0, cur = 0, emitted = 0;
    int32_t *out = a.out_tokens + (int64_t)b * SS_OUT_WIDTH, *nodes = a.accepted_nodes + (int64_t)b * SS_MAX_DEPTH;
    float *lp = a.logprobs ? a.logprobs + (int64_t)b * SS_OUT_WIDTH : nullptr;
    if (rows_of(a, b, r0, rows)) {
        for (;;) {
            const Draw d = w.draw[r0 + cur];
            if (tid == 0) {
                out[emitted] = d.token;
                if (lp) lp[emitted] = d.logprob;
            }
            ++emitted;
            if (n == a.max_depth) break;
            const int c = child_with(a, r0, rows, cur, d.token, sh);
            if (c == 0x7fffffff) break;
            if (tid == 0) nodes[n] = c;
            ++n;
            cur = c;
        }
    }
    if (tid == 0) a.accepted_len[b] = n;
    if (tid < SS_OUT_WIDTH) {
        if (tid >= emitted) {
            out[tid] = -1;
            if (lp) lp[tid] = 0.f;
        }
        if (tid < SS_MAX_DEPTH && tid >= n) nodes[tid] = -1;
    }
}

}  // namespace

int64_t tree_verify_workgroups(int batch, int total_rows, int vocab)
{
    const int64_t n = (int64_t)total_rows * num_sub(vocab);
    return n > batch ? n : batch;
}

size_t tree_verify_workspace_bytes(int batch, int total_rows, int vocab)
{
    const size_t n = (size_t)total_rows * num_sub(vocab);
    return align_up(sizeof(double) * n, 256) + align_up(sizeof(float) * n, 256) + align_up(sizeof(Draw) * (size_t)total_rows, 256) +
           align_up(sizeof(int32_t) * (size_t)total_rows, 256) + 256;
}

int32_t tree_verify_launch(const TreeVerifyArgs &a, hipStream_t stream)
{
    const VerifyWorkspace w = carve_verify(a.workspace, a.total_rows, a.vocab);
    const dim3 wg(kThreads);
    if (a.total_rows > 0) {
        hipLaunchKernelGGL(verify_rows_kernel, dim3((unsigned)(a.total_rows + kThreads - 1) / kThreads), wg, 0, stream, a, w);
        hipLaunchKernelGGL(verify_requests_kernel, dim3((unsigned)a.batch), wg, 0, stream, a, w);
        const dim3 sums((unsigned)a.total_rows * (unsigned)w.nsub), rows((unsigned)a.total_rows);
        if (a.logit_dtype == SS_BF16) {
            hipLaunchKernelGGL(verify_sums_kernel<SS_BF16>, sums, wg, 0, stream, a, w);
            hipLaunchKernelGGL(verify_draw_kernel<SS_BF16>, rows, wg, 0, stream, a, w);
        } else {
            hipLaunchKernelGGL(verify_sums_kernel<SS_F32>, sums, wg, 0, stream, a, w);
            hipLaunchKernelGGL(verify_draw_kernel<SS_F32>, rows, wg, 0, stream, a, w);
        }
    }
    hipLaunchKernelGGL(verify_walk_kernel, dim3((unsigned)a.batch), wg, 0, stream, a, w);
    SS_HIP_CHECK(hipGetLastError(), "launch tree_verify kernels");
    return SS_OK;
}

}  // namespace ss
