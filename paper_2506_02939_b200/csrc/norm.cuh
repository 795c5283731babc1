// Layer norm and its root-mean-square form, forward and backward, optionally with the residual
// addition on both ways.
//
//   h = x (+ r);  mu = mean(h) (0 in the RMS form);  v = mean((h - mu)^2);  s = 1 / sqrt(v + eps)
//   y = (h - mu) s w (+ c)
//   u = (h - mu) s;  g = dy w;  dx = s (g - mean(g) - u mean(g u)) (+ dh), without mean(g) in the RMS form
//   dw = sum over rows of dy u;  dc = sum over rows of dy
//
// All of it is bound by memory: about 10 operations an element against 4 to 8 bytes.  The forward pass
// holds its row in registers, so that x is read once and the variance is taken around the true mean.
// mu and s are those of h before it is rounded to its storage type: y then carries one rounding.
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"

namespace pamm {

constexpr int64_t NORM_MAX_N = 32768;

// Sum over the block (warps = blockDim.x / 32); `part` has 32 floats and is not used again by the
// caller before another barrier.  Fixed order: the same sum in every thread, every time.
__device__ __forceinline__ float block_sum(float x, float* part, int warps) {
    x = warp_sum(x);
    if (warps == 1) return x;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    return warp_sum((threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0.f);
}

struct NormForwardArgs {
    const void *x, *r, *w, *c;
    void *y, *h;
    float *mean, *rstd;
    int64_t ldx, ldr, ldy, ldh, b;
    int n, warps;           // warps of the block that share a row; 1: every warp of the block has a row
    float eps;
    bool rms, w_bf16, w_vec;
};

// EPT elements of a row per thread, in EPT / V pieces of V that lie 32 * warps * V apart.
template <typename T, int V, int EPT>
__global__ void __launch_bounds__(1024)
norm_forward_kernel(const NormForwardArgs a) {
    __shared__ float s_sum[32], s_sq[32];
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr int P = EPT / V;
    const int lane_threads = 32 * a.warps;
    const int t = a.warps == 1 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t row = a.warps == 1 ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= a.b) return;          // whole warps, and whole blocks where a row has more than one warp
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
    float h[P][V];
#pragma unroll
    for (int p = 0; p < P; ++p) RowIo<T, V>::load(x, (t + p * lane_threads) * V, a.n, h[p]);
    if (r) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float q[V];
            RowIo<T, V>::load(r, (t + p * lane_threads) * V, a.n, q);
#pragma unroll
            for (int e = 0; e < V; ++e) h[p][e] += q[e];
        }
    }
    const float inv_n = 1.f / (float)a.n;
    float mean = 0.f;
    if (!a.rms) {
        float sum = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) sum += h[p][e];
        mean = block_sum(sum, s_sum, a.warps) * inv_n;
    }
    float sq = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = (t + p * lane_threads) * V + e < a.n ? h[p][e] - mean : 0.f;
            sq = fmaf(d, d, sq);
        }
    const float rstd = 1.f / sqrtf(block_sum(sq, s_sq, a.warps) * inv_n + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    T* ho = a.h ? static_cast<T*>(a.h) + row * a.ldh : nullptr;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int col = (t + p * lane_threads) * V;
        if (col >= a.n) continue;
        if (ho) RowIo<T, V>::store(ho, col, a.n, h[p]);
        float w[V], c[V];
        load_weights<V>(a.w, a.w_bf16, a.w_vec, col, a.n, 1.f, w);
        load_weights<V>(a.c, a.w_bf16, a.w_vec, col, a.n, 0.f, c);
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = fmaf((h[p][e] - mean) * rstd, w[e], c[e]);
        RowIo<T, V>::store(y, col, a.n, w);
    }
}

struct NormBackwardArgs {
    const void *dy, *x, *w, *dh;
    const float *mean, *rstd;
    void *dx, *dw, *dc;
    float *part;            // [splits][2][n]: partial sums of dw and dc
    int64_t lddy, ldx, lddh, lddx, b, rows_per_split;
    int n, splits;
    bool rms, w_bf16, w_vec, dw_bf16;
};

constexpr int NB_WIDE_THREADS = 256;

// One row per block, read twice (the second time from the caches): the two sums, then dx.
template <typename T, int V>
__global__ void __launch_bounds__(NB_WIDE_THREADS)
norm_backward_row_kernel(const NormBackwardArgs a) {
    __shared__ float s_gu[32], s_g[32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float mean = a.rms ? 0.f : a.mean[row], rstd = a.rstd[row];
    float gu = 0.f, g = 0.f;
    for (int col = threadIdx.x * V; col < a.n; col += NB_WIDE_THREADS * V) {
        float xv[V], dv[V], w[V];
        RowIo<T, V>::load(x, col, a.n, xv);
        RowIo<T, V>::load(dy, col, a.n, dv);
        load_weights<V>(a.w, a.w_bf16, a.w_vec, col, a.n, 1.f, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float q = dv[e] * w[e];
            g += q;
            gu = fmaf(q, (xv[e] - mean) * rstd, gu);
        }
    }
    const float inv_n = 1.f / (float)a.n;
    gu = block_sum(gu, s_gu, NB_WIDE_THREADS / 32) * inv_n;
    g = a.rms ? 0.f : block_sum(g, s_g, NB_WIDE_THREADS / 32) * inv_n;
    T* dx = static_cast<T*>(a.dx) + row * a.lddx;
    const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.lddh : nullptr;
    for (int col = threadIdx.x * V; col < a.n; col += NB_WIDE_THREADS * V) {
        float xv[V], dv[V], w[V], hv[V] = {};
        RowIo<T, V>::load(x, col, a.n, xv);
        RowIo<T, V>::load(dy, col, a.n, dv);
        load_weights<V>(a.w, a.w_bf16, a.w_vec, col, a.n, 1.f, w);
        if (dh) RowIo<T, V>::load(dh, col, a.n, hv);
#pragma unroll
        for (int e = 0; e < V; ++e)
            dv[e] = fmaf(rstd, dv[e] * w[e] - g - (xv[e] - mean) * rstd * gu, hv[e]);
        RowIo<T, V>::store(dx, col, a.n, dv);
    }
}

// Column sums over a range of rows: thread = one column, block.y = one range.
constexpr int NB_COL_THREADS = 128;
template <typename T>
__global__ void __launch_bounds__(NB_COL_THREADS)
norm_backward_columns_kernel(const NormBackwardArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int col = blockIdx.x * NB_COL_THREADS + threadIdx.x;
    if (col >= a.n) return;
    const int64_t begin = (int64_t)blockIdx.y * a.rows_per_split;
    const int64_t end = begin + a.rows_per_split < a.b ? begin + a.rows_per_split : a.b;
    float dw = 0.f, dc = 0.f;
    for (int64_t row = begin; row < end; ++row) {
        const float d = to_float(static_cast<const T*>(a.dy)[row * a.lddy + col]);
        const float mean = a.rms ? 0.f : a.mean[row];
        const float u = (to_float(static_cast<const T*>(a.x)[row * a.ldx + col]) - mean) * a.rstd[row];
        dw = fmaf(d, u, dw);
        dc += d;
    }
    float* part = a.part + (int64_t)blockIdx.y * 2 * a.n + col;
    part[0] = dw;
    part[a.n] = dc;
}

// The partial sums of all ranges, added in their order.
__global__ void __launch_bounds__(NB_COL_THREADS)
norm_backward_finish_kernel(const NormBackwardArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int col = blockIdx.x * NB_COL_THREADS + threadIdx.x;
    if (col >= a.n) return;
    float dw = 0.f, dc = 0.f;
    for (int s = 0; s < a.splits; ++s) {
        const float* part = a.part + (int64_t)s * 2 * a.n + col;
        dw += part[0];
        dc += part[a.n];
    }
    if (a.dw) {
        if (a.dw_bf16) static_cast<__nv_bfloat16*>(a.dw)[col] = __float2bfloat16_rn(dw);
        else static_cast<float*>(a.dw)[col] = dw;
    }
    if (a.dc) {
        if (a.dw_bf16) static_cast<__nv_bfloat16*>(a.dc)[col] = __float2bfloat16_rn(dc);
        else static_cast<float*>(a.dc)[col] = dc;
    }
}

}  // namespace pamm
