// The global norm of a list of gradients, and their clipping:
//   N = sqrt(sum over all elements of g^2);  g <- g min(1, max_norm / (N + 1e-6))
//
// Two passes, both bound by memory: the squares' sum reads every element once, the scaling reads and
// writes it once more (or, in place and below the limit, does nothing).  The list travels in the
// kernels' parameters, so that a call needs no copy and no allocation and can be captured; lists
// longer than one launch holds take several.  The work is cut into chunks of about 8192 elements that
// every block takes a consecutive range of; squares are summed in 64 bits, whose range no bf16 or fp32
// gradient leaves, and joined in a fixed order.
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"

namespace pamm {

constexpr int GC_THREADS = 256;
constexpr int GC_CHUNK = 8192;          // elements
constexpr int GC_BLOCKS_PER_SM = 8;
constexpr int GC_SMALL = 24, GC_LARGE = 448;      // list entries per launch: parameters of 1.5 and 28 KB

struct GradEntry {
    const void* in;
    void* out;
    int64_t rows, cols, ld_in, ld_out;
    int64_t first_chunk;
    int in_bf16, out_bf16;
};
template <int CAP>
struct GradList {
    int count, add;                     // add: the partial sums continue those of an earlier launch
    int64_t chunks;
    GradEntry e[CAP];
};

// Rows of at most GC_CHUNK columns are put together until a chunk is full, wider rows are cut.
__host__ __device__ inline int64_t grad_rows_per_chunk(int64_t cols) { return cols < GC_CHUNK ? GC_CHUNK / cols : 1; }
__host__ __device__ inline int64_t grad_pieces(int64_t cols) { return (cols + GC_CHUNK - 1) / GC_CHUNK; }
__host__ __device__ inline int64_t grad_chunks(int64_t rows, int64_t cols) {
    if (rows == 0 || cols == 0) return 0;
    const int64_t rpc = grad_rows_per_chunk(cols);
    return cols < GC_CHUNK ? (rows + rpc - 1) / rpc : rows * grad_pieces(cols);
}

// Squares of `len` consecutive elements, by `step` threads of which this is number t.
template <typename T>
__device__ __forceinline__ double span_squares(const T* p, int len, int t, int step) {
    constexpr int V = Vec16<T>::N;
    double acc = 0.0;
    const int lead = min(len, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    const int vecs = (len - lead) / V;
    for (int i = t; i < vecs; i += step) {
        float v[V];
        unpack_vec<T>(ld16(p + lead + i * V), v);
#pragma unroll
        for (int e = 0; e < V; ++e) acc += (double)v[e] * (double)v[e];
    }
    if (t < lead) {
        const double v = to_float(p[t]);
        acc += v * v;
    }
    const int done = lead + vecs * V;
    if (t < len - done) {
        const double v = to_float(p[done + t]);
        acc += v * v;
    }
    return acc;
}

// The factor as a product of two, so that one below fp32's normal range keeps its digits.
struct GradFactor {
    float first, second;
    __device__ __forceinline__ float operator()(float g) const { return g * first * second; }
};

template <typename TI, typename TO>
__device__ __forceinline__ void span_scale(const TI* p, TO* q, int len, GradFactor f, int t, int step) {
    constexpr int V = Vec16<TI>::N, W = Vec16<TO>::N;
    const int lead = min(len, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(TI));
    // vector access where both sides reach a 16-byte boundary (of 16-bit and 32-bit elements alike) together
    constexpr int G = V > W ? V : W;
    if ((reinterpret_cast<uintptr_t>(q + lead) & 15) != 0) {
        for (int i = t; i < len; i += step) q[i] = from_float<TO>(f(to_float(p[i])));
        return;
    }
    const int groups = (len - lead) / G;
    for (int i = t; i < groups; i += step) {
        float v[G];
#pragma unroll
        for (int k = 0; k < G; k += V) unpack_vec<TI>(ld16(p + lead + i * G + k), *reinterpret_cast<float(*)[V]>(v + k));
#pragma unroll
        for (int e = 0; e < G; ++e) v[e] = f(v[e]);
#pragma unroll
        for (int k = 0; k < G; k += W) st16(q + lead + i * G + k, round_vec<TO>(*reinterpret_cast<float(*)[W]>(v + k)));
    }
    if (t < lead) q[t] = from_float<TO>(f(to_float(p[t])));
    const int done = lead + groups * G;
    if (t < len - done) q[done + t] = from_float<TO>(f(to_float(p[done + t])));
}

__device__ __forceinline__ double block_sum_double(double x, double* part) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < GC_THREADS / 32; ++w) x += part[w];
    return x;
}

// Calls body(entry, row, column, length, thread, threads) for every span of the block's chunks.
template <int CAP, typename F>
__device__ __forceinline__ void for_each_span(const GradList<CAP>& list, F body) {
    const int64_t per = (list.chunks + gridDim.x - 1) / gridDim.x;
    const int64_t begin = (int64_t)blockIdx.x * per;
    const int64_t end = begin + per < list.chunks ? begin + per : list.chunks;
    if (begin >= end) return;
    int lo = 0, hi = list.count - 1;            // the last entry that starts at or before `begin`
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (list.e[mid].first_chunk <= begin) lo = mid;
        else hi = mid - 1;
    }
    int k = lo;
    for (int64_t chunk = begin; chunk < end; ++chunk) {
        while (k + 1 < list.count && list.e[k + 1].first_chunk <= chunk) ++k;
        const GradEntry& g = list.e[k];
        const int64_t local = chunk - g.first_chunk;
        if (g.cols >= GC_CHUNK) {
            const int64_t pieces = grad_pieces(g.cols), row = local / pieces, col = (local - row * pieces) * GC_CHUNK;
            body(g, row, col, (int)(g.cols - col < GC_CHUNK ? g.cols - col : GC_CHUNK), (int)threadIdx.x, GC_THREADS);
        } else {
            const int64_t rpc = grad_rows_per_chunk(g.cols), first = local * rpc;
            const int64_t last = first + rpc < g.rows ? first + rpc : g.rows;
            if (last - first == 1) {
                body(g, first, 0, (int)g.cols, (int)threadIdx.x, GC_THREADS);
            } else {
                for (int64_t row = first + (threadIdx.x >> 5); row < last; row += GC_THREADS / 32)
                    body(g, row, 0, (int)g.cols, (int)(threadIdx.x & 31), 32);
            }
        }
    }
}

template <int CAP>
__global__ void __launch_bounds__(GC_THREADS)
grad_squares_kernel(const __grid_constant__ GradList<CAP> list, double* partial) {
    __shared__ double s_part[GC_THREADS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    double acc = 0.0;
    for_each_span(list, [&](const GradEntry& g, int64_t row, int64_t col, int len, int t, int step) {
        const int64_t at = row * g.ld_in + col;
        acc += g.in_bf16 ? span_squares(static_cast<const __nv_bfloat16*>(g.in) + at, len, t, step)
                         : span_squares(static_cast<const float*>(g.in) + at, len, t, step);
    });
    acc = block_sum_double(acc, s_part);
    if (threadIdx.x == 0) partial[blockIdx.x] = (list.add ? partial[blockIdx.x] : 0.0) + acc;
}

// The norm from the partial sums, in every block alike.
__device__ __forceinline__ double norm_of(const double* partial, int parts, double* s_part) {
    double acc = 0.0;
    for (int i = threadIdx.x; i < parts; i += GC_THREADS) acc += partial[i];
    return sqrt(block_sum_double(acc, s_part));
}

__global__ void __launch_bounds__(GC_THREADS)
grad_norm_finish_kernel(const double* partial, int parts, float* norm) {
    __shared__ double s_part[GC_THREADS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    const double total = norm_of(partial, parts, s_part);
    if (threadIdx.x == 0) *norm = (float)total;
}

template <int CAP>
__global__ void __launch_bounds__(GC_THREADS)
grad_scale_kernel(const __grid_constant__ GradList<CAP> list, const double* partial, int parts, double max_norm, float* norm) {
    __shared__ double s_part[GC_THREADS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    const double total = norm_of(partial, parts, s_part);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const double limited = max_norm / (total + 1e-6);
    // no limit at all, or one that is kept: 1; a NaN norm gives NaN, as in the formula
    const bool keep = isinf(max_norm) || limited >= 1.0;
    GradFactor f = {1.f, keep ? 1.f : (float)limited};
    if (!keep && limited < 0x1p-100) f = {0x1p-64f, (float)(limited * 0x1p64)};
    for_each_span(list, [&](const GradEntry& g, int64_t row, int64_t col, int len, int t, int step) {
        if (keep && g.in == g.out && g.in_bf16 == g.out_bf16) return;     // g * 1 is there already
        const int64_t i = row * g.ld_in + col, o = row * g.ld_out + col;
        if (g.in_bf16) {
            const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(g.in) + i;
            if (g.out_bf16) span_scale(p, static_cast<__nv_bfloat16*>(g.out) + o, len, f, t, step);
            else span_scale(p, static_cast<float*>(g.out) + o, len, f, t, step);
        } else {
            const float* p = static_cast<const float*>(g.in) + i;
            if (g.out_bf16) span_scale(p, static_cast<__nv_bfloat16*>(g.out) + o, len, f, t, step);
            else span_scale(p, static_cast<float*>(g.out) + o, len, f, t, step);
        }
    });
}

}  // namespace pamm
