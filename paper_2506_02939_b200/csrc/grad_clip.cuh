// The global norm of a list of gradients, and their clipping:
//   N = sqrt(sum over all elements of g^2);  g <- g min(1, max_norm / (N + 1e-6))
//
// Three launches, the first and the last bound by memory: every block sums the squares of its share; one block
// joins the sums in a fixed order (of a small list, every block of the last launch); and the scaling reads and writes every element once more (or, in place and below the
// limit, returns at once).  The list travels in the kernels' parameters, so that a call needs no copy and no allocation
// and can be captured; lists longer than one launch holds take several.  The work is cut into chunks of 4096 to 65536
// elements, block after block; the scaling goes through them backwards, and so finds in L2 what the sum read last.
// Squares are summed in 64 bits, whose range no bf16 or fp32 gradient leaves (B200 has half as many 64-bit as 32-bit
// lanes; the sum stays bound by memory).
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"

namespace pamm {

constexpr int GC_THREADS = 256;
constexpr int GC_UNROLL = 4;            // vectors in flight per thread
constexpr int GC_BLOCKS_PER_SM = 8;     // of the sum: one wave
// elements of a chunk: of the sum, by the size of the list; of the scaling
constexpr int GC_MIN_CHUNK = 4096, GC_MAX_CHUNK = 65536, GC_SCALE_CHUNK = 16384;
// List entries per launch: a power of two, four times as many, and as many as the parameters of a launch hold (2.3, 9 and 32 KB).  What
// a list has no use for still goes to the device with every launch.  Calls in place one after the other, of 4 and 28 small
// tensors: with room for 32 4.7 and 5.3 us, for 128 5.1 and 5.7, for 448 7.0 and 7.7; of 40 and 120: for 128 6.0 and 8.3, for 448 8.0 and 10.0.
constexpr int GC_SMALL = 32, GC_MEDIUM = 128, GC_LARGE = 448;

struct GradEntry {
    const void* in;
    void* out;
    int64_t rows, cols, ld_in, ld_out;
    int64_t first_chunk, pieces;          // chunks before this entry; of a wide row
    short in_bf16, out_bf16;
    int off;                            // one row: elements from the 16-byte boundary below its start, on which chunks are cut
};
template <int CAP>
struct GradList {
    int count;
    int add;                            // the partial sums continue those of an earlier launch
    int in_place;                       // every output is its input
    int chunk;                          // elements
    int64_t chunks;
    GradEntry e[CAP];
};

// Rows of fewer columns than a chunk has elements are put together until it is full, wider rows are cut.
inline int64_t grad_chunks(int64_t rows, int64_t cols, int64_t chunk) {
    if (rows == 0 || cols == 0) return 0;
    return rows > 1 && cols < chunk ? (rows + chunk / cols - 1) / (chunk / cols) : rows * ((cols + chunk - 1) / chunk);
}

// Elements before the first 16-byte boundary at or after p, at most len.
template <typename T>
__device__ __forceinline__ int lead_elements(const T* p, int len) {
    return min(len, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
}

// A square in 64 bits.  Conversions and products keep up with memory (bf16 from HBM: 6.0 TB/s with them, 6.5 without).
__device__ __forceinline__ void add_square(double& acc, float x) { acc = fma((double)x, (double)x, acc); }

// The up to V - 1 elements of a span before its first and behind its last 16-byte vector (or group of G elements): thread t has one
// of each.  Loaded before the vectors and used after them.
template <typename T, int G>
struct Ends {
    using One = Piece<T, 1>;
    int lead, groups, done, len, t;
    typename One::Raw a, b;
    __device__ __forceinline__ Ends(const T* p, int len_, int t_) : lead(lead_elements(p, len_)), len(len_), t(t_), a(One::zero()), b(One::zero()) {
        groups = (len - lead) / G;
        done = lead + groups * G;
        if (t < lead) a = One::load(p + t);
        if (t < len - done) b = One::load(p + done + t);
    }
    template <typename F>
    __device__ __forceinline__ void use(F f) const {          // f(element, its place)
        float v;
        if (t < lead) {
            One::unpack(a, &v);
            f(v, t);
        }
        if (t < len - done) {
            One::unpack(b, &v);
            f(v, done + t);
        }
    }
};

// load(k, first element) and use(k, first element) for a span's groups of G elements by STEP threads: U of them at a time, then half
// as many, at last one.  (With U loads under a condition each, every load is waited for by itself: half the speed.)
template <int G, int U, int STEP, typename Load, typename Use>
__device__ __forceinline__ void walk_span(int lead, int groups, int t, Load load, Use use) {
    int i = t;
    for (; i + (U - 1) * STEP < groups; i += U * STEP) {
#pragma unroll
        for (int k = 0; k < U; ++k) load(k, lead + (i + k * STEP) * G);
#pragma unroll
        for (int k = 0; k < U; ++k) use(k, lead + (i + k * STEP) * G);
    }
    if constexpr (U > 1) walk_span<G, U / 2, STEP>(lead, groups, i, load, use);
}

template <typename T, int STEP>
__device__ __forceinline__ void add_squares(const T* p, int len, int t, double& sum) {
    constexpr int V = Vec16<T>::N, U = STEP > 32 ? GC_UNROLL : 1;
    using P = Piece<T, V>;
    const Ends<T, V> ends(p, len, t);
    typename P::Raw r[U];
    walk_span<V, U, STEP>(ends.lead, ends.groups, t, [&](int k, int at) { r[k] = P::load(p + at); },
                          [&](int k, int) {
                              float v[V];
                              P::unpack(r[k], v);
#pragma unroll
                              for (int e = 0; e < V; ++e) add_square(sum, v[e]);
                          });
    ends.use([&](float v, int) { add_square(sum, v); });
}

// The factor as a product of two, so that one below fp32's normal range keeps its digits; and whether it is 1.
struct GradFactor {
    float first, second;
    int keep;
    __device__ __forceinline__ float operator()(float g) const { return g * first * second; }
};

template <typename TI, typename TO, int STEP>
__device__ __forceinline__ void scale_span(const TI* p, TO* q, int len, const GradFactor& f, int t) {
    // G elements at a time: 16 bytes on the side of the wider type, so that a warp's accesses have no gaps on either
    constexpr int G = Vec16<TI>::N < Vec16<TO>::N ? Vec16<TI>::N : Vec16<TO>::N, U = STEP > 32 ? GC_UNROLL : 1;
    if ((reinterpret_cast<uintptr_t>(q + lead_elements(p, len)) & 15) != 0) {        // the output is not on a 16-byte boundary there
        for (int i = t; i < len; i += STEP) q[i] = from_float<TO>(f(to_float(p[i])));
        return;
    }
    const Ends<TI, G> ends(p, len, t);
    const uint64_t policy = evict_first_policy();       // what is yet to be read stays in L2
    typename Piece<TI, G>::Raw r[U];
    walk_span<G, U, STEP>(ends.lead, ends.groups, t, [&](int k, int at) { r[k] = Piece<TI, G>::load(p + at); },
                          [&](int k, int at) {
                              float v[G];
                              Piece<TI, G>::unpack(r[k], v);
#pragma unroll
                              for (int e = 0; e < G; ++e) v[e] = f(v[e]);
                              Piece<TO, G>::store(q + at, v, policy);
                          });
    ends.use([&](float v, int at) { q[at] = from_float<TO>(f(v)); });
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

template <int N> struct Threads { static constexpr int value = N; };

// Calls wide(entry, row, column, length) for every span of the block's chunks (which lie gridDim.x apart) that the whole block
// takes, narrow(entry, row, 0, length) for those that a warp takes.
template <int CAP, typename F, typename G>
__device__ __forceinline__ void for_each_span(const GradList<CAP>& list, bool backwards, F wide, G narrow) {
    for (int64_t n = blockIdx.x; n < list.chunks; n += gridDim.x) {
        const int64_t at = backwards ? list.chunks - 1 - n : n;
        int lo = 0, hi = list.count - 1;            // the last entry that starts at or before the chunk
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (list.e[mid].first_chunk <= at) lo = mid;
            else hi = mid - 1;
        }
        const GradEntry& g = list.e[lo];
        const int64_t local = at - g.first_chunk;
        if (g.rows == 1) {
            const int64_t from = local * list.chunk - g.off, to = from + list.chunk, col = from < 0 ? 0 : from;
            wide(g, (int64_t)0, col, (int)((to < g.cols ? to : g.cols) - col));
        } else if (g.cols >= list.chunk) {
            const int64_t row = local / g.pieces, col = (local - row * g.pieces) * list.chunk;
            wide(g, row, col, (int)(g.cols - col < list.chunk ? g.cols - col : list.chunk));
        } else {                                    // whole rows
            const int64_t rows = list.chunk / (int)g.cols, first = local * rows;
            const int64_t last = first + rows < g.rows ? first + rows : g.rows;
            for (int64_t row = first + (threadIdx.x >> 5); row < last; row += GC_THREADS / 32) narrow(g, row, (int64_t)0, (int)g.cols);
        }
    }
}

template <int CAP>
__global__ void __launch_bounds__(GC_THREADS, GC_BLOCKS_PER_SM)
grad_squares_kernel(const __grid_constant__ GradList<CAP> list, double* partial) {
    __shared__ double s_part[GC_THREADS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    double sum = 0.0;
    const auto span = [&](auto step, int t, const GradEntry& g, int64_t row, int64_t col, int len) {
        const int64_t at = row * g.ld_in + col;
        if (g.in_bf16) add_squares<__nv_bfloat16, decltype(step)::value>(static_cast<const __nv_bfloat16*>(g.in) + at, len, t, sum);
        else add_squares<float, decltype(step)::value>(static_cast<const float*>(g.in) + at, len, t, sum);
    };
    for_each_span(list, false,
                  [&](const GradEntry& g, int64_t row, int64_t col, int len) { span(Threads<GC_THREADS>(), threadIdx.x, g, row, col, len); },
                  [&](const GradEntry& g, int64_t row, int64_t col, int len) { span(Threads<32>(), threadIdx.x & 31, g, row, col, len); });
    const double acc = block_sum_double(sum, s_part);
    if (threadIdx.x == 0) partial[blockIdx.x] = (list.add ? partial[blockIdx.x] : 0.0) + acc;
}

// The norm, and the factor, from the blocks' sums: the same in every block that asks.
__device__ __forceinline__ GradFactor join_sums(const double* partial, int parts, double max_norm, double* s_part, double& total) {
    double acc = 0.0;
    for (int i = threadIdx.x; i < parts; i += GC_THREADS) acc += partial[i];
    total = sqrt(block_sum_double(acc, s_part));
    const double limited = max_norm / (total + 1e-6);
    // no limit at all, or one that is kept: 1; a NaN norm gives NaN, as in the formula
    const bool keep = isinf(max_norm) || limited >= 1.0;
    GradFactor f = {1.f, keep ? 1.f : (float)limited, keep ? 1 : 0};
    if (!keep && limited < 0x1p-100) {
        f.first = 0x1p-64f;
        f.second = (float)(limited * 0x1p64);
    }
    return f;
}

__global__ void __launch_bounds__(GC_THREADS)
grad_norm_finish_kernel(const double* partial, int parts, double max_norm, float* norm, GradFactor* factor) {
    __shared__ double s_part[GC_THREADS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    double total;
    const GradFactor f = join_sums(partial, parts, max_norm, s_part, total);
    if (threadIdx.x != 0) return;
    *norm = (float)total;
    *factor = f;
}

// The sums have been joined (parts = 0), or are few and every block does it for itself, which saves a launch: 2 us of a small list's 9.
template <int CAP>
__global__ void __launch_bounds__(GC_THREADS, 6)
grad_scale_kernel(const __grid_constant__ GradList<CAP> list, const GradFactor* factor, const double* partial, int parts, double max_norm,
                  float* norm) {
    __shared__ double s_part[GC_THREADS / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    GradFactor f;
    if (parts) {
        double total;
        f = join_sums(partial, parts, max_norm, s_part, total);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    } else {
        f = *factor;
    }
    if (f.keep && list.in_place) return;            // g * 1 is there already
    const auto span = [&](auto step, int t, const GradEntry& g, int64_t row, int64_t col, int len) {
        constexpr int STEP = decltype(step)::value;
        const int64_t i = row * g.ld_in + col, o = row * g.ld_out + col;
        if (g.in_bf16) {
            const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(g.in) + i;
            if (g.out_bf16) scale_span<__nv_bfloat16, __nv_bfloat16, STEP>(p, static_cast<__nv_bfloat16*>(g.out) + o, len, f, t);
            else scale_span<__nv_bfloat16, float, STEP>(p, static_cast<float*>(g.out) + o, len, f, t);
        } else {
            const float* p = static_cast<const float*>(g.in) + i;
            if (g.out_bf16) scale_span<float, __nv_bfloat16, STEP>(p, static_cast<__nv_bfloat16*>(g.out) + o, len, f, t);
            else scale_span<float, float, STEP>(p, static_cast<float*>(g.out) + o, len, f, t);
        }
    };
    for_each_span(list, true,
                  [&](const GradEntry& g, int64_t row, int64_t col, int len) { span(Threads<GC_THREADS>(), threadIdx.x, g, row, col, len); },
                  [&](const GradEntry& g, int64_t row, int64_t col, int len) { span(Threads<32>(), threadIdx.x & 31, g, row, col, len); });
}

}  // namespace pamm
