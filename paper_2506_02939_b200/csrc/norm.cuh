// Layer norm and its root-mean-square form, forward and backward, optionally with the residual
// addition on both ways.
//
//   h = x (+ r);  mu = mean(h) (0 in the RMS form);  v = mean((h - mu)^2);  s = 1 / sqrt(v + eps)
//   y = (h - mu) s w (+ c)
//   u = (h - mu) s;  g = dy w;  dx = s (g - mean(g) - u mean(g u)) (+ dh), without mean(g) in the RMS form
//   dw = sum over rows of dy u;  dc = sum over rows of dy
//
// All of it is bound by memory: about 10 operations an element against 4 to 8 bytes.  A row stays in
// registers between its one reading and its one writing, and the variance is taken around the true mean.
// mu and s are those of h before it is rounded to its storage type: y then carries one rounding.
//
// Values from 1e19 on (a masked row holds its type's lowest, -3e38) have squares, and sums, beyond fp32, and h - mu
// reaches twice the type's range.  The forward pass takes such a row a second time, its values times 2^-80; the
// backward pass takes differences as h / 4 - mu / 4, with the same bits (a multiply-add with a power of two in place of
// an addition).
//
// A thread holds EPT elements of its row in EPT / V pieces; V is a 16-byte vector or one element:
//   vectors, whole   every row 16-byte aligned, n a multiple of V
//   vectors, RAGGED  any n and any alignment that all matrices of the call share row by row: the row's whole vectors
//                    on the 16-byte grid of memory, and its up to V - 1 elements before and behind them, which the
//                    row's first 16 threads take one each
//   elements         matrices whose rows are aligned differently
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"
#include "sm100_ptx.cuh"
#include <cfloat>

namespace pamm {

constexpr int64_t NORM_MAX_N = 32768;
constexpr float NORM_SHRINK = 0x1p-80f;       // 32768 squares of 2 x 2^128 x 2^-80 fit fp32

// A row's whole vectors and this thread's element outside them.
struct RowShape {
    int lead, whole;        // elements before the first whole vector, and in the whole ones
    int extra;              // this thread's element outside them (-1: none)
};
template <typename T, int V, bool RAGGED>
__device__ __forceinline__ RowShape row_shape(const T* row, int n, int t) {
    if constexpr (!RAGGED) {
        return {0, n, -1};
    } else {
        const int lead = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T));
        const int whole = (n - lead) / V * V, behind = lead + whole + t - 8;
        return {lead, whole, t < lead ? t : t >= 8 && t < 16 && behind < n ? behind : -1};
    }
}

// The row's pieces: PIECES vectors (or elements) at distance `step` from `at`; zero at and beyond `end`.
template <typename T, int V, int PIECES>
__device__ __forceinline__ void load_row(const T* p, int at, int step, int end, typename Piece<T, V>::Raw (&raw)[PIECES]) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        if (at + i * step < end) raw[i] = Piece<T, V>::load(p + at + i * step);
        else raw[i] = Piece<T, V>::zero();
    }
}
// V weights from element `col` on, whose distance from the vector grid, `OFF`, is the same for the whole row: the aligned vectors that hold
// them, unpacked from the place they lie at.
template <typename W, int V, int OFF>
__device__ __forceinline__ void load_shifted(const W* aligned, float* out) {
    constexpr int A = V < 16 / (int)sizeof(W) ? V : 16 / (int)sizeof(W);      // elements of a vector
    constexpr int COUNT = V / A + (OFF > 0), WORDS = A * (int)sizeof(W) / 4;
    uint32_t w[COUNT * WORDS];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        if constexpr (WORDS == 4) {
            const uint4 t = __ldg(reinterpret_cast<const uint4*>(aligned + i * A));
            w[4 * i] = t.x; w[4 * i + 1] = t.y; w[4 * i + 2] = t.z; w[4 * i + 3] = t.w;
        } else {
            const uint2 t = __ldg(reinterpret_cast<const uint2*>(aligned + i * A));
            w[2 * i] = t.x; w[2 * i + 1] = t.y;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int j = OFF + e;
        if constexpr (sizeof(W) == 4) out[e] = __uint_as_float(w[j]);
        else out[e] = j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
    }
}
template <typename W, int V, int OFF = 0>
__device__ __forceinline__ void load_at_offset(const W* aligned, int off, float* out) {
    constexpr int A = V < 16 / (int)sizeof(W) ? V : 16 / (int)sizeof(W);
    if constexpr (OFF < A) {
        if (off == OFF) load_shifted<W, V, OFF>(aligned, out);
        else load_at_offset<W, V, OFF + 1>(aligned, off, out);
    }
}
// Weights col .. col + V - 1 of the n at `w`.
template <typename W, int V, bool RAGGED>
__device__ __forceinline__ void load_row_weights(const W* w, int col, int n, float* out) {
    if constexpr (!RAGGED) {
        load_weights<W, V>(w + col, out);
    } else {
        constexpr int A = V < 16 / (int)sizeof(W) ? V : 16 / (int)sizeof(W);
        const int off = (int)(reinterpret_cast<uintptr_t>(w + col) / sizeof(W) % A);
        if (off == 0 || (col >= off && col - off + V + A <= n)) {
            load_at_offset<W, V>(w + col - off, off, out);
        } else {            // the vectors would leave the weights
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = to_float(w[col + e]);
        }
    }
}

struct NormForwardArgs {
    const void *x, *r, *w, *c;
    void *y, *h;
    float *mean, *rstd;
    int64_t ldx, ldr, ldy, ldh, b;
    int n, warps;           // warps of the block that share a row; 1: LANES lanes have a row
    float eps;
    bool rms, h_over_input; // H takes the place of X or R
};

// Sums over the warps of a block's rows (all of the block's); every thread gets them.  `part`: [ROWS][32] floats that the
// caller does not use again before another barrier.
template <int LANES, int ROWS>
__device__ __forceinline__ void row_sums(float (&x)[ROWS], float (*part)[32], int warps) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) x[r] = warp_sum<LANES>(x[r]);
    if (LANES < 32 || warps == 1) return;
    const int lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) part[r][threadIdx.x >> 5] = x[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) x[r] = warp_sum(lane < warps ? part[r][lane] : 0.f);
}

// A row whose sum of squares is infinite or NaN, from the start with its values times NORM_SHRINK: NaN and infinities among them
// give what the formulas give, large values their statistics.  Every value is read again for each of the three passes: from H,
// rounded to its type, where that has taken the place of X or R.  Threads without such a row (`active`) go along for the shuffles.
// Rare: the hot path pays a comparison and a branch, up to 1% of its time (3% for rows of 257 to 512, whose lanes are half a warp);
// scaling the sums of every row instead cost up to 4% and more registers, this row kept in registers up to 3%.
template <typename T, typename W, int V, int LANES, bool RAGGED>
__device__ __forceinline__ void norm_forward_shrunk_row(const NormForwardArgs& a, int64_t row, bool active, int at, int step, const RowShape& shape,
                                                        float (*s_sum)[32], float (*s_sq)[32]) {
    using P = Piece<T, V>;
    const float inv_n = 1.f / (float)a.n, to = 1.f / NORM_SHRINK;
    const T* x = a.h_over_input ? static_cast<const T*>(a.h) + row * a.ldh : static_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.r && !a.h_over_input ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
    const int end = active ? shape.whole : 0, extra = RAGGED && active ? shape.extra : -1;
    const auto values = [&](int col, float* v) {
        P::unpack(P::load(x + col), v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] *= NORM_SHRINK;
        if (r) {
            float q[V];
            P::unpack(P::load(r + col), q);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = fmaf(q[e], NORM_SHRINK, v[e]);
        }
    };
    float hx = 0.f, v[V], mean = 0.f;
    if (extra >= 0) hx = fmaf(r ? to_float(r[extra]) : 0.f, NORM_SHRINK, to_float(x[extra]) * NORM_SHRINK);
    const bool barriers = LANES == 32 && a.warps > 1;
    if (barriers) __syncthreads();          // every warp has read the parts of the first time
    if (!a.rms) {
        float sum[1] = {hx};
#pragma unroll 1
        for (int i = at; i < end; i += step) {
            values(shape.lead + i, v);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[0] += v[e];
        }
        row_sums<LANES>(sum, s_sum, a.warps);
        mean = sum[0] * inv_n;
    }
    if (extra >= 0) hx -= mean;
    float sq[1] = {hx * hx};
#pragma unroll 1
    for (int i = at; i < end; i += step) {
        values(shape.lead + i, v);
#pragma unroll
        for (int e = 0; e < V; ++e) sq[0] = fmaf(v[e] - mean, v[e] - mean, sq[0]);
    }
    row_sums<LANES>(sq, s_sq, a.warps);
    if (barriers) __syncthreads();          // the caller may come with another row
    if (!active) return;
    const float small = sq[0] * inv_n, var = small * to * to;
    float rstd = rsqrtf(var + a.eps), factor = rstd * to;
    if (!(var <= FLT_MAX)) {                // beside which eps is nothing
        factor = rsqrtf(small);
        rstd = factor * NORM_SHRINK;
    }
    if (at == 0) {
        const float m = mean * to;          // rounded, it may lie above the largest value
        if (a.mean) a.mean[row] = isinf(m) && !isinf(mean) ? copysignf(FLT_MAX, m) : m;
        if (a.rstd) a.rstd[row] = rstd;
    }
    const W *w = static_cast<const W*>(a.w), *c = static_cast<const W*>(a.c);
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    if (extra >= 0) y[extra] = from_float<T>(fmaf(hx * factor, w ? to_float(w[extra]) : 1.f, c ? to_float(c[extra]) : 0.f));
#pragma unroll 1
    for (int i = at; i < end; i += step) {
        const int col = shape.lead + i;
        values(col, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = fmaf((v[e] - mean) * factor, w ? to_float(w[col + e]) : 1.f, c ? to_float(c[col + e]) : 0.f);
        P::store(y + col, v);
    }
}

// Measured on 65536 x 2048 bf16 (268 MB a matrix): the 16-byte copy of the same streams in one-shot blocks runs at 6.5 to
// 6.7 TB/s, in persistent ones at 6.0, hence a block (or a part of one) for its rows and no loop over rows.
// 158 us with the residual addition (6.8 TB/s), 85 without.  A thread may have ROWS = 2 rows, which share its weights (the launch says when).  8 elements a thread repeat the row's
// overhead in more threads and are for calls with few rows, where the time is one row's latency.
template <typename T, typename W, int V, int EPT, int LANES, int ROWS, bool RAGGED>
__global__ void __launch_bounds__(1024)
norm_forward_kernel(const __grid_constant__ NormForwardArgs a) {
    static_assert(ROWS == 1 || !RAGGED, "rows of one thread share their offset");
    using P = Piece<T, V>;
    constexpr int PIECES = EPT / V;
    __shared__ float s_sum[ROWS][32], s_sq[ROWS][32];
    grid_dependency_wait();
    grid_launch_dependents();
    const bool one = a.warps == 1;
    const int step = (LANES < 32 ? LANES : 32 * a.warps) * V;
    const int at = (LANES < 32 ? threadIdx.x & (LANES - 1) : one ? threadIdx.x & 31 : threadIdx.x) * V;
    const int64_t row0 = (one ? (int64_t)blockIdx.x * (blockDim.x / LANES) + threadIdx.x / LANES : blockIdx.x) * ROWS;
    // the lanes behind the last row go along with it, so that shuffles have all of their warp, and write nothing
    int64_t row[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) row[r] = row0 + r < a.b ? row0 + r : a.b - 1;
    const T* x0 = static_cast<const T*>(a.x) + row[0] * a.ldx;
    const RowShape shape = row_shape<T, V, RAGGED>(x0, a.n, at / V);
    const int lead = shape.lead, end = shape.whole, extra = shape.extra;
    float h[ROWS][EPT], hx = 0.f;
    {
        typename P::Raw xr[ROWS][PIECES];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) load_row<T, V, PIECES>(static_cast<const T*>(a.x) + row[r] * a.ldx + lead, at, step, end, xr[r]);
        using One = Piece<T, 1>;
        typename One::Raw x1 = One::zero(), r1 = One::zero();
        if (RAGGED && extra >= 0) x1 = One::load(x0 + extra);
        if (a.r) {
            typename P::Raw rr[ROWS][PIECES];
            const T* r0 = static_cast<const T*>(a.r) + row[0] * a.ldr;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) load_row<T, V, PIECES>(static_cast<const T*>(a.r) + row[r] * a.ldr + lead, at, step, end, rr[r]);
            if (RAGGED && extra >= 0) r1 = One::load(r0 + extra);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
#pragma unroll
                for (int p = 0; p < PIECES; ++p) {
                    float q[V];
                    P::unpack(xr[r][p], h[r] + p * V);
                    P::unpack(rr[r][p], q);
#pragma unroll
                    for (int e = 0; e < V; ++e) h[r][p * V + e] += q[e];
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int p = 0; p < PIECES; ++p) P::unpack(xr[r][p], h[r] + p * V);
        }
        if (RAGGED) {
            float q;
            One::unpack(x1, &hx);
            One::unpack(r1, &q);
            hx += q;
        }
    }
    if (a.h) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row0 + r >= a.b) continue;
            T* ho = static_cast<T*>(a.h) + row[r] * a.ldh;
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
                if (at + p * step < end) P::store(ho + lead + at + p * step, h[r] + p * V);
            if (RAGGED && extra >= 0) ho[extra] = from_float<T>(hx);
        }
    }
    const float inv_n = 1.f / (float)a.n;
    float mean[ROWS], rstd[ROWS];
    if (!a.rms) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float2 sum = make_float2(RAGGED ? hx : 0.f, 0.f);
#pragma unroll
            for (int e = 0; e < EPT; e += 2) sum = add2(sum, make_float2(h[r][e], h[r][e + 1]));
            mean[r] = sum.x + sum.y;
        }
        row_sums<LANES>(mean, s_sum, a.warps);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mean[r] *= inv_n;
            const float2 minus = twice(-mean[r]);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                if (at + p * step < end) {          // what lies outside the row stays 0
                    if constexpr (V == 1) {
                        h[r][p] -= mean[r];
                    } else {
#pragma unroll
                        for (int e = p * V; e < p * V + V; e += 2) {
                            const float2 d = add2(make_float2(h[r][e], h[r][e + 1]), minus);
                            h[r][e] = d.x; h[r][e + 1] = d.y;
                        }
                    }
                }
            }
        }
        if (extra >= 0) hx -= mean[0];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float2 sq = make_float2(RAGGED ? hx * hx : 0.f, 0.f);
#pragma unroll
        for (int e = 0; e < EPT; e += 2) {
            const float2 d = make_float2(h[r][e], h[r][e + 1]);
            sq = fma2(d, d, sq);
        }
        rstd[r] = sq.x + sq.y;
    }
    row_sums<LANES>(rstd, s_sq, a.warps);
    bool beyond[ROWS], any = false;          // fp32's range: the row is taken again in the end
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        beyond[r] = !(rstd[r] <= FLT_MAX);
        any = any || beyond[r];
        rstd[r] = rsqrtf(rstd[r] * inv_n + a.eps);
        if (at == 0 && row0 + r < a.b) {
            if (a.mean) a.mean[row[r]] = a.rms ? 0.f : mean[r];
            if (a.rstd) a.rstd[row[r]] = rstd[r];
        }
    }
    constexpr bool ALONE = LANES == 32 && ROWS == 1;         // all of the warp has one row, the same answer with it
    if (ALONE && any) {
        norm_forward_shrunk_row<T, W, V, LANES, RAGGED>(a, row[0], row0 < a.b, at, step, shape, s_sum, s_sq);
        return;
    }
    const W *w = static_cast<const W*>(a.w), *c = static_cast<const W*>(a.c);
    if (RAGGED && extra >= 0 && row0 < a.b && (ALONE || !beyond[0]))
        static_cast<T*>(a.y)[row[0] * a.ldy + extra] =
            from_float<T>(fmaf(hx * rstd[0], w ? to_float(w[extra]) : 1.f, c ? to_float(c[extra]) : 0.f));
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int col = lead + at + p * step;
        if (at + p * step >= end) continue;
        float q[V], k[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            q[e] = 1.f;
            k[e] = 0.f;
        }
        if (w) load_row_weights<W, V, RAGGED>(w, col, a.n, q);
        if (c) load_row_weights<W, V, RAGGED>(c, col, a.n, k);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float y[V];
            if constexpr (V == 1) {
                y[0] = fmaf(h[r][p] * rstd[r], q[0], k[0]);
            } else {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float2 u = mul2(make_float2(h[r][p * V + e], h[r][p * V + e + 1]), twice(rstd[r]));
                    const float2 v = fma2(u, make_float2(q[e], q[e + 1]), make_float2(k[e], k[e + 1]));
                    y[e] = v.x; y[e + 1] = v.y;
                }
            }
            if (row0 + r < a.b && (ALONE || !beyond[r])) P::store(static_cast<T*>(a.y) + row[r] * a.ldy + col, y);
        }
    }
    if (LANES < 32) any = __any_sync(0xffffffffu, any);          // rows that share a warp go along
    if (!ALONE && any) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            norm_forward_shrunk_row<T, W, V, LANES, RAGGED>(a, row[r], beyond[r] && row0 + r < a.b, at, step, shape, s_sum, s_sq);
    }
}

struct NormBackwardArgs {
    const void *dy, *x, *w, *dh;
    const float *mean, *rstd;
    void *dx, *dw, *dc;
    float *part;            // [splits][2][pitch]: partial sums of dw and dc; the pitch is n in whole sectors
    int64_t lddy, ldx, lddh, lddx, b, rows_per_split;
    int n, pitch, splits, warps, groups, period;
    int cluster, slice;     // blocks that share a row, and the elements of it that each has
    bool rms, w_bf16, dw_bf16;
};

// V weights (1 where there are none) of either type.
template <int V, bool RAGGED>
__device__ __forceinline__ void load_any_weights(const void* w, bool is_bf16, int col, int n, float* out) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = 1.f;
    } else if (is_bf16) {
        load_row_weights<__nv_bfloat16, V, RAGGED>(static_cast<const __nv_bfloat16*>(w), col, n, out);
    } else {
        load_row_weights<float, V, RAGGED>(static_cast<const float*>(w), col, n, out);
    }
}

__device__ __forceinline__ void copy16_async(uint32_t smem, const void* p) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(p) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 load_shared16(uint32_t smem) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem) : "memory");
    return v;
}

constexpr int NB_WARPS = 8;             // of a block, but where a row has more
// Rows in shared memory: four of at most 32 bytes a thread and matrix (98 KB for three matrices and 256 threads, two blocks an
// SM), two where the rows are wider.
template <typename T, int EPT> __host__ __device__ constexpr int norm_stages() { return EPT * (int)sizeof(T) > 32 ? 2 : 4; }

// Floats between the two vectors of a block's sums in shared memory.
__host__ __device__ constexpr int norm_sums_pitch(int n) { return (n + n / 32 + 4) & ~3; }

// dx and the partial sums of dw (and, SHIFT, of dc) in one pass.  A block has `groups` groups of `warps` warps; a group takes
// row after row, so that a thread's columns stay the same and their sums stay in its registers.  The rows that follow are
// copied ahead into shared memory, STAGES - 1 of them: every thread fetches what it will read itself, so that no barrier is
// needed for it (elements, V = 1, are loaded when they are needed).  Rows whose offset into the 16-byte grid differs go to
// different blocks (`period` of them: the row distance's phase repeats after so many rows), which keeps the columns of
// a thread fixed there too.
// LANES < 32: narrow rows, several to a warp, each a group.
// CLUSTER: rows wider than a block holds, over the blocks of a cluster, which have a slice of the columns each.  Every warp sends its part of a
// row's two sums to all blocks (st.async, counted on an mbarrier; a cluster barrier a row instead waits for the stores of dx too:
// 4096 x 16384 bf16 121 us).
// SHIFT: layer norm, or a bias in the RMS form; otherwise there is neither a mean nor dc.
template <typename T, int V, int EPT, int LANES, bool SHIFT, bool RAGGED, bool CLUSTER>
__global__ void __launch_bounds__(512)
norm_backward_kernel(const __grid_constant__ NormBackwardArgs a) {
    using P = Piece<T, V>;
    constexpr int PIECES = EPT / V, STAGES = norm_stages<T, EPT>();
    __shared__ __align__(8) float2 s_part[2][NB_WARPS][16];         // of the groups' or the cluster's blocks' warps
    __shared__ uint64_t s_bar[2];
    __shared__ int s_abort;
    extern __shared__ __align__(16) unsigned char s_ring[];       // [stage][array][piece][thread] 16 bytes; in the end [2][n] sums
    grid_dependency_wait();
    grid_launch_dependents();
    const int width = LANES < 32 ? LANES : 32 * a.warps;         // threads of a group
    const int group = threadIdx.x / width, t = threadIdx.x - group * width;
    const int step = width * V, at = t * V, lane = threadIdx.x & 31, warp = t >> 5;
    const int rank = CLUSTER ? (int)ptx::cluster_ctarank() : 0;
    const unsigned unit = CLUSTER ? blockIdx.x / a.cluster : blockIdx.x, units = CLUSTER ? gridDim.x / a.cluster : gridDim.x;
    const int64_t cls = unit % a.period;
    const int64_t stride = (int64_t)a.period * a.groups * (units / a.period);
    const int64_t first = cls + a.period * ((int64_t)(unit / a.period) * a.groups);      // of the block
    const T *X = static_cast<const T*>(a.x), *DY = static_cast<const T*>(a.dy), *DH = static_cast<const T*>(a.dh);
    const RowShape shape = row_shape<T, V, RAGGED>(X + cls * a.ldx, a.n, t);
    // of a cluster's blocks each has the vectors of its slice, the first the elements before them, the last those behind
    const int lead = shape.lead + (CLUSTER ? rank * a.slice : 0);
    const int end = CLUSTER ? max(0, min(shape.whole - rank * a.slice, a.slice)) : shape.whole;
    const int extra = CLUSTER && rank != (t < 8 ? 0 : a.cluster - 1) ? -1 : shape.extra;
    const float inv_n = 1.f / (float)a.n;
    const uint32_t sent = a.cluster * a.warps * sizeof(float2);         // to a block of a cluster, for a row
    if constexpr (CLUSTER) {
        if (threadIdx.x == 0) {
            s_abort = 0;
            for (int k = 0; k < 2; ++k) {
                ptx::mbar_init(&s_bar[k], 1);
                ptx::mbar_arrive_expect_tx(&s_bar[k], sent);
            }
            ptx::fence_barrier_init();
        }
        ptx::cluster_sync_all();            // every block's barriers are there before anything is sent to them
    }
    float w[EPT], dw[EPT], dc[SHIFT ? EPT : 1];
    float wx = 0.f, dwx = 0.f, dcx = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
#pragma unroll
        for (int e = 0; e < V; ++e) w[p * V + e] = 0.f;
        if (at + p * step < end) load_any_weights<V, RAGGED>(a.w, a.w_bf16, lead + at + p * step, a.n, w + p * V);
    }
    if (RAGGED && extra >= 0) load_any_weights<1, false>(a.w, a.w_bf16, extra, a.n, &wx);
#pragma unroll
    for (int e = 0; e < EPT; ++e) dw[e] = 0.f;
#pragma unroll
    for (int e = 0; e < (SHIFT ? EPT : 1); ++e) dc[e] = 0.f;

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + threadIdx.x * 16;
    const uint32_t piece_bytes = blockDim.x * 16, array_bytes = PIECES * piece_bytes, stage_bytes = (DH ? 3 : 2) * array_bytes;
    auto fetch = [&](int64_t r, int stage) {
        if constexpr (V > 1) {
            if (r < a.b) {
                const uint32_t to = ring + stage * stage_bytes;
                const T *x = X + r * a.ldx + lead + at, *dy = DY + r * a.lddy + lead + at, *dh = DH + r * a.lddh + lead + at;
#pragma unroll
                for (int p = 0; p < PIECES; ++p) {
                    if (at + p * step < end) {
                        copy16_async(to + p * piece_bytes, x + p * step);
                        copy16_async(to + array_bytes + p * piece_bytes, dy + p * step);
                        if (DH) copy16_async(to + 2 * array_bytes + p * piece_bytes, dh + p * step);
                    }
                }
            }
            copy_commit();
        }
    };
    auto taken = [&](int stage, int array, int p) {
        typename P::Raw r = P::zero();
        if constexpr (V > 1) {
            if (at + p * step < end) {
                const uint4 v = load_shared16(ring + stage * stage_bytes + array * array_bytes + p * piece_bytes);
                r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
            }
        }
        return r;
    };
    // statistics and the element outside the vectors: one row ahead, in registers
    using One = Piece<T, 1>;
    float next_mean = 0.f, next_rstd = 0.f;
    typename One::Raw next_x = One::zero(), next_y = One::zero(), next_h = One::zero();
    auto fetch_scalars = [&](int64_t r) {
        if (r >= a.b) return;
        next_rstd = a.rstd[r];
        if (SHIFT && !a.rms) next_mean = a.mean[r];
        if (RAGGED && extra >= 0) {
            next_x = One::load(X + r * a.ldx + extra);
            next_y = One::load(DY + r * a.lddy + extra);
            if (DH) next_h = One::load(DH + r * a.lddh + extra);
        }
    };
    int64_t row = first + a.period * group;
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k) fetch(row + k * stride, k);
    fetch_scalars(row);
    int stage = 0, parity = 0, phase = 0;
    bool fine = true;
    // a group's threads go the same rounds; where a warp has several groups, all of them as many as its block's first
    for (; row - (LANES < 32 ? a.period * group : 0) < a.b; row += stride, parity ^= 1) {
        const bool mine = LANES == 32 || row < a.b;
        const float s = mine ? next_rstd : 0.f, m = mine ? next_mean : 0.f;
        float ux, yx, hx;
        One::unpack(next_x, &ux);
        One::unpack(next_y, &yx);
        One::unpack(next_h, &hx);
        float u[EPT], g[EPT];
        if constexpr (V > 1) {
            copy_wait<STAGES - 2>();
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                P::unpack(mine ? taken(stage, 0, p) : P::zero(), u + p * V);
                P::unpack(mine ? taken(stage, 1, p) : P::zero(), g + p * V);
            }
        } else {
            typename P::Raw raw[PIECES];
            load_row<T, V, PIECES>(X + row * a.ldx, at, step, end, raw);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) P::unpack(raw[p], u + p);
            load_row<T, V, PIECES>(DY + row * a.lddy, at, step, end, raw);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) P::unpack(raw[p], g + p);
        }
        // the stage that the last round read is free
        fetch(row + (STAGES - 1) * stride, stage == 0 ? STAGES - 1 : stage - 1);
        fetch_scalars(row + stride);
        float2 gu2 = twice(0.f), g2 = twice(0.f);
        const float quarter = -0.25f * m, grown = SHIFT ? 4.f * s : s;
        // what a thread holds outside the row counts for nothing, where the mean times s is infinite too
        const auto times = [&](int e) { return at + e / V * step < end ? grown : 0.f; };
#pragma unroll
        for (int e = 0; e < EPT; e += 2) {
            float2 uu = make_float2(u[e], u[e + 1]);
            const float2 dd = make_float2(g[e], g[e + 1]);
            if (SHIFT) uu = fma2(uu, twice(0.25f), twice(quarter));
            uu = mul2(uu, make_float2(times(e), times(e + 1)));
            const float2 ww = fma2(dd, uu, make_float2(dw[e], dw[e + 1]));
            dw[e] = ww.x; dw[e + 1] = ww.y;
            if (SHIFT) {
                const float2 cc = add2(dd, make_float2(dc[e], dc[e + 1]));
                dc[e] = cc.x; dc[e + 1] = cc.y;
            }
            const float2 gg = mul2(dd, make_float2(w[e], w[e + 1]));
            gu2 = fma2(gg, uu, gu2);
            if (SHIFT) g2 = add2(g2, gg);
            u[e] = uu.x; u[e + 1] = uu.y; g[e] = gg.x; g[e + 1] = gg.y;
        }
        float gu = gu2.x + gu2.y, gs = g2.x + g2.y, gx = 0.f;
        if (RAGGED && extra >= 0 && mine) {
            ux = (SHIFT ? fmaf(ux, 0.25f, quarter) : ux) * grown;
            dwx = fmaf(yx, ux, dwx);
            dcx += yx;
            gx = yx * wx;
            gu = fmaf(gx, ux, gu);
            gs += gx;
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
            gu += __shfl_xor_sync(0xffffffffu, gu, o);
            if (SHIFT) gs += __shfl_xor_sync(0xffffffffu, gs, o);
        }
        if constexpr (CLUSTER) {
            if (lane < a.cluster)
                ptx::store_async_pair(ptx::map_to_rank(&s_part[parity][rank][warp], lane), gu, gs, ptx::map_to_rank(&s_bar[parity], lane));
            fine = __all_sync(0xffffffffu, ptx::mbar_wait_cluster(&s_bar[parity], phase, &s_abort));
            if (!fine) break;
            if (threadIdx.x == 0) ptx::mbar_arrive_expect_tx(&s_bar[parity], sent);         // for the row after the next
            phase ^= parity;
            // two buffers: a warp writes one again when it has every warp's part of the row between, sent after this one was read
            float2 v = twice(0.f);
            if ((lane & 15) < a.warps)
                for (int r = 0; r < a.cluster; ++r) v = add2(v, s_part[parity][r][lane & 15]);
            gu = v.x; gs = v.y;
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) {
                gu += __shfl_xor_sync(0xffffffffu, gu, o);
                if (SHIFT) gs += __shfl_xor_sync(0xffffffffu, gs, o);
            }
        } else if (LANES == 32 && a.warps > 1) {          // at most 16; two buffers, so that one barrier a row is enough
            if (lane == 0) s_part[parity][group][warp] = make_float2(gu, gs);
            asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(32 * a.warps) : "memory");
            const float2 v = (lane & 15) < a.warps ? s_part[parity][group][lane & 15] : twice(0.f);
            gu = v.x; gs = v.y;
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) {
                gu += __shfl_xor_sync(0xffffffffu, gu, o);
                if (SHIFT) gs += __shfl_xor_sync(0xffffffffu, gs, o);
            }
        }
        const float mu = -gu * inv_n, mg = SHIFT && !a.rms ? -gs * inv_n : 0.f;
        T* dx = static_cast<T*>(a.dx) + row * a.lddx;
        typename P::Raw hr[PIECES];
        if constexpr (V == 1) {
            if (DH) load_row<T, V, PIECES>(DH + row * a.lddh, at, step, end, hr);
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (at + p * step >= end || !mine) continue;
            float q[V], hv[V];
#pragma unroll
            for (int e = 0; e < V; ++e) hv[e] = 0.f;
            if (DH) {
                if constexpr (V > 1) P::unpack(taken(stage, 2, p), hv);
                else P::unpack(hr[p], hv);
            }
            if constexpr (V == 1) {
                q[0] = fmaf(fmaf(u[p], mu, g[p] + mg), s, hv[0]);
            } else {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const int j = p * V + e;
                    float2 gg = make_float2(g[j], g[j + 1]);
                    if (SHIFT) gg = add2(gg, twice(mg));
                    const float2 d = fma2(fma2(make_float2(u[j], u[j + 1]), twice(mu), gg), twice(s), make_float2(hv[e], hv[e + 1]));
                    q[e] = d.x; q[e + 1] = d.y;
                }
            }
            P::store(dx + lead + at + p * step, q);
        }
        if (RAGGED && extra >= 0 && mine) dx[extra] = from_float<T>(fmaf(fmaf(ux, mu, gx + mg), s, hx));
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    if constexpr (CLUSTER) {
        copy_wait<0>();
        ptx::cluster_sync_all();            // nothing is sent to a block that has left
        if (!fine && lane == 0) raise_status(DEV_TIMEOUT);
    }
    if (!a.part) return;
    if (LANES < 32) {           // a warp's groups have the same columns
#pragma unroll
        for (int o = LANES; o < 32; o *= 2) {
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                dw[e] += __shfl_xor_sync(0xffffffffu, dw[e], o);
                if (SHIFT) dc[e] += __shfl_xor_sync(0xffffffffu, dc[e], o);
            }
            dwx += __shfl_xor_sync(0xffffffffu, dwx, o);
            dcx += __shfl_xor_sync(0xffffffffu, dcx, o);
        }
    }
    // the groups' sums one after the other, in the place of the ring, whose last copies (of no row) are through; from there they
    // go out in whole sectors
    float* cols = reinterpret_cast<float*>(s_ring);
    // the block's columns: all of them, or from its slice's first (and the row's first) to the next slice's (and the row's last)
    const int from = CLUSTER && rank > 0 ? lead : 0, behind = CLUSTER && rank < a.cluster - 1 ? lead + a.slice : a.n;
    // by vectors where the row's offset allows it; else element by element, with a gap every 32 so that lanes hit different banks
    const bool vec = V % 4 == 0 && (lead - from) % 4 == 0;
    const auto place = [vec](int col) { return vec ? col : col + (col >> 5); };
    float* cols_c = cols + norm_sums_pitch(CLUSTER ? a.slice + 16 : a.n);
    copy_wait<0>();
    __syncthreads();
    const auto put = [&](float* to, int col, const float* x, bool add) {
        if (V % 4 == 0 && vec) {
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                float4* q = reinterpret_cast<float4*>(to + col + e);
                const float4 old = add ? *q : make_float4(0.f, 0.f, 0.f, 0.f);
                *q = make_float4(old.x + x[e], old.y + x[e + 1], old.z + x[e + 2], old.w + x[e + 3]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float* q = to + place(col + e);
                *q = (add ? *q : 0.f) + x[e];
            }
        }
    };
    const int parts = LANES < 32 ? (int)blockDim.x / 32 : a.groups, mine_of = LANES == 32 ? group : lane < LANES ? (int)threadIdx.x / 32 : -1;
    for (int k = 0; k < parts; ++k) {
        if (k == mine_of) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int col = lead - from + at + p * step;
                if (at + p * step >= end) continue;
                put(cols, col, dw + p * V, k > 0);
                if (SHIFT) put(cols_c, col, dc + p * V, k > 0);
            }
            if (RAGGED && extra >= 0) {
                const int q = place(extra - from);
                cols[q] = dwx + (k ? cols[q] : 0.f);
                if (SHIFT) cols_c[q] = dcx + (k ? cols_c[q] : 0.f);
            }
        }
        __syncthreads();
    }
    float* part = a.part + (int64_t)unit * 2 * a.pitch + from;
    for (int i = threadIdx.x; i < behind - from; i += blockDim.x) {
        part[i] = cols[place(i)];
        if (SHIFT) part[a.pitch + i] = cols_c[place(i)];
    }
}

constexpr int NB_WIDE_THREADS = 512;

// Matrices whose rows are aligned differently, in rows too wide for a block's registers: three launches, element by element.
// One row per block, read twice (the second time from the caches): the two sums, then dx.
template <typename T>
__global__ void __launch_bounds__(NB_WIDE_THREADS)
norm_backward_row_kernel(const __grid_constant__ NormBackwardArgs a) {
    __shared__ float s_sums[2][32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float quarter = a.rms ? 0.f : -0.25f * a.mean[row], rstd = a.rstd[row];
    const auto unit = [&](int col) { return fmaf(to_float(x[col]), 0.25f, quarter) * (4.f * rstd); };
    float sums[2] = {0.f, 0.f};
    for (int col = threadIdx.x; col < a.n; col += NB_WIDE_THREADS) {
        float w;
        load_any_weights<1, false>(a.w, a.w_bf16, col, a.n, &w);
        const float g = to_float(dy[col]) * w;
        sums[0] = fmaf(g, unit(col), sums[0]);
        sums[1] += g;
    }
    row_sums<32>(sums, s_sums, NB_WIDE_THREADS / 32);
    const float gu = sums[0] / (float)a.n, g = a.rms ? 0.f : sums[1] / (float)a.n;
    T* dx = static_cast<T*>(a.dx) + row * a.lddx;
    const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.lddh : nullptr;
    for (int col = threadIdx.x; col < a.n; col += NB_WIDE_THREADS) {
        float w;
        load_any_weights<1, false>(a.w, a.w_bf16, col, a.n, &w);
        const float d = to_float(dy[col]) * w - g - unit(col) * gu;
        dx[col] = from_float<T>(fmaf(rstd, d, dh ? to_float(dh[col]) : 0.f));
    }
}

// Column sums over a range of rows: thread = one column, block.y = one range.
constexpr int NB_COL_THREADS = 128;
template <typename T>
__global__ void __launch_bounds__(NB_COL_THREADS)
norm_backward_columns_kernel(const __grid_constant__ NormBackwardArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int col = blockIdx.x * NB_COL_THREADS + threadIdx.x;
    if (col >= a.n) return;
    const int64_t begin = (int64_t)blockIdx.y * a.rows_per_split;
    const int64_t end = begin + a.rows_per_split < a.b ? begin + a.rows_per_split : a.b;
    float dw = 0.f, dc = 0.f;
    for (int64_t row = begin; row < end; ++row) {
        const float d = to_float(static_cast<const T*>(a.dy)[row * a.lddy + col]);
        const float quarter = a.rms ? 0.f : -0.25f * a.mean[row];
        const float u = fmaf(to_float(static_cast<const T*>(a.x)[row * a.ldx + col]), 0.25f, quarter) * (4.f * a.rstd[row]);
        dw = fmaf(d, u, dw);
        dc += d;
    }
    float* part = a.part + (int64_t)blockIdx.y * 2 * a.pitch + col;
    part[0] = dw;
    part[a.pitch] = dc;
}

// The partial sums of all ranges, added in a fixed order: COLS columns (whole sectors) a block, whose other threads are strands of the ranges.
constexpr int NB_FINISH_THREADS = 512;
template <int COLS>
__global__ void __launch_bounds__(NB_FINISH_THREADS)
norm_backward_finish_kernel(const __grid_constant__ NormBackwardArgs a) {
    constexpr int STRANDS = NB_FINISH_THREADS / COLS, WARPS = NB_FINISH_THREADS / 32;
    __shared__ float2 s_part[WARPS][COLS];
    grid_dependency_wait();
    grid_launch_dependents();
    const int c = threadIdx.x % COLS, strand = threadIdx.x / COLS, col = blockIdx.x * COLS + c;
    float dw = 0.f, dc = 0.f;
    if (col < a.n) {
#pragma unroll 4
        for (int s = strand; s < a.splits; s += STRANDS) {
            const float* part = a.part + (int64_t)s * 2 * a.pitch + col;
            dw += part[0];
            if (a.dc) dc += part[a.pitch];
        }
    }
#pragma unroll
    for (int o = COLS; o < 32; o *= 2) {          // the strands of a warp
        dw += __shfl_xor_sync(0xffffffffu, dw, o);
        dc += __shfl_xor_sync(0xffffffffu, dc, o);
    }
    if ((threadIdx.x & 31) < COLS) s_part[threadIdx.x >> 5][c] = make_float2(dw, dc);
    __syncthreads();
    if (threadIdx.x >= COLS || col >= a.n) return;
    dw = dc = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        dw += s_part[w][c].x;
        dc += s_part[w][c].y;
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
