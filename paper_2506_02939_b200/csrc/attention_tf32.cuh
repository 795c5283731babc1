// Attention in fp32 on the tensor cores' tf32 products: heads of up to 128, rows of whole 16-byte vectors.  Every factor is a sum of two
// numbers of 11 bits, x = h + l with |x - h - l| <= 2^-23 |x|, and a product x y is h h' + h l' + l h' (what is left out is at most
// 2^-22 |x y|), so sums come out as fp32 sums do; a product takes three of the tensor cores'.
//
// One warp owns 16 rows and goes over tiles of 64 streamed rows (mma.sync, 16 x 8 x 8: tiles of 128 rows for tcgen05 would leave most SMs
// without work in the batches that are computed in fp32).  Scores stay in registers from product to product: as the accumulators of
// one they are the first operand of the next.  That, and vector loads without bank conflicts (rows DP + 4 words apart), need an order of
// rows and columns of our own, which sums do not notice:
//   within 16 columns along the head, lane q = lane % 4 has the four neighbours 4 q ..: two steps of 8;
//   row m of an operand's 16 is tf_row(m % 8) + m / 8, and streamed row n of tile j of 8 is 16 (j / 2) + tf_row(n) + j % 2.
// 8 x 256 causal tokens of 8 heads of 64: bound by the products (8.7 clocks each, three a term) and by their operands' splitting.
#pragma once
#include "attention.cuh"

namespace pamm {

constexpr int TF_ROWS = 32, TF_THREADS = 64;           // two warps

__device__ __forceinline__ int tf_row(int n) { return n & 1 ? 8 + ((n - 1) ^ 4) : n; }
// The first number is x rounded to 11 bits (NaN and infinities as they are), the second what is left (nothing of an infinity); the products
// drop what is behind the second's 11 bits, so that half a step is added to it.
__device__ __forceinline__ void tf_split(float x, uint32_t& high, uint32_t& low) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(high) : "f"(x));
    const float h = __uint_as_float(high);
    low = h == x ? 0u : __float_as_uint(x - h) + 0x1000u;
}
__device__ __forceinline__ void tf_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d += a b of split operands
__device__ __forceinline__ void tf_mma3(float (&d)[4], const uint32_t (&ah)[4], const uint32_t (&al)[4], const uint32_t (&bh)[2], const uint32_t (&bl)[2]) {
    tf_mma(d, al, bh[0], bh[1]);
    tf_mma(d, ah, bl[0], bl[1]);
    tf_mma(d, ah, bh[0], bh[1]);
}
// c[j]: the warp's 16 rows of A (from `row` on) times the 64 rows of B, over d columns (rounded up to 16; tiles are zero behind d).
template <int DP>
__device__ __forceinline__ void tf_scores(const float* A, const float* B, int row, int d, float (&c)[8][4]) {
    constexpr int LD = DP + 4;
    const int g = (threadIdx.x & 31) >> 2, q = threadIdx.x & 3, rb = tf_row(g);
    const float *a = A + (row + rb) * LD + 4 * q, *b = B + rb * LD + 4 * q;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[j][e] = 0.f;
#pragma unroll 1
    for (int k = 0; k < d; k += 16) {
        const float4 x = *reinterpret_cast<const float4*>(a + k), y = *reinterpret_cast<const float4*>(a + LD + k);
        uint32_t h[2][4], l[2][4];
        tf_split(x.x, h[0][0], l[0][0]); tf_split(y.x, h[0][1], l[0][1]); tf_split(x.y, h[0][2], l[0][2]); tf_split(y.y, h[0][3], l[0][3]);
        tf_split(x.z, h[1][0], l[1][0]); tf_split(y.z, h[1][1], l[1][1]); tf_split(x.w, h[1][2], l[1][2]); tf_split(y.w, h[1][3], l[1][3]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float4 z = *reinterpret_cast<const float4*>(b + (16 * (j >> 1) + (j & 1)) * LD + k);
            uint32_t u[2], v[2];
            tf_split(z.x, u[0], v[0]); tf_split(z.y, u[1], v[1]);
            tf_mma3(c[j], h[0], l[0], u, v);
            tf_split(z.z, u[0], v[0]); tf_split(z.w, u[1], v[1]);
            tf_mma3(c[j], h[1], l[1], u, v);
        }
    }
}
// acc += P B: P as tf_scores leaves scores, B its 64 streamed rows.  acc[4 b + t][.]: a lane's columns 32 b + 8 q + t (entries 0 and 2) and
// + 4 (1 and 3), of its rows tf_row(g) (0 and 1) and the next.
template <int DP>
__device__ __forceinline__ void tf_accumulate(const float (&p)[8][4], const float* B, int d, float (&acc)[DP / 8][4]) {
    constexpr int LD = DP + 4;
    const int g = (threadIdx.x & 31) >> 2, q = threadIdx.x & 3;
    const float *b0 = B + 2 * q * LD + 4 * g, *b1 = B + (8 + ((2 * q) ^ 4)) * LD + 4 * g;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t h[4], l[4];
        tf_split(p[j][0], h[0], l[0]); tf_split(p[j][2], h[1], l[1]); tf_split(p[j][1], h[2], l[2]); tf_split(p[j][3], h[3], l[3]);
        const int row = (16 * (j >> 1) + (j & 1)) * LD;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b) {
            if (32 * b >= d) break;
            const float4 x = *reinterpret_cast<const float4*>(b0 + row + 32 * b), y = *reinterpret_cast<const float4*>(b1 + row + 32 * b);
            const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t u[2], v[2];
                tf_split(xs[t], u[0], v[0]);
                tf_split(ys[t], u[1], v[1]);
                tf_mma3(acc[4 * b + t], h, l, u, v);
            }
        }
    }
}
// Where a lane's entry e of score tile j stands: row (within the warp's 16) and streamed row.
__device__ __forceinline__ int tf_own(int e) { return tf_row((threadIdx.x & 31) >> 2) + (e >> 1); }
__device__ __forceinline__ int tf_streamed(int j, int e) {
    const int q = threadIdx.x & 3;
    return 16 * (j >> 1) + (j & 1) + (e & 1 ? 8 + ((2 * q) ^ 4) : 2 * q);
}
// The warp's rows times `factor` (of the lane's two rows), zero from the sequence's end on.
template <int DP>
__device__ __forceinline__ void tf_store(const HeadsView& y, const Tile& t, int64_t head, int d, int row, const float (&acc)[DP / 8][4], const float (&factor)[2]) {
    const int q = threadIdx.x & 3;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int at = t.at + row + tf_own(2 * r);
        if (at >= t.rows) continue;
        float* p = y.at<float>(t.b, t.first + at, head);
        const float f = at < t.len ? factor[r] : 0.f;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int col = 32 * b + 8 * q + 4 * s;
                float4 v = make_float4(acc[4 * b][2 * r + s] * f, acc[4 * b + 1][2 * r + s] * f, acc[4 * b + 2][2 * r + s] * f, acc[4 * b + 3][2 * r + s] * f);
                if (at >= t.len) v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (col < d) *reinterpret_cast<float4*>(p + col) = v;
            }
    }
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

// Owned tiles (Q, or two), the two streamed ones, and two numbers a streamed row.
template <int DP, bool BACK>
constexpr size_t tf_smem = (size_t)(((BACK ? 2 : 1) * TF_ROWS + 2 * AG_TILE) * (DP + 4) + (BACK ? 2 * AG_TILE : 0)) * 4;

template <int DP>
__global__ void __launch_bounds__(TF_THREADS, DP <= 64 ? 5 : 2)
attention_forward_tf32_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionOrder order) {
    extern __shared__ __align__(16) float ag_shared[];
    float *Q = ag_shared, *K = Q + TF_ROWS * (DP + 4), *V = K + AG_TILE * (DP + 4);
    grid_dependency_wait();
    grid_launch_dependents();
    int h, item;
    order.at((int)blockIdx.x, item, h);
    const Tile t = find_tile<TF_ROWS>(a.s, item);
    if (!t.any) return;
    const int row = (threadIdx.x >> 5) * 16;
    const float c = a.scale * LOG2E;
    float acc[DP / 8][4], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
    const int end = t.at < t.len ? (a.causal ? min(t.len, t.at + TF_ROWS) : t.len) : 0;
    const auto load = [&](float* to, const HeadsView& x, int k0) { ag_load<float, DP, AG_TILE, TF_THREADS>(to, x, t, h / a.group, k0, t.len, a.d, true); };
    if (end > 0) {
        ag_load<float, DP, TF_ROWS, TF_THREADS>(Q, a.q, t, h, t.at, t.len, a.d, true);
        load(K, a.k, 0);
        load(V, a.v, 0);
    }
    for (int k0 = 0; k0 < end; k0 += AG_TILE) {
        const bool more = k0 + AG_TILE < end;
        ag_wait<1>();
        __syncthreads();
        float s[8][4];
        tf_scores<DP>(Q, K, row, a.d, s);
        __syncthreads();
        if (more) load(K, a.k, k0 + AG_TILE);
        else ag_commit();                                       // as many groups, so that V's is the last but one
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int me = t.at + row + tf_own(2 * r), last = (a.causal ? min(me, t.len - 1) : t.len - 1) - k0;
            float m = top[r];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    s[j][e] = tf_streamed(j, e) <= last ? s[j][e] : -INFINITY;
                    m = fmaxf(m, s[j][e]);
                }
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const float mc = m == -INFINITY ? 0.f : m * c;                   // a row that sees no finite score so far
            const float keep = exp2f(fmaf(top[r], c, -mc));
            sum[r] *= keep;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
                acc[i][2 * r] *= keep;
                acc[i][2 * r + 1] *= keep;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    s[j][e] = exp2f(fmaf(s[j][e], c, -mc));
                    sum[r] += s[j][e];
                }
            top[r] = m;
        }
        ag_wait<1>();
        __syncthreads();
        tf_accumulate<DP>(s, V, a.d, acc);
        if (more) {
            __syncthreads();
            load(V, a.v, k0 + AG_TILE);
        }
    }
    float factor[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const float l = quad_sum(sum[r]);
        const int me = t.at + row + tf_own(2 * r);
        factor[r] = 1.f / l;
        if ((threadIdx.x & 3) == 0 && me < t.rows && a.lse)
            a.lse[a.row_number(t, h) + me] = me < t.len ? fmaf(top[r], a.scale, logf(l)) : -INFINITY;
    }
    tf_store<DP>(a.o, t, h, a.d, row, acc, factor);
}

// As the backward kernel for every order of memory.
template <int DP, bool KEYS>
__global__ void __launch_bounds__(TF_THREADS, DP <= 64 ? 4 : 2)
attention_backward_tf32_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionOrder order) {
    constexpr int OWNED = TF_ROWS * (DP + 4), TILE = AG_TILE * (DP + 4);
    extern __shared__ __align__(16) float ag_shared[];
    float *A0 = ag_shared, *A1 = A0 + OWNED, *X0 = A1 + OWNED, *X1 = X0 + TILE, *lse = X1 + TILE, *delta = lse + AG_TILE;
    grid_dependency_wait();
    grid_launch_dependents();
    int owner, item;                                          // query head or key head
    order.at((int)blockIdx.x, item, owner);
    const Tile t = find_tile<TF_ROWS>(a.s, item);
    if (!t.any) return;
    const int row = (threadIdx.x >> 5) * 16, q = threadIdx.x & 3;
    const float c = a.scale * LOG2E;
    float acc0[DP / 8][4], acc1[KEYS ? DP / 8 : 1][4], row_lse[2] = {0.f, 0.f}, row_delta[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < DP / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            acc0[i][e] = 0.f;
            if (KEYS) acc1[KEYS ? i : 0][e] = 0.f;
        }
    // step i of n: tile i % per of the streamed rows, of head i / per of those that share the keys
    const int begin = KEYS && a.causal ? t.at : 0;
    const int end = t.at >= t.len ? begin : !KEYS && a.causal ? min(t.len, t.at + TF_ROWS) : t.len;
    const int per = (end - begin + AG_TILE - 1) / AG_TILE, n = per * (KEYS ? a.group : 1);
    const auto head_of = [&](int i) { return KEYS ? owner * a.group + i / per : owner / a.group; };
    const auto at_of = [&](int i) { return begin + i % per * AG_TILE; };
    const auto load0 = [&](int i) { ag_load<float, DP, AG_TILE, TF_THREADS>(X0, KEYS ? a.q : a.k, t, head_of(i), at_of(i), t.len, a.d, true); };
    const auto load1 = [&](int i) { ag_load<float, DP, AG_TILE, TF_THREADS>(X1, KEYS ? a.d_o : a.v, t, head_of(i), at_of(i), t.len, a.d, true); };
    float next_lse = 0.f, next_delta = 0.f;                   // of the next step's streamed rows, on their way
    const auto numbers = [&](int i) {
        if (!KEYS) return;
        const int at = at_of(i) + (int)threadIdx.x;
        const int64_t number = a.row_number(t, head_of(i)) + at;
        next_lse = at < t.len ? a.lse_in[number] * LOG2E : 0.f;
        next_delta = at < t.len ? a.delta[number] : 0.f;
    };
    static_assert(TF_THREADS == AG_TILE, "a thread a streamed row");
    if (n > 0) {
        ag_load<float, DP, TF_ROWS, TF_THREADS>(A0, KEYS ? a.k : a.q, t, owner, t.at, t.len, a.d, true);
        ag_load<float, DP, TF_ROWS, TF_THREADS>(A1, KEYS ? a.v : a.d_o, t, owner, t.at, t.len, a.d, true);
        numbers(0);
        load0(0);
        load1(0);
    }
    if (!KEYS) {
        const int64_t number = a.row_number(t, owner);
        ag_wait<2>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int own = row + tf_own(2 * r), me = t.at + own;
            float sum = 0.f;
            if (me < t.len) {
                const float* o = a.o.at<float>(t.b, t.first + me, owner);
                for (int e = 4 * q; e < a.d; e += 16) {
                    const float4 x = *reinterpret_cast<const float4*>(o + e), y = *reinterpret_cast<const float4*>(A1 + own * (DP + 4) + e);
                    sum = fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, sum))));
                }
                row_lse[r] = a.lse_in[number + me] * LOG2E;
            }
            row_delta[r] = quad_sum(sum);
            if (q == 0 && me < t.rows) a.delta[number + me] = row_delta[r];
        }
    }
    for (int i = 0; i < n; ++i) {
        const bool more = i + 1 < n;
        const int x0 = at_of(i);
        if (KEYS) {
            lse[threadIdx.x] = next_lse;
            delta[threadIdx.x] = next_delta;
        }
        ag_wait<1>();
        __syncthreads();
        if (more) numbers(i + 1);
        float p[8][4], dp[8][4];
        tf_scores<DP>(A0, X0, row, a.d, p);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int own = t.at + row + tf_own(e), col = tf_streamed(j, e), other = x0 + col;
                const bool sees = other < t.len && (!a.causal || (KEYS ? other >= own : other <= own));
                p[j][e] = sees ? exp2f(fmaf(p[j][e], c, -(KEYS ? lse[col] : row_lse[e >> 1]))) : 0.f;
            }
        ag_wait<0>();
        __syncthreads();
        tf_scores<DP>(A1, X1, row, a.d, dp);
        if constexpr (KEYS) tf_accumulate<DP>(p, X1, a.d, acc1);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)      // a masked place stays 0 whatever dp is there
                p[j][e] = p[j][e] == 0.f ? 0.f : p[j][e] * (dp[j][e] - (KEYS ? delta[tf_streamed(j, e)] : row_delta[e >> 1]));
        tf_accumulate<DP>(p, X0, a.d, acc0);
        if (more) {
            __syncthreads();
            load0(i + 1);
            load1(i + 1);
        }
    }
    const float factor[2] = {a.scale, a.scale}, one[2] = {1.f, 1.f};
    tf_store<DP>(KEYS ? a.dk : a.dq, t, owner, a.d, row, acc0, factor);
    if constexpr (KEYS) tf_store<DP>(a.dv, t, owner, a.d, row, acc1, one);
}

}  // namespace pamm
