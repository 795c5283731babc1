// Rotary positions on the heads of a row: pair i of a head at position p is turned by the angle p f_i,
//   (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin),
// with the pairs (i, i + rot/2) or (2i, 2i + 1) of the head's first `rot` elements.  The transposed
// turn (sin -> -sin) is the backward pass: the rotation is linear, and orthogonal up to the amplitude.
// cos and sin come from a table in fp32, one row [cos f_0 .. | sin f_0 ..] per position, computed in
// 64 bits: p f_i in fp32 alone would be off by 0.01 radian at position 130,000.
//
// The operator is a copy with six operations a pair; bound by memory.  The table of the positions in
// use stays in L2 (4 rot bytes a position), and a row's heads share its table row through L1.
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"

namespace pamm {

constexpr int ROTARY_MAX_ROT = 512;
constexpr int64_t ROTARY_MAX_ROW = 1 << 24;       // heads times head_dim
constexpr int ROTARY_THREADS = 256;

// Division of 0 <= n < 2^31 by a fixed 1 <= d < 2^31 as a product with a rounded-up reciprocal: Granlund and Montgomery, Division by
// Invariant Integers using Multiplication (PLDI 1994), theorem 4.2 for N = 31.  With l = ceil(log2 d) and m = ceil(2^(31 + l) / d), which
// fits 32 bits, n / d = n m >> (31 + l); of 2 n, which fits as well, the product's upper half has 32 of those places off.
struct Divisor {
    uint32_t d, reciprocal, shift;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return __umulhi(2 * n, reciprocal) >> shift; }
};
inline Divisor make_divisor(uint32_t d) {
    uint32_t log = 0;
    while ((uint64_t)d > (1ull << log)) ++log;
    const uint64_t dividend = 1ull << (31 + log);
    return {d, (uint32_t)((dividend + d - 1) / d), log};
}

struct RotaryArgs {
    const void* x;
    void* y;
    const float* table;
    const void* positions;      // null: first + token
    int64_t xb, xs, xh, yb, ys, yh, pb, ps, table_rows, first;
    int64_t tokens;             // of all sequences
    Divisor seq, units, per_turned, per_whole;      // tokens of a sequence; units of a token, of a turned head and of one that passes
    int tokens_per_block, turned_units, turns, rot;
    int heads, rotated, turned_step, whole_step;    // distances between the heads that a thread takes
    bool transposed, pos64;
};

// One pair.  The products' order is written out, so that every access width gives the same bits.
__device__ __forceinline__ void turn_pair(float& x1, float& x2, float c, float s) {
    const float y1 = fmaf(x1, c, -__fmul_rn(x2, s));
    x2 = fmaf(x2, c, __fmul_rn(x1, s));
    x1 = y1;
}

template <int N>
__device__ __forceinline__ void load_table(const float* p, float (&out)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 t = __ldg(reinterpret_cast<const float4*>(p + i));
            out[i] = t.x; out[i + 1] = t.y; out[i + 2] = t.z; out[i + 3] = t.w;
        }
    } else if constexpr (N == 2) {
        const float2 t = __ldg(reinterpret_cast<const float2*>(p));
        out[0] = t.x; out[1] = t.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = __ldg(p + i);
    }
}

// A unit is what a thread turns of one head: V pairs of a half-split head (two vectors), or the V / 2 pairs of one vector of
// adjacent ones; V = 1: one pair, element by element.  What passes through is copied in units of V elements; a call in place has
// no such units.  A thread takes the same unit of HEADS heads, which share its index arithmetic, position and table entries;
// a block takes a few tokens, or, along y and z, a part of one.
// Measured on 65536 tokens of 32 heads of 128 bf16 in a row of 48 (537 MB read, as much written), halves: 202 us with a
// unit a thread and table entries one by one, 170 us with an index division less costly, 160 us (6.7 TB/s) with four heads a
// thread; adjacent pairs 269, 198 and 160 us with eight heads.
template <typename T, int V, bool ADJACENT, int HEADS>
__global__ void __launch_bounds__(256)
rotary_kernel(const __grid_constant__ RotaryArgs a) {
    using P = Piece<T, V>;
    constexpr int PAIRS = ADJACENT ? (V == 1 ? 1 : V / 2) : V;      // of a unit
    constexpr bool TWO = !ADJACENT || V == 1;                       // pieces of a turned unit
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t token0 = (int64_t)blockIdx.x * a.tokens_per_block;
    const uint32_t here = (uint32_t)(a.tokens - token0 < a.tokens_per_block ? a.tokens - token0 : a.tokens_per_block) * a.units.d;
    const uint32_t i = threadIdx.x + (blockIdx.z * gridDim.y + blockIdx.y) * blockDim.x;
    if (i >= here) return;
    const uint32_t local = a.units(i), u = i - local * a.units.d;
    const uint32_t token = (uint32_t)token0 + local, b = a.seq(token), s = token - b * a.seq.d;
    const bool in_turned = u < (uint32_t)a.turned_units;
    const uint32_t v = in_turned ? u : u - a.turned_units;
    const uint32_t slot = in_turned ? a.per_turned(v) : a.per_whole(v);
    const int k = (int)(v - slot * (in_turned ? a.per_turned.d : a.per_whole.d));
    const bool turned = in_turned && k < a.turns;
    const int col = turned ? k * (ADJACENT ? 2 * PAIRS : V) : in_turned ? a.rot + (k - a.turns) * V : k * V;
    int head = in_turned ? (int)slot : a.rotated + (int)slot;
    const int last = in_turned ? a.rotated : a.heads, step = in_turned ? a.turned_step : a.whole_step;
    const int half = a.rot / 2, second = ADJACENT ? 1 : half;       // distance of a turned unit's second piece
    const T* x = static_cast<const T*>(a.x) + (b * a.xb + s * a.xs + col);
    T* y = static_cast<T*>(a.y) + (b * a.yb + s * a.ys + col);
    typename P::Raw r1[HEADS], r2[HEADS];
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        if (head + j * step < last) {
            const T* p = x + (head + j * step) * a.xh;
            r1[j] = P::load(p);
            if (TWO && turned) r2[j] = P::load(p + second);
        }
    }
    float c[PAIRS], sn[PAIRS];
    bool known = false;
    if (turned) {
        int64_t pos = a.first + s;
        if (a.positions) {
            const int64_t at = b * a.pb + s * a.ps;
            pos = a.pos64 ? static_cast<const int64_t*>(a.positions)[at] : (int64_t)static_cast<const int32_t*>(a.positions)[at];
        }
        known = pos >= 0 && pos < a.table_rows;
        if (known) {
            const float* row = a.table + pos * a.rot + k * PAIRS;
            load_table(row, c);
            load_table(row + half, sn);
            if (a.transposed) {
#pragma unroll
                for (int e = 0; e < PAIRS; ++e) sn[e] = -sn[e];
            }
        } else if (u == 0) {
            raise_status(DEV_BAD_INDEX);
        }
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
        if (head + j * step >= last) continue;
        T* q = y + (head + j * step) * a.yh;
        float f[TWO ? 2 * V : V];
        P::unpack(r1[j], f);
        if (TWO && turned) P::unpack(r2[j], f + V);
        if (known) {
#pragma unroll
            for (int e = 0; e < PAIRS; ++e) {
                if constexpr (TWO) turn_pair(f[e], f[V + e], c[e], sn[e]);
                else turn_pair(f[2 * e], f[2 * e + 1], c[e], sn[e]);
            }
        }
        P::store(q, f);
        if (TWO && turned) P::store(q + second, f + V);
    }
}

struct RotaryFrequencies { double f[ROTARY_MAX_ROT / 2]; };

// Angles, cosines and sines in 64 bits, rounded once.
__global__ void __launch_bounds__(ROTARY_THREADS)
rotary_table_kernel(const RotaryFrequencies freq, int half, double amplitude, int64_t first, int64_t length, float* table) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t total = length * half;
    for (int64_t k = (int64_t)blockIdx.x * ROTARY_THREADS + threadIdx.x; k < total; k += (int64_t)gridDim.x * ROTARY_THREADS) {
        const int64_t p = k / half;
        const int i = (int)(k - p * half);
        double s, c;
        sincos((double)(first + p) * freq.f[i], &s, &c);
        table[p * 2 * half + i] = (float)(amplitude * c);
        table[p * 2 * half + half + i] = (float)(amplitude * s);
    }
}

}  // namespace pamm
