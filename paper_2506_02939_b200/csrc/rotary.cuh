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
constexpr int ROTARY_THREADS = 256;

struct RotaryArgs {
    const void* x;
    void* y;
    const float* table;
    const void* positions;      // null: first + token
    int64_t xb, xs, xh, yb, ys, yh, pb, ps, table_rows, first;
    int seq, heads, rotated, head_dim, rot;
    bool adjacent, transposed, pos64, in_place;
};

template <typename T, int V>
__device__ __forceinline__ void load_unit(const T* p, float* out) {
    Piece<T, V>::unpack(Piece<T, V>::load(p), out);
}

// One pair.  The products' order is written out, so that every access width gives the same bits.
__device__ __forceinline__ void turn_pair(float& x1, float& x2, float c, float s) {
    const float y1 = fmaf(x1, c, -__fmul_rn(x2, s));
    x2 = fmaf(x2, c, __fmul_rn(x1, s));
    x1 = y1;
}

// One block per token.  A unit is V pairs of a half-split head, or V consecutive elements (V / 2 pairs of
// adjacent ones; the part of a head or the heads that are not turned).  V = 1: a unit is one pair or one element.
template <typename T, int V>
__global__ void __launch_bounds__(ROTARY_THREADS)
rotary_kernel(const RotaryArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t token = blockIdx.x;
    const int64_t b = token / a.seq, s = token % a.seq;
    int64_t pos = a.first + s;
    if (a.positions) {
        const int64_t at = b * a.pb + s * a.ps;
        pos = a.pos64 ? static_cast<const int64_t*>(a.positions)[at] : (int64_t)static_cast<const int32_t*>(a.positions)[at];
    }
    const bool known = pos >= 0 && pos < a.table_rows;
    if (!known && threadIdx.x == 0) raise_status(DEV_BAD_INDEX);
    const T* x = static_cast<const T*>(a.x) + b * a.xb + s * a.xs;
    T* y = static_cast<T*>(a.y) + b * a.yb + s * a.ys;
    const int half = a.rot / 2;
    const float* cs = a.table + (known ? pos : 0) * a.rot;
    const int per_turn = a.adjacent ? (V == 1 ? 2 : V) : 2 * V;      // elements of a turned unit
    const int turns = a.rot / per_turn;                              // turned units of a head
    const int rest = (a.head_dim - a.rot) / V, whole = a.head_dim / V;
    // units of the turned heads first, then those of the heads that pass through
    const int units_t = a.rotated * (turns + (a.in_place ? 0 : rest));
    const int units = units_t + (a.in_place ? 0 : (a.heads - a.rotated) * whole);
    for (int u = threadIdx.x; u < units; u += ROTARY_THREADS) {
        int head, col;
        bool turn = false;
        if (u < units_t) {
            const int per = turns + (a.in_place ? 0 : rest);
            head = u / per;
            const int k = u - head * per;
            turn = k < turns;
            col = turn ? k : a.rot + (k - turns) * V;
        } else {
            const int k = u - units_t;
            head = k / whole;
            col = (k - head * whole) * V;
            head += a.rotated;
        }
        const T* xr = x + (int64_t)head * a.xh;
        T* yr = y + (int64_t)head * a.yh;
        if (!turn) {
            float v[V];
            load_unit<T, V>(xr + col, v);
            Piece<T, V>::store(yr + col, v);
            continue;
        }
        if (a.adjacent) {
            constexpr int E = V == 1 ? 2 : V;
            float v[E];
            if constexpr (V == 1) {
                v[0] = to_float(xr[2 * col]);
                v[1] = to_float(xr[2 * col + 1]);
            } else {
                load_unit<T, V>(xr + col * V, v);
            }
            if (known) {
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const int i = col * (E / 2) + e / 2;
                    const float c = cs[i], sn = a.transposed ? -cs[half + i] : cs[half + i];
                    turn_pair(v[e], v[e + 1], c, sn);
                }
            }
            if constexpr (V == 1) {
                yr[2 * col] = from_float<T>(v[0]);
                yr[2 * col + 1] = from_float<T>(v[1]);
            } else {
                Piece<T, V>::store(yr + col * V, v);
            }
        } else {
            float v1[V], v2[V];
            load_unit<T, V>(xr + col * V, v1);
            load_unit<T, V>(xr + half + col * V, v2);
            if (known) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int i = col * V + e;
                    const float c = cs[i], sn = a.transposed ? -cs[half + i] : cs[half + i];
                    turn_pair(v1[e], v2[e], c, sn);
                }
            }
            Piece<T, V>::store(yr + col * V, v1);
            Piece<T, V>::store(yr + half + col * V, v2);
        }
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
