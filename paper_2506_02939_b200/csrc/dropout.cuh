// Dropout with a residual, y = r + (kept ? x / (1 - p) : 0), whose mask comes from a counter-based generator and is never
// stored: the backward pass makes it again.  Element e (in the rows' order) has word e % 4 of block
// (e / 4, offset) of Philox 4x32 with ten rounds under the key `seed` (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011); it is kept where the word is not below floor(p 2^32).
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"

namespace pamm {

struct DropoutArgs {
    const void *x, *r;
    void* y;
    int64_t rows, n, ldx, ldr, ldy, total;
    const int64_t* counter;         // null, or a device number that is added to the offset
    uint64_t offset;
    uint32_t keys[20];              // of the ten rounds, from the seed: constants to the kernel
    uint32_t threshold;
    bool none;                      // nothing is kept
    float factor;
};

inline void dropout_keys(uint64_t seed, uint32_t (&keys)[20]) {
    for (uint32_t round = 0; round < 10; ++round) {
        keys[2 * round] = (uint32_t)seed + round * 0x9E3779B9u;
        keys[2 * round + 1] = (uint32_t)(seed >> 32) + round * 0xBB67AE85u;
    }
}
// Two products with 64-bit results and two three-way exclusive ors a round: bound by instructions rather than memory if there are many more.
__device__ __forceinline__ uint4 random_block(uint64_t block, uint64_t offset, const uint32_t (&keys)[20]) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ keys[2 * round];
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ keys[2 * round + 1];
        c3 = (uint32_t)p0;
    }
    return make_uint4(c0, c1, c2, c3);
}

template <typename T, bool RESIDUAL>
__device__ __forceinline__ void dropout_element(const DropoutArgs& a, int64_t e, bool kept) {
    const int64_t row = a.rows == 1 ? 0 : e / a.n, col = e - row * a.n;
    float f = kept ? to_float(static_cast<const T*>(a.x)[row * a.ldx + col]) : 0.f;
    f = RESIDUAL ? fmaf(f, a.factor, to_float(static_cast<const T*>(a.r)[row * a.ldr + col])) : f * a.factor;
    static_cast<T*>(a.y)[row * a.ldy + col] = from_float<T>(f);
}

// A thread takes V elements that follow each other (V = 4 or 8: whole vectors on memory's grid, in rows of whole vectors or in one
// row of any length, whose last elements go one by one), or (V = 1) the up to four elements of one block, one by one.
template <typename T, int V, bool RESIDUAL>
__global__ void __launch_bounds__(256)
dropout_kernel(const __grid_constant__ DropoutArgs a) {
    grid_dependency_wait();
    grid_launch_dependents();
    const uint64_t offset = a.offset + (a.counter ? (uint64_t)*a.counter : 0ull);
    const auto kept = [&](uint32_t w) { return w >= a.threshold && !a.none; };
    if constexpr (V > 1) {
        using P = Piece<T, V>;
        const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
        if (e + V > a.total) {
            for (int64_t i = e; i < a.total; ++i) {
                const uint4 w = random_block((uint64_t)i / 4, offset, a.keys);
                dropout_element<T, RESIDUAL>(a, i, kept(i % 4 == 0 ? w.x : i % 4 == 1 ? w.y : i % 4 == 2 ? w.z : w.w));
            }
            return;
        }
        const int64_t row = a.rows == 1 ? 0 : e / a.n, col = e - row * a.n;
        const auto x = P::load(static_cast<const T*>(a.x) + row * a.ldx + col);
        auto r = P::zero();
        if (RESIDUAL) r = P::load(static_cast<const T*>(a.r) + row * a.ldr + col);
        float f[V], g[V];
        P::unpack(x, f);
        P::unpack(r, g);
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const uint4 w = random_block((uint64_t)(e + i) / 4, offset, a.keys);
            f[i] = kept(w.x) ? f[i] : 0.f;
            f[i + 1] = kept(w.y) ? f[i + 1] : 0.f;
            f[i + 2] = kept(w.z) ? f[i + 2] : 0.f;
            f[i + 3] = kept(w.w) ? f[i + 3] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = RESIDUAL ? fmaf(f[i], a.factor, g[i]) : f[i] * a.factor;
        P::store(static_cast<T*>(a.y) + row * a.ldy + col, f);
    } else {
        const int64_t e0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
        if (e0 >= a.total) return;
        const uint4 w = random_block((uint64_t)e0 / 4, offset, a.keys);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e0 + i < a.total) dropout_element<T, RESIDUAL>(a, e0 + i, kept(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w));
    }
}

}  // namespace pamm
