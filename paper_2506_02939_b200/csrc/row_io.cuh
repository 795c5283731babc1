// Row access shared by the operators around the projection (norm, rotary positions, gradient
// clipping): plain (coherent) loads and stores of 16 bytes or of one element, because these
// operators may write where they read.  A value is read once by the thread that later writes its
// place, so in-place calls need no more than program order.
#pragma once
#include "pamm_common.cuh"

namespace pamm {

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st16(void* p, const uint4& v) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A store whose lines leave L2 first (a policy of evict_first_policy).
__device__ __forceinline__ uint64_t evict_first_policy() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void st16(void* p, const uint4& v, uint64_t policy) {
    asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1,%2,%3,%4}, %5;" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "l"(policy)
                 : "memory");
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {       // to nearest even
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// V consecutive elements of a row as they lie in memory, aligned to their size of 2, 4, 8 or 16 bytes.  Loading and unpacking
// are apart, so that all of a thread's loads are in flight before the first is waited for.
template <typename T, int V>
struct Piece {
    static constexpr int BYTES = V * (int)sizeof(T), WORDS = BYTES < 4 ? 1 : BYTES / 4;
    static_assert(BYTES == 2 || BYTES == 4 || BYTES == 8 || BYTES == 16, "a power of two up to 16 bytes");
    struct Raw { uint32_t w[WORDS]; };

    static __device__ __forceinline__ Raw zero() {
        Raw r;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) r.w[i] = 0;
        return r;
    }
    static __device__ __forceinline__ Raw load(const T* p) {
        Raw r;
        if constexpr (BYTES == 2) {
            r.w[0] = *reinterpret_cast<const unsigned short*>(p);
        } else if constexpr (BYTES == 4) {
            r.w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (BYTES == 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            r.w[0] = v.x; r.w[1] = v.y;
        } else {
            const uint4 v = ld16(p);
            r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
        }
        return r;
    }
    static __device__ __forceinline__ void unpack(const Raw& r, float* out) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = __uint_as_float(r.w[e]);
        } else if constexpr (V == 1) {
            out[0] = bf16_lo(r.w[0]);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                out[2 * i] = bf16_lo(r.w[i]);
                out[2 * i + 1] = bf16_hi(r.w[i]);
            }
        }
    }
    static __device__ __forceinline__ void pack(const float* x, uint32_t (&w)[WORDS]) {       // rounded to nearest even
        if constexpr (BYTES == 2) {
            w[0] = round_bf16x2(x[0], 0.f);
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = __float_as_uint(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = round_bf16x2(x[2 * i], x[2 * i + 1]);
        }
    }
    static __device__ __forceinline__ void store(T* p, const float* x) {
        uint32_t w[WORDS];
        pack(x, w);
        if constexpr (BYTES == 2) *reinterpret_cast<unsigned short*>(p) = (unsigned short)w[0];
        else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
        else if constexpr (BYTES == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else st16(p, make_uint4(w[0], w[1], w[2], w[3]));
    }
    static __device__ __forceinline__ void store(T* p, const float* x, uint64_t policy) {     // the policy is for 16 bytes only
        if constexpr (BYTES == 16) {
            uint32_t w[WORDS];
            pack(x, w);
            st16(p, make_uint4(w[0], w[1], w[2], w[3]), policy);
        } else {
            store(p, x);
        }
    }
};

// V consecutive entries of a vector of weights (V > 1: 16-byte aligned base, col a multiple of V).
template <typename W, int V>
__device__ __forceinline__ void load_weights(const W* w, float* out) {
    if constexpr (V == 1) {
        out[0] = to_float(*w);
    } else if constexpr (sizeof(W) == 4) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 t = __ldg(reinterpret_cast<const float4*>(w + e));
            out[e] = t.x; out[e + 1] = t.y; out[e + 2] = t.z; out[e + 3] = t.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const uint2 t = __ldg(reinterpret_cast<const uint2*>(w + e));
            out[e] = bf16_lo(t.x); out[e + 1] = bf16_hi(t.x); out[e + 2] = bf16_lo(t.y); out[e + 3] = bf16_hi(t.y);
        }
    }
}

// Two fp32 operations in one instruction (each rounded as the single one).
__device__ __forceinline__ float2 fma2(const float2 a, const float2 b, const float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(const float2 a, const float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(const float2 a, const float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
template <int LANES = 32>
__device__ __forceinline__ float warp_sum(float x) {       // over LANES neighbouring lanes, the same sum in each
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}
__device__ __forceinline__ float2 twice(float x) { return make_float2(x, x); }

}  // namespace pamm
