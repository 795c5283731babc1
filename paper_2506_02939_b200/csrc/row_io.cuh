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

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// floats -> 16 bytes of T, rounded to nearest even
template <typename T>
__device__ __forceinline__ uint4 round_vec(const float (&x)[Vec16<T>::N]);
template <>
__device__ __forceinline__ uint4 round_vec<float>(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <>
__device__ __forceinline__ uint4 round_vec<__nv_bfloat16>(const float (&x)[8]) {
    return make_uint4(round_bf16x2(x[0], x[1]), round_bf16x2(x[2], x[3]), round_bf16x2(x[4], x[5]), round_bf16x2(x[6], x[7]));
}

// V consecutive elements of a row of `n`, V = one 16-byte vector (row 16-byte aligned, col a
// multiple of V) or one element (any alignment of the type).  Elements at or beyond n read as zero
// and are not written.
template <typename T, int V>
struct RowIo {
    static_assert(V == 1 || V == Vec16<T>::N, "one element or 16 bytes");
    static __device__ __forceinline__ void load(const T* row, int64_t col, int64_t n, float (&out)[V]) {
        if constexpr (V == 1) {
            out[0] = col < n ? to_float(row[col]) : 0.f;
        } else {
            if (col + V <= n) {
                unpack_vec<T>(ld16(row + col), out);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) out[e] = col + e < n ? to_float(row[col + e]) : 0.f;
            }
        }
    }
    static __device__ __forceinline__ void store(T* row, int64_t col, int64_t n, const float (&x)[V]) {
        if constexpr (V == 1) {
            if (col < n) row[col] = from_float<T>(x[0]);
        } else {
            if (col + V <= n) {
                st16(row + col, round_vec<T>(x));
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (col + e < n) row[col + e] = from_float<T>(x[e]);
            }
        }
    }
};

// V consecutive entries of a vector of weights (fp32 or bf16, a runtime choice), zero at and beyond
// n.  A null vector stands for `missing` in every place.  Vector access where the base is 16-byte
// aligned (`vec`); col is a multiple of V and V at most 8.
template <int V>
__device__ __forceinline__ void load_weights(const void* w, bool is_bf16, bool vec, int col, int n, float missing, float (&out)[V]) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = missing;
        return;
    }
    if (V > 1 && vec && col + V <= n) {
        if constexpr (V == 8) {
            if (is_bf16) {
                unpack_vec<__nv_bfloat16>(__ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + col)), out);
            } else {
                const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + col);
                const float4 a = __ldg(p), b = __ldg(p + 1);
                out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w;
                out[4] = b.x; out[5] = b.y; out[6] = b.z; out[7] = b.w;
            }
        } else if constexpr (V == 4) {
            if (is_bf16) {
                const uint2 t = __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(w) + col));
                out[0] = bf16_lo(t.x); out[1] = bf16_hi(t.x); out[2] = bf16_lo(t.y); out[3] = bf16_hi(t.y);
            } else {
                const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + col));
                out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w;
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int i = col + e;
        out[e] = i >= n ? 0.f : is_bf16 ? to_float(static_cast<const __nv_bfloat16*>(w)[i]) : static_cast<const float*>(w)[i];
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

}  // namespace pamm
