// Eight neighbouring elements of a row, as they are stored (16 bytes, fp32: 32) and as fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cstdint>

#include "ptx.cuh"

namespace precog {

template <typename T> struct Raw8 { uint4 q[1]; };
template <> struct Raw8<float> { uint4 q[2]; };

template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T *p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) r.q[i] = reinterpret_cast<const uint4 *>(p)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const Raw8<T> &r) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = r.q[i];
}

__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(r.q[i].x), v[4 * i + 1] = __uint_as_float(r.q[i].y);
        v[4 * i + 2] = __uint_as_float(r.q[i].z), v[4 * i + 3] = __uint_as_float(r.q[i].w);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16> &r, float (&v)[8]) {
    const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ Raw8<float> pack8(const float *, const float (&v)[8]) {
    Raw8<float> r;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        r.q[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                            __float_as_uint(v[4 * i + 3]));
    return r;
}
__device__ __forceinline__ Raw8<__nv_bfloat16> pack8(const __nv_bfloat16 *, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&p);
    }
    Raw8<__nv_bfloat16> r;
    r.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
    return r;
}

// x / (1 + e^-x); NaN stays, and -infinity gives NaN as the formula does. For rows that are stored in 16 bits
// the quick exponential and reciprocal (together within 2^-19 of the value while |x| < 10) are far below the
// rounding; where e^-x leaves 2^126 they give 0. Rows in fp32 get the exact ones.
constexpr float kMinusLog2e = -1.4426950408889634f;
__device__ __forceinline__ float rcp_quick(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <typename T>
__device__ __forceinline__ float silu(float x) {
    if constexpr (sizeof(T) == 4) return x / (1.f + expf(-x));
    return x * rcp_quick(1.f + ex2(x * kMinusLog2e));
}
// two at once
template <typename T>
__device__ __forceinline__ f2 silu2(f2 x) {
    float a, b;
    if constexpr (sizeof(T) == 4) {
        unpack2(x, a, b);
        return pack2(silu<T>(a), silu<T>(b));
    }
    unpack2(mul2(x, pack2(kMinusLog2e, kMinusLog2e)), a, b);
    return mul2(x, pack2(rcp_quick(1.f + ex2(a)), rcp_quick(1.f + ex2(b))));
}

// the same eight as four pairs
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T> &r, f2 (&v)[4]) {
    float e[8];
    unpack8(r, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(e[2 * i], e[2 * i + 1]);
}
template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const T *, const f2 (&v)[4]) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(v[i], e[2 * i], e[2 * i + 1]);
    return pack8(static_cast<const T *>(nullptr), e);
}

}  // namespace precog
