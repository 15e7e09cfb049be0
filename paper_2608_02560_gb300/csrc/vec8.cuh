// Eight neighbouring elements of a row, as they are stored (16 bytes, fp32: 32) and as fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cstdint>

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
// the quick exponential and quotient (together within 2^-19 of the value while |x| < 10) are far below the
// rounding; where e^-x leaves 2^126 they give 0. Rows in fp32 get the exact ones.
template <typename T>
__device__ __forceinline__ float silu(float x) {
    if constexpr (sizeof(T) == 4) return x / (1.f + expf(-x));
    return __fdividef(x, 1.f + __expf(-x));
}

}  // namespace precog
