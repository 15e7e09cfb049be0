// Neighbouring elements of a row, as they are stored and as fp32; and SiLU.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cstdint>
#include <type_traits>

#include "ptx.cuh"

namespace precog {

// Four neighbouring elements, as they are stored (8 bytes, fp32: 16) and as fp32.
template <typename T> struct Raw4 { using type = uint2; };
template <> struct Raw4<float> { using type = uint4; };
template <typename T>
__device__ __forceinline__ typename Raw4<T>::type load4(const T *p) { return *reinterpret_cast<const typename Raw4<T>::type *>(p); }
__device__ __forceinline__ void unpack4(const uint4 &q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y), v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack4(const uint2 &q, float (&v)[4]) {   // bf16
    v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xffff0000u);
    v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xffff0000u);
}

// V of them, in pieces of 16 bytes (four of bf16: 8).
template <typename T, int V> struct Piece { uint4 q[V * static_cast<int>(sizeof(T)) / 16]; };
template <> struct Piece<__nv_bfloat16, 4> { uint2 q[1]; };

template <int V, typename T>
__device__ __forceinline__ Piece<T, V> load_piece(const T *p) {
    Piece<T, V> r;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r.q) / sizeof(r.q[0])); ++i)
        r.q[i] = reinterpret_cast<const std::remove_extent_t<decltype(r.q)> *>(p)[i];
    return r;
}
template <int V>
__device__ __forceinline__ void unpack(const Piece<float, V> &r, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        v[4 * i] = __uint_as_float(r.q[i].x), v[4 * i + 1] = __uint_as_float(r.q[i].y);
        v[4 * i + 2] = __uint_as_float(r.q[i].z), v[4 * i + 3] = __uint_as_float(r.q[i].w);
    }
}
__device__ __forceinline__ void unpack(const Piece<__nv_bfloat16, 4> &r, float (&v)[4]) { unpack4(r.q[0], v); }
__device__ __forceinline__ void unpack(const Piece<__nv_bfloat16, 8> &r, float (&v)[8]) {
    const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
template <int V>
__device__ __forceinline__ void store_piece(float *p, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) reinterpret_cast<float4 *>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    return make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7]));
}
__device__ __forceinline__ void store_piece(__nv_bfloat16 *p, const float (&v)[8]) { *reinterpret_cast<uint4 *>(p) = pack(v); }
__device__ __forceinline__ void store_piece(__nv_bfloat16 *p, const float (&v)[4]) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack(v[0], v[1]), pack(v[2], v[3]));
}

// x / (1 + e^-x); NaN stays, and -infinity gives NaN as the formula does. T is the type of the rows that x is from, TO the
// widest that the value goes into. Rows in fp32 get expf and the quotient. 16-bit rows:
//   into 16 bits: the quick exponential and reciprocal, together within (5 + 1.2 |x|) 2^-23 of the value (2^-19 while
//   |x| < 10), far below the rounding; where e^-x leaves 2^126 they give 0;
//   into fp32: the same two with their errors taken back, within 7 * 2^-24 of the value. What -x log2(e) loses is an fma's
//   difference (Dekker's product in two parts), and enters as 2^low = 1 + low ln 2 (|low| < 2^-17); the quotient is
//   q + (x - d q) r (Markstein's correction by the residual). 4 for the exponential, and one each for its product with 1 + low ln 2, for d, and for the quotient. (65,521 rows of 2048, gate,
//   norm, fp32 residual, next norm: 276 us; with the 16-bit form 267, with expf and a quotient 292.)
constexpr float kMinusLog2e = -1.4426950408889634f;
constexpr float kMinusLog2eLow = -1.9259629911266175e-8f;   // what the constant above lacks
constexpr float kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float rcp_quick(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <typename T, typename TO = T>
__device__ __forceinline__ float silu(float x) {
    if constexpr (sizeof(T) == 4) return x / (1.f + expf(-x));
    const float z = x * kMinusLog2e;
    if constexpr (sizeof(TO) != 4) return x * rcp_quick(1.f + ex2(z));
    const bool near = fabsf(x) <= 87.f;   // beyond, e^-x is nothing beside 1, or the value nothing beside any other (e infinite)
    const float low = fmaf(x, kMinusLog2eLow, fmaf(x, kMinusLog2e, -z));
    const float e = ex2(z), d = 1.f + (near ? fmaf(e, low * kLn2, e) : e), r = rcp_quick(d), q = x * r;
    return near ? fmaf(fmaf(-d, q, x), r, q) : q;
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

}  // namespace precog
