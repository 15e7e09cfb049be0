// Norms of query and key heads with the position rotation, in one pass over the projection.
//
//   n = rsqrt(sum x^2 [/ dim] + eps) ;  x <- x n w ;  (a, b) <- (a cos - b sin, b cos + a sin)
//
// A vector of `dim` numbers belongs to a group of G lanes (the least power of two that leaves a
// lane at most 8 numbers), its sum of squares to log2(G) shuffles. A lane's 8 numbers are two
// quads chosen so that both partners of every rotated pair are its own: eight neighbours where
// pairs are neighbours, else four of the lower half and the same four of the upper one; outputs
// may therefore be the inputs. A group keeps its token's rotations and the weights in registers
// and takes kHeads heads, kFly of them in flight. What bounds it is memory: each number is read
// once and written once (65,521 tokens of 16 + 8 heads of 128 bf16, slices of a projection, weights, pairs
// of neighbours: 146 us, 5.64 TB/s, 0.83 of the measured copy rate; the same of whole tensors, no weights,
// pairs of halves, 134; a single token its launch). A group of lanes a head, rather than a warp, keeps
// every lane's loads 16 bytes wide: a first kernel of 32 scalar lanes a head took 468 us.
#include <type_traits>

#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_qk_status;

constexpr int kThreads = 256;
constexpr int kHeads = 8, kFly = 4;

// Eight numbers as they are stored: two quads, or one 16-byte (fp32: 32-byte) piece if they are
// neighbours.
template <typename T> struct Raw { uint2 q[2]; };
template <> struct Raw<float> { uint4 q[2]; };
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_raw(const T *base, int e0, int e1, Raw<T> &r) {
    if constexpr (WHOLE && sizeof(T) == 2) {
        const uint4 v = *reinterpret_cast<const uint4 *>(base + e0);
        r.q[0] = make_uint2(v.x, v.y), r.q[1] = make_uint2(v.z, v.w);
    } else {
        using Q = std::remove_reference_t<decltype(r.q[0])>;
        r.q[0] = *reinterpret_cast<const Q *>(base + e0), r.q[1] = *reinterpret_cast<const Q *>(base + e1);
    }
}
__device__ __forceinline__ void unpack(const Raw<float> &r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(r.q[i].x), v[4 * i + 1] = __uint_as_float(r.q[i].y);
        v[4 * i + 2] = __uint_as_float(r.q[i].z), v[4 * i + 3] = __uint_as_float(r.q[i].w);
    }
}
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16> &r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(r.q[i].x << 16), v[4 * i + 1] = __uint_as_float(r.q[i].x & 0xffff0000u);
        v[4 * i + 2] = __uint_as_float(r.q[i].y << 16), v[4 * i + 3] = __uint_as_float(r.q[i].y & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw<__half> &r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&r.q[i].x)), b = __half22float2(*reinterpret_cast<const __half2 *>(&r.q[i].y));
        v[4 * i] = a.x, v[4 * i + 1] = a.y, v[4 * i + 2] = b.x, v[4 * i + 3] = b.y;
    }
}
__device__ __forceinline__ uint32_t two(const __nv_bfloat16 *, float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ uint32_t two(const __half *, float a, float b) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void store8(T *base, int e0, int e1, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(base + e0) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(base + e1) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        const uint2 a = make_uint2(two(base, v[0], v[1]), two(base, v[2], v[3])), b = make_uint2(two(base, v[4], v[5]), two(base, v[6], v[7]));
        if constexpr (WHOLE) {
            *reinterpret_cast<uint4 *>(base + e0) = make_uint4(a.x, a.y, b.x, b.y);
        } else {
            *reinterpret_cast<uint2 *>(base + e0) = a;
            *reinterpret_cast<uint2 *>(base + e1) = b;
        }
    }
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_f(float *p, float v) { *p = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f(__half *p, float v) { *p = __float2half_rn(v); }

// `per` heads of a token's q or k a group: `qparts` groups a token for q, `parts` in all.
// HALF: pair i is (i, i + rot / 2) with rot / 2 a multiple of 4; else (2 i, 2 i + 1).
template <typename T, int G, bool HALF, bool WEIGHT>
__global__ void __launch_bounds__(kThreads, 3) qk_norm_kernel(const QkNormParams p, int qparts, int parts, int per, int64_t items) {
    const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / G;
    const int lane = threadIdx.x % G;
    if (item >= items) return;   // whole groups: the shuffles below stay within one
    const unsigned mask = G == 32 ? 0xffffffffu : ((1u << G) - 1u) << ((threadIdx.x & 31) / G * G);
    const int64_t t = item / parts;
    int h0 = static_cast<int>(item - t * parts);
    const int which = h0 >= qparts;
    h0 = (h0 - (which ? qparts : 0)) * per;
    const int h1 = h0 + per < p.heads[which] ? h0 + per : p.heads[which];
    const int64_t pos = p.rot == 0 ? 0 : p.positions ? p.positions[t] : t;
    if (p.rot != 0 && (pos < 0 || pos >= p.n_positions)) {
        if (lane == 0) atomicOr(&g_qk_status, PRECOG_DEV_BAD_INDEX);
        return;
    }
    // this lane's quads
    const int pairs = HALF ? p.rot / 8 : 0;
    const int e0 = HALF && lane < pairs ? 4 * lane : 8 * lane;
    const int e1 = HALF && lane < pairs ? p.rot / 2 + 4 * lane : 8 * lane + 4;
    const bool live = 8 * lane < p.dim;
    const T *in = static_cast<const T *>(p.in[which]) + t * p.in_stride[which];
    T *out = static_cast<T *>(p.out[which]) + t * p.out_stride[which];
    float cs[4], sn[4];          // of the lane's four pairs
    bool turn[4];                // (not by 1 and 0: 0 times a partner that is infinite is NaN)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        turn[i] = HALF ? lane < pairs : 4 * lane + i < p.rot / 2;
        cs[i] = turn[i] ? p.cos[pos * (p.rot / 2) + 4 * lane + i] : 1.f;
        sn[i] = turn[i] ? p.sin[pos * (p.rot / 2) + 4 * lane + i] : 0.f;
    }
    float w[8];
    if constexpr (WEIGHT) {
        const float *weight = p.weight[which];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = live && weight ? weight[(i < 4 ? e0 : e1 - 4) + i] : 1.f;
    }
    const float inv = p.norm == PRECOG_NORM_RMS ? 1.f / static_cast<float>(p.dim) : 1.f;
#pragma unroll 1
    for (int h = h0; h < h1; h += kFly) {
        Raw<T> raw[kFly];
#pragma unroll
        for (int f = 0; f < kFly; ++f) {
            raw[f] = Raw<T>{};
            if (live && h + f < h1) load_raw<!HALF>(in + static_cast<int64_t>(h + f) * p.dim, e0, e1, raw[f]);
        }
        float n[kFly];
#pragma unroll
        for (int f = 0; f < kFly; ++f) {
            float x[8];
            unpack(raw[f], x);
            n[f] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) n[f] = fmaf(x[i], x[i], n[f]);
        }
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1)
#pragma unroll
            for (int f = 0; f < kFly; ++f) n[f] += __shfl_xor_sync(mask, n[f], o);
#pragma unroll
        for (int f = 0; f < kFly; ++f) {
            if (!live || h + f >= h1) continue;
            const float m = p.norm == PRECOG_NORM_NONE ? 1.f : rsqrtf(fmaf(n[f], inv, p.eps));
            float x[8];
            unpack(raw[f], x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= m;
            if constexpr (WEIGHT) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float &a = x[HALF ? i : 2 * i], &b = x[HALF ? i + 4 : 2 * i + 1];
                const float a0 = a;
                if (turn[i]) a = a0 * cs[i] - b * sn[i], b = b * cs[i] + a0 * sn[i];
            }
            store8<!HALF>(out + static_cast<int64_t>(h + f) * p.dim, e0, e1, x);
        }
    }
}

// Every entry alone, for pairs (i, i + rot / 2) with rot / 2 not a multiple of 4: lane l of 16 has the
// pairs l, l + 16, ...
template <typename T, int G>
__global__ void __launch_bounds__(kThreads) qk_norm_any_kernel(const QkNormParams p, int64_t vectors) {
    const int64_t vec = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / G;
    const int lane = threadIdx.x % G;
    const int heads = p.heads[0] + p.heads[1];
    if (vec >= vectors) return;   // whole groups: the shuffles below stay within one
    const int64_t t = vec / heads;
    int head = static_cast<int>(vec % heads);
    const int which = head >= p.heads[0];
    head -= which ? p.heads[0] : 0;
    const int64_t pos = p.rot == 0 ? 0 : p.positions ? p.positions[t] : t;
    if (p.rot != 0 && (pos < 0 || pos >= p.n_positions)) {
        if (lane == 0) atomicOr(&g_qk_status, PRECOG_DEV_BAD_INDEX);
        return;
    }
    const T *in = static_cast<const T *>(p.in[which]) + t * p.in_stride[which] + static_cast<int64_t>(head) * p.dim;
    T *out = static_cast<T *>(p.out[which]) + t * p.out_stride[which] + static_cast<int64_t>(head) * p.dim;
    const unsigned mask = G == 32 ? 0xffffffffu : ((1u << G) - 1u) << ((threadIdx.x & 31) / G * G);
    float sum = 0.f;
    for (int i = lane; i < p.dim; i += G) sum = fmaf(to_f(in[i]), to_f(in[i]), sum);
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
    const float n = p.norm == PRECOG_NORM_NONE ? 1.f : rsqrtf((p.norm == PRECOG_NORM_RMS ? sum / p.dim : sum) + p.eps);
    const float *w = p.weight[which];
    const int half = p.rot / 2;
    // both partners are read before either is written, by the one lane that has them: in place is fine
    for (int i = lane; i < half; i += G) {
        const int ia = p.interleaved ? 2 * i : i, ib = p.interleaved ? 2 * i + 1 : i + half;
        const float c = p.cos[pos * half + i], s = p.sin[pos * half + i];
        const float a = to_f(in[ia]) * n * (w ? w[ia] : 1.f), b = to_f(in[ib]) * n * (w ? w[ib] : 1.f);
        from_f(out + ia, a * c - b * s);
        from_f(out + ib, b * c + a * s);
    }
    for (int i = p.rot + lane; i < p.dim; i += G) from_f(out + i, to_f(in[i]) * n * (w ? w[i] : 1.f));
}

template <typename T, int G, bool HALF, bool WEIGHT>
cudaError_t launch_lanes(const QkNormParams &p, cudaStream_t stream) {
    // Eight heads a group reuse its rotations and weights (16 + 8 heads of 128, whole tensors, halves: 65,521
    // tokens 134 us, one head a group 380; 1000 tokens 3.5 and 6.8); fewer where that would leave SMs with
    // less than two CTAs.
    int per = kHeads;
    auto parts_of = [&](int heads) { return (heads + per - 1) / per; };
    while (per > 1 && p.T * (parts_of(p.heads[0]) + parts_of(p.heads[1])) * G < 2LL * device_sm_count() * kThreads) per /= 2;
    const int qparts = parts_of(p.heads[0]), parts = qparts + parts_of(p.heads[1]);
    const int64_t items = p.T * parts, blocks = (items * G + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    qk_norm_kernel<T, G, HALF, WEIGHT><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p, qparts, parts, per, items);
    return cudaGetLastError();
}

template <typename T, int G>
cudaError_t launch_group(const QkNormParams &p, cudaStream_t stream) {
    const bool weight = p.weight[0] != nullptr || p.weight[1] != nullptr, half = p.rot != 0 && !p.interleaved;
    if (half) return weight ? launch_lanes<T, G, true, true>(p, stream) : launch_lanes<T, G, true, false>(p, stream);
    return weight ? launch_lanes<T, G, false, true>(p, stream) : launch_lanes<T, G, false, false>(p, stream);
}

template <typename T>
cudaError_t launch_typed(const QkNormParams &p, cudaStream_t stream) {
    cudaError_t e;
    if (p.rot != 0 && !p.interleaved && p.rot % 8 != 0) {
        // (slower where both could run: the same 65,521 tokens take 415 us, the other kernel 134)
        const int64_t vectors = p.T * (static_cast<int64_t>(p.heads[0]) + p.heads[1]), blocks = (vectors * 16 + kThreads - 1) / kThreads;
        if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
        qk_norm_any_kernel<T, 16><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p, vectors);
        e = cudaGetLastError();
    } else if (p.dim <= 64) {
        e = launch_group<T, 8>(p, stream);
    } else if (p.dim <= 128) {
        e = launch_group<T, 16>(p, stream);
    } else {
        e = launch_group<T, 32>(p, stream);
    }
    if (e == cudaSuccess) count_launches(1);
    return e;
}

}  // namespace

cudaError_t launch_qk_norm(const QkNormParams &p, cudaStream_t stream) {
    switch (p.dtype) {
        case PRECOG_F32: return launch_typed<float>(p, stream);
        case PRECOG_F16: return launch_typed<__half>(p, stream);
        default: return launch_typed<__nv_bfloat16>(p, stream);
    }
}

cudaError_t qk_norm_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_qk_status); }

}  // namespace precog
