// Norms of query and key heads with the position rotation, in one pass over the projection.
//
//   n = rsqrt(sum x^2 [/ dim] + eps) ;  x <- x n w ;  (a, b) <- (a cos - b sin, b cos + a sin)
//
// A vector of `dim` numbers belongs to a group of G lanes; both partners of a rotated pair are
// read and written by one lane, so outputs may be the inputs.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_qk_status;

constexpr int kThreads = 256;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_f(float *p, float v) { *p = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f(__half *p, float v) { *p = __float2half_rn(v); }

// One vector a group of G lanes, every entry alone: any rot_dim. Lane l has entries l, l + G, ...
template <typename T, int G>
__global__ void __launch_bounds__(kThreads) qk_norm_kernel(const QkNormParams p, int64_t vectors) {
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

template <typename T>
cudaError_t launch_typed(const QkNormParams &p, cudaStream_t stream) {
    const int64_t vectors = p.T * (static_cast<int64_t>(p.heads[0]) + p.heads[1]);
    const int64_t blocks = (vectors * 16 + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    qk_norm_kernel<T, 16><<<static_cast<unsigned>(blocks), kThreads, 0, stream>>>(p, vectors);
    cudaError_t e = cudaGetLastError();
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

cudaError_t qk_norm_status_word_read_clear(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_qk_status, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_qk_status, &zero, sizeof(uint32_t));
}

}  // namespace precog
