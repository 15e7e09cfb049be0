// Logits before a token is chosen: penalties for tokens that the text has already, biases, grammar masks.
//
//   z = x ;  seen:  z <- z > 0 ? z / repetition : z repetition
//   n = times in the counted part > 0:  z <- z - n frequency - presence
//   biased:  z <- z + bias ;  not allowed by the mask:  z <- -infinity
//
// A CTA has a slice of one row's vocabulary. It counts the slice's tokens of the row's history in shared
// memory (a word a token: the top bit for a token seen before the counted part, the count below it; integer
// atomics, so the order does not matter), notes the last bias of each token the same way, and then passes
// over the slice's logits once.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_adjust_status;

constexpr int kThreads = 256;
constexpr uint32_t kSeen = 0x80000000u;

template <typename T> __device__ __forceinline__ T stored(float v) { return from_f32<T>(v); }
template <> __device__ __forceinline__ __half stored<__half>(float v) { return __float2half_rn(v); }

// The range [a, b) of row r in a list of `total` entries; empty (and flagged) where the offsets are broken.
__device__ __forceinline__ void list_of(const int64_t *offsets, int64_t r, int64_t total, bool flag, int64_t &a, int64_t &b) {
    a = offsets[r], b = offsets[r + 1];
    if (a < 0 || b < a || b > total) {
        if (flag) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_OFFSETS);
        a = b = 0;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) adjust_kernel(const AdjustParams p, int slice, int slices) {
    grid_dependency_wait();
    extern __shared__ uint32_t shared[];
    uint32_t *const counts = shared, *const biased = shared + (p.history ? slice : 0);
    const int64_t r = blockIdx.x / static_cast<unsigned>(slices);
    const int part = static_cast<int>(blockIdx.x % static_cast<unsigned>(slices));
    const int lo = part * slice, hi = min(static_cast<int>(p.vocab), lo + slice);
    const bool first = part == 0 && threadIdx.x == 0;
    int64_t ba = 0, bb = 0;
    if (p.history || p.bias) {
        for (int i = threadIdx.x; i < slice * ((p.history != nullptr) + (p.bias != nullptr)); i += kThreads) shared[i] = 0;
        __syncthreads();
        if (p.history) {
            int64_t a, b;
            list_of(p.history_offsets, r, p.n_history, first, a, b);
            const int64_t from = a + (p.count_from ? min(b - a, max(static_cast<int64_t>(0), p.count_from[r])) : 0);
            for (int64_t j = a + threadIdx.x; j < b; j += kThreads) {
                const int64_t tok = p.history[j];
                if (tok >= lo && tok < hi) {
                    if (j < from) atomicOr(&counts[tok - lo], kSeen);
                    else atomicAdd(&counts[tok - lo], 1u);
                } else if (part == 0 && (tok < -1 || tok >= p.vocab)) {
                    atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
                }
            }
        }
        if (p.bias) {
            list_of(p.bias_offsets, r, p.n_bias, first, ba, bb);
            for (int64_t j = ba + threadIdx.x; j < bb; j += kThreads) {
                const int64_t tok = p.bias_idx[j];
                if (tok >= lo && tok < hi) atomicMax(&biased[tok - lo], static_cast<uint32_t>(j - ba) + 1u);
                else if (part == 0 && (tok < -1 || tok >= p.vocab)) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
            }
        }
        __syncthreads();
    }
    const uint32_t *mask = nullptr;
    if (p.mask || p.mask_rows) {
        const int64_t m = p.mask_rows ? p.mask_rows[r] : r;
        if (m >= 0 && m < p.n_masks) mask = p.mask + m * ((p.vocab + 31) / 32);
        else if (m != -1 && first) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
    }
    const float rep = p.repetition ? p.repetition[r] : 1.f, freq = p.frequency ? p.frequency[r] : 0.f;
    const float pres = p.presence ? p.presence[r] : 0.f;
    const T *x = static_cast<const T *>(p.logits) + r * p.stride;
    T *out = static_cast<T *>(p.out) + r * p.out_stride;
    for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
        float z = to_f32(x[i]);
        if (p.history) {
            const uint32_t n = counts[i - lo];
            if (n != 0) {
                if (p.repetition) z = z > 0.f ? z / rep : z * rep;
                if ((n & ~kSeen) != 0) z = z - freq * static_cast<float>(n & ~kSeen) - pres;
            }
        }
        if (p.bias) {
            const uint32_t j = biased[i - lo];
            if (j != 0) z += p.bias[ba + j - 1];
        }
        if (mask && ((mask[i >> 5] >> (i & 31)) & 1u) == 0) z = __int_as_float(0xff800000);
        out[i] = stored<T>(z);
    }
}

template <typename T>
cudaError_t launch_typed(const AdjustParams &p, cudaStream_t stream) {
    const int slice = 8192;
    const int slices = static_cast<int>((p.vocab + slice - 1) / slice);
    const int64_t blocks = p.rows * slices;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const int words = slice * ((p.history != nullptr) + (p.bias != nullptr));
    cudaError_t e = ensure_smem(reinterpret_cast<const void *>(adjust_kernel<T>), words * 4);
    if (e != cudaSuccess) return e;
    e = launch_dependent(adjust_kernel<T>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), words * 4, stream, p, slice, slices);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

}  // namespace

cudaError_t launch_adjust(const AdjustParams &p, cudaStream_t stream) {
    switch (p.dtype) {
        case PRECOG_F32: return launch_typed<float>(p, stream);
        case PRECOG_F16: return launch_typed<__half>(p, stream);
        default: return launch_typed<__nv_bfloat16>(p, stream);
    }
}

cudaError_t adjust_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_adjust_status); }

}  // namespace precog
