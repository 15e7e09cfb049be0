// The short causal convolution in front of a selective scan, over ragged sequences and for single tokens.
//
//   y[t, d] = act(bias[d] + sum_{j < K} w[d, j] x[t - K + 1 + j, d]),   act = SiLU or none
//
// Inputs before a sequence's first token come from its window, K - 1 rows [oldest .. newest] that the
// sequence's past left (a bank's entry, a table's slot), or are zero. A thread has eight channels and rolls
// over a segment of tokens with the last K - 1 inputs in registers, so a row is read once and, at the start
// of a segment, K - 1 rows again.
//
// Segments of S tokens of ragged sequences need no prefix sums: item i belongs to the sequence c with
// base(c) <= i < base(c + 1), base(c) = offsets[c] / S + c, because base(c + 1) - base(c) is at least
// ceil(len / S) and at least 1. Items without tokens end at once.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"
#include "vec8.cuh"

namespace precog {
namespace {

__device__ uint32_t g_conv_status;

constexpr int kThreads = 128;

template <typename T, int K>
struct Lane {
    float w[K][8], bias[8];
    __device__ __forceinline__ void weights(const ConvParams &p, int d) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            bias[i] = p.bias ? p.bias[d + i] : 0.f;
#pragma unroll
            for (int j = 0; j < K; ++j) w[j][i] = p.weight[static_cast<int64_t>(d + i) * K + j];
        }
    }
    // y of the inputs before[0 .. K - 2] and now
    __device__ __forceinline__ Raw8<T> out(const float (&before)[K - 1][8], const float (&now)[8], bool act) const {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float a = bias[i];
#pragma unroll
            for (int j = 0; j < K - 1; ++j) a = fmaf(w[j][i], before[j][i], a);
            a = fmaf(w[K - 1][i], now[i], a);
            y[i] = act ? silu<T>(a) : a;
        }
        return pack8(static_cast<const T *>(nullptr), y);
    }
};

template <typename T, int K>
__global__ void __launch_bounds__(kThreads) conv_kernel(const ConvParams p, int segment, int64_t items) {
    grid_dependency_wait();
    const int groups = p.dim / 8;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t item = at / groups;
    if (item >= items) return;
    const int d = static_cast<int>(at - item * groups) * 8;
    // (in every thread of an item, so that every sequence is looked at whichever way the search goes)
    if (item < p.n_seqs) {
        const int64_t a = p.offsets[item], b = p.offsets[item + 1];
        if (a < 0 || b < a || b > p.T_tot) {
            if (d == 0) atomicOr(&g_conv_status, PRECOG_DEV_BAD_OFFSETS);
        }
    }
    int64_t lo = 0, hi = p.n_seqs;   // base(lo) <= item < base(hi)
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (p.offsets[mid] / segment + mid <= item) lo = mid;
        else hi = mid;
    }
    const int64_t c = lo, a = p.offsets[c], b = p.offsets[c + 1];
    if (a < 0 || b < a || b > p.T_tot) return;
    const int64_t part = item - (a / segment + c);
    int64_t t = a + part * segment;
    if (part < 0 || t > b || (t == b && part > 0)) return;   // (an empty sequence leaves its window all the same)
    const int64_t end = t + segment < b ? t + segment : b;

    const T *x = static_cast<const T *>(p.x) + d;
    float before[K - 1][8];
    const T *window = nullptr;
    if ((p.bank != nullptr || p.idx != nullptr) && t - (K - 1) < a) {
        const int64_t row = p.idx ? p.idx[c] : c;
        if (row < -1 || row >= p.bank_entries) {
            if (d == 0 && part == 0) atomicOr(&g_conv_status, PRECOG_DEV_BAD_INDEX);
        } else if (row >= 0) {
            window = static_cast<const T *>(p.bank) + ((row * p.L_total + p.layer) * (K - 1)) * p.dim + d;
        }
    }
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int64_t s = t - (K - 1) + j;
        Raw8<T> r = {};
        if (s >= a) r = load8(x + s * p.x_stride);
        else if (window != nullptr) r = load8(window + (s - a + K - 1) * p.dim);
        unpack8(r, before[j]);
    }
    Lane<T, K> lane;
    lane.weights(p, d);
    T *y = static_cast<T *>(p.y) + d;
    for (; t < end; ++t) {
        float now[8];
        unpack8(load8(x + t * p.x_stride), now);
        store8(y + t * p.y_stride, lane.out(before, now, p.silu != 0));
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) before[j][i] = j + 1 < K - 1 ? before[j + 1 < K - 1 ? j + 1 : 0][i] : now[i];
    }
    if (end == b && p.windows != nullptr) {
        T *out = static_cast<T *>(p.windows) + ((c * p.L_total + p.layer) * (K - 1)) * p.dim + d;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) store8(out + static_cast<int64_t>(j) * p.dim, pack8(out, before[j]));
    }
}

template <typename T, int K>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(const ConvParams p) {
    grid_dependency_wait();
    const int groups = p.dim / 8;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t row = at / groups;
    if (row >= p.n_seqs) return;
    const int d = static_cast<int>(at - row * groups) * 8;
    const int64_t slot = p.idx ? p.idx[row] : row;
    T *y = static_cast<T *>(p.y) + row * p.y_stride + d;
    if (slot < 0 || slot >= p.bank_entries) {
        if (slot != -1 && d == 0) atomicOr(&g_conv_status, PRECOG_DEV_BAD_INDEX);
        store8(y, Raw8<T>{});
        return;
    }
    T *window = static_cast<T *>(p.windows) + ((slot * p.L_total + p.layer) * (K - 1)) * p.dim + d;
    Raw8<T> raw[K];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) raw[j] = load8(window + static_cast<int64_t>(j) * p.dim);
    raw[K - 1] = load8(static_cast<const T *>(p.x) + row * p.x_stride + d);
    Lane<T, K> lane;
    lane.weights(p, d);
    float before[K - 1][8], now[8];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) unpack8(raw[j], before[j]);
    unpack8(raw[K - 1], now);
    store8(y, lane.out(before, now, p.silu != 0));
#pragma unroll
    for (int j = 0; j < K - 1; ++j) store8(window + static_cast<int64_t>(j) * p.dim, raw[j + 1]);
}

template <typename T, int K>
cudaError_t launch_k(const ConvParams &p, bool step, cudaStream_t stream) {
    const int segment = 32;
    const int64_t groups = p.dim / 8, items = step ? p.n_seqs : (p.T_tot + segment - 1) / segment + p.n_seqs;
    const int64_t blocks = (items * groups + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const cudaError_t e = step ? launch_dependent(conv_step_kernel<T, K>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, p)
                               : launch_dependent(conv_kernel<T, K>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, p, segment, items);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T>
cudaError_t launch_typed(const ConvParams &p, bool step, cudaStream_t stream) {
    switch (p.kernel) {
        case 2: return launch_k<T, 2>(p, step, stream);
        case 3: return launch_k<T, 3>(p, step, stream);
        default: return launch_k<T, 4>(p, step, stream);
    }
}

}  // namespace

cudaError_t launch_conv(const ConvParams &p, bool step, cudaStream_t stream) {
    return p.dtype == PRECOG_F32 ? launch_typed<float>(p, step, stream) : launch_typed<__nv_bfloat16>(p, step, stream);
}

cudaError_t conv_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_conv_status); }

}  // namespace precog
