// Logits before a token is chosen: penalties for tokens that the text has already, biases, grammar masks.
//
//   z = x ;  seen:  z <- z > 0 ? z / repetition : z repetition
//   n = times in the counted part > 0:  z <- z - n frequency - presence
//   biased:  z <- z + bias ;  not allowed by the mask:  z <- -infinity
//
// A CTA has a slice of one row's vocabulary. It asks for the slice's logits, counts the slice's tokens of the
// row's history in shared memory meanwhile (a word a token: seen, biased, and the count; integer atomics, so
// the order does not matter), and passes over the logits once, 16 bytes of output at a time. Rows of any
// alignment: a 16-byte piece of output is cut from the two pieces of input that it lies in. Most pieces have
// no token of the history, and only their mask is looked at.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_adjust_status;

constexpr int kThreads = 256;
constexpr uint32_t kSeen = 0x80000000u, kBiased = 0x40000000u, kCount = 0x3fffffffu;   // (lists are shorter than 2^30)
constexpr int kShortList = 128;   // biases that are looked through where a token is biased

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

// 16 bytes that begin `shift` bytes (even) into the 32 of a and b.
__device__ __forceinline__ uint4 cut(const uint4 &a, const uint4 &b, int shift) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (shift & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (shift & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const int bits = (shift & 2) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Row {
    float rep, freq, pres;
    bool penalised;
    int64_t first, n;          // its biases
    const int64_t *bias_idx;
    const float *bias;
};

// z of a token with word `n`
__device__ __forceinline__ float adjusted(float z, uint32_t n, const Row &row, int token, const uint32_t *last) {
    if ((n & (kSeen | kCount)) != 0 && row.penalised) z = z > 0.f ? z / row.rep : z * row.rep;
    if ((n & kCount) != 0) z = z - row.freq * static_cast<float>(n & kCount) - row.pres;
    if ((n & kBiased) != 0) {
        if (last != nullptr) return z + row.bias[row.first + *last - 1];
        for (int64_t j = row.n - 1; j >= 0; --j)
            if (row.bias_idx[row.first + j] == token) return z + row.bias[row.first + j];
    }
    return z;
}

// PIECES 16-byte pieces a thread and slice. LIST: there are histories or biases.
template <typename T, int PIECES, bool LIST>
__global__ void __launch_bounds__(kThreads, 4) adjust_kernel(const AdjustParams p, unsigned slices) {
    grid_dependency_wait();
    constexpr int sz = static_cast<int>(sizeof(T)), E = 16 / sz, kSlice = kThreads * PIECES * E, kHalf = kSlice / 2;
    extern __shared__ uint4 raw[];                            // the slice's logits, in the input's pieces
    uint32_t *const words = reinterpret_cast<uint32_t *>(raw + kThreads * PIECES + 1);
    __shared__ uint32_t allowed[kSlice / 32 + 1];             // its mask
    const int64_t r = blockIdx.x / slices;
    const int vocab = static_cast<int>(p.vocab), lo = static_cast<int>(blockIdx.x % slices) * kSlice, hi = min(vocab, lo + kSlice);
    const bool first_slice = lo == 0, flag = first_slice && threadIdx.x == 0;
    const T *const x = static_cast<const T *>(p.logits) + r * p.stride;
    T *const out = static_cast<T *>(p.out) + r * p.out_stride;
    // pieces of output begin at `head`; tokens [lo, head) and those behind the last whole piece go one by one
    const int head = min(hi, lo + ((16 - static_cast<int>(reinterpret_cast<uintptr_t>(out + lo) & 15)) & 15) / sz);
    const int pieces = (hi - head) / E;
    const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(x + head) & 15), before = shift / sz;
    for (int k = threadIdx.x; k < pieces + (shift != 0); k += kThreads) {
        const int e = head - before + k * E;
        if (e >= 0 && e + E <= vocab) {
            cp_async16(&raw[k], x + e);
        } else {   // at the row's ends nothing beside it is read
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (e + i >= 0 && e + i < vocab) reinterpret_cast<T *>(&raw[k])[i] = x[e + i];
        }
    }
    bool masked = false;
    if (p.mask || p.mask_rows) {
        const int64_t m = p.mask_rows ? p.mask_rows[r] : r;
        masked = m >= 0 && m < p.n_masks;
        if (!masked && m != -1 && flag) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
        const int n_words = (vocab + 31) / 32;
        if (masked) {
            for (int i = threadIdx.x; i < kSlice / 32 + 1; i += kThreads)
                if (lo / 32 + i < n_words) allowed[i] = p.mask[m * n_words + lo / 32 + i];
        }
    }

    Row row = {};
    int64_t ha = 0, hb = 0, from = 0;
    if constexpr (LIST) {
        if (p.history) {
            list_of(p.history_offsets, r, p.n_history, flag, ha, hb);
            from = ha + (p.count_from ? min(hb - ha, max(static_cast<int64_t>(0), p.count_from[r])) : 0);
            row.penalised = p.repetition != nullptr;
            row.rep = p.repetition ? p.repetition[r] : 1.f, row.freq = p.frequency ? p.frequency[r] : 0.f;
            row.pres = p.presence ? p.presence[r] : 0.f;
        }
        if (p.bias) {
            int64_t b;
            list_of(p.bias_offsets, r, p.n_bias, flag, row.first, b);
            row.n = b - row.first;
            row.bias_idx = p.bias_idx, row.bias = p.bias;
        }
    }
    // With a long list of biases half of the words hold the biased tokens' last places, and the slice goes in halves.
    const bool places = LIST && row.n > kShortList;
    for (int half = 0; half < (places ? 2 : 1); ++half) {
        const int begin = half == 0 ? lo : min(hi, head + kHalf), end = places && half == 0 ? min(hi, head + kHalf) : hi;
        const int place = E - half * kHalf - head;   // token i's word is words[place + i]; a piece's are 16-byte aligned
        if constexpr (LIST) {
            if (half != 0) __syncthreads();
            for (int i = threadIdx.x; i < (kSlice + 2 * E) / 4; i += kThreads) reinterpret_cast<uint4 *>(words)[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            constexpr int kAtOnce = 8;
            for (int64_t j0 = ha + threadIdx.x; j0 < hb; j0 += kAtOnce * kThreads) {
                int64_t tok[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) tok[k] = j0 + k * kThreads < hb ? p.history[j0 + k * kThreads] : -1;
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (tok[k] >= begin && tok[k] < end) {
                        uint32_t *w = words + (place + static_cast<int>(tok[k]));
                        if (j0 + k * kThreads < from) atomicOr(w, kSeen);
                        else atomicAdd(w, 1u);
                    } else if (first_slice && (tok[k] < -1 || tok[k] >= vocab)) {
                        atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
                    }
                }
            }
            for (int64_t j = threadIdx.x; j < row.n; j += kThreads) {
                const int64_t tok = row.bias_idx[row.first + j];
                if (tok >= begin && tok < end) {
                    uint32_t *w = words + (place + static_cast<int>(tok));
                    atomicOr(w, kBiased);
                    if (places) atomicMax(w + kHalf + E, static_cast<uint32_t>(j) + 1u);
                } else if (first_slice && (tok < -1 || tok >= vocab)) {
                    atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
                }
            }
        }
        if (half == 0) {
            cp_async_commit();
            cp_async_wait<0>();
        }
        __syncthreads();
        auto finish = [&](int i, T v, bool may) {
            if constexpr (LIST) {
                const uint32_t *w = words + (place + i);
                if (*w != 0) v = stored<T>(adjusted(to_f32(v), *w, row, i, places ? w + kHalf + E : nullptr));
            }
            return may ? v : stored<T>(__int_as_float(0xff800000));
        };
        for (int k = threadIdx.x; k < pieces; k += kThreads) {
            const int e = head + k * E;
            if (e < begin || e >= end) continue;
            const uint4 q = shift == 0 ? raw[k] : cut(raw[k], raw[k + 1], shift);
            uint32_t may = 0xffffffffu;   // (the low E bits; one word twice: its bits are the low ones)
            if (masked) may = __funnelshift_r(allowed[(e - lo) >> 5], allowed[(e - lo + E - 1) >> 5], (e - lo) & 31);
            uint32_t any = 0;
            if constexpr (LIST) {
#pragma unroll
                for (int i = 0; i < E / 4; ++i) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(words + (place + e) + 4 * i);
                    any |= w.x | w.y | w.z | w.w;
                }
            }
            T v[E];
            memcpy(v, &q, 16);
            if (any == 0) {
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] = (may >> i) & 1u ? v[i] : stored<T>(__int_as_float(0xff800000));
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] = finish(e + i, v[i], (may >> i) & 1u);
            }
            uint4 o;
            memcpy(&o, v, 16);
            *reinterpret_cast<uint4 *>(out + e) = o;
        }
        if (threadIdx.x < 2 * E) {   // the ends
            const int at = static_cast<int>(threadIdx.x) % E;
            const int i = threadIdx.x < E ? lo + at : head + pieces * E + at;
            if (i < (threadIdx.x < E ? head : hi) && i >= begin && i < end)
                out[i] = finish(i, x[i], !masked || ((allowed[(i - lo) >> 5] >> ((i - lo) & 31)) & 1u) != 0);
        }
    }
}

template <typename T, int PIECES, bool LIST>
cudaError_t launch_pieces(const AdjustParams &p, cudaStream_t stream) {
    constexpr int E = 16 / static_cast<int>(sizeof(T)), kSlice = kThreads * PIECES * E;
    constexpr int kBytes = 16 * (kThreads * PIECES + 1) + (LIST ? 4 * (kSlice + 2 * E) : 0);
    const int64_t slices = (p.vocab + kSlice - 1) / kSlice, blocks = p.rows * slices;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    cudaError_t e = ensure_smem(reinterpret_cast<const void *>(adjust_kernel<T, PIECES, LIST>), kBytes);
    if (e != cudaSuccess) return e;
    e = launch_dependent(adjust_kernel<T, PIECES, LIST>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), kBytes, stream, p,
                         static_cast<unsigned>(slices));
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T>
cudaError_t launch_typed(const AdjustParams &p, cudaStream_t stream) {
    const bool many = p.rows * p.vocab * static_cast<int64_t>(sizeof(T)) >= static_cast<int64_t>(device_sm_count()) * kThreads * 16 * 4;
    if (p.history || p.bias) return many ? launch_pieces<T, 4, true>(p, stream) : launch_pieces<T, 1, true>(p, stream);
    return many ? launch_pieces<T, 4, false>(p, stream) : launch_pieces<T, 1, false>(p, stream);
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
