// Logits before a token is chosen: penalties for tokens that the text has already, biases, grammar masks.
//
//   z = x ;  seen:  z <- z > 0 ? z / repetition : z repetition
//   n = times in the counted part > 0:  z <- z - n frequency - presence
//   biased:  z <- z + bias ;  not allowed by the mask:  z <- -infinity
//
// A CTA has a slice of one row's vocabulary. It copies the slice's logits to shared memory and meanwhile counts
// the slice's tokens of the row's history there (a word a token: seen, biased, and the count; integer atomics,
// so the order does not matter). The first to count a token lists it; the listed tokens' logits are then
// adjusted where they lie, a thread each, so that a few tokens do not hold up the many. What is left is a copy
// with the mask, 16 bytes of output at a time. Rows of any alignment: a piece of output is cut from the two
// pieces of input that it lies in.
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

// 16 bytes that begin `shift` bytes (even, the same for all) into the 32 of a and b.
__device__ __forceinline__ uint4 cut(const uint4 &a, const uint4 &b, int shift) {
    const int bits = (shift & 2) * 8;
    auto words = [&](uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t w4) {
        return make_uint4(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits), __funnelshift_r(w2, w3, bits),
                          __funnelshift_r(w3, w4, bits));
    };
    switch (shift / 4) {
        case 0: return words(a.x, a.y, a.z, a.w, b.x);
        case 1: return words(a.y, a.z, a.w, b.x, b.y);
        case 2: return words(a.z, a.w, b.x, b.y, b.z);
        default: return words(a.w, b.x, b.y, b.z, b.w);
    }
}

struct Row {
    float rep, freq, pres;
    bool penalised;
    int64_t first, n;          // its biases
    const int64_t *bias_idx;
    const float *bias;
};

// z of a token with word `n`; `last`: 1 + the place of its bias, if that is known
__device__ __forceinline__ float adjusted(float z, uint32_t n, const Row &row, int token, uint32_t last) {
    if ((n & (kSeen | kCount)) != 0 && row.penalised) z = z > 0.f ? z / row.rep : z * row.rep;
    if ((n & kCount) != 0) z = z - row.freq * static_cast<float>(n & kCount) - row.pres;
    if ((n & kBiased) != 0) {
        if (last != 0) return z + row.bias[row.first + last - 1];
        for (int64_t j = row.n - 1; j >= 0; --j)
            if (row.bias_idx[row.first + j] == token) return z + row.bias[row.first + j];
    }
    return z;
}

// 32 bits, each a 16-bit half's or (WIDE) a whole word's: words i, as masks
template <bool WIDE>
__device__ __forceinline__ uint32_t mask_of(uint32_t bits, int i) {
    if constexpr (WIDE) return (bits >> i) & 1u ? 0xffffffffu : 0u;
    return ((bits >> (2 * i)) & 1u ? 0xffffu : 0u) | ((bits >> (2 * i)) & 2u ? 0xffff0000u : 0u);
}
template <typename T> constexpr uint32_t kBanned = 0xff80ff80u;   // -infinity, twice where it is a half
template <> constexpr uint32_t kBanned<__half> = 0xfc00fc00u;
template <> constexpr uint32_t kBanned<float> = 0xff800000u;

// PIECES 16-byte pieces a thread and slice. LIST: there are histories or biases.
template <typename T, int PIECES, bool LIST>
__global__ void __launch_bounds__(kThreads, LIST ? 4 : 1) adjust_kernel(const AdjustParams p, unsigned slices) {
    grid_dependency_wait();
    constexpr int sz = static_cast<int>(sizeof(T)), E = 16 / sz, kSlice = kThreads * PIECES * E, kHalf = kSlice / 2;
    constexpr int kTouched = kSlice / 4;                      // tokens that are listed; more are found by their words
    extern __shared__ uint4 raw[];                            // the slice's logits, in the input's pieces
    uint32_t *const words = reinterpret_cast<uint32_t *>(raw + kThreads * PIECES + 1);
    uint16_t *const touched = reinterpret_cast<uint16_t *>(words + kSlice);
    __shared__ uint32_t allowed[kSlice / 32 + 1], n_touched;  // its mask
    const int64_t r = blockIdx.x / slices;
    const int vocab = static_cast<int>(p.vocab), lo = static_cast<int>(blockIdx.x % slices) * kSlice, hi = min(vocab, lo + kSlice);
    const bool first_slice = lo == 0, flag = first_slice && threadIdx.x == 0;
    const T *const x = static_cast<const T *>(p.logits) + r * p.stride;
    T *const out = static_cast<T *>(p.out) + r * p.out_stride;
    // token i is logit `before` + i - lo of `raw`
    const int before = static_cast<int>(reinterpret_cast<uintptr_t>(x + lo) & 15) / sz;
    for (int k = threadIdx.x; k * E < before + hi - lo; k += kThreads) {
        const int e = lo - before + k * E;
        if (e >= 0 && e + E <= vocab) {
            cp_async16(&raw[k], x + e);
        } else {   // at the row's ends nothing beside it is read
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (e + i >= 0 && e + i < vocab) reinterpret_cast<T *>(&raw[k])[i] = x[e + i];
        }
    }
    cp_async_commit();
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

    if constexpr (LIST) {
        Row row = {};
        int64_t ha = 0, hb = 0, from = 0;
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
        // With a long list of biases half of the words hold the biased tokens' last places, and the slice goes in halves.
        const bool places = row.n > kShortList;
        for (int begin = lo; begin < hi; begin += places ? kHalf : kSlice) {
            const unsigned size = static_cast<unsigned>(min(hi - begin, places ? kHalf : kSlice));
            for (int i = threadIdx.x; i < kSlice / 4; i += kThreads) reinterpret_cast<uint4 *>(words)[i] = make_uint4(0, 0, 0, 0);
            if (threadIdx.x == 0) n_touched = 0;
            __syncthreads();
            auto touch = [&](unsigned i, uint32_t was) {   // the first to come lists the token
                if (was == 0) {
                    const uint32_t at = atomicAdd(&n_touched, 1u);
                    if (at < kTouched) touched[at] = static_cast<uint16_t>(i);
                }
            };
            auto check = [&](int64_t tok) {
                if (first_slice && (tok < -1 || tok >= vocab)) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
            };
            constexpr int kAtOnce = 8;
            for (int64_t j0 = ha + threadIdx.x; j0 < hb; j0 += kAtOnce * kThreads) {
                int64_t tok[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) tok[k] = j0 + k * kThreads < hb ? p.history[j0 + k * kThreads] : -1;
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const uint64_t i = static_cast<uint64_t>(tok[k] - begin);
                    if (i < size) touch(static_cast<unsigned>(i), j0 + k * kThreads < from ? atomicOr(&words[i], kSeen) : atomicAdd(&words[i], 1u));
                    else check(tok[k]);
                }
            }
            for (int64_t j = threadIdx.x; j < row.n; j += kThreads) {
                const int64_t tok = row.bias_idx[row.first + j];
                const uint64_t i = static_cast<uint64_t>(tok - begin);
                if (i < size) {
                    touch(static_cast<unsigned>(i), atomicOr(&words[i], kBiased));
                    if (places) atomicMax(&words[kHalf + i], static_cast<uint32_t>(j) + 1u);
                } else {
                    check(tok);
                }
            }
            cp_async_wait<0>();
            __syncthreads();
            auto put = [&](unsigned i) {
                T *v = reinterpret_cast<T *>(raw) + before + (begin - lo) + i;
                *v = stored<T>(adjusted(to_f32(*v), words[i], row, begin + static_cast<int>(i), places ? words[kHalf + i] : 0u));
            };
            if (n_touched <= kTouched) {
                for (unsigned k = threadIdx.x; k < n_touched; k += kThreads) put(touched[k]);
            } else {
                for (unsigned i = threadIdx.x; i < size; i += kThreads)
                    if (words[i] != 0) put(i);
            }
            __syncthreads();
        }
    } else {
        cp_async_wait<0>();
        __syncthreads();
    }

    // tokens [lo, head) and those behind the last whole piece of output go one by one
    const int head = min(hi, lo + ((16 - static_cast<int>(reinterpret_cast<uintptr_t>(out + lo) & 15)) & 15) / sz);
    const int pieces = (hi - head) / E, skew = (before + head - lo) * sz, shift = skew & 15;
    const uint4 *const from = raw + skew / 16;
    for (int k = threadIdx.x; k < pieces; k += kThreads) {
        const int e = head + k * E;
        const uint4 q = shift == 0 ? from[k] : cut(from[k], from[k + 1], shift);
        uint32_t w[4] = {q.x, q.y, q.z, q.w};
        if (masked) {   // (one word twice: its bits are the low ones)
            const uint32_t may = __funnelshift_r(allowed[(e - lo) >> 5], allowed[(e - lo + E - 1) >> 5], (e - lo) & 31);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t m = mask_of<sizeof(T) == 4>(may, i);
                w[i] = (w[i] & m) | (kBanned<T> & ~m);
            }
        }
        *reinterpret_cast<uint4 *>(out + e) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (threadIdx.x < 2 * E) {   // the ends
        const int at = static_cast<int>(threadIdx.x) % E;
        const int i = threadIdx.x < E ? lo + at : head + pieces * E + at;
        if (i < (threadIdx.x < E ? head : hi)) {
            const bool may = !masked || ((allowed[(i - lo) >> 5] >> ((i - lo) & 31)) & 1u) != 0;
            out[i] = may ? reinterpret_cast<const T *>(raw)[before + i - lo] : stored<T>(__int_as_float(0xff800000));
        }
    }
}

template <typename T, int PIECES, bool LIST>
cudaError_t launch_pieces(const AdjustParams &p, cudaStream_t stream) {
    constexpr int kSlice = kThreads * PIECES * 16 / static_cast<int>(sizeof(T));
    constexpr int kBytes = 16 * (kThreads * PIECES + 1) + (LIST ? 4 * kSlice + 2 * (kSlice / 4) : 0);
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
