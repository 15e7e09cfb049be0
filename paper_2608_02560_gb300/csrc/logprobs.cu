// Log probabilities of given tokens, the entropy of their distribution and the k best entries,
// in one pass over the logits.
//
// With z = x / temperature, m = max z, d_i = z_i - m:
//   S = sum e^{d_i},  W = sum d_i e^{d_i}
//   log p(token) = d_token - log S,   H = log S - W / S.
// Every thread keeps (m, S, W) of what it has seen; when its maximum grows by c, S becomes
// S e^-c and W becomes (W - c S) e^-c, and two threads' sums join the same way. The maximum
// is tracked on x itself, and d is formed as (x - max x) / temperature: no product overflows
// where the logits are the type's lowest value, and equal logits differ by exactly 0.
// Exponentials below 2^-150 of the largest count as zero, -infinity among them.
#include <climits>

#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_logprob_status;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFloor = -150.f;      // exponents below it count as e^d = 0
using u64 = unsigned long long;

// Maximum and sums of a thread, in units of log2 for d.
struct Sums {
    float mx, s, w;
};

__device__ __forceinline__ float clamped(float d) {
    float r;   // NaN stays NaN
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(d), "f"(kFloor));
    return r;
}

// The sums seen from the maximum `mx` >= a.mx. c: log2(e) / temperature.
__device__ __forceinline__ Sums moved(const Sums a, float mx, float c) {
    if (mx == a.mx) return a;
    const float d = clamped((a.mx - mx) * c), f = ex2(d);
    return Sums{mx, a.s * f, fmaf(d, a.s, a.w) * f};
}
__device__ __forceinline__ Sums joined(const Sums a, const Sums b, float c) {
    const float mx = fmaxf(a.mx, b.mx);
    const Sums x = moved(a, mx, c), y = moved(b, mx, c);
    return Sums{mx, x.s + y.s, x.w + y.w};
}

// Ordered bits of a comparable value above, the complement of the index below: larger keys come
// first, ties go to the lower index. 0: nothing (NaN has no key).
__device__ __forceinline__ u64 key_of(float x, uint32_t index) {
    if (isnan(x)) return 0ull;
    const uint32_t u = __float_as_uint(x + 0.0f);
    const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return (static_cast<u64>(o) << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ float value_of(u64 key) {
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

// Insert `v` (the same in every lane) into the warp's descending list, lane i's entry the i-th.
__device__ __forceinline__ void insert(u64 &mine, u64 v, int lane) {
    const int at = __popc(__ballot_sync(0xffffffffu, mine > v));
    const u64 up = __shfl_up_sync(0xffffffffu, mine, 1);
    mine = lane < at ? mine : lane == at ? v : up;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const LogprobParams p) {
    __shared__ Sums warp_sums[kWarps];
    __shared__ u64 lists[kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(p.logits) + row * p.stride;
    const float c = p.inv_temp * kLog2e;
    const int vocab = static_cast<int>(p.vocab);
    Sums a{kLowest, 0.f, 0.f};
    u64 mine = 0ull, least = 0ull;     // the warp's list and its k-th entry
    for (int i0 = warp * 32; i0 < vocab; i0 += kThreads) {
        const int i = i0 + lane;
        const bool in = i < vocab;
        const float v = in ? to_f32(x[i]) : -__int_as_float(0x7f800000);
        if (v > a.mx) a = moved(a, v, c);
        const float d = clamped((v - a.mx) * c), e = ex2(d);
        a.s += e;
        a.w = fmaf(d, e, a.w);
        if (p.k > 0) {
            const u64 key = in ? key_of(v, static_cast<uint32_t>(i)) : 0ull;
            unsigned todo = __ballot_sync(0xffffffffu, key > least);
            while (todo) {
                const int from = __ffs(static_cast<int>(todo)) - 1;
                todo &= todo - 1;
                const u64 one = __shfl_sync(0xffffffffu, key, from);
                if (one > least) {
                    insert(mine, one, lane);
                    least = __shfl_sync(0xffffffffu, mine, p.k - 1);
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Sums b{__shfl_xor_sync(0xffffffffu, a.mx, o), __shfl_xor_sync(0xffffffffu, a.s, o),
                     __shfl_xor_sync(0xffffffffu, a.w, o)};
        a = joined(a, b, c);
    }
    if (lane == 0) warp_sums[warp] = a;
    lists[warp][lane] = mine;
    __syncthreads();
    if (warp != 0) return;
    a = warp_sums[0];
    for (int w = 1; w < kWarps; ++w) a = joined(a, warp_sums[w], c);
    const float nan = __int_as_float(0x7fffffff);
    const float log_s = log2f(a.s);                        // NaN where the row holds one
    const bool empty = a.s == 0.f;
    if (lane == 0) {
        const int64_t token = p.tokens[row];
        float lp = 0.f;
        if (token >= 0 && token < p.vocab) {
            const float v = to_f32(x[token]);
            lp = empty ? nan : (v - a.mx) * p.inv_temp - log_s * kLn2;
        } else if (token != -1) {
            atomicOr(&g_logprob_status, PRECOG_DEV_BAD_INDEX);
            lp = nan;
        }
        p.logprob[row] = lp;
        if (p.entropy) p.entropy[row] = empty ? nan : (log_s - a.w / a.s) * kLn2;
    }
    if (p.k > 0) {
        for (int w = 1; w < kWarps; ++w)
            for (int j = 0; j < p.k; ++j) {
                const u64 one = lists[w][j];
                if (one <= least) break;                   // sorted: nothing better follows
                insert(mine, one, lane);
                least = __shfl_sync(0xffffffffu, mine, p.k - 1);
            }
        if (lane < p.k) {
            const bool some = mine != 0ull;
            p.top_idx[row * p.k + lane] = some ? static_cast<int64_t>(0xffffffffu - static_cast<uint32_t>(mine)) : -1;
            p.top_logprob[row * p.k + lane] = some && !empty ? (value_of(mine) - a.mx) * p.inv_temp - log_s * kLn2 : nan;
        }
    }
}

template <typename T>
cudaError_t launch_typed(const LogprobParams &p, cudaStream_t stream) {
    logprobs_kernel<T><<<static_cast<unsigned>(p.rows), kThreads, 0, stream>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launches(1);
    return e;
}

}  // namespace

cudaError_t launch_logprobs(const LogprobParams &p, cudaStream_t stream) {
    switch (p.dtype) {
        case PRECOG_F32: return launch_typed<float>(p, stream);
        case PRECOG_F16: return launch_typed<__half>(p, stream);
        default: return launch_typed<__nv_bfloat16>(p, stream);
    }
}

cudaError_t logprobs_status_word_read_clear(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_logprob_status, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_logprob_status, &zero, sizeof(uint32_t));
}

}  // namespace precog
