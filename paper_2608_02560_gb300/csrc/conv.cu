// The short causal convolution in front of a selective scan, over ragged sequences and for single tokens.
//
//   y[t, d] = act(bias[d] + sum_{j < K} w[d, j] x[t - K + 1 + j, d]),   act = SiLU or none
//
// Inputs before a sequence's first token come from its window, K - 1 rows [oldest .. newest] that the
// sequence's past left (a bank's entry, a table's slot), or are zero. A thread has 16 bytes of channels and rolls
// over a segment of tokens with the last K - 1 inputs in registers, so a row is read once and, at the start
// of a segment, K - 1 rows again. Copies run eight tokens ahead of the arithmetic.
//
// Memory bounds it where there is enough: 557,000 tokens of 256 sequences, 2048 bf16 channels, K = 4 with SiLU (4.57 GB,
// 673 us at the measured copy rate): 670 to 673 us. (1999 us with one token at a time, 798 with four ahead in registers, which
// left room for 16 warps an SM and 32 KB on the way; eight ahead in shared memory are 64 KB.) 96 sequences of up to 200
// tokens (13.2 us): 19.2 us, one round of CTAs with 4 warps a scheduler (20.5 with half the channels a thread and six).
// 64 tokens: 3.3 us.
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
constexpr int kAhead = 8;   // tokens whose loads are in flight together
template <typename T> constexpr int kResident = sizeof(T) == 2 ? 4 : 5;   // CTAs an SM, by their registers

// A thread has the channels of 16 bytes of a row, eight of bf16 or four of fp32, as pairs.
template <typename T> constexpr int kChannels = 16 / static_cast<int>(sizeof(T));
template <typename T>
__device__ __forceinline__ uint4 load16(const T *p) { return *reinterpret_cast<const uint4 *>(p); }
template <typename T>
__device__ __forceinline__ void store16(T *p, const uint4 &q) { *reinterpret_cast<uint4 *>(p) = q; }
template <typename T>
__device__ __forceinline__ void unpack16(const uint4 &q, f2 (&v)[kChannels<T> / 2]) {
    if constexpr (sizeof(T) == 4) {
        v[0] = pack2(__uint_as_float(q.x), __uint_as_float(q.y)), v[1] = pack2(__uint_as_float(q.z), __uint_as_float(q.w));
    } else {
        float e[8];
        unpack(Piece<T, 8>{{q}}, e);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack2(e[2 * i], e[2 * i + 1]);
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack16(const f2 (&v)[kChannels<T> / 2]) {
    float e[kChannels<T>];
#pragma unroll
    for (int i = 0; i < kChannels<T> / 2; ++i) unpack2(v[i], e[2 * i], e[2 * i + 1]);
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(e[0]), __float_as_uint(e[1]), __float_as_uint(e[2]), __float_as_uint(e[3]));
    else return pack(e);
}

template <typename T, int K>
struct Taps {
    static constexpr int C = kChannels<T>, P = C / 2;
    f2 w[K][P], bias[P];
    __device__ __forceinline__ void load(const ConvParams &p, int d) {
        __align__(16) float flat[C * K], b[C] = {};
        const float4 *from = reinterpret_cast<const float4 *>(p.weight + static_cast<int64_t>(d) * K);
#pragma unroll
        for (int i = 0; i < C * K / 4; ++i) *reinterpret_cast<float4 *>(flat + 4 * i) = __ldg(from + i);
        if (p.bias) {
#pragma unroll
            for (int i = 0; i < C / 4; ++i) *reinterpret_cast<float4 *>(b + 4 * i) = __ldg(reinterpret_cast<const float4 *>(p.bias + d) + i);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            bias[i] = pack2(b[2 * i], b[2 * i + 1]);
#pragma unroll
            for (int j = 0; j < K; ++j) w[j][i] = pack2(flat[2 * i * K + j], flat[(2 * i + 1) * K + j]);
        }
    }
    // y of inputs in[0 .. K - 1], oldest first
    __device__ __forceinline__ uint4 out(const f2 (*const (&in)[K])[P], bool act) const {
        f2 y[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            y[i] = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) y[i] = fma2(w[j][i], (*in[j])[i], y[i]);
            if (act) y[i] = silu2<T>(y[i]);
        }
        return pack16<T>(y);
    }
};

// The sequence with base(c) <= item < base(c + 1), by all lanes of a warp: 32 places are looked at together where they
// have one item (two loads one behind the other for 1000 sequences, not ten). Within [0, n_seqs) whatever the offsets.
__device__ __forceinline__ int sequence_of(const ConvParams &p, int64_t item, int segment) {
    int lo = 0, hi = static_cast<int>(p.n_seqs);
    auto begins = [&](int c) { return p.offsets[c] / segment + c <= item; };
    if (__all_sync(0xffffffffu, item == __shfl_sync(0xffffffffu, item, 0))) {
        const int lane = threadIdx.x % 32;
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, mid = lo + step * (lane + 1);
            lo += step * __popc(__ballot_sync(0xffffffffu, mid < hi && begins(mid)));
            hi = min(hi, lo + step);
        }
        return lo;
    }
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (begins(mid)) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename T, int K>
__global__ void __launch_bounds__(kThreads, kResident<T>) conv_kernel(const ConvParams p, int segment, int64_t items) {
    grid_dependency_wait();
    constexpr int C = kChannels<T>;
    const unsigned groups = static_cast<unsigned>(p.dim) / C;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t item = at >> 32 ? at / groups : static_cast<int64_t>(static_cast<unsigned>(at) / groups);
    const int d = static_cast<int>(at - item * groups) * C;
    if (item < p.n_seqs && d == 0) {   // every sequence is looked at, whichever way the search goes
        const int64_t a = p.offsets[item], b = p.offsets[item + 1];
        if (a < 0 || b < a || b > p.T_tot) atomicOr(&g_conv_status, PRECOG_DEV_BAD_OFFSETS);
    }
    const int lo = sequence_of(p, item, segment);
    if (item >= items) return;
    const int64_t c = lo, a = p.offsets[c], b = p.offsets[c + 1];
    if (a < 0 || b < a || b > p.T_tot) return;
    const int64_t part = item - (a / segment + c);
    const int64_t begin = a + part * segment;
    if (part < 0 || begin > b || (begin == b && part > 0)) return;   // (an empty sequence leaves its window all the same)
    const int n = static_cast<int>(begin + segment < b ? segment : b - begin);

    const T *window = nullptr;
    if ((p.bank != nullptr || p.idx != nullptr) && begin - (K - 1) < a) {
        const int64_t row = p.idx ? p.idx[c] : c;
        if (row < -1 || row >= p.bank_entries) {
            if (d == 0 && part == 0) atomicOr(&g_conv_status, PRECOG_DEV_BAD_INDEX);
        } else if (row >= 0) {
            window = static_cast<const T *>(p.bank) + ((row * p.L_total + p.layer) * (K - 1)) * p.dim + d;
        }
    }
    const T *x = static_cast<const T *>(p.x) + begin * p.x_stride + d;
    // where input t of the segment is, which for t < 0 may be the window's (or nowhere: 0)
    auto place = [&](int t) -> const T * {
        const T *w = window == nullptr ? nullptr : window + (begin - a + t + K - 1) * p.dim;
        return begin + t >= a ? x + t * p.x_stride : w;
    };
    // A thread's next kAhead inputs are on their way to its own places in shared memory (registers for them would
    // cost the warps that hide their latency).
    __shared__ uint4 ring[kAhead][kThreads];
    auto fetch = [&](int place, const T *from, bool there) {
        if (there) cp_async16_exact(&ring[place][threadIdx.x], from);
        cp_async_commit();
    };
    uint4 past[K - 1] = {};
#pragma unroll
    for (int u = 0; u < kAhead; ++u) fetch(u, x + u * p.x_stride, u < n);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const T *at_j = place(j - (K - 1));
        if (at_j != nullptr) past[j] = load16(at_j);
    }
    Taps<T, K> taps;
    taps.load(p, d);
    f2 in[K][C / 2];   // input t in place t mod K
#pragma unroll
    for (int j = 1; j < K; ++j) unpack16<T>(past[j - 1], in[j]);
    T *y = static_cast<T *>(p.y) + begin * p.y_stride + d;
    const T *from = x + kAhead * p.x_stride;
    const bool act = p.silu != 0;
    constexpr int kRound = K == 3 ? 6 : 4;   // tokens after which the inputs' places repeat, two at a time
    int slot = 0;
    for (int t = 0; t < n; t += kRound) {
#pragma unroll
        for (int u = 0; u < kRound; u += 2) {
            if (t + u >= n) break;
            cp_async_wait<kAhead - 2>();
            uint4 raw[2];
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                raw[v] = ring[slot + v][threadIdx.x];
                fetch(slot + v, from + v * p.x_stride, t + u + v + kAhead < n);
            }
            slot = (slot + 2) % kAhead;
            from += 2 * p.x_stride;
            uint4 r[2];
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                unpack16<T>(raw[v], in[(u + v) % K]);
                const f2(*of[K])[C / 2];
#pragma unroll
                for (int j = 0; j < K; ++j) of[j] = &in[(u + v + 1 + j) % K];
                r[v] = taps.out(of, act);
            }
            store16(y, r[0]);
            if (t + u + 1 < n) store16(y + p.y_stride, r[1]);
            y += 2 * p.y_stride;
        }
    }
    if (begin + n == b && p.windows != nullptr) {   // the last inputs, as they are stored
        T *out = static_cast<T *>(p.windows) + ((c * p.L_total + p.layer) * (K - 1)) * p.dim + d;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            const T *at_j = place(n - (K - 1) + j);
            store16(out + static_cast<int64_t>(j) * p.dim, at_j != nullptr ? load16(at_j) : uint4{});
        }
    }
}

// One token of each row: a thread has 16 bytes of the rows first, first + stride, ..., whose taps it keeps. Two
// rows are on their way while one is worked on, their slots a round before. 256 rows of 8448 bf16 channels, K = 4 (34.8
// MB, 5.1 us at the measured copy rate): 8.6 us (39 with a row a thread, whose taps are as many bytes as the row's own;
// 9.5 with two rows a thread in 1.7 rounds of CTAs).
template <typename T, int K>
struct StepRow {
    T *window;   // nullptr: idle
    uint4 in[K];
};
template <typename T, int K, int AHEAD>
__global__ void __launch_bounds__(kThreads, kResident<T>) conv_step_kernel(const ConvParams p, int stride) {
    grid_dependency_wait();
    constexpr int C = kChannels<T>;
    const unsigned groups = static_cast<unsigned>(p.dim) / C;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t first = at >> 32 ? at / groups : static_cast<int64_t>(static_cast<unsigned>(at) / groups);
    if (first >= stride) return;
    const int d = static_cast<int>(at - first * groups) * C;
    auto slot_of = [&](int64_t row) -> int64_t { return row >= p.n_seqs ? -1 : p.idx ? p.idx[row] : row; };
    auto load = [&](StepRow<T, K> &r, int64_t row, int64_t slot) {
        r.window = nullptr;
        if (slot < 0 || slot >= p.bank_entries) {
            if (slot != -1 && d == 0) atomicOr(&g_conv_status, PRECOG_DEV_BAD_INDEX);
            return;
        }
        r.window = static_cast<T *>(p.windows) + ((slot * p.L_total + p.layer) * (K - 1)) * p.dim + d;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) r.in[j] = load16(r.window + static_cast<int64_t>(j) * p.dim);
        r.in[K - 1] = load16(static_cast<const T *>(p.x) + row * p.x_stride + d);
    };
    StepRow<T, K> rows[AHEAD];
    int64_t slot[AHEAD];
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) slot[r] = slot_of(first + static_cast<int64_t>(r) * stride);
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) load(rows[r], first + static_cast<int64_t>(r) * stride, slot[r]);
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) slot[r] = slot_of(first + static_cast<int64_t>(AHEAD + r) * stride);
    Taps<T, K> taps;
    taps.load(p, d);
    for (int64_t row0 = first; row0 < p.n_seqs; row0 += static_cast<int64_t>(AHEAD) * stride) {
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            const int64_t row = row0 + static_cast<int64_t>(r) * stride;
            if (row >= p.n_seqs) break;
            uint4 y = {};
            if (rows[r].window != nullptr) {
                f2 in[K][C / 2];
                const f2(*of[K])[C / 2];
#pragma unroll
                for (int j = 0; j < K; ++j) unpack16<T>(rows[r].in[j], in[j]), of[j] = &in[j];
                y = taps.out(of, p.silu != 0);
#pragma unroll
                for (int j = 0; j < K - 1; ++j) store16(rows[r].window + static_cast<int64_t>(j) * p.dim, rows[r].in[j + 1]);
            }
            store16(static_cast<T *>(p.y) + row * p.y_stride + d, y);
            load(rows[r], row + static_cast<int64_t>(AHEAD) * stride, slot[r]);
            slot[r] = slot_of(row + static_cast<int64_t>(2 * AHEAD) * stride);
        }
    }
}

template <typename T, int K>
cudaError_t launch_k(const ConvParams &p, bool step, cudaStream_t stream) {
    const int64_t groups = p.dim / kChannels<T>, fill = static_cast<int64_t>(device_sm_count()) * kResident<T> * kThreads;
    cudaError_t e;
    auto go = [&](auto kernel, int64_t threads, auto... more) {
        const int64_t blocks = (threads + kThreads - 1) / kThreads;
        if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
        return launch_dependent(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, p, more...);
    };
    if (step) {
        // A row a thread where that fits the GPU at once; otherwise as many threads as do.
        const int64_t at_once = fill / groups < 1 ? 1 : fill / groups;
        if (p.n_seqs <= at_once) e = go(conv_step_kernel<T, K, 1>, p.n_seqs * groups, static_cast<int>(p.n_seqs));
        else e = go(conv_step_kernel<T, K, 2>, at_once * groups, static_cast<int>(at_once));
    } else {
        // As long as the segments fit the GPU at once, with half of one left over a sequence; at most 64 tokens, from
        // where on what a segment's start costs no longer counts (us for 557,000 tokens of 256 sequences, 2048 channels,
        // segments of 16, 32, 64, 128: 933, 727, 672, 674).
        const int64_t at_once = fill / groups - p.n_seqs / 2;
        const int64_t tokens = at_once > 0 ? (p.T_tot + at_once - 1) / at_once : 64;
        const int segment = tokens >= 64 ? 64 : tokens < 4 ? 4 : static_cast<int>((tokens + 3) / 4 * 4);
        const int64_t items = (p.T_tot + segment - 1) / segment + p.n_seqs;
        e = go(conv_kernel<T, K>, items * groups, segment, items);
    }
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
