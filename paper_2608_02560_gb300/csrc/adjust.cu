// Logits before a token is chosen: penalties for tokens that the text has already, biases, grammar masks.
//
//   z = x ;  seen:  z <- z > 0 ? z / repetition : z repetition
//   n = times in the counted part > 0:  z <- z - n frequency - presence
//   biased:  z <- z + bias ;  not allowed by the mask:  z <- -infinity
//
// Most logits are copied with their mask and no more: 16 bytes of output at a time, rows of any alignment (a piece of
// output is cut from the two pieces of input that it lies in). The tokens of the row's history and its biased ones
// are few. They are counted in a table in shared memory (a word a token: seen, biased, and the count, and the place
// of its last bias; integer atomics, so their order does not matter), and then the table's tokens are adjusted and put
// over the copy. In place that is the same: the copy leaves an allowed logit as it was, and a banned one needs none.
// Few logits: one launch; a CTA has 2048 tokens of a row and a word for each. Many: a copy, and a launch behind it whose
// CTAs count whole rows in a hash table, instead of every slice's going through the row's history. Where that table is
// too small, its tokens are taken 8192 at a time, with a word for each, and the row's lists are read again each time: a
// cliff. The rows below with one history alone, of 4000 different tokens: 43 us, of 8000 180, of 20,000 375, of 100,000
// 1600 (256 such histories of 4000 53, of 8000 221, of 20,000 478).
//
// Memory bounds the copy, latency the rest. 256 rows of 128,001 bf16 logits, up to 4096 tokens of history, 16 biases,
// masks that allow a tenth (136 MB, 20.0 us at the measured copy rate): 36.7 us; the copy alone 24.4, without masks
// 22.1. Before: a CTA a slice with a word a token, 240 us (logits one by one), 66 (16 bytes, eight at once looked up
// where one had a word), 55 (with the listed ones apart, whether in the same warps or in others: every slice pays for
// the way from offsets through history and table to scattered logits). A copy by resident CTAs, to make room for the
// second launch's beside it, took 47; with the shared memory for both set aside it loses the L1 that it cuts from.
#include <cstddef>
#include <type_traits>

#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_adjust_status;

constexpr int kThreads = 256;        // of a copy
constexpr uint32_t kSeen = 0x80000000u, kBiased = 0x40000000u, kCount = 0x3fffffffu;   // (lists are shorter than 2^30)
constexpr int kProbes = 64;          // places that the hash table looks at for a token

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
    int64_t begin, end, from;  // its history, and where the counted part begins
};

// z of a token with word `n`; `last`: 1 + the place of its bias
__device__ __forceinline__ float adjusted(float z, uint32_t n, const Row &row, const float *bias, uint32_t last) {
    if ((n & (kSeen | kCount)) != 0 && row.penalised) z = z > 0.f ? z / row.rep : z * row.rep;
    if ((n & kCount) != 0) z = z - row.freq * static_cast<float>(n & kCount) - row.pres;
    return (n & kBiased) != 0 ? z + bias[row.first + last - 1] : z;
}

// Word i of a piece whose entries' bits these are, as a mask: all ones where a bit is set (16-bit entries: a half each).
template <bool WIDE>
__device__ __forceinline__ uint32_t mask_of(uint32_t bits, int i) {
    if constexpr (WIDE) return (bits >> i) & 1u ? 0xffffffffu : 0u;
    // the two bits go to the tops of bytes 0 and 1, which prmt then spreads over a half each
    const uint32_t tops = ((bits >> (2 * i)) & 3u) * 0x4080u;
    uint32_t m;
    asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(m) : "r"(tops));
    return m;
}
template <typename T> constexpr uint32_t kBanned = 0xff80ff80u;   // -infinity, twice where it is a half
template <> constexpr uint32_t kBanned<__half> = 0xfc00fc00u;
template <> constexpr uint32_t kBanned<float> = 0xff800000u;

__device__ __forceinline__ bool allows(const uint32_t *mask, int i) { return mask == nullptr || ((mask[i >> 5] >> (i & 31)) & 1u) != 0; }

// Tokens [begin, end) of a row, with -infinity where its mask (or nullptr) says so.
template <typename T>
__device__ __forceinline__ void copy_range(const T *x, T *out, int begin, int end, int vocab, const uint32_t *mask) {
    constexpr int sz = static_cast<int>(sizeof(T)), E = 16 / sz, kAtOnce = 4;
    const int head = min(end, begin + ((16 - static_cast<int>(reinterpret_cast<uintptr_t>(out + begin) & 15)) & 15) / sz);
    const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(x + head) & 15), before = shift / sz;
    // pieces whose two pieces of input are the row's own; nothing beside the row is read
    int first = 0, last = (end - head) / E;
    if (shift != 0) {
        first = head < before ? min(1, last) : 0;
        last = max(first, min(last, (vocab - head + before) / E - 1));
    }
    const uint4 *const from = reinterpret_cast<const uint4 *>(x + head - before);
    uint4 *const to = reinterpret_cast<uint4 *>(out + head);
    for (int k0 = first + static_cast<int>(threadIdx.x); k0 < last; k0 += kAtOnce * kThreads) {
        uint4 a[kAtOnce], b[kAtOnce];
        uint32_t low[kAtOnce], high[kAtOnce];   // (of one word twice the bits are the low ones)
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int k = k0 + u * kThreads, e = head + k * E;
            if (k < last) a[u] = from[k];
            if (k < last && shift != 0) b[u] = from[k + 1];
            if (k < last && mask != nullptr) low[u] = mask[e >> 5], high[u] = mask[(e + E - 1) >> 5];
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int k = k0 + u * kThreads;
            if (k >= last) break;
            const uint4 q = shift == 0 ? a[u] : cut(a[u], b[u], shift);
            uint32_t w[4] = {q.x, q.y, q.z, q.w};
            if (mask != nullptr) {
                const uint32_t may = __funnelshift_r(low[u], high[u], (head + k * E) & 31);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t m = mask_of<sizeof(T) == 4>(may, i);
                    w[i] = (w[i] & m) | (kBanned<T> & ~m);
                }
            }
            to[k] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // what is left at the ends: fewer than two pieces each
    const int t = static_cast<int>(threadIdx.x), i = t < 2 * E ? begin + t : head + last * E + t - 2 * E;
    if (t < 4 * E && i < (t < 2 * E ? head + first * E : end))
        out[i] = allows(mask, i) ? x[i] : stored<T>(__int_as_float(0xff800000));
}

__device__ __forceinline__ const uint32_t *mask_of_row(const AdjustParams &p, int64_t r, bool flag) {
    if (!p.mask && !p.mask_rows) return nullptr;
    const int64_t m = p.mask_rows ? p.mask_rows[r] : r;
    if (m >= 0 && m < p.n_masks) return p.mask + m * ((p.vocab + 31) / 32);
    if (m != -1 && flag) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
    return nullptr;
}

// SLOTS tokens of a row at once, or, with HASH, the listed ones of any range. The biases' places only where there are any.
template <int SLOTS, bool HASH>
struct Tables {
    uint32_t word[SLOTS];
    uint32_t token[HASH ? SLOTS : 4];   // + 1; 0: free
    uint32_t last[SLOTS];
    static constexpr int bytes(bool biases) { return static_cast<int>(biases ? sizeof(Tables) : offsetof(Tables, last)); }
};

// Listed and biased tokens of [lo, hi) of row r. `before_writing` is called once, when nothing has been written yet.
template <typename T, int SLOTS, bool HASH, int THREADS, typename Wait>
__device__ __forceinline__ void adjust_range(const AdjustParams &p, Tables<SLOTS, HASH> &sh, int64_t r, int lo, int hi, Wait before_writing) {
    const int vocab = static_cast<int>(p.vocab);
    const bool flag = lo == 0 && threadIdx.x == 0;
    Row row = {};
    if (p.history) {
        list_of(p.history_offsets, r, p.n_history, flag, row.begin, row.end);
        row.from = row.begin + (p.count_from ? min(row.end - row.begin, max(static_cast<int64_t>(0), p.count_from[r])) : 0);
        row.penalised = p.repetition != nullptr;
        row.rep = p.repetition ? p.repetition[r] : 1.f, row.freq = p.frequency ? p.frequency[r] : 0.f;
        row.pres = p.presence ? p.presence[r] : 0.f;
    }
    if (p.bias) {
        int64_t b;
        list_of(p.bias_offsets, r, p.n_bias, flag, row.first, b);
        row.n = b - row.first;
    }
    auto clear = [&](bool hash) {
        for (int i = threadIdx.x; i < SLOTS / 4; i += THREADS) {
            reinterpret_cast<uint4 *>(sh.word)[i] = make_uint4(0, 0, 0, 0);
            if (hash) reinterpret_cast<uint4 *>(sh.token)[i] = make_uint4(0, 0, 0, 0);
            if (row.n > 0) reinterpret_cast<uint4 *>(sh.last)[i] = make_uint4(0, 0, 0, 0);
        }
    };
    // Counts tokens [begin, begin + size): slot = token - begin, or (hashed) the token's in the table. False where
    // a token of this thread's found no place.
    auto count = [&](auto hashed, int begin, int size) -> bool {
        bool all = true;
        auto touch = [&](unsigned i, uint32_t flags, uint32_t place) {   // flags: kSeen, kBiased or a count of 1
            unsigned at = i;
            if constexpr (decltype(hashed)::value) {
                at = i * 2654435761u / (0x80000000u / (SLOTS / 2));
                int tries = 0;
                for (; tries < kProbes; ++tries, at = (at + 1) % SLOTS) {
                    uint32_t there = *static_cast<volatile uint32_t *>(&sh.token[at]);
                    if (there == 0) there = atomicCAS(&sh.token[at], 0u, i + 1);
                    if (there == 0 || there == i + 1) break;
                }
                if (tries == kProbes) {
                    all = false;
                    return;
                }
            }
            if (flags == 1u) atomicAdd(&sh.word[at], 1u);
            else atomicOr(&sh.word[at], flags);
            if (flags == kBiased) atomicMax(&sh.last[at], place);
        };
        auto check = [&](int64_t token) {
            if (lo == 0 && (token < -1 || token >= vocab)) atomicOr(&g_adjust_status, PRECOG_DEV_BAD_INDEX);
        };
        constexpr int kAtOnce = 8;
        for (int64_t j0 = row.begin + threadIdx.x; j0 < row.end; j0 += kAtOnce * THREADS) {
            int64_t token[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) token[k] = j0 + k * THREADS < row.end ? p.history[j0 + k * THREADS] : -1;
#pragma unroll 1
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t tok = token[0];
#pragma unroll
                for (int i = 0; i + 1 < kAtOnce; ++i) token[i] = token[i + 1];
                const uint64_t i = static_cast<uint64_t>(tok) - static_cast<uint64_t>(begin);
                if (i < static_cast<unsigned>(size)) touch(static_cast<unsigned>(i), j0 + k * THREADS < row.from ? kSeen : 1u, 0u);
                else check(tok);
            }
        }
        for (int64_t j = threadIdx.x; j < row.n; j += THREADS) {
            const int64_t tok = p.bias_idx[row.first + j];
            const uint64_t i = static_cast<uint64_t>(tok) - static_cast<uint64_t>(begin);
            if (i < static_cast<unsigned>(size)) touch(static_cast<unsigned>(i), kBiased, static_cast<uint32_t>(j) + 1u);
            else check(tok);
        }
        return all;
    };
    const T *const x = static_cast<const T *>(p.logits) + r * p.stride;
    T *const out = static_cast<T *>(p.out) + r * p.out_stride;
    auto put = [&](bool hash, int begin) {
        const uint32_t *const mask = mask_of_row(p, r, false);
        constexpr int kAtOnce = SLOTS / THREADS < 8 ? SLOTS / THREADS : 8;   // slots whose scattered loads are in flight together
        for (int at0 = threadIdx.x; at0 < SLOTS; at0 += kAtOnce * THREADS) {
            int token[kAtOnce];
            uint32_t word[kAtOnce], may[kAtOnce];
            T v[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int at = at0 + u * THREADS;
                word[u] = sh.word[at];
                token[u] = begin + (hash ? static_cast<int>(sh.token[at]) - 1 : at);
                if (word[u] == 0) continue;
                v[u] = x[token[u]];
                may[u] = mask != nullptr ? mask[token[u] >> 5] : 0xffffffffu;
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (word[u] == 0 || ((may[u] >> (token[u] & 31)) & 1u) == 0) continue;
                const uint32_t last = (word[u] & kBiased) != 0 ? sh.last[at0 + u * THREADS] : 0u;
                out[token[u]] = stored<T>(adjusted(to_f32(v[u]), word[u], row, p.bias, last));
            }
        }
    };
    clear(HASH);
    __syncthreads();
    const bool all = count(std::integral_constant<bool, HASH>{}, lo, hi - lo);
    before_writing();
    if (__syncthreads_and(all)) {   // (a copy by this CTA is behind it, too)
        put(HASH, lo);
        return;
    }
    for (int begin = lo; begin < hi; begin += SLOTS) {
        __syncthreads();
        clear(false);
        __syncthreads();
        count(std::false_type{}, begin, min(hi - begin, SLOTS));
        __syncthreads();
        put(false, begin);
    }
}

// A copy with the mask, a CTA `slice` tokens of a row. Of a pair of launches it lets the other in early, whose CTAs read
// no logits and write nothing before the copy has ended (what they do read was there before the copy began).
template <typename T>
__global__ void __launch_bounds__(kThreads, 3) copy_kernel(const AdjustParams p, int slice, unsigned slices, bool pair) {
    grid_dependency_wait();
    if (pair) grid_dependency_launch();
    const int64_t r = blockIdx.x / slices;
    const int vocab = static_cast<int>(p.vocab), lo = static_cast<int>(blockIdx.x % slices) * slice, hi = min(vocab, lo + slice);
    copy_range(static_cast<const T *>(p.logits) + r * p.stride, static_cast<T *>(p.out) + r * p.out_stride, lo, hi, vocab,
               mask_of_row(p, r, lo == 0 && threadIdx.x == 0));
}

constexpr int kHashSlots = 8192, kHashThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kHashThreads, 2) listed_kernel(const AdjustParams p, int slice, unsigned slices) {
    extern __shared__ uint4 shared[];
    const int64_t r = blockIdx.x / slices;
    const int vocab = static_cast<int>(p.vocab), lo = static_cast<int>(blockIdx.x % slices) * slice, hi = min(vocab, lo + slice);
    adjust_range<T, kHashSlots, true, kHashThreads>(p, *reinterpret_cast<Tables<kHashSlots, true> *>(shared), r, lo, hi, [] { grid_dependency_wait(); });
}

constexpr int kSmallSlice = 2048;
template <typename T>
__global__ void __launch_bounds__(kThreads, 3) adjust_kernel(const AdjustParams p, unsigned slices) {
    grid_dependency_wait();
    extern __shared__ uint4 shared[];
    const int64_t r = blockIdx.x / slices;
    const int vocab = static_cast<int>(p.vocab), lo = static_cast<int>(blockIdx.x % slices) * kSmallSlice, hi = min(vocab, lo + kSmallSlice);
    copy_range(static_cast<const T *>(p.logits) + r * p.stride, static_cast<T *>(p.out) + r * p.out_stride, lo, hi, vocab,
               mask_of_row(p, r, lo == 0 && threadIdx.x == 0));
    adjust_range<T, kSmallSlice, false, kThreads>(p, *reinterpret_cast<Tables<kSmallSlice, false> *>(shared), r, lo, hi, [] {});
}

template <typename Kernel, typename... More>
cudaError_t launch_slices(Kernel kernel, const AdjustParams &p, int slice, int threads, int smem, cudaStream_t stream, More... more) {
    const int64_t slices = (p.vocab + slice - 1) / slice, blocks = p.rows * slices;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    cudaError_t e = smem > 48 * 1024 ? ensure_smem(reinterpret_cast<const void *>(kernel), smem) : cudaSuccess;
    if (e != cudaSuccess) return e;
    e = launch_dependent(kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), smem, stream, p, more...);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T>
cudaError_t launch_typed(const AdjustParams &p, cudaStream_t stream) {
    const int64_t tokens = p.rows * p.vocab, sms = device_sm_count();
    const auto slices_of = [&](int slice) { return static_cast<unsigned>((p.vocab + slice - 1) / slice); };
    // One launch or two: 4 rows of 128,001 logits 6.6 against 9.2 us, 16 of 32,000 7.1 against 9.8; 64 of 32,000 16.4
    // against 12.7, 16 of 128,001 14.1 against 10.3, 64 of 128,001 51.7 against 19.4. (Slices of 8192 and 32,768: 39.5 and
    // 37.0 us for the 256 rows above; parts of 65,536: 43.6, rows being few enough to fit the GPU whole.)
    const bool many = tokens >= sms * 8192, biases = p.bias != nullptr;
    if (!p.history && !biases) {
        const int slice = many ? 16384 : 2048;
        return launch_slices(copy_kernel<T>, p, slice, kThreads, 0, stream, slice, slices_of(slice), false);
    }
    if (!many)
        return launch_slices(adjust_kernel<T>, p, kSmallSlice, kThreads, Tables<kSmallSlice, false>::bytes(biases), stream, slices_of(kSmallSlice));
    const int slice = 16384, part = 131072;
    const cudaError_t e = launch_slices(copy_kernel<T>, p, slice, kThreads, 0, stream, slice, slices_of(slice), true);
    if (e != cudaSuccess) return e;
    return launch_slices(listed_kernel<T>, p, part, kHashThreads, Tables<kHashSlots, true>::bytes(biases), stream, part, slices_of(part));
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
