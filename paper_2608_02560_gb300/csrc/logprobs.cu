// Log probabilities of given tokens, the entropy of their distribution and the k best entries,
// in one pass over the logits.
//
// With z = x / temperature, m = max z, d_i = z_i - m:
//   S = sum e^{d_i},  W = sum d_i e^{d_i}
//   log p(token) = d_token - log S,   H = log S - W / S.
// Every thread keeps (max, S, W) of what it has seen; when its maximum grows by c, S becomes
// S e^-c and W becomes (W - c S) e^-c, and two threads' sums join the same way. Exponentials below
// 2^-150 of the largest count as zero, -infinity among them. d is one FMA, x c - rn(max c), and sums move
// to another maximum by the difference of the rounded products: so every term carries the rounding of the
// last maximum's product and no other's, and the result is freed of it. Where max c is so large that its
// rounding itself would count (2^28 and more: rows of the type's lowest value among them) the row is summed
// again with d = (x - max) c.
//
// The best entries: each warp keeps its k best in its lanes, sorted, as keys (value, complement of
// the index). The CTA's first batches give a bound that at least k entries reach (the k-th of all
// lanes' maxima), and later the warps share the largest of their k-th values, so few entries are
// ever inserted. Batches whose maximum does not reach the bound cost one comparison.
//
// Memory and the instructions, 5 to 8 an entry, bound it alike: 2048 rows of 50,257 bf16 logits, 5 best,
// take 53 us (3.87 TB/s, 0.57 of the measured copy rate, schedulers 66 % busy); 61 rows of 128,001 fp32
// ones with nine tenths at -infinity, 20 best, 22.5 us, by the latency of the joins; one row of 32,000
// 8.2 us. A CTA takes a row; with few rows a cluster of up to 8 shares one and joins over distributed
// shared memory.
#include <cmath>
#include <cstddef>

#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {
namespace {

__device__ uint32_t g_logprob_status;

constexpr int kFly = 4;               // 16-byte vectors of a batch a lane
constexpr int kStages = 3;            // batches of a warp in shared memory
constexpr int kMaxParts = 8;          // CTAs of a row
constexpr float kFar = 268435456.f;   // 2^28: up to there the rounding of max c is at most 16, e^d far from fp32's ends
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

// The sums seen from the maximum `mx` >= a.mx. c: log2(e) / temperature. (__fmul_rn: never part of an
// FMA. FAR: without the products, for maxima whose own leave fp32's range.)
template <bool FAR = false>
__device__ __forceinline__ Sums moved(const Sums a, float mx, float c) {
    if (mx == a.mx) return a;
    const float d = clamped(FAR ? (a.mx - mx) * c : __fmul_rn(a.mx, c) - __fmul_rn(mx, c)), f = ex2(d);
    return Sums{mx, a.s * f, fmaf(d, a.s, a.w) * f};
}
template <bool FAR = false>
__device__ __forceinline__ Sums joined(const Sums a, const Sums b, float c) {
    const float mx = fmaxf(a.mx, b.mx);
    const Sums x = moved<FAR>(a, mx, c), y = moved<FAR>(b, mx, c);
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

// What a CTA has found.
struct Found {
    Sums sums;
    u64 best[32];
};

__device__ __forceinline__ uint32_t word(const uint32_t (&r)[4], int i) {
    const uint32_t a = i & 1 ? r[1] : r[0], b = i & 1 ? r[3] : r[2];
    return i & 2 ? b : a;
}

template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kN = 4;
    static constexpr uint32_t kNone = 0xff800000u;   // -infinity
    static constexpr bool kRaised = false;           // finite() keeps -infinity out
    static __device__ __forceinline__ float get(const uint32_t (&r)[4], int i) { return __uint_as_float(r[i]); }
    static __device__ __forceinline__ uint32_t lowest(float) { return 0u; }
    static __device__ __forceinline__ f2 finite(const uint32_t (&r)[4], int i, uint32_t) { return pack2(get(r, i), get(r, i + 1)); }
    // The largest entry; NaN is none.
    static __device__ __forceinline__ float most(const uint32_t (&r)[4]) {
        return fmaxf(fmaxf(get(r, 0), get(r, 1)), fmaxf(get(r, 2), get(r, 3)));
    }
    // Bit i: entry i is above thr, or (not `strict`) equals it.
    static __device__ __forceinline__ unsigned reach(const uint32_t (&r)[4], float thr, bool strict) {
        unsigned m = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) m |= get(r, i) > thr || (!strict && get(r, i) == thr) ? 1u << i : 0u;
        return m;
    }
    static __device__ __forceinline__ float at(const uint32_t (&r)[4], int i) { return __uint_as_float(word(r, i)); }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static constexpr uint32_t kNone = 0xff80ff80u;
    static constexpr bool kRaised = true;
    static __device__ __forceinline__ float get(const uint32_t (&r)[4], int i) {
        return __uint_as_float(i % 2 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
    }
    // Entries i, i + 1, not below `low` (two of the same): so that d is finite and d e^d no NaN.
    static __device__ __forceinline__ f2 finite(const uint32_t (&r)[4], int i, uint32_t low) {
        const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&r[i / 2]), *reinterpret_cast<const __nv_bfloat162 *>(&low));
        const uint32_t w = *reinterpret_cast<const uint32_t *>(&m);
        return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t lowest(float v) {
        const __nv_bfloat162 m = __float2bfloat162_rn(v);
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    static __device__ __forceinline__ float most(const uint32_t (&r)[4]) {
        auto two = [&](int i) { return *reinterpret_cast<const __nv_bfloat162 *>(&r[i]); };
        const __nv_bfloat162 m = __hmax2(__hmax2(two(0), two(1)), __hmax2(two(2), two(3)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ unsigned reach(const uint32_t (&r)[4], float thr, bool strict) {
        const __nv_bfloat162 t = __float2bfloat162_rn(thr);   // (an entry's value: exact)
        unsigned m = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 w = *reinterpret_cast<const __nv_bfloat162 *>(&r[i]);
            m |= ((strict ? __hgt2_mask(w, t) : __hge2_mask(w, t)) & 0x00020001u) << (2 * i);
        }
        return (m | m >> 16) & 0xffu;
    }
    static __device__ __forceinline__ float at(const uint32_t (&r)[4], int i) {
        return __uint_as_float(i % 2 ? word(r, i / 2) & 0xffff0000u : word(r, i / 2) << 16);
    }
};
template <> struct Vec<__half> {
    static constexpr int kN = 8;
    static constexpr uint32_t kNone = 0xfc00fc00u;
    static constexpr bool kRaised = false;
    static __device__ __forceinline__ float get(const uint32_t (&r)[4], int i) {
        return __half2float(__ushort_as_half(static_cast<unsigned short>(i % 2 ? r[i / 2] >> 16 : r[i / 2] & 0xffffu)));
    }
    // (no entry of fp16 is low enough at every temperature)
    static __device__ __forceinline__ uint32_t lowest(float) { return 0u; }
    static __device__ __forceinline__ f2 finite(const uint32_t (&r)[4], int i, uint32_t) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&r[i / 2]));
        return pack2(v.x, v.y);
    }
    static __device__ __forceinline__ float most(const uint32_t (&r)[4]) {
        auto two = [&](int i) { return *reinterpret_cast<const __half2 *>(&r[i]); };
        const __half2 m = __hmax2(__hmax2(two(0), two(1)), __hmax2(two(2), two(3)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ unsigned reach(const uint32_t (&r)[4], float thr, bool strict) {
        const __half2 t = __float2half2_rn(thr);
        unsigned m = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 w = *reinterpret_cast<const __half2 *>(&r[i]);
            m |= ((strict ? __hgt2_mask(w, t) : __hge2_mask(w, t)) & 0x00020001u) << (2 * i);
        }
        return (m | m >> 16) & 0xffu;
    }
    static __device__ __forceinline__ float at(const uint32_t (&r)[4], int i) {
        return __half2float(__ushort_as_half(static_cast<unsigned short>(word(r, i / 2) >> (i % 2 * 16))));
    }
};

// Descending over the lanes.
__device__ __forceinline__ float sorted(float v, int lane) {
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int o = size / 2; o > 0; o /= 2) {
            const float u = __shfl_xor_sync(0xffffffffu, v, o);
            const bool first = (lane & o) == 0, down = (lane & size) == 0 || size == 32;
            v = first == down ? fmaxf(u, v) : fminf(u, v);
        }
    return v;
}

// The 32 largest of two descending lists, descending; `reversed`: the second, last entry first. (The
// larger of each pair makes a sequence that falls and rises, which five steps sort.)
__device__ __forceinline__ u64 merged(u64 v, u64 reversed, int lane) {
    v = v > reversed ? v : reversed;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        const u64 u = __shfl_xor_sync(0xffffffffu, v, o);
        v = ((lane & o) == 0) == (u > v) ? u : v;
    }
    return v;
}

// The same of two lists of plain values.
__device__ __forceinline__ float merged(float v, float reversed, int lane) {
    v = fmaxf(v, reversed);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = (lane & o) == 0 ? fmaxf(u, v) : fminf(u, v);
    }
    return v;
}

// The k best entries of a warp. Entries come in the order of their indices: once the warp has k, only
// ones above the k-th enter; those of a bound that others found may also equal it.
// (thr and strict are the same in every lane: whole warps branch on them around shuffles.)
struct Best {
    u64 mine = 0ull;             // entry `lane`, best first
    float thr = -INFINITY;
    bool strict = false;
    __device__ __forceinline__ bool enters(float x) const { return x > thr || (!strict && x == thr); }
    __device__ __forceinline__ void bound(float v) {
        if (v > thr) thr = v, strict = false;
    }
    __device__ __forceinline__ void add(u64 key, int k, int lane) {
        insert(mine, key, lane);
        const u64 last = __shfl_sync(0xffffffffu, mine, k - 1);
        if (last != 0ull && value_of(last) >= thr) thr = value_of(last), strict = true;
    }
};

// One entry a lane (`in`: there is one), in the order of the lanes.
template <bool TOP>
__device__ __forceinline__ void take_one(float x, uint32_t index, bool in, float c, int k, int lane, Sums &a, Best &b) {
    if (in) {
        if (x > a.mx) a = moved(a, x, c);
        const float d = clamped(fmaf(x, c, -__fmul_rn(a.mx, c))), e = ex2(d);
        a.s += e;
        a.w = fmaf(d, e, a.w);
    }
    if constexpr (TOP) {
        unsigned todo = __ballot_sync(0xffffffffu, in && b.enters(x));
        while (todo) {
            const int from = __ffs(static_cast<int>(todo)) - 1;
            const float v = __shfl_sync(0xffffffffu, x, from);
            if (b.enters(v)) b.add(key_of(v, __shfl_sync(0xffffffffu, index, from)), k, lane);
            todo &= todo - 1;
        }
    }
}

// The sums of a row by one warp, d as a difference: for maxima that are too large for the product.
// (A second pass: rows that are all masked take 41 us where an ordinary one of 32,000 takes 9, 64 of
// 128,001 fp32 143 and 18, 2048 of 50,257 187 and 55.)
template <typename T>
__device__ __noinline__ Sums sums_far(const T *x, int vocab, float c, int lane) {
    Sums a{kLowest, 0.f, 0.f};
    for (int i = lane; i < vocab; i += 32) {
        const float v = to_f32(x[i]);
        if (v > a.mx) a = moved<true>(a, v, c);
        const float d = clamped((v - a.mx) * c), e = ex2(d);
        a.s += e;
        a.w = fmaf(d, e, a.w);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        a = joined<true>(a, Sums{__shfl_xor_sync(0xffffffffu, a.mx, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.w, o)}, c);
    return a;
}

template <typename T, bool TOP, int kWarps>
__global__ void __launch_bounds__(kWarps * 32) logprobs_kernel(const LogprobParams p, int parts) {
    using V = Vec<T>;
    constexpr int N = V::kN;
    __shared__ Found found[kWarps];                // of the warps; the first becomes the CTA's
    __shared__ float tops[kWarps][32];             // the lanes' maxima of the first batches, sorted
    __shared__ uint32_t shared_bound;              // the warps' largest k-th value, as ordered bits
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x / parts;
    const int part = static_cast<int>(blockIdx.x % parts);
    const T *x = static_cast<const T *>(p.logits) + row * p.stride;
    const float c = p.inv_temp * kLog2e;
    const int vocab = static_cast<int>(p.vocab), k = p.k;
    // entries before the row's first 16-byte boundary, whole vectors, entries after the last
    const int past = static_cast<int>(reinterpret_cast<uintptr_t>(x) & 15u) / static_cast<int>(sizeof(T));
    const int head = past == 0 ? 0 : N - past < vocab ? N - past : vocab;
    const int vecs = (vocab - head) / N, tail = vocab - head - vecs * N;
    const uint4 *xv = reinterpret_cast<const uint4 *>(x + head);
    const int gw = part * kWarps + warp, warps = parts * kWarps;

    const float far = fminf(kFar / c, 1e37f);      // a maximum within it: |max c| < kFar
    Sums a{-far, 0.f, 0.f};
    float nmc = __fmul_rn(far, c);                 // -max c, rounded
    f2 s2 = pack2(0.f, 0.f), w2 = s2;
    Best b;
    if (gw == 0 && head > 0) {
        take_one<TOP>(lane < head ? to_f32(x[lane < head ? lane : 0]) : 0.f, lane, lane < head, c, k, lane, a, b);
        nmc = -__fmul_rn(a.mx, c);
    }
    const f2 cc = pack2(c, c);
    const uint32_t low = V::lowest(-2.f * far);    // below any maximum, and low c finite
    bool first = true;
    // A lane copies its own vectors to shared memory, two batches ahead, and reads its own: registers
    // held too few loads in flight (2048 x 50,257 bf16: 57 us).
    extern __shared__ __align__(16) uint4 ring[];
    uint4 *mine = ring + static_cast<size_t>(warp) * kStages * kFly * 32 + lane;
    const int step = warps * 32 * kFly;
    auto fetch = [&](int v0, int stage) {
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int v = v0 + u * warps * 32 + lane;
            if (v < vecs) cp_async16(mine + (stage * kFly + u) * 32, xv + v);
        }
        cp_async_commit();
    };
    int stage = 0;
    for (int i = 0; i < kStages - 1; ++i) fetch(gw * 32 + i * step, i);
    if (TOP && threadIdx.x == 0) shared_bound = 0u;
#pragma unroll 1
    for (int v0 = gw * 32; v0 < vecs || (TOP && first); v0 += step) {
        cp_async_wait<kStages - 2>();
        fetch(v0 + (kStages - 1) * step, stage == 0 ? kStages - 1 : stage - 1);
        uint32_t r[kFly][4];
        float top[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const uint4 q = mine[(stage * kFly + u) * 32];
            r[u][0] = q.x, r[u][1] = q.y, r[u][2] = q.z, r[u][3] = q.w;
        }
        if (v0 + (kFly - 1) * warps * 32 + 32 > vecs) {   // (one branch a batch: the rest is straight)
#pragma unroll
            for (int u = 0; u < kFly; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) r[u][i] = v0 + u * warps * 32 + lane < vecs ? r[u][i] : V::kNone;
        }
        stage = stage == kStages - 1 ? 0 : stage + 1;
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            top[u] = fmaxf(-INFINITY, V::most(r[u]));
            most = fmaxf(most, top[u]);
        }
        if (most > a.mx) {
            const float next = -__fmul_rn(most, c), d = clamped(next - nmc), f = ex2(d);
            w2 = mul2(fma2(pack2(d, d), s2, w2), pack2(f, f));
            s2 = mul2(s2, pack2(f, f));
            const Sums m = moved(a, most, c);
            a = m;
            nmc = next;
        }
        const f2 nm = pack2(nmc, nmc);
#pragma unroll
        for (int u = 0; u < kFly; ++u)
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                float d0, d1;
                unpack2(fma2(V::finite(r[u], i, low), cc, nm), d0, d1);
                if constexpr (!V::kRaised) d0 = clamped(d0), d1 = clamped(d1);
                const f2 e = pack2(ex2(d0), ex2(d1));
                s2 = fma2(e, pack2(1.f, 1.f), s2);
                w2 = fma2(pack2(d0, d1), e, w2);
            }
        if constexpr (TOP) {
            if (first) {   // k of the CTA's lanes hold an entry as large as the k-th of their maxima
                first = false;
                float v = sorted(most, lane);
                tops[warp][lane] = v;
                __syncthreads();   // every warp comes here once
#pragma unroll
                for (int w = 1; w < kWarps; ++w) v = merged(v, tops[(warp + w) % kWarps][31 - lane], lane);
                b.bound(__shfl_sync(0xffffffffu, v, k - 1));
            } else {   // one lane's reading for all: others may raise it between two lanes' own
                const uint32_t others = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t *>(&shared_bound), 0);
                if (others != 0u) b.bound(value_of(static_cast<u64>(others) << 32));
            }
            if (__any_sync(0xffffffffu, b.enters(most))) {
#pragma unroll
                for (int u = 0; u < kFly; ++u) {
                    const int v = v0 + u * warps * 32 + lane;
                    if (!__any_sync(0xffffffffu, b.enters(top[u]))) continue;
                    unsigned left = v < vecs ? V::reach(r[u], b.thr, b.strict) : 0u;   // this lane's entries that may enter
                    unsigned todo;
                    while ((todo = __ballot_sync(0xffffffffu, left != 0u)) != 0u) {
                        const int from = __ffs(static_cast<int>(todo)) - 1;
                        const int at = __ffs(static_cast<int>(left)) - 1;
                        const float value = __shfl_sync(0xffffffffu, V::at(r[u], at), from);
                        const int index = __shfl_sync(0xffffffffu, head + v * N + at, from);
                        b.add(key_of(value, static_cast<uint32_t>(index)), k, lane);
                        if (lane == from) left &= left - 1u;
                        if (b.strict) left &= V::reach(r[u], b.thr, true);
                    }
                }
                if (b.strict && lane == 0) atomicMax(&shared_bound, static_cast<uint32_t>(key_of(b.thr, 0u) >> 32));
            }
        }
    }
    {
        float lo, hi;
        unpack2(s2, lo, hi);
        a.s += lo + hi;
        unpack2(w2, lo, hi);
        a.w += lo + hi;
    }
    if (gw == warps - 1 && tail > 0) {
        const int i = head + vecs * N + lane;
        take_one<TOP>(lane < tail ? to_f32(x[lane < tail ? i : 0]) : 0.f, i, lane < tail, c, k, lane, a, b);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        a = joined(a, Sums{__shfl_xor_sync(0xffffffffu, a.mx, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.w, o)}, c);
    // ---- join the warps, then the row's CTAs ----
    auto publish = [&] {
        if (lane == 0) found[warp].sums = a;
        if (TOP) found[warp].best[lane] = b.mine;
    };
    publish();
    for (int o = kWarps / 2; o > 0; o /= 2) {
        __syncthreads();
        if (warp < o) {
            a = joined(a, found[warp + o].sums, c);
            if (TOP) b.mine = merged(b.mine, found[warp + o].best[31 - lane], lane);
            publish();
        }
    }
    if (parts > 1) {
        cluster_sync_all();
        if (warp == 0 && part == 0) {
            Sums sums[kMaxParts - 1];
            u64 its[kMaxParts - 1];   // lane j reads the other's entry 31 - j
#pragma unroll
            for (int o = 1; o < kMaxParts; ++o) {
                if (o >= parts) break;
                const uint32_t other = mapa_shared(&found[0], static_cast<uint32_t>(o));
                sums[o - 1] = Sums{__uint_as_float(ld_cluster_u32(other)), __uint_as_float(ld_cluster_u32(other + 4)),
                                   __uint_as_float(ld_cluster_u32(other + 8))};
                if constexpr (TOP) {
                    const uint32_t at = other + static_cast<uint32_t>(offsetof(Found, best)) + 8u * (31 - lane);
                    its[o - 1] = static_cast<u64>(ld_cluster_u32(at)) | static_cast<u64>(ld_cluster_u32(at + 4)) << 32;
                }
            }
#pragma unroll
            for (int o = 1; o < kMaxParts; ++o) {
                if (o >= parts) break;
                a = joined(a, sums[o - 1], c);
                if (TOP) b.mine = merged(b.mine, its[o - 1], lane);
            }
        }
        cluster_sync_all();   // the others' shared memory has been read
    }
    if (warp != 0 || part != 0) return;
    // (nor at temperatures where entries below -far would still count)
    const bool near = fabsf(a.mx) < far && far * c > 1e3f;
    if (!near) a = sums_far(x, vocab, c, lane);
    const float nan = __int_as_float(0x7fffffff);
    const float log_s = log2f(a.s);                        // NaN where the row holds one
    const bool empty = a.s == 0.f;
    auto log_p = [&](float v) {
        // (what the rounding of max c has added to every d)
        const float off = near ? fmaf(a.mx, c, -__fmul_rn(a.mx, c)) : 0.f;
        return empty ? nan : (v - a.mx) * p.inv_temp - (log_s - off) * kLn2;
    };
    if (lane == 0) {
        const int64_t token = p.tokens[row];
        float lp = 0.f;
        if (token >= 0 && token < p.vocab) {
            lp = log_p(to_f32(x[token]));
        } else if (token != -1) {
            atomicOr(&g_logprob_status, PRECOG_DEV_BAD_INDEX);
            lp = nan;
        }
        p.logprob[row] = lp;
        if (p.entropy) p.entropy[row] = empty ? nan : (log_s - a.w / a.s) * kLn2;
    }
    if (TOP && lane < k) {
        const bool some = b.mine != 0ull;
        p.top_idx[row * k + lane] = some ? static_cast<int64_t>(0xffffffffu - static_cast<uint32_t>(b.mine)) : -1;
        p.top_logprob[row * k + lane] = some ? log_p(value_of(b.mine)) : nan;
    }
}

template <typename T, bool TOP, int kWarps>
cudaError_t launch_warps(const LogprobParams &p, int parts, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.rows * parts));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = static_cast<size_t>(kWarps) * kStages * kFly * 32 * 16;
    const cudaError_t s = ensure_smem(reinterpret_cast<const void *>(logprobs_kernel<T, TOP, kWarps>), static_cast<int>(cfg.dynamicSmemBytes));
    if (s != cudaSuccess) return s;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, logprobs_kernel<T, TOP, kWarps>, p, parts);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T, bool TOP>
cudaError_t launch_parts(const LogprobParams &p, cudaStream_t stream) {
    // Each warp pays for its own first entries, so a row gets only the warps that keep an SM's loads
    // in flight. 50,257 bf16 logits, 5 best, two / four / eight warps a row: 2048 rows 52 / 55 / 60 us,
    // 1500 rows 39 / 45 / 47, 1000 rows 34 / 31 / 33, 700 rows 30 / 25 / 28, 300 rows 26 / 18 / 15; 2048
    // rows without a list, whose first entries cost nothing, 42 / 37 / 39.
    const int64_t sms = device_sm_count();
    if (TOP && p.rows >= 8 * sms) return launch_warps<T, TOP, 2>(p, 1, stream);
    if (p.rows >= 4 * sms) return launch_warps<T, TOP, 4>(p, 1, stream);
    // With fewer rows than fill the SMs and rows long enough to be shared, up to eight CTAs a row, of at
    // least 4096 entries each: 300 rows of 50,257 15.2 us (a CTA each 15.4), 16 rows 8.0 (12.1), 61
    // rows of 128,001 fp32 20 (33), one of 152,000 8.8 (17.9).
    int parts = 1;
    while (parts < kMaxParts && p.rows * parts * 2 <= 4 * sms && p.vocab >= 4096LL * parts * 2) parts *= 2;
    return launch_warps<T, TOP, 8>(p, parts, stream);
}

template <typename T>
cudaError_t launch_typed(const LogprobParams &p, cudaStream_t stream) {
    return p.k > 0 ? launch_parts<T, true>(p, stream) : launch_parts<T, false>(p, stream);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobParams &p, cudaStream_t stream) {
    switch (p.dtype) {
        case PRECOG_F32: return launch_typed<float>(p, stream);
        case PRECOG_F16: return launch_typed<__half>(p, stream);
        default: return launch_typed<__nv_bfloat16>(p, stream);
    }
}

cudaError_t logprobs_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_logprob_status); }

}  // namespace precog
