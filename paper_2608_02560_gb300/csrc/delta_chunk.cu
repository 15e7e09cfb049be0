// The gated delta rule in chunks of 64 tokens on the 5th-generation tensor cores (bf16 inputs).
//
// With b the running sum of the log decays within a chunk and S the state before it,
//   A[i][j] = beta_i e^{b_i-b_j} k_i.k_j (j < i),   T = (I + A)^-1 diag(beta),
//   U = T (v - e^b S k),
//   y_i = scale (e^{b_i} S q_i + sum_{j<=i} e^{b_i-b_j} (q_i.k_j) U_j),
//   S  <- e^{b_C} S + sum_j e^{b_C-b_j} U_j k_j^T.
// A CTA owns 128 value channels of one (sequence, head): S^T's rows are the lanes of tensor
// memory, so every product has M = 128 and everything that follows a product (scales, the splits
// below) is a thread's own row. K, Q and V tiles enter the MMAs as the TMA laid them down, K both as
// [token][key] (k.q products, S k) and as [key][token] (the update).
//
// Precision: the inputs are exact bf16 operands; S, S k, U, T and P, which are not, enter as pairs
// hi + lo of bf16 numbers (16 significant bits). Sums and the state itself stay fp32. A single bf16 would
// put 2^-9 of S into every y. P U goes without lo * lo. (S k) T has it: where keys repeat, its terms are
// large and cancel (one key, dk = 8, beta = 1: 1.6e-4 of the largest without, 6e-5 with; a corpus takes
// 2 % longer). Ordinary keys: 5e-6. Where betas pass 1 the terms do not shrink along the chunk, and what
// T's 16 bits leave out adds up, 1e-2 for one key and betas of 2 throughout.
//
// Warps 0-7, the chain: what each chunk needs of the chunk before it, half the columns each
// group of four. Per chunk: split S (each half of it goes to the MMAs as it is done), [S k], y of the
// chunk before leaves, [S q, V T], split S k, [S k T], split U, [update], [P U]; [..] are MMAs.
// Warps 8-15, two teams that take chunks by turns, one or two ahead of the chain (one team of eight
// was no faster than one of four; a third team, at 80 registers a thread, slowed a corpus by 12 %):
// A and P with their decays, the inverse T in fp32: blocks of 16 by substitution (a product form would
// lose its digits where keys repeat), then joined twice, T10 = -(T1 A10) T0, a thread 4 x 2 entries of
// each product (16 x 16 and 32 x 32: too small for an MMA of 128 rows; on mma.sync with pairs of tf32 a
// corpus took 3 % longer).
// Warp 16: K and Q in, three chunks ahead (K alone six), the chunks' gates, and the MMAs of k.k and
// q.k, which the teams wait for. Warp 17: issues every other MMA, so that no working warp waits in the
// queue of the tensor cores. Warp 18: V in and y rows out.
//
// What bounds it: in full rounds the chain and the teams alike, 2.42 us or some 4700 cycles a chunk (3.6
// us, 7000 with a readout) at 0.45 instructions a cycle of each scheduler, the tensor cores' pipe 33 to 35 %
// busy, DRAM at 16 to 21 % of its rate; in rounds of a chunk or two the 13 us from a CTA's start to its
// end, most of them one chunk's way through a team. Measured, bf16, 128 x 128 a head: 256 sequences of 256
// to 4096 tokens, 8 heads, states alone, 1327 to 1351 us (218 TFLOP/s of the recurrence's operations); 96
// sequences of 1 to 200 tokens, 16 heads, with a readout, 176 to 178 us; one of 64 tokens 15 us; one of
// 32,768 tokens, cut into segments, 688 us.
// Loops over columns are rolled where they can be: fully unrolled, the roles' code was several times
// the instruction cache and warps waited for instructions 40 % of the time (25,000 cycles a chunk).
// Tokens beyond a sequence's end have beta 0 and zeroed rows: whatever the memory holds, nothing
// of them enters a sum.
// NaN and infinity among the inputs of a token reach its whole chunk, 0 * NaN being NaN in the products
// with T and P, and leave the channel's state not finite, from then on. So the state is looked at once, at
// the end, and a channel that broke is done again token by token (once_more): sequences that stay finite
// pay two barriers for it. So is every channel where gates grow more than e-fold over a chunk: rounding
// grows with them in the differences that make T (g = 0.1 a token, beta = 1: 3e-3 of the largest entry; g = 0.5:
// anything), though the correction may hold the state itself back.
//
// Few sequences leave SMs idle, and a chain is as long as its sequence. Then each sequence is cut into
// segments: a state passes through one as S M + B, M a product of e^g (I - beta k k^T) over its tokens.
// First B (from the zero state, or for the first segment from the initial one) and M (the rows of the
// identity, with v = 0) of all segments but the last; then the segments' initial states one after
// another (delta_join_kernel); then the segments themselves, with their readout. Where a segment's gates
// grow, or B or M is not finite, the join rolls rows over the segment itself.
//
// Tensor memory: S [128 columns]; a pair area [128]: S's pair, then U, whose place its decayed pair
// takes; places [64] by turns: a chunk's k.k and q.k, then its S k, then that one's pair, then U's
// (three; four without a readout); and S q [64], then y.
#include <cuda.h>

#include "../../include/precog.h"
#include "delta.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {

__device__ uint32_t g_delta_chunk_status;

namespace {

constexpr int kC = 64;                 // tokens of a chunk
constexpr int kM = 128;                // value channels of a CTA
constexpr int kVStages = 2;
constexpr int kChain = 256, kTeam = 128;   // threads
constexpr int kThreads = kChain + 2 * kTeam + 96;
constexpr int kCopyWarp = (kChain + 2 * kTeam) / 32, kMmaWarp = kCopyWarp + 1, kValueWarp = kCopyWarp + 2;
constexpr int kH = kC / 2, kB = kC / 4;    // the inverse: blocks of 16, joined to halves, joined
constexpr int kBlock = kH * kH;            // a quarter of A
constexpr uint32_t kTile = kC * 128;   // bytes of a [64 tokens][64 keys] bf16 tile
constexpr float kLeastGate = -128.f;   // e^-128 is 0 in fp32
// Growth (sums of positive gates) up to which chunks and segments keep their digits. The entries of T and of
// M are differences of e^growth, so what rounding leaves of them is that much larger than their own.
constexpr float kMostGrowth = 1.f;

// tensor memory columns
constexpr uint32_t kColS = 0, kColPair = 128, kColK = 256, kColQ = 448;

constexpr int kBarTeam = 1;            // and 2
constexpr int kBarChain = 3, kBarAgain = 4;

// A sum of logs as an unevaluated pair: differences of large sums keep their digits.
struct Log {
    float h, l;
};
__device__ __forceinline__ Log operator+(Log a, Log b) {
    const float s = a.h + b.h, t = s - a.h;
    const float e = ((a.h - (s - t)) + (b.h - t)) + (a.l + b.l);
    const float h = s + e;
    return Log{h, e - (h - s)};
}
__device__ __forceinline__ float exp_diff(Log a, Log b) { return ex2((a.h - b.h) + (a.l - b.l)); }
__device__ __forceinline__ Log shfl_up(Log a, int o) {
    return Log{__shfl_up_sync(0xffffffffu, a.h, o), __shfl_up_sync(0xffffffffu, a.l, o)};
}
__device__ __forceinline__ Log shfl(Log a, int from) {
    return Log{__shfl_sync(0xffffffffu, a.h, from), __shfl_sync(0xffffffffu, a.l, from)};
}

// What the gates of a chunk become.
struct alignas(16) Gates {
    float bh[kC], bl[kC]; // b in units of log2, a pair
    Log last[4];          // b of the last token of each 16
    float to_last[kC];    // e^{last - b_j}
    float beta[kC];
    float ek[kC];         // -e^{b_j}
    float eq[kC];         // scale e^{b_j}
    float ec[kC];         // e^{b_C - b_j}
    float whole;          // e^{b_C}
};

// States of one head.
struct States {
    void *base;                // nullptr: zeros
    int dtype;
    int64_t at;                // elements before row 0
};

// A CTA's tokens, the state before them and where the one behind them goes (nowhere: nullptr); in shared
// memory for the end, since in registers they made the chunks' own spill (one long sequence: 714 us).
struct Job {
    int64_t begin, end;
    States from, to;
    int head;
    bool m;                    // it is M
    bool again;                // what breaks is done again (else: by the join)
};

template <int NA, bool Y>
struct Smem {
    // chunks of K and Q on their way, places for k.k in tensor memory: more where no Q and no S q need theirs
    static constexpr int kStages = Y ? 3 : 6, kSlots = Y ? 3 : 4, kSides = Y ? 2 : 1;
    // V's two tiles, where the chunk's bf16 y rows lie on their way out; per stage, [K][Q] tiles of key
    // columns 0..63, then of 64..127, [Q][K] for the second team
    uint8_t v[kVStages][2 * kTile];
    uint8_t kq[kStages][NA * kSides * kTile];
    uint8_t tp[2][2 * kSides][kTile]; // T hi, T lo, P hi, P lo
    float a[2][3 * kBlock];           // a team's A, by columns in quarters 11, 21, 22, and what becomes of it
    Gates gates[kStages];
    uint64_t full_kq[kStages], free_kq[kStages], gated[kStages];
    uint64_t full_v[kVStages], through[kVStages];
    uint64_t zeroed_kq, zeroed_v, taken_y;
    uint64_t done_prep[kSlots], free_slot[kSlots], ready[2], done_o[2];
    uint64_t have_s[2], have_k, have_d, have_u;   // the chain's operands are in tensor memory
    uint64_t done_ks, done_qs, done_u, done_s;
    uint32_t broken[kM / 32];         // bit: a value channel that the chunks cannot be trusted with
    uint32_t growing;                 // a gate above 0 was seen
    Job job;
    uint32_t tmem_base;
};

__device__ __forceinline__ uint64_t desc_base(const void *tile) {
    uint64_t d = (smem_u32(tile) & 0x3ffffu) >> 4;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;     // 8-row groups
    d |= static_cast<uint64_t>(kTile >> 4) << 16;    // V's two tiles (others are one tile wide)
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;             // 128-byte swizzle
    return d;
}

// bf16 operands, fp32 sums, M = 128; `mn_a`, `mn_b`: the operand's rows run along K.
__host__ __device__ constexpr uint32_t idesc(int n, bool mn_a, bool mn_b) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((mn_a ? 1u : 0u) << 15) | ((mn_b ? 1u : 0u) << 16) |
           (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(kM >> 4) << 24);
}

// Bounded wait. A thread whose wait gives up records it and waits for nothing more than a moment
// from then on: it runs to the end on whatever is there, so that every barrier below is met.
__device__ __forceinline__ void wait_one(uint64_t *bar, uint32_t parity, uint32_t &patience) {
    uint32_t i = 0;
    bool ok;
    do {
        ok = mbar_try_wait(bar, parity);
    } while (!ok && ++i < patience);
    if (!ok) {
        patience = 1;
        atomicOr(&g_delta_chunk_status, PRECOG_DEV_TIMEOUT);
    }
}
// The same by all lanes of a warp, which go on together (tensor-memory accesses are a warp's).
__device__ __forceinline__ void wait(uint64_t *bar, uint32_t parity, uint32_t &patience) {
    wait_one(bar, parity, patience);
    __syncwarp();
}

__device__ __forceinline__ uint32_t bits2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
// Rows n .. 63 of `tiles` tiles, by a warp; MMAs see it.
__device__ __forceinline__ void zero_rows(uint8_t *first, int tiles, int n, int lane) {
    const int pieces = (kC - n) * 8;
    for (int e = lane; e < tiles * pieces; e += 32)
        *reinterpret_cast<uint4 *>(first + e / pieces * kTile + n * 128 + e % pieces * 16) = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    __syncwarp();
}

// Two numbers as bf16 in h and what that leaves, again in bf16, in l.
__device__ __forceinline__ void split(f2 ab, uint32_t &h, uint32_t &l) {
    float a, b;
    unpack2(ab, a, b);
    h = bits2(a, b);
    unpack2(fma2(pack2(__uint_as_float(h << 16), __uint_as_float(h & 0xffff0000u)), pack2(-1.f, -1.f), ab), a, b);
    l = bits2(a, b);
}
__device__ __forceinline__ void split(float a, float b, uint32_t &h, uint32_t &l) { split(pack2(a, b), h, l); }
__device__ __forceinline__ f2 pair_of(const uint32_t (&r)[32], int e) {
    return pack2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]));
}
__device__ __forceinline__ f2 load2(const float *p) { return *reinterpret_cast<const f2 *>(p); }

// Column j, row i of a quarter of A and later of T: the rows of four neighbouring columns begin in
// different banks.
__device__ __forceinline__ int place(int j, int i) { return j * kH + (i ^ ((j & 3) << 3)); }
// Rows r .. r + 3 of columns n, n + 1 of a product over K: L's columns from lc on, R's rows from rr on.
template <int K>
__device__ __forceinline__ void product(f2 (&sum)[2][2], const float *l, int lc, int r, const float *right, int rr, int n) {
    sum[0][0] = sum[0][1] = sum[1][0] = sum[1][1] = pack2(0.f, 0.f);
#pragma unroll 2
    for (int k = 0; k < K; k += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(right + place(n, rr + k));
        const float4 y = *reinterpret_cast<const float4 *>(right + place(n + 1, rr + k));
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 w = *reinterpret_cast<const float4 *>(l + place(lc + k + e, r));
            const f2 lo = pack2(w.x, w.y), hi = pack2(w.z, w.w), xx = pack2(xs[e], xs[e]), yy = pack2(ys[e], ys[e]);
            sum[0][0] = fma2(lo, xx, sum[0][0]);
            sum[0][1] = fma2(hi, xx, sum[0][1]);
            sum[1][0] = fma2(lo, yy, sum[1][0]);
            sum[1][1] = fma2(hi, yy, sum[1][1]);
        }
    }
}
__device__ __forceinline__ void store_product(const f2 (&sum)[2][2], float sign, float *to, int r, int n) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float4 w;
        unpack2(mul2(sum[j][0], pack2(sign, sign)), w.x, w.y);
        unpack2(mul2(sum[j][1], pack2(sign, sign)), w.z, w.w);
        *reinterpret_cast<float4 *>(to + place(n + j, r)) = w;
    }
}

// Segments of `len` tokens (0: whole sequences). Sequence c's first is slot begin / len + c: no two
// sequences' slots meet, and there are at most T_tot / len + n_seqs.
struct Cut {
    int len, slots;
    int joined;                // 0: B and M; 1: the segments from their initial states
    float *states;             // [slots][Hv][dv][dk]: B, then the state after the segment
    float *moves;              // [slots][Hv][dk][dk]: M
    float *begins;             // [n_seqs][Hv][dv][dk]: initial states of sequences of several segments
};
__device__ __forceinline__ int64_t segments(int64_t tokens, int len) { return tokens <= len ? 1 : (tokens + len - 1) / len; }

// Whether a job's gates grow too far for the chunks, or its whole length's for M; by a warp.
__device__ __noinline__ bool too_far(const DeltaParams &p, const Job &job) {
    const int lane = threadIdx.x & 31;
    float growth = 0.f;
    for (int64_t t0 = job.begin; t0 < job.end; t0 += kC) {
        float up = 0.f;
        for (int64_t t = t0 + lane; t < t0 + kC && t < job.end; t += 32) up += fmaxf(p.g[t * p.hv + job.head], 0.f);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) up += __shfl_xor_sync(0xffffffffu, up, o);
        growth = job.m ? growth + up : up;
        if (growth > kMostGrowth) return true;
    }
    return false;
}

// A job's tokens once more, one after another as the recurrence is defined, for the value channels whose
// state the chunks left not finite: there the zeros of T and P met NaN or infinity, 0 * NaN being NaN, and
// tokens before the broken one lost their readouts with it; and for all of them where gates grow. The first
// 16 warps, 8 channels each from `first` on (`broken`: bits), 8 lanes
// two channels: lane l of the 8 has the four-number groups l, l + 8, ... of both ones' keys. Tokens pass
// through `room`, 64 at a time, as fp32, keys padded with zeros. Once nothing of a warp's states is finite
// nothing will be again, and the rest of its readouts is NaN. No sequence comes here that stays finite and
// whose gates decay.
// 152 heads of 128 x 128, 4096 tokens, 247 us: all broken by their first token 545 us, by their last, or with
// gates that grow, 3.6 ms.
constexpr int kAgain = 512;
__host__ __device__ constexpr int again_bytes(int keys) { return 4 * (2 * kC * keys + kC * kM + 3 * kC); }
template <int NA, bool Y>
__device__ __noinline__ void once_more(const DeltaParams &p, const Job &job, float *room, int first, const uint32_t *broken) {
    constexpr int kKeys = NA * 64, kGroups = kKeys / 32, R = 2;   // four-number groups and channels a lane
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lane8 = lane & 7;
    const int row = warp * 8 + lane / 8, dk = p.dk, qk = job.head / (p.hv / p.hk);   // and row + 4, counted from `first`
    const int channels = p.dv - first < kM ? p.dv - first : kM;
    bool mine[R];                                  // (then the channel is one of the head's)
#pragma unroll
    for (int r = 0; r < R; ++r) mine[r] = (broken[warp / 4] >> (warp % 4 * 8 + lane / 8 + 4 * r) & 1u) != 0u;
    float *ks = room, *qs = ks + kC * kKeys, *vs = qs + kC * kKeys, *as = vs + kC * kM, *bs = as + kC, *kqs = bs + kC;
    f2 s[R][kGroups][2];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const int col = 4 * (lane8 + 8 * j);
            s[r][j][0] = s[r][j][1] = pack2(0.f, 0.f);
            if (!mine[r] || job.from.base == nullptr || col >= dk) continue;
            const int64_t at = job.from.at + static_cast<int64_t>(first + row + 4 * r) * dk + col;
            if (job.from.dtype == PRECOG_F32) {
                const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(job.from.base) + at);
                s[r][j][0] = pack2(v.x, v.y), s[r][j][1] = pack2(v.z, v.w);
            } else {
                const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(job.from.base) + at);
                s[r][j][0] = pack2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u));
                s[r][j][1] = pack2(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
            }
        }
    auto write_y = [&](int64_t t, int r, float v) {
        const int64_t at = (t * p.hv + job.head) * p.dv + first + row + 4 * r;
        if (p.y_dtype == PRECOG_F32) static_cast<float *>(p.y)[at] = v;
        else static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(v);
    };
    auto no_more = [&](int64_t t, int64_t end) {   // NaN from t on
#pragma unroll
        for (int r = 0; r < R; ++r)
            for (int64_t u = t + lane8; Y && mine[r] && u < end; u += 8) write_y(u, r, __int_as_float(0x7fffffff));
    };
    auto open = [&] {                              // anything finite left in the warp
        bool left = false;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < kGroups; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x, y;
                    unpack2(s[r][j][i], x, y);
                    left |= mine[r] && 4 * (lane8 + 8 * j) < dk && (isfinite(x) || isfinite(y));
                }
        return __any_sync(0xffffffffu, left);
    };
    // 64 rows of `width` numbers from column `col` on, `pitch` apart, zeros beyond the width and the last token
    auto bring = [&](float *to, int pitch, const void *base, int64_t stride, int64_t col, int width, int64_t t0) {
        uint4 v[2];                                     // (kC x pitch / 8 pieces: at most two a thread)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = (threadIdx.x + i * kAgain) * 8, t = e / pitch, c = e % pitch;
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (t < kC && t0 + t < job.end && c < width)
                v[i] = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(base) + (t0 + t) * stride + col + c);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = (threadIdx.x + i * kAgain) * 8;
            if (e >= kC * pitch) continue;
            float4 lo, hi;
            lo.x = __uint_as_float(v[i].x << 16), lo.y = __uint_as_float(v[i].x & 0xffff0000u);
            lo.z = __uint_as_float(v[i].y << 16), lo.w = __uint_as_float(v[i].y & 0xffff0000u);
            hi.x = __uint_as_float(v[i].z << 16), hi.y = __uint_as_float(v[i].z & 0xffff0000u);
            hi.z = __uint_as_float(v[i].w << 16), hi.w = __uint_as_float(v[i].w & 0xffff0000u);
            *reinterpret_cast<float4 *>(to + e) = lo;
            *reinterpret_cast<float4 *>(to + e + 4) = hi;
        }
    };
    bool going = open();
    int64_t t0 = job.begin;
#pragma unroll 1
    for (; t0 < job.end; t0 += kC) {
        if (!named_any(kBarAgain, kAgain, going)) break;   // (and the last tokens have been read)
        bring(ks, kKeys, p.k, p.k_stride, static_cast<int64_t>(qk) * dk, dk, t0);
        if (Y) bring(qs, kKeys, p.q, p.q_stride, static_cast<int64_t>(qk) * dk, dk, t0);
        bring(vs, kM, p.v, p.v_stride, static_cast<int64_t>(job.head) * p.dv + first, channels, t0);
        if (threadIdx.x < kC && t0 + threadIdx.x < job.end) {
            const float g = p.g[(t0 + threadIdx.x) * p.hv + job.head];
            as[threadIdx.x] = g < kLeastGate ? 0.f : expf(g);
            bs[threadIdx.x] = p.beta[(t0 + threadIdx.x) * p.hv + job.head];
        }
        named_sync(kBarAgain, kAgain);
        if (Y) {   // k.q of 4 tokens a warp
            for (int t = warp * 4; t < warp * 4 + 4; ++t) {
                float sum = 0.f;
                for (int c = lane; c < kKeys; c += 32) sum = fmaf(ks[t * kKeys + c], qs[t * kKeys + c], sum);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (lane == 0) kqs[t] = sum;
            }
            named_sync(kBarAgain, kAgain);
        }
        const int n = job.end - t0 < kC ? static_cast<int>(job.end - t0) : kC;
        if (!going) {
            no_more(t0, t0 + n);
            continue;
        }
#pragma unroll 1
        for (int t = 0; t < n; ++t) {
            const float4 *k = reinterpret_cast<const float4 *>(ks + t * kKeys) + lane8, *q = reinterpret_cast<const float4 *>(qs + t * kKeys) + lane8;
            float4 key[kGroups];
            f2 x[R][2], y[R][2];
#pragma unroll
            for (int r = 0; r < R; ++r) x[r][0] = x[r][1] = y[r][0] = y[r][1] = pack2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                key[j] = k[8 * j];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    x[r][0] = fma2(s[r][j][0], pack2(key[j].x, key[j].y), x[r][0]);
                    x[r][1] = fma2(s[r][j][1], pack2(key[j].z, key[j].w), x[r][1]);
                }
            }
            if (Y) {
#pragma unroll
                for (int j = 0; j < kGroups; ++j) {
                    const float4 v = q[8 * j];
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        y[r][0] = fma2(s[r][j][0], pack2(v.x, v.y), y[r][0]);
                        y[r][1] = fma2(s[r][j][1], pack2(v.z, v.w), y[r][1]);
                    }
                }
            }
            auto total = [](const f2 (&v)[2]) {
                float a, b, c, d;
                unpack2(v[0], a, b);
                unpack2(v[1], c, d);
                return (a + b) + (c + d);
            };
            float sk[R], sq[R];
#pragma unroll
            for (int r = 0; r < R; ++r) sk[r] = total(x[r]), sq[r] = total(y[r]);
#pragma unroll
            for (int o = 4; o > 0; o >>= 1)
#pragma unroll
                for (int r = 0; r < R; ++r) sk[r] += __shfl_xor_sync(0xffffffffu, sk[r], o), sq[r] += __shfl_xor_sync(0xffffffffu, sq[r], o);
            const float a = as[t], beta = bs[t];
            const f2 aa = pack2(a, a);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float u = beta * fmaf(-a, sk[r], vs[t * kM + row + 4 * r]);
                const f2 uu = pack2(u, u);
#pragma unroll
                for (int j = 0; j < kGroups; ++j) {
                    s[r][j][0] = fma2(uu, pack2(key[j].x, key[j].y), mul2(aa, s[r][j][0]));
                    s[r][j][1] = fma2(uu, pack2(key[j].z, key[j].w), mul2(aa, s[r][j][1]));
                }
                if (Y && mine[r] && lane8 == 0) write_y(t0 + t, r, p.scale * fmaf(u, kqs[t], a * sq[r]));
            }
        }
        going = open();
    }
    no_more(t0, job.end);
    if (job.to.base == nullptr) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const int col = 4 * (lane8 + 8 * j);
            if (!mine[r] || col >= dk) continue;
            const int64_t at = job.to.at + static_cast<int64_t>(first + row + 4 * r) * dk + col;
            float4 v;
            unpack2(s[r][j][0], v.x, v.y);
            unpack2(s[r][j][1], v.z, v.w);
            if (job.to.dtype == PRECOG_F32) *reinterpret_cast<float4 *>(static_cast<float *>(job.to.base) + at) = v;
            else *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(job.to.base) + at) = make_uint2(bits2(v.x, v.y), bits2(v.z, v.w));
        }
}

template <int NA, bool Y, bool CUT>
__global__ void __launch_bounds__(kThreads, 1)
    delta_chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const __grid_constant__ DeltaParams p, int slices, const Cut cut) {
    constexpr int kKeys = NA * 64;               // key coordinates, padded
    // Where K and Q lie in chunk c's stage: the second team has k.k in the tensor memory of its third
    // and fourth warps, so that the teams' work on A falls to all four schedulers.
    auto tile_of = [](int c, int side) { return Y ? static_cast<int>(kTile) * ((c & 1) ^ side) : 0; };
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // (an offset, not a rounded address: the compiler would lose that it is shared memory)
    using S = Smem<NA, Y>;
    constexpr int kStages = S::kStages, kSlots = S::kSlots, kSides = S::kSides;
    S &sm = *reinterpret_cast<S *>(smem_raw + ((0u - smem_u32(smem_raw)) & 1023u));
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint32_t patience = kWaitLimit;

    int64_t item = blockIdx.x;
    const bool kept = CUT && !cut.joined;        // B and M: states go to the workspace
    const int kinds = slices + (kept ? 1 : 0);
    const int slice = static_cast<int>(item % kinds);
    const bool ident = kept && slice == slices;  // M
    item /= kinds;
    const int head = static_cast<int>(item % p.hv);
    int64_t seq = item / p.hv;
    int64_t slot = seq, begin, end;
    bool first = true, last = true;
    if constexpr (CUT) {
        // the sequence that has this slot: found by the lanes, each warp for itself
        int64_t found = -1;
        for (int64_t c0 = 0; c0 < p.n_seqs && found < 0; c0 += 32) {
            const int64_t c = c0 + lane;
            bool mine = false, bad = false;
            if (c < p.n_seqs) {
                const int64_t b = p.offsets[c], e = p.offsets[c + 1], base = b / cut.len + c;
                bad = b < 0 || e < b || e > p.T_tot;
                mine = !bad && slot >= base && slot < base + segments(e - b, cut.len);
            }
            const unsigned who = __ballot_sync(0xffffffffu, mine), bads = __ballot_sync(0xffffffffu, bad);
            if (who && (!bads || __ffs(static_cast<int>(who)) < __ffs(static_cast<int>(bads)))) found = c0 + __ffs(static_cast<int>(who)) - 1;
            else if (bads) {   // what follows may overlap what came before: skipped
                if (threadIdx.x == 0) atomicOr(&g_delta_chunk_status, PRECOG_DEV_BAD_OFFSETS);
                return;
            }
        }
        if (found < 0) return;
        seq = found;
        begin = p.offsets[seq], end = p.offsets[seq + 1];
        const int64_t seg = slot - (begin / cut.len + seq), segs = segments(end - begin, cut.len);
        first = seg == 0, last = seg + 1 == segs;
        begin += seg * cut.len;
        end = last ? end : begin + cut.len;
        // no segment follows the last, the first begins from its state itself; without a readout the
        // others are done with
        if (cut.joined ? !Y && !last : last || (ident && first)) return;
    } else {
        begin = p.offsets[seq], end = p.offsets[seq + 1];
        if (begin < 0 || end < begin || end > p.T_tot) {
            if (threadIdx.x == 0) atomicOr(&g_delta_chunk_status, PRECOG_DEV_BAD_OFFSETS);
            return;
        }
    }
    const int len = static_cast<int>(end - begin);
    const int chunks = (len + kC - 1) / kC;
    const int qk = head / (p.hv / p.hk);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full_kq[s], 1);
            mbar_init(&sm.free_kq[s], 1);
            mbar_init(&sm.gated[s], 1);
        }
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(&sm.done_prep[s], 1);
            mbar_init(&sm.free_slot[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.full_v[i], 1);
            mbar_init(&sm.through[i], kChain / 32);
            mbar_init(&sm.ready[i], kTeam / 32);
            mbar_init(&sm.done_o[i], 1);
            mbar_init(&sm.have_s[i], kChain / 32);
        }
        mbar_init(&sm.zeroed_kq, 1);
        mbar_init(&sm.zeroed_v, 1);
        mbar_init(&sm.taken_y, kChain / 32);
        mbar_init(&sm.have_k, kChain / 32);
        mbar_init(&sm.have_d, kChain / 32);
        mbar_init(&sm.have_u, kChain / 32);
        mbar_init(&sm.done_ks, 1);
        mbar_init(&sm.done_qs, 1);
        mbar_init(&sm.done_u, 1);
        mbar_init(&sm.done_s, 1);
        for (int i = 0; i < kM / 32; ++i) sm.broken[i] = 0u;
        sm.growing = 0u;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&sm.tmem_base, 512);
        tmem_relinquish();
    }
    // the blocks of T and P right of the diagonal are zero for good
    for (int e = threadIdx.x; e < 4 * kSides * static_cast<int>(kTile) / 16; e += kThreads)
        reinterpret_cast<uint4 *>(sm.tp[0][0])[e] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // all 512 columns: they begin at 0, and addresses are constants below
    constexpr uint32_t tmem = 0;

    if (warp == kMmaWarp) {
        // ---------------- MMAs ----------------
        if (elect_one()) {
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                const uint32_t ph = static_cast<uint32_t>(c) & 1u;
                const uint32_t col_k = tmem + kColK + c % kSlots * 64, col_q = tmem + kColQ;
                const uint64_t d = desc_base(sm.kq[c % kStages] + tile_of(c, 0)), past = desc_base(sm.kq[c % kStages] + tile_of(c, 1)) - d;
                const uint64_t dv = desc_base(sm.v[c % kVStages]), dt = desc_base(sm.tp[ph][0]);
                wait_one(&sm.full_kq[c % kStages], static_cast<uint32_t>(c / kStages) & 1u, patience);
                if (len - c * kC < kC) wait_one(&sm.zeroed_kq, 0, patience);   // rows beyond the end
                wait_one(&sm.ready[ph], static_cast<uint32_t>(c >> 1) & 1u, patience);
                // 16 keys of S, hi and lo, onto S k or S q; the first sets it
                auto read_out = [&](uint32_t col, int kk, int q, bool onto) {
#pragma unroll
                    for (int l = 0; l < 2; ++l)
                        tc_mma_f16_ts(col, tmem + kColPair + l * (kKeys / 2) + kk * 8,
                                      d + q * past + (kk / 4) * (kSides * kTile / 16) + 2 * (kk % 4), idesc(kC, false, false), onto || l);
                };
#pragma unroll
                for (int part = 0; part < NA; ++part) {   // 32 keys of each half as they come
                    wait_one(&sm.have_s[part], ph, patience);
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) read_out(col_k, k / 2 * (2 * NA) + part * 2 + k % 2, 0, part + k > 0);
                }
                tc_commit(&sm.done_ks);
                if (Y) {
                    if (c > 0) {   // y of the chunk before has been read
                        wait_one(&sm.taken_y, ph ^ 1u, patience);
                        tc_fence_after();
                    }
#pragma unroll
                    for (int k = 0; k < kKeys / 16; ++k) read_out(col_q, k, 1, k > 0);
                    tc_commit(&sm.done_qs);
                }
                wait_one(Y ? &sm.done_qs : &sm.done_ks, ph, patience);   // S's pair has been read: U takes its place
                if (!ident) {
                    wait_one(&sm.full_v[c % kVStages], static_cast<uint32_t>(c / kVStages) & 1u, patience);
                    if (len - c * kC < kC) wait_one(&sm.zeroed_v, 0, patience);
                }
#pragma unroll
                for (int k = 0; k < 8 && !ident; ++k)   // V T hi, V T lo
                    tc_mma_f16(tmem + kColPair, dv + (k % 4) * (2048 / 16), dt + (k / 4) * (kTile / 16) + 2 * (k % 4),
                               idesc(kC, true, false), k > 0);
                wait_one(&sm.have_k, ph, patience);
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < 16; ++k) {   // (S k) hi T hi, lo T hi, hi T lo, lo T lo
                    const int part = k / 4, kk = k % 4;
                    tc_mma_f16_ts(tmem + kColPair, col_k + (kk / 2) * 32 + (kk % 2) * 8 + (part % 2 ? 16 : 0),
                                  dt + (part / 2 ? kTile / 16 : 0) + 2 * kk, idesc(kC, false, false), !ident || k > 0);
                }
                tc_commit(&sm.done_u);
                wait_one(&sm.have_d, ph, patience);
                tc_fence_after();
                constexpr uint64_t kPast = static_cast<uint64_t>((kSides - 1) * kTile >> 4) << 16;   // Q lies between K's tiles
#pragma unroll
                for (int k = 0; k < 8; ++k) {   // hi, then lo; 16 tokens = two 8-row groups of K
                    const int kk = k % 4;
                    tc_mma_f16_ts(tmem + kColS, tmem + kColPair + (kk / 2) * 32 + (kk % 2) * 8 + (k / 4) * 16,
                                  d + kPast + kk * (2048 / 16), idesc(kKeys, false, true), true);
                }
                tc_commit(&sm.done_s);
                tc_commit(&sm.free_kq[c % kStages]);
                if (Y) {
                    wait_one(&sm.have_u, ph, patience);
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 12; ++k) {   // U hi P hi, U lo P hi, U hi P lo, onto S q
                        const int part = k / 4, kk = k % 4;
                        tc_mma_f16_ts(col_q, col_k + (kk / 2) * 32 + (kk % 2) * 8 + (part == 1 ? 16 : 0),
                                      dt + (part == 2 ? 3 : 2) * (kTile / 16) + 2 * kk, idesc(kC, false, false), true);
                    }
                }
                tc_commit(&sm.free_slot[c % kSlots]);
                tc_commit(&sm.done_o[ph]);
            }
        }
        __syncwarp();
    } else if (warp == kCopyWarp) {
        // ---------------- copies and gates ----------------
        auto load_kq = [&](int c) {
            uint8_t *st = sm.kq[c % kStages];
            uint64_t *full = &sm.full_kq[c % kStages];
            mbar_arrive_expect_tx(full, NA * kSides * kTile);
            const int row = static_cast<int>(begin) + c * kC;
            for (int a = 0; a < NA; ++a) {
                tma_load_3d(st + a * kSides * kTile + tile_of(c, 0), &map_k, a * 64, qk, row, full);
                if (Y) tma_load_3d(st + a * kSides * kTile + tile_of(c, 1), &map_q, a * 64, qk, row, full);
                // the stages alone do not hide DRAM's latency: the next one's load finds its rows in L2
                if (c + 1 >= kStages && c + 1 < chunks) {
                    tma_prefetch_3d(&map_k, a * 64, qk, row + kC);
                    if (Y) tma_prefetch_3d(&map_q, a * 64, qk, row + kC);
                }
            }
        };
        float g[2], bt[2];   // of tokens 2 lane, 2 lane + 1 of a chunk to come
        auto load_gates = [&](int c) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = c * kC + 2 * lane + e;
                g[e] = bt[e] = 0.f;
                if (t < len) {
                    g[e] = p.g[(begin + t) * p.hv + head];
                    bt[e] = p.beta[(begin + t) * p.hv + head];
                }
            }
        };
        auto gate = [&](int c) {
            constexpr float kL = 1.44269502f, kLl = 1.92596303e-8f;   // log2 e
            Gates &to = sm.gates[c % kStages];
            if (g[0] > 0.f || g[1] > 0.f) sm.growing = 1u;
            Log x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v;   // NaN stays NaN
                asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(g[e]), "f"(kLeastGate));
                x[e].h = v * kL;
                x[e].l = fmaf(v, kL, -x[e].h) + v * kLl;
            }
            Log sum = x[0] + x[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const Log up = shfl_up(sum, o);
                if (lane >= o) sum = up + sum;
            }
            const Log before = shfl_up(sum, 1), total = shfl(sum, 31), last = shfl(sum, lane | 7);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const Log b = e ? sum : lane ? before + x[0] : x[0];
                const int t = 2 * lane + e;
                const float eb = ex2(b.h + b.l);
                to.bh[t] = b.h;
                to.bl[t] = b.l;
                to.to_last[t] = exp_diff(last, b);
                to.beta[t] = bt[e];
                to.ek[t] = -eb;
                to.eq[t] = p.scale * eb;
                to.ec[t] = exp_diff(total, b);
            }
            if ((lane & 7) == 7) to.last[lane / 8] = sum;
            if (lane == 31) to.whole = ex2(sum.h + sum.l);
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.gated[c % kStages]);
            __syncwarp();
        };
        for (int c = 0; c < kStages && c < chunks && lane == 0; ++c) load_kq(c);
        __syncwarp();
        load_gates(0);
#pragma unroll 1
        for (int c = 0; c < chunks; ++c) {
            if (c >= kStages) {   // its stage and its gates' place: the update of the chunk there before has read them
                wait(&sm.free_kq[c % kStages], static_cast<uint32_t>(c / kStages - 1) & 1u, patience);
                if (lane == 0) load_kq(c);
                __syncwarp();
            }
            gate(c);
            load_gates(c + 1);
            wait(&sm.full_kq[c % kStages], static_cast<uint32_t>(c / kStages) & 1u, patience);
            if (len - c * kC < kC) {   // rows beyond the end, whatever they are
                zero_rows(sm.kq[c % kStages], NA * kSides, len - c * kC, lane);
                if (lane == 0) mbar_arrive(&sm.zeroed_kq);
                __syncwarp();
            }
            // [K; Q] K^T or [Q; K] K^T, for the warps that work ahead, where the chunk there before has left
            // its place. (Where there is no Q, those 64 rows are of whatever lies before or behind K.)
            if (c >= kSlots) wait(&sm.free_slot[c % kSlots], static_cast<uint32_t>(c / kSlots - 1) & 1u, patience);
            tc_fence_after();
            if (elect_one()) {
                const uint64_t d = desc_base(sm.kq[c % kStages] + tile_of(c, 0)), up = (c & 1) * (kTile / 16);
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k) {
                    const uint64_t dk = d + (k / 4) * (kSides * kTile / 16) + 2 * (k % 4);
                    tc_mma_f16(tmem + kColK + c % kSlots * 64, dk - up, dk, idesc(kC, false, false), k > 0);
                }
                tc_commit(&sm.done_prep[c % kSlots]);
            }
            __syncwarp();
        }
    } else if (warp == kValueWarp) {
        // ---------------- V in, y out ----------------
        const int channels = p.dv - slice * kM < kM ? p.dv - slice * kM : kM;
        auto load_v = [&](int c) {
            if (ident) return;
            uint64_t *full = &sm.full_v[c % kVStages];
            const int tiles = channels > 64 ? 2 : 1;
            mbar_arrive_expect_tx(full, tiles * kTile);
            for (int a = 0; a < tiles; ++a)
                tma_load_3d(sm.v[c % kVStages] + a * kTile, &map_v, slice * kM + a * 64, head, static_cast<int>(begin) + c * kC, full);
            for (int a = 0; a < tiles && c + 1 >= kVStages && c + 1 < chunks; ++a)
                tma_prefetch_3d(&map_v, slice * kM + a * 64, head, static_cast<int>(begin) + (c + 1) * kC);
        };
#pragma unroll 1
        for (int c = 0; c < chunks + kVStages; ++c) {
            if (const int o = c - kVStages; o >= 0) {
                // the chunk before in this stage: its y
                wait(&sm.through[o % kVStages], static_cast<uint32_t>(o / kVStages) & 1u, patience);
                if (Y && p.y_dtype == PRECOG_BF16) {
                    const int n = len - o * kC < kC ? len - o * kC : kC;
                    for (int t = lane; t < n; t += 32)
                        bulk_s2g(static_cast<__nv_bfloat16 *>(p.y) + (begin + o * kC + t) * p.hv * p.dv + static_cast<int64_t>(head) * p.dv + slice * kM,
                                 sm.v[o % kVStages] + t * kM * 2, channels * 2);
                    bulk_commit();
                    bulk_wait_read<0>();
                    __syncwarp();
                }
            }
            if (c >= chunks) continue;
            if (lane == 0) load_v(c);
            __syncwarp();
            if (c + 1 == chunks && len - c * kC < kC && !ident) {
                wait(&sm.full_v[c % kVStages], static_cast<uint32_t>(c / kVStages) & 1u, patience);
                zero_rows(sm.v[c % kVStages], 2, len - c * kC, lane);
                if (lane == 0) mbar_arrive(&sm.zeroed_v);
            }
        }
        if (Y) bulk_wait_all();
        __syncwarp();
    } else if (warp >= 8) {
        // ---------------- T and P, ahead of the chain ----------------
        const int team = (warp >> 2) & 1, quarter = warp & 3, tid = threadIdx.x & (kTeam - 1);
        const int half = quarter & 1, i = half * kH + lane;   // this thread's row: of A or P
        const bool is_a = quarter / 2 == team;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        float *a11 = sm.a[team], *a21 = a11 + kBlock, *a22 = a21 + kBlock;
#pragma unroll 1
        for (int c = team; c < chunks; c += 2) {
            const uint32_t col = tmem + kColK + c % kSlots * 64;
            const Gates &gt = sm.gates[c % kStages];
            wait(&sm.done_prep[c % kSlots], static_cast<uint32_t>(c / kSlots) & 1u, patience);
            wait(&sm.gated[c % kStages], static_cast<uint32_t>(c / kStages) & 1u, patience);
            tc_fence_after();
            const Log bi{gt.bh[i], gt.bl[i]};
            const f2 bih = pack2(bi.h, bi.h), bil = pack2(bi.l, bi.l), minus = pack2(-1.f, -1.f);
            const float mine = is_a ? gt.beta[i] : p.scale;
            // two chunks ago: through with T and P
            if (Y && !is_a && c >= 2) wait(&sm.done_o[team], static_cast<uint32_t>((c - 2) >> 1) & 1u, patience);
            // Columns of 16. Left of the diagonal half the decay from j to i goes by the last token of the
            // 16, both factors at most 1 where nothing grows; on it each entry has its exponential.
#pragma unroll 1
            for (int j0 = 0; j0 < (is_a || Y ? (half + 1) * kH : 0); j0 += kB) {
                float v[16];
                tmem_ld16(col + lanes + j0, v);
                if (j0 < half * kH) {
                    const float f = exp_diff(bi, gt.last[j0 / 16]) * mine;
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] *= f * gt.to_last[j0 + e];
                } else {
                    const int lim = i + (is_a ? 0 : 1) - j0;
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        float x, y;
                        unpack2(fma2(load2(gt.bl + j0 + e), minus, fma2(fma2(load2(gt.bh + j0 + e), minus, bih), pack2(1.f, 1.f), bil)), x, y);
                        v[e] = e < lim ? v[e] * (ex2(x) * mine) : 0.f;
                        v[e + 1] = e + 1 < lim ? v[e + 1] * (ex2(y) * mine) : 0.f;
                    }
                }
                if (is_a) {
                    float *to = (half == 0 ? a11 : j0 < kH ? a21 : a22) + (j0 & (kH - 1)) * kH;
#pragma unroll
                    for (int e = 0; e < 16; ++e) to[e * kH + (lane ^ ((e & 3) << 3))] = v[e];
                } else if constexpr (Y) {
#pragma unroll
                    for (int o = 0; o < 16; o += 8) {
                        uint32_t h[4], l[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) split(v[o + 2 * e], v[o + 2 * e + 1], h[e], l[e]);
                        const int to = i * 128 + (((j0 + o) / 8) ^ (i & 7)) * 16;
                        *reinterpret_cast<uint4 *>(sm.tp[team][2] + to) = make_uint4(h[0], h[1], h[2], h[3]);
                        *reinterpret_cast<uint4 *>(sm.tp[team][3] + to) = make_uint4(l[0], l[1], l[2], l[3]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            // ---- (I + A)^-1 of one half a warp: two blocks of 16, a column a lane ----
            f2 sum[2][2];
            if (is_a) {
                float *a = half == 0 ? a11 : a22;
                const int b = lane & 16, cc = lane & 15;
                f2 x[kB / 2];
#pragma unroll
                for (int e = 0; e < kB / 2; ++e) x[e] = pack2(2 * e == cc ? 1.f : 0.f, 2 * e + 1 == cc ? 1.f : 0.f);
                // from I, rows below l lose A[.][l] T[l], l = 0, 1, ..
#pragma unroll
                for (int l = 0; l < kB - 1; ++l) {
                    float even, odd;
                    unpack2(x[l / 2], even, odd);
                    const float m = -(l % 2 ? odd : even);
                    const f2 mm = pack2(m, m);
#pragma unroll
                    for (int e = (l + 1) / 4 * 4; e < kB; e += 4) {
                        const float4 w = *reinterpret_cast<const float4 *>(a + (b + l) * kH + ((b + e) ^ ((l & 3) << 3)));
                        x[e / 2] = fma2(pack2(w.x, w.y), mm, x[e / 2]);
                        x[e / 2 + 1] = fma2(pack2(w.z, w.w), mm, x[e / 2 + 1]);
                    }
                }
                __syncwarp();
#pragma unroll
                for (int e = 0; e < kB; e += 4) {
                    float4 w;
                    unpack2(x[e / 2], w.x, w.y);
                    unpack2(x[e / 2 + 1], w.z, w.w);
                    *reinterpret_cast<float4 *>(a + (b + cc) * kH + ((b + e) ^ ((cc & 3) << 3))) = w;
                }
                __syncwarp();
                // -(T1 A10) T0 in the place of A10
                const int r = kB + (lane & 3) * 4, n = (lane >> 2) * 2;
                product<kB>(sum, a, kB, r, a, kB, n);
                __syncwarp();   // A10 has been read
                store_product(sum, 1.f, a, r, n);
                __syncwarp();
                product<kB>(sum, a, 0, r, a, 0, n);
                __syncwarp();
                store_product(sum, -1.f, a, r, n);
            }
            named_sync(kBarTeam + team, kTeam);
            // ---- joined: 8 columns a warp, T22 A21 in the place of A21 and then T21 in its place ----
            {
                const int r = (lane & 7) * 4, n = quarter * 8 + (lane >> 3) * 2;
                product<kH>(sum, a22, 0, r, a21, 0, n);
                __syncwarp();   // these columns have been read
                store_product(sum, 1.f, a21, r, n);
                named_sync(kBarTeam + team, kTeam);
                product<kH>(sum, a21, 0, r, a11, 0, n);
                named_sync(kBarTeam + team, kTeam);
                store_product(sum, -1.f, a21, r, n);
            }
            if (is_a && c >= 2) wait(&sm.done_o[team], static_cast<uint32_t>((c - 2) >> 1) & 1u, patience);
            named_sync(kBarTeam + team, kTeam);
            // ---- T diag(beta) as a pair: a row's 32 columns a thread ----
            const int row = tid & (kC - 1), j1 = tid / kC * kH;
            if (j1 <= row) {   // (whole warps)
                const float *from = row < kH ? a11 : j1 ? a22 : a21;
#pragma unroll 1
                for (int j0 = 0; j0 < kH; j0 += kB) {
                    uint32_t h[8], l[8];
#pragma unroll
                    for (int e = 0; e < kB; e += 2)
                        split(mul2(pack2(from[(j0 + e) * kH + (lane ^ ((e & 3) << 3))], from[(j0 + e + 1) * kH + (lane ^ (((e + 1) & 3) << 3))]),
                                   load2(gt.beta + j1 + j0 + e)),
                              h[e / 2], l[e / 2]);
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const int to = row * 128 + (((j1 + j0) / 8 + o) ^ (row & 7)) * 16;
                        *reinterpret_cast<uint4 *>(sm.tp[team][0] + to) = make_uint4(h[4 * o], h[4 * o + 1], h[4 * o + 2], h[4 * o + 3]);
                        *reinterpret_cast<uint4 *>(sm.tp[team][1] + to) = make_uint4(l[4 * o], l[4 * o + 1], l[4 * o + 2], l[4 * o + 3]);
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.ready[team]);
            named_sync(kBarTeam + team, kTeam);   // A may be written again
        }
    } else {
        // ---------------- the chain ----------------
        const int half = warp >> 2, quarter = warp & 3;
        const int row = quarter * 32 + lane;             // value channel within the slice
        const int ch = slice * kM + row;                 // and within the head
        const uint32_t tm = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        const bool live = ident ? row < p.dk : ch < p.dv;
        constexpr int kHalf = kKeys / 2;                 // S's columns of this half of the warps
        const uint32_t col_s = tm + kColS + half * kHalf;
        {   // initial state
            const int64_t head_elems = static_cast<int64_t>(p.dv) * p.dk;
            Job job = {begin, end, {nullptr, PRECOG_F32, 0}, {nullptr, PRECOG_F32, 0}, head, ident, !kept || (first && !ident)};
            if (CUT && first && !last && cut.joined) {   // (the bank may be where the last segment's state goes)
                job.from = States{cut.begins, PRECOG_F32, (seq * p.hv + head) * head_elems};
            } else if (first && p.bank && !ident) {
                const int64_t entry = p.idx ? p.idx[seq] : seq;
                if (entry < -1 || entry >= p.bank_entries) {
                    if (threadIdx.x == 0) atomicOr(&g_delta_chunk_status, PRECOG_DEV_BAD_INDEX);
                } else if (entry >= 0) {
                    job.from = States{const_cast<void *>(p.bank), p.bank_dtype, ((entry * p.L_total + p.layer) * p.hv + head) * head_elems};
                }
            } else if (CUT && !first && cut.joined) {
                job.from = States{cut.states, PRECOG_F32, ((slot - 1) * p.hv + head) * head_elems};
            }
            if (ident) job.to = States{cut.moves, PRECOG_F32, (slot * p.hv + head) * p.dk * p.dk};
            else if (kept) job.to = States{cut.states, PRECOG_F32, (slot * p.hv + head) * head_elems};
            else if (last && p.states) job.to = States{p.states, p.state_dtype, ((seq * p.L_total + p.layer) * p.hv + head) * head_elems};
            if (threadIdx.x == 0) sm.job = job;     // (for the end)
            const States from = job.from;
            const int64_t at = from.at + static_cast<int64_t>(ch) * p.dk;
#pragma unroll
            for (int g = 0; g < kHalf; g += 32) {
                uint32_t r[32];
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    const int col = half * kHalf + g + e;
                    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    if (from.base && live && col < p.dk) delta_load8(from.base, from.dtype, at + col, v);
                    if (ident && row >= col && row < col + 8) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = row == col + x ? 1.f : 0.f;
                    }
                    if (kept && first && !ident && live && col < p.dk)
                        delta_store8(cut.begins, PRECOG_F32, ((seq * p.hv + head) * p.dv + ch) * static_cast<int64_t>(p.dk) + col, v);
#pragma unroll
                    for (int x = 0; x < 8; ++x) r[e + x] = __float_as_uint(v[x]);
                }
                __syncwarp();
                tmem_st32(col_s + g, r);
            }
            tmem_st_wait();
        }
        // What this warp stored into tensor memory is there for the MMAs.
        auto hand_over = [&](uint64_t *bar) {
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            __syncwarp();
        };
        const int64_t y_row = static_cast<int64_t>(p.hv) * p.dv;
        if (chunks > 0) wait(&sm.gated[0], 0, patience);
#pragma unroll 1
        for (int c = 0; c <= chunks; ++c) {   // the last turn only leaves the last chunk
            const int buf = c & 1;
            const uint32_t ph = static_cast<uint32_t>(c) & 1u;
            const Gates &gt = sm.gates[c % kStages];
            const uint32_t col_k = tm + kColK + c % kSlots * 64 + half * 32, col_q = tm + kColQ + half * 32;
            if (c < chunks) {
                // ---- S as a pair ----
#pragma unroll 1
                for (int g = 0; g < kHalf; g += 32) {
                    uint32_t r[32], h[16], l[16];
                    tmem_ld32_async(col_s + g, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int e = 0; e < 16; ++e) split(pair_of(r, e), h[e], l[e]);
                    tmem_st16(tm + kColPair + (half * kHalf + g) / 2, h);
                    tmem_st16(tm + kColPair + kHalf + (half * kHalf + g) / 2, l);
                    hand_over(&sm.have_s[g / 32]);
                }
            }
            if (c > 0) {
                wait(&sm.done_o[buf ^ 1], static_cast<uint32_t>((c - 1) >> 1) & 1u, patience);
                tc_fence_after();
                // ---- y of the chunk before, tokens 32 half .. , while S k is formed ----
                if (Y) {
                    uint32_t r[32];
                    tmem_ld32_async(col_q, r);
                    tmem_ld_wait(r);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.taken_y);
                    const int t0 = (c - 1) * kC + half * 32;
                    if (p.y_dtype == PRECOG_F32) {
                        float *to = static_cast<float *>(p.y) + (begin + t0) * y_row + static_cast<int64_t>(head) * p.dv + ch;
                        if (live) {
#pragma unroll
                            for (int e = 0; e < 32; ++e, to += y_row)
                                if (t0 + e < len) *to = __uint_as_float(r[e]);
                        }
                    } else {   // rows of 128 channels, for the copies
                        uint16_t *to = reinterpret_cast<uint16_t *>(sm.v[(c - 1) % kVStages]) + half * 32 * kM + row;
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const uint32_t w = bits2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]));
                            to[2 * e * kM] = static_cast<uint16_t>(w);
                            to[(2 * e + 1) * kM] = static_cast<uint16_t>(w >> 16);
                        }
                        fence_proxy_async_smem();
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.through[(c - 1) % kVStages]);
                __syncwarp();
            }
            if (c == chunks) break;
            // ---- -e^b S k as a pair in its own place: hi of this half's 32 tokens, then lo ----
            wait(&sm.done_ks, ph, patience);
            tc_fence_after();
            {
                uint32_t r[32], h[16], l[16];
                tmem_ld32_async(col_k, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) split(mul2(load2(gt.ek + half * 32 + 2 * e), pair_of(r, e)), h[e], l[e]);
                tmem_st16(col_k, h);
                tmem_st16(col_k + 16, l);
            }
            hand_over(&sm.have_k);
            // ---- S decayed, while U is formed ----
            const f2 whole = pack2(gt.whole, gt.whole);
#pragma unroll 1
            for (int g = 0; g < kHalf; g += 32) {
                uint32_t r[32];
                tmem_ld32_async(col_s + g, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float a, b;
                    unpack2(mul2(pair_of(r, e), whole), a, b);
                    r[2 * e] = __float_as_uint(a);
                    r[2 * e + 1] = __float_as_uint(b);
                }
                tmem_st32(col_s + g, r);
            }
            if (Y) {   // scale e^b S q: P U adds to it
                wait(&sm.done_qs, ph, patience);
                tc_fence_after();
                uint32_t r[32];
                tmem_ld32_async(col_q, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float a, b;
                    unpack2(mul2(load2(gt.eq + half * 32 + 2 * e), pair_of(r, e)), a, b);
                    r[2 * e] = __float_as_uint(a);
                    r[2 * e + 1] = __float_as_uint(b);
                }
                tmem_st32(col_q, r);
            }
            // ---- U decayed to the chunk's end, as a pair in U's place, for the update; then U's pair ----
            wait(&sm.done_u, ph, patience);
            tc_fence_after();
            {
                uint32_t r[32], h[16], l[16];
                tmem_ld32_async(tm + kColPair + half * 32, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) split(mul2(load2(gt.ec + half * 32 + 2 * e), pair_of(r, e)), h[e], l[e]);
                tmem_st16(tm + kColPair + half * 32, h);
                tmem_st16(tm + kColPair + half * 32 + 16, l);
                hand_over(&sm.have_d);
                if (Y) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) split(pair_of(r, e), h[e], l[e]);
                    tmem_st16(col_k, h);
                    tmem_st16(col_k + 16, l);
                    hand_over(&sm.have_u);
                }
            }
            if (c + 1 < chunks) wait(&sm.gated[(c + 1) % kStages], static_cast<uint32_t>((c + 1) / kStages) & 1u, patience);
            wait(&sm.done_s, ph, patience);
            tc_fence_after();
        }
        // ---- the state leaves; broken rows are left to once_more ----
        {
            named_sync(kBarChain, kChain);   // (thread 0 wrote the job, which a sequence without chunks waits for here alone)
            const bool again = !kept || (first && !ident), grown = sm.growing != 0u && too_far(p, sm.job);
            uint32_t r[NA][32];
            f2 zeros = pack2(0.f, 0.f);      // 0 x, summed
#pragma unroll
            for (int g = 0; g < NA; ++g) {
                tmem_ld32_async(col_s + g * 32, r[g]);
                tmem_ld_wait(r[g]);
#pragma unroll
                for (int e = 0; e < 16; ++e) zeros = fma2(pair_of(r[g], e), pack2(0.f, 0.f), zeros);
            }
            float x, y;
            unpack2(zeros, x, y);
            if (live && (grown || (again && !(x + y == 0.f)))) atomicOr(&sm.broken[quarter], 1u << lane);
            named_sync(kBarChain, kChain);
            const States to = sm.job.to;
            const int64_t at = to.at + static_cast<int64_t>(ident ? row : ch) * p.dk;
            const bool broke = (sm.broken[quarter] >> lane & 1u) != 0u;
            if (to.base && live && !(broke && again)) {
#pragma unroll
                for (int e = 0; e < kHalf; e += 8)
                    if (const int col = half * kHalf + e; col < p.dk) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = ident && broke ? __int_as_float(0x7fffffff) : __uint_as_float(r[e / 32][e % 32 + i]);
                        delta_store8(to.base, to.dtype, at + col, v);   // (NaN for M: the join goes without it)
                    }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    static_assert(again_bytes(kKeys) <= static_cast<int>(sizeof(sm.v) + sizeof(sm.kq)), "the tokens' room");
    if (sm.job.again && warp < kAgain / 32 && (sm.broken[0] | sm.broken[1] | sm.broken[2] | sm.broken[3]) != 0u)
        once_more<NA, Y>(p, sm.job, reinterpret_cast<float *>(sm.v), slice * kM, sm.broken);
}

// The segments' initial states: state after segment s = state before it * M + B, in the place of B,
// for 16 value channels a CTA. M comes through shared memory, the next one while this one is used.
constexpr int kJoinRows = 16, kJoinThreads = 128;

// Four rows of a state, a lane 4 columns of each, rolled over tokens t .. end - 1 as the recurrence is
// defined: where B or M is not finite, or M was given up because the segment's gates grow. Four tokens' loads
// are in flight at a time (32,768 tokens of 16 heads whose gates grow throughout: 8.8 ms, decaying 0.69).
__device__ __noinline__ void rolled(const DeltaParams &p, float4 (&s)[4], int head, int row, int64_t t, int64_t end) {
    const int c = (threadIdx.x & 31) * 4, qk = head / (p.hv / p.hk);
    const __nv_bfloat16 *kp = static_cast<const __nv_bfloat16 *>(p.k) + static_cast<int64_t>(qk) * p.dk + c;
    const __nv_bfloat16 *vp = static_cast<const __nv_bfloat16 *>(p.v) + static_cast<int64_t>(head) * p.dv + row;
#pragma unroll 1
    for (; t < end; t += 4) {
        uint2 k[4];
        float g[4], beta[4], v[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // (beyond the end: nothing decays, nothing enters)
            const bool there = t + u < end;
            k[u] = there && c < p.dk ? *reinterpret_cast<const uint2 *>(kp + (t + u) * p.k_stride) : make_uint2(0u, 0u);
            g[u] = there ? p.g[(t + u) * p.hv + head] : 0.f;
            beta[u] = there ? p.beta[(t + u) * p.hv + head] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[u][i] = there && row + i < p.dv ? to_f32(vp[(t + u) * p.v_stride + i]) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (t + u >= end) break;
            const float x = __uint_as_float(k[u].x << 16), y = __uint_as_float(k[u].x & 0xffff0000u);
            const float z = __uint_as_float(k[u].y << 16), w = __uint_as_float(k[u].y & 0xffff0000u);
            const float a = g[u] < kLeastGate ? 0.f : expf(g[u]);
            float sk[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sk[i] = fmaf(s[i].w, w, fmaf(s[i].z, z, fmaf(s[i].y, y, s[i].x * x)));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) sk[i] += __shfl_xor_sync(0xffffffffu, sk[i], o);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float n = beta[u] * fmaf(-a, sk[i], v[u][i]);
                s[i] = make_float4(fmaf(n, x, a * s[i].x), fmaf(n, y, a * s[i].y), fmaf(n, z, a * s[i].z), fmaf(n, w, a * s[i].w));
            }
        }
    }
}

__global__ void __launch_bounds__(kJoinThreads) delta_join_kernel(const __grid_constant__ DeltaParams p, const Cut cut) {
    extern __shared__ __align__(16) float join_smem[];
    const int dk = p.dk, pitch = dk + 4;
    float *move[2] = {join_smem, join_smem + dk * dk};
    float *rows = join_smem + 2 * dk * dk;                 // [16][pitch]
    const int tiles = (p.dv + kJoinRows - 1) / kJoinRows;
    int64_t item = blockIdx.x;
    const int r0 = static_cast<int>(item % tiles) * kJoinRows;
    item /= tiles;
    const int head = static_cast<int>(item % p.hv);
    const int64_t seq = item / p.hv;
    const int64_t begin = p.offsets[seq], end = p.offsets[seq + 1];
    for (int64_t c = 0; c <= seq; ++c)                     // as the segments' own kernel: up to the first bad one
        if (p.offsets[c] < 0 || p.offsets[c + 1] < p.offsets[c] || p.offsets[c + 1] > p.T_tot) return;
    const int64_t base = begin / cut.len + seq, segs = segments(end - begin, cut.len);
    if (segs < 3) return;                                  // the second begins where the first ended
    const int quads = dk / 4;
    auto fetch = [&](int64_t seg) {
        const float *from = cut.moves + ((base + seg) * p.hv + head) * dk * dk;
        for (int e = threadIdx.x; e < dk * quads; e += kJoinThreads) cp_async16(move[seg & 1] + 4 * e, from + 4 * e);
        cp_async_commit();
    };
    auto state = [&](int64_t seg, int r) { return cut.states + (((base + seg) * p.hv + head) * p.dv + r0 + r) * dk; };
    fetch(1);
    for (int e = threadIdx.x; e < kJoinRows * quads; e += kJoinThreads) {
        const int r = e / quads, c = e % quads;
        const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
        *reinterpret_cast<float4 *>(rows + r * pitch + 4 * c) = r0 + r < p.dv ? *reinterpret_cast<const float4 *>(state(0, r) + 4 * c) : zero;
    }
    // thread: 4 rows of warp `threadIdx.x / 32`, 4 columns
    const int r = threadIdx.x / 32 * 4, c = threadIdx.x % 32 * 4;
    // The rows behind segment `seg`, from what they were before it: those that broke in it.
    auto mend = [&](float4 (&now)[4], int64_t seg) {
        auto whole = [&](float4 v) { return __all_sync(0xffffffffu, c >= dk || (isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w))); };
        float4 was[4];
        bool broke[4], any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            was[i] = c < dk ? *reinterpret_cast<const float4 *>(rows + (r + i) * pitch + c) : make_float4(0.f, 0.f, 0.f, 0.f);
            broke[i] = r0 + r + i < p.dv && !whole(now[i]) && whole(was[i]);
            any |= broke[i];
        }
        if (!any) return;
        rolled(p, was, head, r0 + r, begin + seg * cut.len, begin + (seg + 1) * cut.len);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (broke[i]) now[i] = was[i];
    };
    for (int64_t seg = 1; seg + 1 < segs; ++seg) {
        if (seg + 2 < segs) fetch(seg + 1);
        else cp_async_commit();
        float4 b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            b[i] = c < dk && r0 + r + i < p.dv ? *reinterpret_cast<const float4 *>(state(seg, r + i) + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        cp_async_wait<1>();
        __syncthreads();
        f2 acc[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][0] = pack2(b[i].x, b[i].y), acc[i][1] = pack2(b[i].z, b[i].w);
        const float *m = move[seg & 1];
        if (c < dk) {
#pragma unroll 2
            for (int k = 0; k < dk; k += 4) {
                float4 s[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = *reinterpret_cast<const float4 *>(rows + (r + i) * pitch + k);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 x = *reinterpret_cast<const float4 *>(m + (k + e) * dk + c);
                    const f2 lo = pack2(x.x, x.y), hi = pack2(x.z, x.w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = e == 0 ? s[i].x : e == 1 ? s[i].y : e == 2 ? s[i].z : s[i].w;
                        acc[i][0] = fma2(pack2(v, v), lo, acc[i][0]);
                        acc[i][1] = fma2(pack2(v, v), hi, acc[i][1]);
                    }
                }
            }
        }
        __syncthreads();
        float4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unpack2(acc[i][0], x[i].x, x[i].y);
            unpack2(acc[i][1], x[i].z, x[i].w);
        }
        mend(x, seg);
        if (c < dk) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                *reinterpret_cast<float4 *>(rows + (r + i) * pitch + c) = x[i];
                if (r0 + r + i < p.dv) *reinterpret_cast<float4 *>(state(seg, r + i) + c) = x[i];
            }
        }
        __syncthreads();
    }
}

struct Maps {
    CUtensorMap q, k, v;
};

template <int NA, bool Y, bool CUT>
cudaError_t launch(const DeltaParams &p, const Maps &maps, int slices, const Cut &cut, cudaStream_t stream) {
    auto kern = delta_chunk_kernel<NA, Y, CUT>;
    const int smem = static_cast<int>(sizeof(Smem<NA, Y>) + 1024);
    static_assert(sizeof(Smem<NA, Y>) + 1024 <= 227 * 1024, "one CTA's shared memory");
    cudaError_t e = ensure_smem(reinterpret_cast<const void *>(kern), smem);
    if (e != cudaSuccess) return e;
    const int64_t ctas = (CUT ? cut.slots : p.n_seqs) * p.hv * (slices + (CUT && !cut.joined ? 1 : 0));
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    kern<<<static_cast<unsigned>(ctas), kThreads, smem, stream>>>(maps.q, maps.k, maps.v, p, slices, cut);
    e = cudaGetLastError();
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <int NA>
cudaError_t launch_all(const DeltaParams &p, const Maps &maps, int slices, Cut cut, cudaStream_t stream) {
    cudaError_t e;
    if (cut.len) {
        e = launch<NA, false, true>(p, maps, slices, cut, stream);
        if (e != cudaSuccess) return e;
        const int smem = (2 * p.dk * p.dk + kJoinRows * (p.dk + 4)) * 4;
        e = ensure_smem(reinterpret_cast<const void *>(delta_join_kernel), smem);
        if (e != cudaSuccess) return e;
        const int64_t ctas = p.n_seqs * p.hv * ((p.dv + kJoinRows - 1) / kJoinRows);
        delta_join_kernel<<<static_cast<unsigned>(ctas), kJoinThreads, smem, stream>>>(p, cut);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        count_launches(1);
        cut.joined = 1;
        return p.y ? launch<NA, true, true>(p, maps, slices, cut, stream) : launch<NA, false, true>(p, maps, slices, cut, stream);
    }
    return p.y ? launch<NA, true, false>(p, maps, slices, cut, stream) : launch<NA, false, false>(p, maps, slices, cut, stream);
}

// The segments' length for these sizes, or 0. In chunks of 64 tokens, of which a CTA takes one after
// another: whole sequences are as long as their rounds of CTAs; segments go in one pass for B and M,
// one step of the join each, and one pass for themselves. Cut only where that is a third shorter: the
// estimate knows the sequences' mean length alone. One sequence, 16 heads of 128 x 128, with a readout:
// 2048 tokens 89 us (whole 116), 4096 tokens 130 (222), 32,768 tokens 681 (1702).
int cut_length(const DeltaParams &p) {
    const int64_t sms = device_sm_count(), slices = (p.dv + kM - 1) / kM, items = p.n_seqs * p.hv * slices;
    if (items > sms || p.T_tot / p.n_seqs < 16 * kC) return 0;
    const int64_t chunks = p.T_tot / kC;
    auto rounds = [&](int64_t ctas) { return (ctas + sms - 1) / sms; };
    int64_t best = chunks / p.n_seqs, len = 0;
    for (int64_t per = 4; per < chunks / p.n_seqs; per += 1 + per / 16) {   // chunks of a segment
        const int64_t segs = (chunks / p.n_seqs + per - 1) / per;            // of a mean sequence
        const int64_t cost = per * (rounds((items + p.n_seqs * p.hv) * (segs - 1)) + rounds(items * segs)) + segs;
        if (cost * 3 < best * 2 || (len && cost < best)) best = cost, len = per;
    }
    return static_cast<int>(len * kC);
}

// [rows][heads][dim] bf16 with `stride` elements between rows, in boxes of 64 columns of 64
// rows of one head.
bool rows_map(CUtensorMap *map, const void *base, int dim, int heads, int64_t rows, int64_t stride) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
    if (rows == 1) stride = static_cast<int64_t>(heads) * dim;
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(dim) * 2, static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t box[3] = {64, 1, kC};
    return encode_tiled_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box,
                            CU_TENSOR_MAP_SWIZZLE_128B);
}

}  // namespace

size_t delta_chunk_workspace_size(const DeltaParams &p) {
    const int64_t len = cut_length(p);
    if (len == 0) return 0;
    return (static_cast<size_t>(p.T_tot / len + p.n_seqs) * (p.dv + p.dk) + static_cast<size_t>(p.n_seqs) * p.dv) * p.hv * p.dk * sizeof(float);
}

cudaError_t launch_delta_chunk(const DeltaParams &p, cudaStream_t stream) {
    const bool want_y = p.y != nullptr;
    const int slices = (p.dv + kM - 1) / kM;
    Maps maps;
    if (!rows_map(&maps.k, p.k, p.dk, p.hk, p.T_tot, p.k_stride) ||
        !rows_map(&maps.q, want_y ? p.q : p.k, p.dk, p.hk, p.T_tot, want_y ? p.q_stride : p.k_stride) ||
        !rows_map(&maps.v, p.v, p.dv, p.hv, p.T_tot, p.v_stride))
        return cudaErrorInvalidValue;
    Cut cut = {};
    cut.len = cut_length(p);
    if (cut.len) {
        cut.slots = static_cast<int>(p.T_tot / cut.len + p.n_seqs);
        cut.states = static_cast<float *>(p.workspace);
        cut.moves = cut.states + static_cast<int64_t>(cut.slots) * p.hv * p.dv * p.dk;
        cut.begins = cut.moves + static_cast<int64_t>(cut.slots) * p.hv * p.dk * p.dk;
    }
    return p.dk <= 64 ? launch_all<1>(p, maps, slices, cut, stream) : launch_all<2>(p, maps, slices, cut, stream);
}

cudaError_t delta_chunk_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_delta_chunk_status); }

}  // namespace precog
