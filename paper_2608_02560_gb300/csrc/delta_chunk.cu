// The gated delta rule in chunks of 64 tokens on the 5th-generation tensor cores (bf16 inputs).
//
// With b the running sum of the log decays within a chunk and S the state before it,
//   A[i][j] = beta_i e^{b_i-b_j} k_i.k_j (j < i),   T = (I + A)^-1,
//   X_i = beta_i (v_i - e^{b_i} S k_i),             U = T X,
//   y_i = scale (e^{b_i} S q_i + sum_{j<=i} e^{b_i-b_j} (q_i.k_j) U_j),
//   S  <- e^{b_C} S + sum_j e^{b_C-b_j} U_j k_j^T.
// A CTA owns 128 value channels of one (sequence, head): S^T's rows are the lanes of tensor
// memory, so every product has M = 128 and everything that follows a product (scales, the
// correction X, the splits below) is a thread's own row. K and Q tiles enter the MMAs as the TMA
// laid them down, both as [token][key] (k.q products, S k, S q) and as [key][token] (the update).
//
// Precision: the inputs are exact bf16 operands; S, X, U, T and P, which are not, enter as pairs
// hi + lo of bf16 numbers (16 significant bits), products of two pairs without lo * lo. Sums and
// the state itself stay fp32. A single bf16 would put 2^-9 of S into every y.
//
// Warps 0-7, the chain: what each chunk needs of the chunk before it, half the columns each
// group of four. Per chunk: split S, [S k], [S q], X, [U], split U, [update], [P U]; [..] are
// MMAs that one thread issues. y of a chunk leaves while the next one's first MMAs run.
// Warps 8-11, one chunk ahead: [k.k, q.k], A and P with their decays, the inverse T by
// substitution in fp32 (a product form of the inverse would lose its digits where keys repeat).
// Warp 12: copies, three chunks deep, and y rows out.
// All loops over columns are kept rolled: fully unrolled, the three roles' code was several times
// the instruction cache and warps waited for instructions 40 % of the time (25,000 cycles a chunk).
// Tokens beyond a sequence's end have beta 0 and zeroed rows: whatever the memory holds, nothing
// of them enters a sum.
//
// Tensor memory: S [128 columns]; a pair area [128]: S's pair, then U (whose place its decayed pair
// takes) and U's pair; two places [64 + 64] by the chunk's parity: S k, in its place X's pair, then
// P U | S q. The chunk after next's k.k and q.k products lie where P U was.
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
constexpr int kStages = 3;
constexpr int kChain = 256, kPrep = 128;   // threads
constexpr int kThreads = kChain + kPrep + 32;
constexpr int kH = kC / 2;             // T is solved for in halves
constexpr int kPad = kH + 4;
constexpr uint32_t kTile = kC * 128;   // bytes of a [64 tokens][64 keys] bf16 tile
constexpr float kLeastGate = -128.f;   // e^-128 is 0 in fp32

// tensor memory columns
constexpr uint32_t kColS = 0, kColPair = 128, kColK = 256, kColQ = kColK + 64, kPlace = 128;

constexpr int kBarChain = 1, kBarPrep = 2;

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

template <int NA>
struct Smem {
    // per stage: [K][Q] tiles of key columns 0..63, then of 64..127, then V rows; the chunk's y rows
    // lie there on their way out
    uint8_t ring[kStages][NA * 2 * kTile + kC * kM * 2];
    // T hi, T lo, P hi, P lo; while T is solved for, A^T in fp32 fills the place of T
    uint8_t tp[2][4][kTile];
    float eb[2][kC];      // e^{b_j}
    float ec[2][kC];      // e^{b_C - b_j}
    float beta[2][kC];
    float bk[2][kC];      // -beta_j e^{b_j}
    Log b[kC];            // in units of log2
    Log last[4];          // b of the last token of each 16
    float to_last[kC];    // e^{last - b_j}
    float t11[kH][kH];    // [row][column]
    float t22[kH][kPad];  // [column][row]
    float mid[kH][kH];    // A21 T11
    uint64_t full[kStages], through[kStages];
    uint64_t ready[2];
    uint64_t done_prep, done_ks, done_qs, done_u, done_s, done_o;
    uint32_t tmem_base;
};

__device__ __forceinline__ uint64_t desc_base(const void *tile) {
    uint64_t d = (smem_u32(tile) & 0x3ffffu) >> 4;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;     // 8-row groups
    d |= static_cast<uint64_t>(1) << 16;             // leading offset (one atom wide: unused)
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;             // 128-byte swizzle
    return d;
}

// bf16 operands, fp32 sums, M = 128; `mn`: B's rows run along K.
__host__ __device__ constexpr uint32_t idesc(int n, bool mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((mn ? 1u : 0u) << 16) | (static_cast<uint32_t>(n >> 3) << 17) |
           (static_cast<uint32_t>(kM >> 4) << 24);
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
// (a, b) as a pair of bf16 in h and what that leaves, again in bf16, in l.
__device__ __forceinline__ void split(float a, float b, uint32_t &h, uint32_t &l) {
    h = bits2(a, b);
    l = bits2(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xffff0000u));
}

template <int NA, bool Y>
__global__ void __launch_bounds__(kThreads, 1)
    delta_chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const DeltaParams p, int slices, int v_cols) {
    constexpr int kKeys = NA * 64;               // key coordinates, padded
    constexpr uint32_t kVOff = NA * 2 * kTile;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // (an offset, not a rounded address: the compiler would lose that it is shared memory)
    Smem<NA> &sm = *reinterpret_cast<Smem<NA> *>(smem_raw + ((0u - smem_u32(smem_raw)) & 1023u));
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint32_t patience = kWaitLimit;

    int64_t item = blockIdx.x;
    const int slice = static_cast<int>(item % slices);
    item /= slices;
    const int head = static_cast<int>(item % p.hv);
    const int64_t seq = item / p.hv;
    const int64_t begin = p.offsets[seq], end = p.offsets[seq + 1];
    if (begin < 0 || end < begin || end > p.T_tot) {
        if (threadIdx.x == 0) atomicOr(&g_delta_chunk_status, PRECOG_DEV_BAD_OFFSETS);
        return;
    }
    const int len = static_cast<int>(end - begin);
    const int chunks = (len + kC - 1) / kC;
    const int qk = head / (p.hv / p.hk);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.through[s], kChain / 32);
        }
        for (int i = 0; i < 2; ++i) mbar_init(&sm.ready[i], kPrep);
        mbar_init(&sm.done_prep, 1);
        mbar_init(&sm.done_ks, 1);
        mbar_init(&sm.done_qs, 1);
        mbar_init(&sm.done_u, 1);
        mbar_init(&sm.done_s, 1);
        mbar_init(&sm.done_o, 1);
        fence_barrier_init();
    }
    if (warp == 12) {
        tmem_alloc(&sm.tmem_base, 512);
        tmem_relinquish();
    }
    // P's upper 16 x 16 blocks are zero for good
    for (int e = threadIdx.x; e < 4 * static_cast<int>(kTile) / 16; e += kThreads) {
        const int buf = e / (2 * kTile / 16);
        reinterpret_cast<uint4 *>(sm.tp[buf][2])[e % (2 * kTile / 16)] = make_uint4(0u, 0u, 0u, 0u);
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // all 512 columns: they begin at 0, and addresses are constants below
    constexpr uint32_t tmem = 0;

    if (warp == 12) {
        // ---------------- copies ----------------
        const uint32_t y_size = p.y_dtype == PRECOG_F32 ? 4 : 2;
        const uint32_t y_pitch = v_cols * y_size;
        const int y_cols = p.dv - slice * kM < v_cols ? p.dv - slice * kM : v_cols;
        auto load = [&](int c) {
            uint8_t *st = sm.ring[c % kStages];
            uint64_t *full = &sm.full[c % kStages];
            const int row = static_cast<int>(begin) + c * kC;
            mbar_arrive_expect_tx(full, NA * (Y ? 2 : 1) * kTile + kC * v_cols * 2);
            for (int a = 0; a < NA; ++a) {
                tma_load_3d(st + a * 2 * kTile, &map_k, a * 64, qk, row, full);
                if (Y) tma_load_3d(st + a * 2 * kTile + kTile, &map_q, a * 64, qk, row, full);
            }
            tma_load_3d(st + kVOff, &map_v, slice * kM, head, row, full);
        };
        for (int c = 0; c < kStages && c < chunks && lane == 0; ++c) load(c);
        for (int c = 0; c < chunks; ++c) {
            wait(&sm.through[c % kStages], static_cast<uint32_t>(c / kStages) & 1u, patience);
            if (Y) {
                const int n = len - c * kC < kC ? len - c * kC : kC;
                for (int t = lane; t < n; t += 32)
                    bulk_s2g(static_cast<char *>(p.y) + ((begin + c * kC + t) * p.hv * p.dv + static_cast<int64_t>(head) * p.dv + slice * kM) * y_size,
                             sm.ring[c % kStages] + t * y_pitch, y_cols * y_size);
                bulk_commit();
                bulk_wait_read<0>();
                __syncwarp();
            }
            if (lane == 0 && c + kStages < chunks) load(c + kStages);
        }
        if (Y) bulk_wait_all();
        __syncwarp();
    } else if (warp >= 8) {
        // ---------------- T and P, one chunk ahead of the chain ----------------
        const int tid = threadIdx.x - kChain, pw = warp - 8;
        const int half = pw & 1, i = half * kH + lane;   // this thread's row: of A (warps 8, 9) or P
        const bool is_a = pw < 2;
        const uint32_t lanes = static_cast<uint32_t>(pw * 32) << 16;
        float g[2], bt[2];                               // of tokens 2 lane, 2 lane + 1 of the next chunk (warp 8)
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
        if (pw == 0) load_gates(0);
        for (int c = 0; c < chunks; ++c) {
            const int s = c % kStages, buf = c & 1;
            const int n = len - c * kC < kC ? len - c * kC : kC;
            uint8_t *st = sm.ring[s];
            const uint32_t col = tmem + kColK + buf * kPlace;
            wait(&sm.full[s], static_cast<uint32_t>(c / kStages) & 1u, patience);
            if (n < kC) {   // rows beyond the end, whatever they are
                for (int e = tid; e < NA * 2 * (kC - n) * 8; e += kPrep)
                    *reinterpret_cast<uint4 *>(st + e / ((kC - n) * 8) * kTile + n * 128 + e % ((kC - n) * 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
                for (int e = tid; e < (kC - n) * v_cols / 8; e += kPrep)
                    *reinterpret_cast<uint4 *>(st + kVOff + n * v_cols * 2 + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async_smem();
            }
            // two chunks ago: through with T, P, the gates and the place in tensor memory
            if (c >= 2) wait(&sm.through[(c - 2) % kStages], static_cast<uint32_t>((c - 2) / kStages) & 1u, patience);
            tc_fence_before();
            named_sync(kBarPrep, kPrep);
            if (pw == 0 && elect_one()) {
                tc_fence_after();
                const uint64_t d = desc_base(st);
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k) {   // [K; Q] K^T
                    const uint64_t dk = d + (k / 4) * (2 * kTile / 16) + 2 * (k % 4);
                    tc_mma_f16(col, dk, dk, idesc(kC, false), k > 0);
                }
                tc_commit(&sm.done_prep);
            }
            __syncwarp();
            if (pw == 0) {
                constexpr float kL = 1.44269502f, kLl = 1.92596303e-8f;   // log2 e
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
                    sm.b[t] = b;
                    sm.to_last[t] = exp_diff(last, b);
                    sm.eb[buf][t] = eb;
                    sm.ec[buf][t] = exp_diff(total, b);
                    sm.beta[buf][t] = bt[e];
                    sm.bk[buf][t] = -bt[e] * eb;
                }
                if ((lane & 7) == 7) sm.last[lane / 8] = sum;
                if (c + 1 < chunks) load_gates(c + 1);
            }
            named_sync(kBarPrep, kPrep);
            const Log bi = sm.b[i];
            const float beta = sm.beta[buf][i];
            wait(&sm.done_prep, static_cast<uint32_t>(c) & 1u, patience);
            tc_fence_after();
            float *at = reinterpret_cast<float *>(sm.tp[buf][0]);   // A^T[j][i]
            // Columns of 16. Left of the diagonal the decay from j to i goes by the last token of
            // the 16, both factors at most 1 where nothing grows; on it each has its exponential.
#pragma unroll 1
            for (int j0 = 0; j0 < (half + 1) * kH; j0 += 16) {
                float v[16];
                tmem_ld16(col + lanes + j0, v);
                if (j0 < half * kH) {
                    const float f = exp_diff(bi, sm.last[j0 / 16]) * (is_a ? beta : 1.f);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] *= f * sm.to_last[j0 + e];
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float f = exp_diff(bi, sm.b[j0 + e]) * (is_a ? beta : 1.f);
                        v[e] = j0 + e < i + (is_a ? 0 : 1) ? v[e] * f : 0.f;
                    }
                }
                if (is_a) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) at[(j0 + e) * kC + i] = v[e];
                } else {
#pragma unroll
                    for (int o = 0; o < 16; o += 8) {
                        uint32_t h[4], l[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) split(v[o + 2 * e], v[o + 2 * e + 1], h[e], l[e]);
                        const int to = i * 128 + (((j0 + o) / 8) ^ (i & 7)) * 16;
                        *reinterpret_cast<uint4 *>(sm.tp[buf][2] + to) = make_uint4(h[0], h[1], h[2], h[3]);
                        *reinterpret_cast<uint4 *>(sm.tp[buf][3] + to) = make_uint4(l[0], l[1], l[2], l[3]);
                    }
                }
            }
            tc_fence_before();
            named_sync(kBarPrep, kPrep);
            // ---- T = (I + A)^-1 in halves of 32: T11 and T22, then T21 = -T22 (A21 T11) ----
            f2 t[kH / 2];
            if (is_a) {
                // column `lane` of T11 or T22: from I, rows below l lose A[.][l] T[l], l = 0, 1, ..
#pragma unroll
                for (int e = 0; e < kH / 2; ++e) t[e] = pack2(2 * e == lane ? 1.f : 0.f, 2 * e + 1 == lane ? 1.f : 0.f);
                const float *a = at + half * (kH * kC + kH);
#pragma unroll
                for (int l = 0; l < kH - 1; ++l) {
                    float lo, hi;
                    unpack2(t[l / 2], lo, hi);
                    const float m = -(l % 2 ? hi : lo);
                    const f2 mm = pack2(m, m);
#pragma unroll
                    for (int e = (l + 1) / 4 * 4; e < kH; e += 4) {
                        const float4 x = *reinterpret_cast<const float4 *>(a + l * kC + e);
                        t[e / 2] = fma2(pack2(x.x, x.y), mm, t[e / 2]);
                        t[e / 2 + 1] = fma2(pack2(x.z, x.w), mm, t[e / 2 + 1]);
                    }
                }
                if (half == 0) {
#pragma unroll
                    for (int e = 0; e < kH / 2; ++e) unpack2(t[e], sm.t11[2 * e][lane], sm.t11[2 * e + 1][lane]);
                } else {
#pragma unroll
                    for (int e = 0; e < kH / 4; ++e) {
                        float4 x;
                        unpack2(t[2 * e], x.x, x.y);
                        unpack2(t[2 * e + 1], x.z, x.w);
                        *reinterpret_cast<float4 *>(&sm.t22[lane][4 * e]) = x;
                    }
                }
            }
            named_sync(kBarPrep, kPrep);
            // rows 8 pw .. + 7, column `lane`
            f2 acc[4];
            auto product = [&](const float *left, int stride, const float *right) {
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = pack2(0.f, 0.f);
#pragma unroll 8
                for (int l = 0; l < kH; ++l) {
                    const float4 x = *reinterpret_cast<const float4 *>(left + l * stride), z = *reinterpret_cast<const float4 *>(left + l * stride + 4);
                    const float m = right[l * kH + lane];
                    const f2 mm = pack2(m, m);
                    acc[0] = fma2(pack2(x.x, x.y), mm, acc[0]);
                    acc[1] = fma2(pack2(x.z, x.w), mm, acc[1]);
                    acc[2] = fma2(pack2(z.x, z.y), mm, acc[2]);
                    acc[3] = fma2(pack2(z.z, z.w), mm, acc[3]);
                }
            };
            product(at + kH + 8 * pw, kC, &sm.t11[0][0]);
#pragma unroll
            for (int e = 0; e < 4; ++e) unpack2(acc[e], sm.mid[8 * pw + 2 * e][lane], sm.mid[8 * pw + 2 * e + 1][lane]);
            named_sync(kBarPrep, kPrep);   // A has been read: T takes its place
            auto put = [&](int row, int col_, float a, float b) {   // T[row .. row + 1][col_]
                uint32_t h, l;
                split(a, b, h, l);
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const int to = (row + o) * 128 + ((col_ / 8) ^ ((row + o) & 7)) * 16 + (col_ % 8) * 2;
                    *reinterpret_cast<uint16_t *>(sm.tp[buf][0] + to) = static_cast<uint16_t>(o ? h >> 16 : h);
                    *reinterpret_cast<uint16_t *>(sm.tp[buf][1] + to) = static_cast<uint16_t>(o ? l >> 16 : l);
                }
            };
            if (is_a) {
#pragma unroll
                for (int e = 0; e < kH / 2; ++e) {
                    float a, b;
                    unpack2(t[e], a, b);
                    put(half * kH + 2 * e, half * kH + lane, a, b);
                }
            } else {   // T12 = 0: rows 0 .. 31, 64 bytes each, of T hi (warp 10) or T lo
#pragma unroll
                for (int e = 4; e < 8; ++e)
                    *reinterpret_cast<uint4 *>(sm.tp[buf][half] + lane * 128 + (e ^ (lane & 7)) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            product(&sm.t22[0][8 * pw], kPad, &sm.mid[0][0]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a, b;
                unpack2(acc[e], a, b);
                put(kH + 8 * pw + 2 * e, lane, -a, -b);
            }
            fence_proxy_async_smem();
            mbar_arrive(&sm.ready[buf]);
        }
    } else {
        // ---------------- the chain ----------------
        const int half = warp >> 2, quarter = warp & 3;
        const int row = quarter * 32 + lane;             // value channel within the slice
        const int ch = slice * kM + row;                 // and within the head
        const uint32_t tm = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        const bool live = ch < p.dv, has_v = row < v_cols;
        constexpr int kHalf = kKeys / 2;                 // S's columns of this half of the warps
        const uint32_t col_s = tm + kColS + half * kHalf;
        const int64_t head_elems = static_cast<int64_t>(p.dv) * p.dk;
        {   // initial state
            int64_t entry = -1;
            if (p.bank) {
                entry = p.idx ? p.idx[seq] : seq;
                if (entry < -1 || entry >= p.bank_entries) {
                    if (threadIdx.x == 0) atomicOr(&g_delta_chunk_status, PRECOG_DEV_BAD_INDEX);
                    entry = -1;
                }
            }
            const int64_t at = ((entry * p.L_total + p.layer) * p.hv + head) * head_elems + static_cast<int64_t>(ch) * p.dk;
#pragma unroll
            for (int g = 0; g < kHalf; g += 32) {
                uint32_t r[32];
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    const int col = half * kHalf + g + e;
                    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    if (entry >= 0 && live && col < p.dk) delta_load8(p.bank, p.bank_dtype, at + col, v);
#pragma unroll
                    for (int x = 0; x < 8; ++x) r[e + x] = __float_as_uint(v[x]);
                }
                __syncwarp();
                tmem_st32(col_s + g, r);
            }
            tmem_st_wait();
        }
        // Chunk c is done with: y of this thread's channel and tokens 32 half .. into the chunk's stage,
        // and word to the other warps.
        auto leave = [&](int c) {
            if (Y) {
                wait(&sm.done_o, static_cast<uint32_t>(c) & 1u, patience);
                tc_fence_after();
                const uint32_t place = tm + (c & 1) * kPlace + half * 32;
                uint32_t r[32], q[32];
                tmem_ld32_async(place + kColK, r);
                tmem_ld32_async(place + kColQ, q);
                tmem_ld_wait(r);
                tmem_ld_wait(q);
                const float *eb = &sm.eb[c & 1][half * 32];
                uint8_t *to = sm.ring[c % kStages] + (half * 32 * v_cols + row) * (p.y_dtype == PRECOG_F32 ? 4 : 2);
                if (has_v) {
                    if (p.y_dtype == PRECOG_F32) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            *reinterpret_cast<float *>(to + e * v_cols * 4) = p.scale * fmaf(eb[e], __uint_as_float(q[e]), __uint_as_float(r[e]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            *reinterpret_cast<__nv_bfloat16 *>(to + e * v_cols * 2) =
                                __float2bfloat16_rn(p.scale * fmaf(eb[e], __uint_as_float(q[e]), __uint_as_float(r[e])));
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.through[c % kStages]);
            __syncwarp();
        };
        for (int c = 0; c <= chunks; ++c) {   // the last turn only leaves the last chunk
            const int s = c % kStages, buf = c & 1;
            const uint32_t ph = static_cast<uint32_t>(c) & 1u;
            const uint8_t *st = sm.ring[s];
            const uint32_t col_k = kColK + buf * kPlace, col_q = kColQ + buf * kPlace;
            if (c < chunks) {
                wait(&sm.ready[buf], static_cast<uint32_t>(c >> 1) & 1u, patience);
                wait(&sm.full[s], static_cast<uint32_t>(c / kStages) & 1u, patience);
                // ---- S as a pair, S decayed ----
                const float whole = sm.eb[buf][kC - 1];
                if (Y && c > 0) {   // P U of the chunk before reads U's pair, which lies there
                    wait(&sm.done_o, ph ^ 1u, patience);
                    tc_fence_after();
                }
#pragma unroll 1
                for (int g = 0; g < kHalf; g += 32) {
                    uint32_t r[32], h[16], l[16];
                    tmem_ld32_async(col_s + g, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        split(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]), h[e], l[e]);
                        r[2 * e] = __float_as_uint(whole * __uint_as_float(r[2 * e]));
                        r[2 * e + 1] = __float_as_uint(whole * __uint_as_float(r[2 * e + 1]));
                    }
                    tmem_st16(tm + kColPair + (half * kHalf + g) / 2, h);
                    tmem_st16(tm + kColPair + kHalf + (half * kHalf + g) / 2, l);
                    tmem_st32(col_s + g, r);
                }
                tmem_st_wait();
                tc_fence_before();
                named_sync(kBarChain, kChain);
                if (warp == 0 && elect_one()) {
                    tc_fence_after();
                    const uint64_t d = desc_base(st);
#pragma unroll
                    for (int q = 0; q < (Y ? 2 : 1); ++q) {
#pragma unroll
                        for (int k = 0; k < kKeys / 8; ++k) {   // hi, then lo
                            const int kk = k % (kKeys / 16);
                            tc_mma_f16_ts(tmem + (q ? col_q : col_k), tmem + kColPair + k * 8,
                                          d + ((kk / 4) * 2 + q) * (kTile / 16) + 2 * (kk % 4), idesc(kC, false), k > 0);
                        }
                        tc_commit(q ? &sm.done_qs : &sm.done_ks);
                    }
                }
                __syncwarp();
            }
            if (c > 0) leave(c - 1);
            if (c == chunks) break;
            // ---- X, in the place of S k: hi of this half's 32 tokens, then lo ----
            wait(&sm.done_ks, ph, patience);
            tc_fence_after();
            {
                uint32_t r[32], h[16], l[16];
                tmem_ld32_async(tm + col_k + half * 32, r);
                const uint8_t *v = st + kVOff + (half * 32 * v_cols + row) * 2;
                const float *beta = &sm.beta[buf][half * 32], *bk = &sm.bk[buf][half * 32];
                float x[32];
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    x[e] = has_v ? beta[e] * __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(v + e * v_cols * 2)) << 16) : 0.f;
                __syncwarp();
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = fmaf(bk[e], __uint_as_float(r[e]), x[e]);
#pragma unroll
                for (int e = 0; e < 16; ++e) split(x[2 * e], x[2 * e + 1], h[e], l[e]);
                tmem_st16(tm + col_k + half * 32, h);
                tmem_st16(tm + col_k + half * 32 + 16, l);
            }
            tmem_st_wait();
            tc_fence_before();
            named_sync(kBarChain, kChain);
            if (warp == 0 && elect_one()) {
                if (Y) wait_one(&sm.done_qs, ph, patience);   // S's pair has been read: U takes its place
                tc_fence_after();
                const uint64_t hi = desc_base(sm.tp[buf][0]), lo = desc_base(sm.tp[buf][1]);
#pragma unroll
                for (int k = 0; k < 12; ++k) {   // X hi T hi, X lo T hi, X hi T lo
                    const int part = k / 4, kk = k % 4;
                    tc_mma_f16_ts(tmem + kColPair, tmem + col_k + (kk / 2) * 32 + (kk % 2) * 8 + (part == 1 ? 16 : 0),
                                  (part == 2 ? lo : hi) + 2 * kk, idesc(kC, false), k > 0);
                }
                tc_commit(&sm.done_u);
            }
            __syncwarp();
            // ---- U: a pair for P U, and decayed to the chunk's end, in U's place, for the update ----
            wait(&sm.done_u, ph, patience);
            tc_fence_after();
            {
                uint32_t r[32], h[16], l[16];
                tmem_ld32_async(tm + kColPair + half * 32, r);
                tmem_ld_wait(r);
                if (Y) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) split(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]), h[e], l[e]);
                    tmem_st16(tm + kColPair + 64 + half * 32, h);
                    tmem_st16(tm + kColPair + 64 + half * 32 + 16, l);
                }
                const float *ec = &sm.ec[buf][half * 32];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    split(ec[2 * e] * __uint_as_float(r[2 * e]), ec[2 * e + 1] * __uint_as_float(r[2 * e + 1]), h[e], l[e]);
                tmem_st16(tm + kColPair + half * 32, h);
                tmem_st16(tm + kColPair + half * 32 + 16, l);
            }
            tmem_st_wait();
            tc_fence_before();
            named_sync(kBarChain, kChain);
            if (warp == 0 && elect_one()) {
                tc_fence_after();
                const uint64_t d = desc_base(st);
#pragma unroll
                for (int a = 0; a < NA; ++a)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {   // hi, then lo; 16 tokens = two 8-row groups of K
                        const int kk = k % 4;
                        tc_mma_f16_ts(tmem + kColS + a * 64, tmem + kColPair + (kk / 2) * 32 + (kk % 2) * 8 + (k / 4) * 16,
                                      d + a * (2 * kTile / 16) + kk * (2048 / 16), idesc(64, true), true);
                    }
                tc_commit(&sm.done_s);
                if (Y) {
                    const uint64_t hi = desc_base(sm.tp[buf][2]), lo = desc_base(sm.tp[buf][3]);
#pragma unroll
                    for (int k = 0; k < 12; ++k) {   // U hi P hi, U lo P hi, U hi P lo
                        const int part = k / 4, kk = k % 4;
                        tc_mma_f16_ts(tmem + col_k, tmem + kColPair + 64 + (kk / 2) * 32 + (kk % 2) * 8 + (part == 1 ? 16 : 0),
                                      (part == 2 ? lo : hi) + 2 * kk, idesc(kC, false), k > 0);
                    }
                    tc_commit(&sm.done_o);
                }
            }
            __syncwarp();
            wait(&sm.done_s, ph, patience);
            tc_fence_after();
        }
        if (p.states) {
            const int64_t at = ((seq * p.L_total + p.layer) * p.hv + head) * head_elems + static_cast<int64_t>(ch) * p.dk;
#pragma unroll
            for (int g = 0; g < kHalf; g += 32) {
                uint32_t r[32];
                tmem_ld32_async(col_s + g, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    if (const int col = half * kHalf + g + e; live && col < p.dk) {
                        float v[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = __uint_as_float(r[e + x]);
                        delta_store8(p.states, p.state_dtype, at + col, v);
                    }
                __syncwarp();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int NA, bool Y>
cudaError_t launch(const DeltaParams &p, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, int slices,
                   int v_cols, cudaStream_t stream) {
    auto kern = delta_chunk_kernel<NA, Y>;
    const int smem = static_cast<int>(sizeof(Smem<NA>) + 1024);
    static_assert(sizeof(Smem<NA>) + 1024 <= 227 * 1024, "one CTA's shared memory");
    cudaError_t e = ensure_smem(reinterpret_cast<const void *>(kern), smem);
    if (e != cudaSuccess) return e;
    kern<<<static_cast<unsigned>(p.n_seqs * p.hv * slices), kThreads, smem, stream>>>(mq, mk, mv, p, slices, v_cols);
    e = cudaGetLastError();
    if (e == cudaSuccess) count_launches(1);
    return e;
}

// [rows][heads][dim] bf16 with `stride` elements between rows, in boxes of 64 rows of one head.
bool rows_map(CUtensorMap *map, const void *base, int dim, int heads, int64_t rows, int64_t stride, int box_cols,
              CUtensorMapSwizzle swizzle) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
    if (rows == 1) stride = static_cast<int64_t>(heads) * dim;
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(dim) * 2, static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), 1, kC};
    return encode_tiled_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, swizzle);
}

}  // namespace

cudaError_t launch_delta_chunk(const DeltaParams &p, cudaStream_t stream) {
    const bool want_y = p.y != nullptr;
    const int v_cols = p.dv < kM ? p.dv : kM;
    const int slices = (p.dv + kM - 1) / kM;
    CUtensorMap mq, mk, mv;
    if (!rows_map(&mk, p.k, p.dk, p.hk, p.T_tot, p.k_stride, 64, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !rows_map(&mq, want_y ? p.q : p.k, p.dk, p.hk, p.T_tot, want_y ? p.q_stride : p.k_stride, 64, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !rows_map(&mv, p.v, p.dv, p.hv, p.T_tot, p.v_stride, v_cols, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorInvalidValue;
    if (p.dk <= 64) return want_y ? launch<1, true>(p, mq, mk, mv, slices, v_cols, stream) : launch<1, false>(p, mq, mk, mv, slices, v_cols, stream);
    return want_y ? launch<2, true>(p, mq, mk, mv, slices, v_cols, stream) : launch<2, false>(p, mq, mk, mv, slices, v_cols, stream);
}

cudaError_t delta_chunk_status_word_read_clear(uint32_t *bits) {
    uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bits, g_delta_chunk_status, sizeof(uint32_t));
    if (e != cudaSuccess) return e;
    return cudaMemcpyToSymbol(g_delta_chunk_status, &zero, sizeof(uint32_t));
}

}  // namespace precog
