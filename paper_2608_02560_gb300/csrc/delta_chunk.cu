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
// Warps 0-3, the chain: what each chunk needs of the chunk before it. Per chunk: split S, [S k,
// S q], X, [U], split U, [update, P U]; [..] are MMAs that warp 0 issues. y of a chunk is
// stored while the next one's first MMAs run.
// Warps 4-7, ahead of it by one chunk: [k.k, q.k], A and P with their decays, the inverse T by
// substitution in fp32 (a product form of the inverse would lose its digits where keys repeat).
// Warp 8: TMA, three chunks deep.
// Tokens beyond a sequence's end have beta 0 and zeroed keys: whatever the rows hold, nothing
// of them enters a sum.
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
constexpr int kThreads = 288;
constexpr uint32_t kTile = kC * 128;   // bytes of a [64 tokens][64 keys] bf16 tile
constexpr double kLog2e = 1.4426950408889634;
constexpr float kLeastGate = -128.f;   // e^-128 is 0 in fp32

// tensor memory columns
constexpr uint32_t kColS = 0, kColSplit = 128, kColKS = 256, kColO = 320, kColPrep = 448;
constexpr uint32_t kColU = kColSplit, kColUSplit = kColSplit + 64;

constexpr int kBarChain = 1, kBarPrep = 2, kBarSolve = 3;

template <int NA>
struct Smem {
    // per stage: [K][Q] tiles of key columns 0..63, then of 64..127, then V rows
    uint8_t ring[kStages][NA * 2 * kTile + kC * kM * 2];
    // T hi, T lo, P hi, P lo; while T is solved for, A^T in fp32 fills the place of T
    uint8_t tp[2][4][kTile];
    float eb[2][kC];      // e^{b_j}
    float ec[2][kC];      // e^{b_C - b_j}
    float beta[2][kC];
    float2 b[kC];         // b in units of log2, as a pair: differences of large sums keep their digits
    uint64_t full[kStages], empty[kStages];
    uint64_t ready[2], used[2];
    uint64_t done_prep, done_ks, done_qs, done_u, done_s, done_o;
    uint32_t tmem_base;
    uint32_t abort_flag;
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

// Bounded wait. Once one has given up, all return at once and the CTA runs to its end on
// whatever is there: every barrier below is still met by all its threads.
template <int NA>
__device__ __forceinline__ void wait_one(uint64_t *bar, uint32_t parity, Smem<NA> &sm) {
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        if (mbar_try_wait(bar, parity)) return;
        if ((i & 255u) == 255u && *reinterpret_cast<volatile uint32_t *>(&sm.abort_flag)) return;
    }
    atomicOr(&g_delta_chunk_status, PRECOG_DEV_TIMEOUT);
    *reinterpret_cast<volatile uint32_t *>(&sm.abort_flag) = 1u;
}
// The same by all lanes of a warp, which go on together (tensor-memory accesses are a warp's).
template <int NA>
__device__ __forceinline__ void wait(uint64_t *bar, uint32_t parity, Smem<NA> &sm) {
    wait_one(bar, parity, sm);
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
    Smem<NA> &sm = *reinterpret_cast<Smem<NA> *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

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
            mbar_init(&sm.empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.ready[i], 128);
            mbar_init(&sm.used[i], 1);
        }
        mbar_init(&sm.done_prep, 1);
        mbar_init(&sm.done_ks, 1);
        mbar_init(&sm.done_qs, 1);
        mbar_init(&sm.done_u, 1);
        mbar_init(&sm.done_s, 1);
        mbar_init(&sm.done_o, 1);
        sm.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 8) {
        tmem_alloc(&sm.tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;

    if (warp == 8) {
        // ---------------- copies ----------------
        if (lane == 0) {
            for (int c = 0; c < chunks; ++c) {
                const int s = c % kStages;
                if (c >= kStages) wait_one(&sm.empty[s], static_cast<uint32_t>(c / kStages - 1) & 1u, sm);
                uint8_t *st = sm.ring[s];
                const int row = static_cast<int>(begin) + c * kC;
                mbar_arrive_expect_tx(&sm.full[s], NA * (Y ? 2 : 1) * kTile + kC * v_cols * 2);
                for (int a = 0; a < NA; ++a) {
                    tma_load_3d(st + a * 2 * kTile, &map_k, a * 64, qk, row, &sm.full[s]);
                    if (Y) tma_load_3d(st + a * 2 * kTile + kTile, &map_q, a * 64, qk, row, &sm.full[s]);
                }
                tma_load_3d(st + kVOff, &map_v, slice * kM, head, row, &sm.full[s]);
            }
            for (int c = chunks > kStages ? chunks - kStages : 0; c < chunks; ++c)   // all have landed
                wait_one(&sm.full[c % kStages], static_cast<uint32_t>(c / kStages) & 1u, sm);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ---------------- T and P, one chunk ahead of the chain ----------------
        const int tid = threadIdx.x - 128;
        const int i = tid & 63;                          // token of this thread's row of A or P
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        for (int c = 0; c < chunks; ++c) {
            const int s = c % kStages, buf = c & 1;
            const int n = len - c * kC < kC ? len - c * kC : kC;
            // gates: lane l of the first warp has tokens 2l and 2l + 1
            float g[2] = {0.f, 0.f}, bt[2] = {0.f, 0.f};
            if (warp == 4)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (2 * lane + e < n) {
                        const int64_t at = (begin + c * kC + 2 * lane + e) * p.hv + head;
                        g[e] = p.g[at];
                        bt[e] = p.beta[at];
                    }
            wait(&sm.full[s], static_cast<uint32_t>(c / kStages) & 1u, sm);
            uint8_t *st = sm.ring[s];
            if (n < kC) {   // keys of rows beyond the end: whatever they are, zero
                for (int e = tid; e < NA * (kC - n) * 8; e += 128) {
                    const int a = e / ((kC - n) * 8), at = e % ((kC - n) * 8);
                    *reinterpret_cast<uint4 *>(st + a * 2 * kTile + n * 128 + at * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_proxy_async_smem();
            }
            tc_fence_before();
            named_sync(kBarPrep, 128);
            if (tid == 0) {
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k) {
                    const uint64_t d = desc_base(st + (k / 4) * 2 * kTile) + 2 * (k % 4);
                    tc_mma_f16(tmem + kColPrep, d, d, idesc(kC, false), k > 0);   // [K; Q] K^T
                }
                tc_commit(&sm.done_prep);
            }
            __syncwarp();
            if (warp == 4) {
                double x0 = 0., x1 = 0.;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float v;   // NaN stays NaN
                    asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(g[e]), "f"(kLeastGate));
                    (e ? x1 : x0) = static_cast<double>(v) * kLog2e;
                }
                double sum = x0 + x1;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double up = __shfl_up_sync(0xffffffffu, sum, o);
                    if (lane >= o) sum += up;
                }
                const double total = __shfl_sync(0xffffffffu, sum, 31);
                if (c >= 2) wait(&sm.used[buf], static_cast<uint32_t>(c / 2 - 1) & 1u, sm);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const double b = e ? sum : sum - x1;
                    const float hi = static_cast<float>(b);
                    sm.b[2 * lane + e] = make_float2(hi, static_cast<float>(b - hi));
                    sm.eb[buf][2 * lane + e] = ex2(hi);
                    sm.ec[buf][2 * lane + e] = ex2(static_cast<float>(total - b));
                    sm.beta[buf][2 * lane + e] = bt[e];
                }
            }
            named_sync(kBarPrep, 128);
            wait(&sm.done_prep, static_cast<uint32_t>(c) & 1u, sm);
            tc_fence_after();
            uint32_t r[2][32];
            tmem_ld32_async(tmem + lanes + kColPrep, r[0]);
            tmem_ld32_async(tmem + lanes + kColPrep + 32, r[1]);
            tmem_ld_wait(r[0]);
            tmem_ld_wait(r[1]);
            const float2 bi = sm.b[i];
            float *at = reinterpret_cast<float *>(sm.tp[buf][0]);   // A^T[j][i]
            if (tid < 64) {
                const float beta = sm.beta[buf][i];
#pragma unroll
                for (int j = 0; j < kC; ++j) {
                    const float2 bj = sm.b[j];
                    const float d = ex2((bi.x - bj.x) + (bi.y - bj.y));
                    at[j * kC + i] = j < i ? beta * d * __uint_as_float(r[j / 32][j % 32]) : 0.f;
                }
            } else {
#pragma unroll
                for (int j8 = 0; j8 < kC; j8 += 8) {
                    uint32_t h[4], l[4];
#pragma unroll
                    for (int j = j8; j < j8 + 8; j += 2) {
                        float v[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float2 bj = sm.b[j + e];
                            const float d = ex2((bi.x - bj.x) + (bi.y - bj.y));
                            v[e] = j + e <= i && i < n ? d * __uint_as_float(r[(j + e) / 32][(j + e) % 32]) : 0.f;
                        }
                        split(v[0], v[1], h[(j - j8) / 2], l[(j - j8) / 2]);
                    }
                    const int to = i * 128 + ((j8 / 8) ^ (i & 7)) * 16;
                    *reinterpret_cast<uint4 *>(sm.tp[buf][2] + to) = make_uint4(h[0], h[1], h[2], h[3]);
                    *reinterpret_cast<uint4 *>(sm.tp[buf][3] + to) = make_uint4(l[0], l[1], l[2], l[3]);
                }
            }
            tc_fence_before();
            named_sync(kBarPrep, 128);
            if (tid < 64) {
                // column i of T: T = I, then for l = 0, 1, ..: rows below l lose A[.][l] T[l]
                f2 t[kC / 2];
#pragma unroll
                for (int e = 0; e < kC / 2; ++e) t[e] = pack2(2 * e == i ? 1.f : 0.f, 2 * e + 1 == i ? 1.f : 0.f);
                auto eliminate = [&](int l) {
                    float lo, hi;
                    unpack2(t[l / 2], lo, hi);
                    const float tl = -(l % 2 ? hi : lo);
                    const f2 m = pack2(tl, tl);
#pragma unroll
                    for (int e = (l + 1) / 4 * 4; e < kC; e += 4) {
                        const float4 a = *reinterpret_cast<const float4 *>(at + l * kC + e);
                        t[e / 2] = fma2(pack2(a.x, a.y), m, t[e / 2]);
                        t[e / 2 + 1] = fma2(pack2(a.z, a.w), m, t[e / 2 + 1]);
                    }
                };
                if (tid < 32) {   // columns from 32 on begin at their own rows
#pragma unroll
                    for (int l = 0; l < 32; ++l) eliminate(l);
                }
#pragma unroll
                for (int l = 32; l < kC - 1; ++l) eliminate(l);
                named_sync(kBarSolve, 64);   // A has been read: T takes its place
#pragma unroll
                for (int e = 0; e < kC / 2; ++e) {
                    float lo, hi;
                    unpack2(t[e], lo, hi);
                    uint32_t h, l;
                    split(lo, hi, h, l);
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const int row = 2 * e + o;
                        const int to = row * 128 + ((i / 8) ^ (row & 7)) * 16 + (i % 8) * 2;
                        *reinterpret_cast<uint16_t *>(sm.tp[buf][0] + to) = static_cast<uint16_t>(o ? h >> 16 : h);
                        *reinterpret_cast<uint16_t *>(sm.tp[buf][1] + to) = static_cast<uint16_t>(o ? l >> 16 : l);
                    }
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(&sm.ready[buf]);
        }
    } else {
        // ---------------- the chain ----------------
        const int row = threadIdx.x;                     // value channel within the slice
        const int ch = slice * kM + row;                 // and within the head
        const uint32_t tm = tmem + (static_cast<uint32_t>(warp * 32) << 16);
        const bool live = ch < p.dv;
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
            for (int g = 0; g < kKeys / 32; ++g) {
                uint32_t r[32];
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    const int col = g * 32 + e;
                    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    if (entry >= 0 && live && col < p.dk) delta_load8(p.bank, p.bank_dtype, at + col, v);
#pragma unroll
                    for (int x = 0; x < 8; ++x) r[e + x] = __float_as_uint(v[x]);
                }
                tmem_st32(tm + kColS + g * 32, r);
            }
            tmem_st_wait();
        }
        const int64_t y_row = static_cast<int64_t>(p.hv) * p.dv;
        const int64_t y_at = static_cast<int64_t>(head) * p.dv + ch;
        // y of chunk c from its sums in tensor memory
        auto store_y = [&](int c) {
            const int n = len - c * kC < kC ? len - c * kC : kC;
            const int64_t at = (begin + c * kC) * y_row + y_at;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                uint32_t r[32];
                tmem_ld32_async(tm + kColO + (c & 1) * 64 + g * 32, r);
                tmem_ld_wait(r);
                if (live) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (g * 32 + e < n) {
                            const float y = p.scale * __uint_as_float(r[e]);
                            const int64_t to = at + (g * 32 + e) * y_row;
                            if (p.y_dtype == PRECOG_F32) static_cast<float *>(p.y)[to] = y;
                            else static_cast<__nv_bfloat16 *>(p.y)[to] = __float2bfloat16_rn(y);
                        }
                }
                __syncwarp();
            }
        };
        for (int c = 0; c < chunks; ++c) {
            const int s = c % kStages, buf = c & 1;
            const uint32_t ph = static_cast<uint32_t>(c) & 1u;
            const int n = len - c * kC < kC ? len - c * kC : kC;
            const uint32_t col_o = kColO + ph * 64;
            const uint8_t *st = sm.ring[s];
            wait(&sm.ready[buf], static_cast<uint32_t>(c >> 1) & 1u, sm);
            wait(&sm.full[s], static_cast<uint32_t>(c / kStages) & 1u, sm);
            // ---- S as a pair, S decayed ----
            const float whole = sm.eb[buf][kC - 1];
#pragma unroll
            for (int g = 0; g < kKeys / 32; ++g) {
                uint32_t r[32], h[16], l[16];
                tmem_ld32_async(tm + kColS + g * 32, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    split(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]), h[e], l[e]);
                    r[2 * e] = __float_as_uint(whole * __uint_as_float(r[2 * e]));
                    r[2 * e + 1] = __float_as_uint(whole * __uint_as_float(r[2 * e + 1]));
                }
                if (Y && g == 0 && c > 0) {   // P U of the chunk before reads U's pair, which lies there
                    wait(&sm.done_o, ph ^ 1u, sm);
                    tc_fence_after();
                }
                tmem_st16(tm + kColSplit + g * 16, h);
                tmem_st16(tm + kColSplit + kKeys / 2 + g * 16, l);
                tmem_st32(tm + kColS + g * 32, r);
            }
            tmem_st_wait();
            tc_fence_before();
            named_sync(kBarChain, 128);
            if (threadIdx.x == 0) {
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < (Y ? 2 : 1); ++q) {
#pragma unroll
                    for (int k = 0; k < kKeys / 8; ++k) {   // hi, then lo
                        const int kk = k % (kKeys / 16);
                        tc_mma_f16_ts(tmem + (q ? col_o : kColKS), tmem + kColSplit + k * 8,
                                      desc_base(st + (kk / 4) * 2 * kTile + q * kTile) + 2 * (kk % 4), idesc(kC, false), k > 0);
                    }
                    tc_commit(q ? &sm.done_qs : &sm.done_ks);
                }
                if (c > 0) {   // nothing of the chunk before is in use any more
                    mbar_arrive(&sm.used[buf ^ 1]);
                    mbar_arrive(&sm.empty[(c - 1) % kStages]);
                }
            }
            __syncwarp();
            if (Y && c > 0) store_y(c - 1);
            // ---- X ----
            wait(&sm.done_ks, ph, sm);
            tc_fence_after();
            {
                const uint8_t *v = st + kVOff + row * 2;
                const bool has_v = row < v_cols;
                uint32_t r[2][32], h[16], l[16];
                tmem_ld32_async(tm + kColKS, r[0]);
                tmem_ld32_async(tm + kColKS + 32, r[1]);
                tmem_ld_wait(r[0]);
                tmem_ld_wait(r[1]);
#pragma unroll
                for (int g = 0; g < 2; ++g) {   // in the place of S k
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const int j = g * 32 + e;
                        const float vj = has_v ? __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(v + j * v_cols * 2)) << 16) : 0.f;
                        const float x = sm.beta[buf][j] * (vj - sm.eb[buf][j] * __uint_as_float(r[g][e]));
                        r[g][e] = __float_as_uint(j < n ? x : 0.f);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) split(__uint_as_float(r[g][2 * e]), __uint_as_float(r[g][2 * e + 1]), h[e], l[e]);
                    tmem_st16(tm + kColKS + g * 16, h);
                    tmem_st16(tm + kColKS + 32 + g * 16, l);
                }
            }
            tmem_st_wait();
            if (Y) wait(&sm.done_qs, ph, sm);   // S's pair has been read: U takes its place
            tc_fence_before();
            named_sync(kBarChain, 128);
            if (threadIdx.x == 0) {
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < 12; ++k) {   // X hi T hi, X lo T hi, X hi T lo
                    const int part = k / 4, kk = k % 4;
                    tc_mma_f16_ts(tmem + kColU, tmem + kColKS + (part == 1 ? 32 : 0) + kk * 8,
                                  desc_base(sm.tp[buf][part == 2 ? 1 : 0]) + 2 * kk, idesc(kC, false), k > 0);
                }
                tc_commit(&sm.done_u);
            }
            __syncwarp();
            if (Y) {   // S q, decayed: P U adds to it
                tc_fence_after();
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    uint32_t r[32];
                    tmem_ld32_async(tm + col_o + g * 32, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(sm.eb[buf][g * 32 + e] * __uint_as_float(r[e]));
                    tmem_st32(tm + col_o + g * 32, r);
                }
            }
            // ---- U, for P U and, decayed to the chunk's end, for the update ----
            wait(&sm.done_u, ph, sm);
            tc_fence_after();
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                uint32_t r[32], h[16], l[16];
                tmem_ld32_async(tm + kColU + g * 32, r);
                tmem_ld_wait(r);
                if (Y) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) split(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]), h[e], l[e]);
                    tmem_st16(tm + kColUSplit + g * 16, h);
                    tmem_st16(tm + kColUSplit + 32 + g * 16, l);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = g * 32 + 2 * e;
                    split(sm.ec[buf][j] * __uint_as_float(r[2 * e]), sm.ec[buf][j + 1] * __uint_as_float(r[2 * e + 1]), h[e], l[e]);
                }
                tmem_st16(tm + kColKS + g * 16, h);
                tmem_st16(tm + kColKS + 32 + g * 16, l);
            }
            tmem_st_wait();
            tc_fence_before();
            named_sync(kBarChain, 128);
            if (threadIdx.x == 0) {
                tc_fence_after();
#pragma unroll
                for (int a = 0; a < NA; ++a)
#pragma unroll
                    for (int k = 0; k < 8; ++k)   // hi, then lo; 16 tokens = two 8-row groups of K
                        tc_mma_f16_ts(tmem + kColS + a * 64, tmem + kColKS + k * 8,
                                      desc_base(st + a * 2 * kTile + (k % 4) * 2048), idesc(64, true), true);
                tc_commit(&sm.done_s);
                if (Y) {
#pragma unroll
                    for (int k = 0; k < 12; ++k) {   // U hi P hi, U lo P hi, U hi P lo
                        const int part = k / 4, kk = k % 4;
                        tc_mma_f16_ts(tmem + col_o, tmem + kColUSplit + (part == 1 ? 32 : 0) + kk * 8,
                                      desc_base(sm.tp[buf][part == 2 ? 3 : 2]) + 2 * kk, idesc(kC, false), true);
                    }
                    tc_commit(&sm.done_o);
                }
            }
            __syncwarp();
            wait(&sm.done_s, ph, sm);
            tc_fence_after();
        }
        if (chunks > 0 && Y) {
            wait(&sm.done_o, static_cast<uint32_t>(chunks - 1) & 1u, sm);
            tc_fence_after();
            store_y(chunks - 1);
        }
        if (p.states) {
            const int64_t at = ((seq * p.L_total + p.layer) * p.hv + head) * head_elems + static_cast<int64_t>(ch) * p.dk;
#pragma unroll
            for (int g = 0; g < kKeys / 32; ++g) {
                uint32_t r[32];
                tmem_ld32_async(tm + kColS + g * 32, r);
                tmem_ld_wait(r);
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    if (live && g * 32 + e < p.dk) {
                        float v[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = __uint_as_float(r[e + x]);
                        delta_store8(p.states, p.state_dtype, at + g * 32 + e, v);
                    }
                __syncwarp();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
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
