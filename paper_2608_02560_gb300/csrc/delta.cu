// The gated delta rule token by token: one token of each sequence of a serving batch on a
// table of fp32 states (precog_delta_step), and the scan of sequences whose inputs are fp32 or
// whose lengths are a few tokens (precog_delta_scan; longer bf16 sequences: delta_chunk.cu).
//
//   S <- e^g S ;  u = beta (v - S k) ;  S <- S + u k^T ;  y = scale S q
//
// A step is bound by memory, each state read and written once: 256 rows x 16 heads of 128 x 128 in
// 89 us, 6.07 TB/s, 0.89 of the measured copy rate; a single row by its launch. A scan is bound by the
// latency of its tokens, 0.17 us each (8 sequences of 129 to 256 tokens, 4 heads of 64 x 64, fp32:
// 43 us).
//
// Rows of S (value channels) are independent given k, q and the gates, so a row belongs to 8
// lanes of a warp and to nobody else: lane l of the 8 holds the four-number groups
// l, l + 8, l + 16, ... of its columns, so a group's loads are whole 128-byte lines, and each of
// the two dot products ends in three shuffles. The readout uses S q = e^g (S_old q) + u (k.q),
// whose shuffles run beside those of S_old k, in place of a second pass over the new state.
#include "../../include/precog.h"
#include "delta.h"
#include "internal.h"
#include "ptx.cuh"

namespace precog {

__device__ uint32_t g_delta_status;

namespace {

constexpr int kLanes = 8;                       // lanes of a row
constexpr int kThreads = 128;
constexpr int kRowSets = kThreads / kLanes;     // rows that a CTA holds at a time

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p) {
    const uint2 r = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16),
                       __uint_as_float(r.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(p) =
        make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store_any(void *base, int dtype, int64_t at, float v) {
    if (dtype == PRECOG_F32) static_cast<float *>(base)[at] = v;
    else static_cast<__nv_bfloat16 *>(base)[at] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ float4 scale4(float a, float4 v) { return make_float4(a * v.x, a * v.y, a * v.z, a * v.w); }
__device__ __forceinline__ float dot4(float4 a, float4 b, float sum) {
    return fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, sum))));
}
__device__ __forceinline__ float4 axpy4(float a, float4 x, float4 y) {
    return make_float4(fmaf(a, x.x, y.x), fmaf(a, x.y, y.y), fmaf(a, x.z, y.z), fmaf(a, x.w, y.w));
}
// Sum over the 8 lanes of a row, in an order that does not depend on the lane.
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// e^g, 0 below -128 (NaN kept). expf, not the SFU alone: its error is of every token that the state
// remembers, and of hundreds the SFU's would show beside the rounding of the products.
__device__ __forceinline__ float decay_of(float g) { return g < -128.f ? 0.f : expf(g); }

// One token. A thread holds one group of columns of R rows, kRowSets apart.
template <typename T, int J, int R>
__global__ void __launch_bounds__(kThreads) delta_step_kernel(const DeltaParams p, int row_tiles) {
    const int lane8 = threadIdx.x % kLanes, row_in = threadIdx.x / kLanes;
    int64_t item = blockIdx.x;
    const int tile = static_cast<int>(item % row_tiles);
    item /= row_tiles;
    const int head = static_cast<int>(item % p.hv);
    const int64_t i = item / p.hv;
    const int64_t slot = p.idx ? p.idx[i] : i;
    const int row0 = tile * kRowSets * R + row_in;
    const bool there = slot >= 0 && slot < p.bank_entries;
    if (!there) {   // an idle row of a padded batch, or a slot outside the table
        if (slot != -1 && threadIdx.x == 0) atomicOr(&g_delta_status, PRECOG_DEV_BAD_INDEX);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (const int row = row0 + r * kRowSets; lane8 == 0 && row < p.dv)
                store_any(p.y, p.y_dtype, (i * p.hv + head) * p.dv + row, 0.f);
        return;
    }
    float *S = static_cast<float *>(p.states) +
               ((slot * p.L_total + p.layer) * p.hv + head) * static_cast<int64_t>(p.dv) * p.dk;
    float4 s[R][J];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = row0 + r * kRowSets, col = 4 * (lane8 + kLanes * j);
            s[r][j] = row < p.dv && col < p.dk ? load4(S + static_cast<int64_t>(row) * p.dk + col)
                                               : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    const int qk = head / (p.hv / p.hk);
    const T *kr = static_cast<const T *>(p.k) + i * p.k_stride + static_cast<int64_t>(qk) * p.dk;
    const T *qr = static_cast<const T *>(p.q) + i * p.q_stride + static_cast<int64_t>(qk) * p.dk;
    const T *vr = static_cast<const T *>(p.v) + i * p.v_stride + static_cast<int64_t>(head) * p.dv;
    float4 k[J], q[J];
    float kq = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int col = 4 * (lane8 + kLanes * j);
        k[j] = col < p.dk ? load4(kr + col) : make_float4(0.f, 0.f, 0.f, 0.f);
        q[j] = col < p.dk ? load4(qr + col) : make_float4(0.f, 0.f, 0.f, 0.f);
        kq = dot4(k[j], q[j], kq);
    }
    kq = row_sum(kq);
    const float a = decay_of(p.g[i * p.hv + head]), b = p.beta[i * p.hv + head];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + r * kRowSets;
        float sk = 0.f, sq = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            s[r][j] = scale4(a, s[r][j]);
            sk = dot4(s[r][j], k[j], sk);
            sq = dot4(s[r][j], q[j], sq);
        }
        sk = row_sum(sk);
        sq = row_sum(sq);
        if (row >= p.dv) continue;
        const float u = b * (to_f32(vr[row]) - sk);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int col = 4 * (lane8 + kLanes * j);
            if (col < p.dk) store4(S + static_cast<int64_t>(row) * p.dk + col, axpy4(u, k[j], s[r][j]));
        }
        if (lane8 == 0) store_any(p.y, p.y_dtype, (i * p.hv + head) * p.dv + row, p.scale * fmaf(u, kq, sq));
    }
}

// The scan: the state of R rows a thread stays in registers, tokens pass through shared memory in
// tiles of kTile, the next tile's loads in flight behind this one's tokens. What bounds it is the
// chain from one token's state to the next's: a dot product over the lane's columns in four parallel
// sums, three shuffles, one update. Everything else runs beside it: S q shares the shuffles' time,
// e^g S is formed meanwhile, and the next token's rows are read a token ahead.
constexpr int kTile = 16;

template <typename T, int J, int R>
__global__ void __launch_bounds__(kThreads) delta_token_scan_kernel(const DeltaParams p, int row_tiles) {
    constexpr int kCols = J * kLanes * 4;       // dk rounded up to whole groups, zeros beyond dk
    constexpr int kRows = kRowSets * R;
    __shared__ float4 sk4[kTile][kCols / 4];
    __shared__ float4 sq4[kTile][kCols / 4];
    __shared__ float sv[kTile][kRows];
    __shared__ float sg[kTile], sb[kTile], skq[kTile];
    const int lane8 = threadIdx.x % kLanes, row_in = threadIdx.x / kLanes;
    int64_t item = blockIdx.x;
    const int tile = static_cast<int>(item % row_tiles);
    item /= row_tiles;
    const int head = static_cast<int>(item % p.hv);
    const int64_t seq = item / p.hv;
    const int row_base = tile * kRows;
    const int64_t begin = p.offsets[seq], end = p.offsets[seq + 1];
    if (begin < 0 || end < begin || end > p.T_tot) {
        if (threadIdx.x == 0) atomicOr(&g_delta_status, PRECOG_DEV_BAD_OFFSETS);
        return;
    }
    // ---- initial state ----
    int64_t entry = -1;
    if (p.bank) {
        entry = p.idx ? p.idx[seq] : seq;
        if (entry < -1 || entry >= p.bank_entries) {
            if (threadIdx.x == 0) atomicOr(&g_delta_status, PRECOG_DEV_BAD_INDEX);
            entry = -1;
        }
    }
    const int64_t head_elems = static_cast<int64_t>(p.dv) * p.dk;
    float4 s[R][J];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = row_base + row_in + r * kRowSets, col = 4 * (lane8 + kLanes * j);
            s[r][j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (entry >= 0 && row < p.dv && col < p.dk) {
                const int64_t at = ((entry * p.L_total + p.layer) * p.hv + head) * head_elems + static_cast<int64_t>(row) * p.dk + col;
                s[r][j] = p.bank_dtype == PRECOG_F32 ? load4(static_cast<const float *>(p.bank) + at)
                                                     : load4(static_cast<const __nv_bfloat16 *>(p.bank) + at);
            }
        }
    const int qk = head / (p.hv / p.hk);
    const bool want_y = p.y != nullptr;
    const T *kg = static_cast<const T *>(p.k) + static_cast<int64_t>(qk) * p.dk;
    const T *qg = want_y ? static_cast<const T *>(p.q) + static_cast<int64_t>(qk) * p.dk : nullptr;
    const T *vg = static_cast<const T *>(p.v) + static_cast<int64_t>(head) * p.dv + row_base;
    const int groups = p.dk / 4;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    float4 nk[J], nq[J];          // the next tile, on its way
    float nv[2 * R], ng = 0.f, nb = 0.f;
    auto fetch = [&](int64_t t0) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int e = threadIdx.x + j * kThreads, t = e / (kCols / 4), c = e % (kCols / 4);
            const bool there = t0 + t < end && c < groups;
            nk[j] = there ? load4(kg + (t0 + t) * p.k_stride + 4 * c) : zero;
            nq[j] = there && want_y ? load4(qg + (t0 + t) * p.q_stride + 4 * c) : zero;
        }
#pragma unroll
        for (int i = 0; i < 2 * R; ++i) {
            const int e = threadIdx.x + i * kThreads, t = e / kRows, c = e % kRows;
            nv[i] = t0 + t < end && row_base + c < p.dv ? to_f32(vg[(t0 + t) * p.v_stride + c]) : 0.f;
        }
        if (threadIdx.x < kTile && t0 + threadIdx.x < end) {
            ng = p.g[(t0 + threadIdx.x) * p.hv + head];
            nb = p.beta[(t0 + threadIdx.x) * p.hv + head];
        }
    };
    if (begin < end) fetch(begin);
    for (int64_t t0 = begin; t0 < end; t0 += kTile) {
        const int n = end - t0 < kTile ? static_cast<int>(end - t0) : kTile;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int e = threadIdx.x + j * kThreads;
            (&sk4[0][0])[e] = nk[j];
            (&sq4[0][0])[e] = nq[j];
        }
#pragma unroll
        for (int i = 0; i < 2 * R; ++i) (&sv[0][0])[threadIdx.x + i * kThreads] = nv[i];
        if (threadIdx.x < kTile) {
            sg[threadIdx.x] = decay_of(ng);
            sb[threadIdx.x] = nb;
        }
        __syncthreads();
        if (t0 + kTile < end) fetch(t0 + kTile);
        if (want_y) {
            // k.q of the tile's tokens: 8 lanes a token
            const int t = threadIdx.x / kLanes;   // kTile == kRowSets
            float kq = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) kq = dot4(sk4[t][lane8 + kLanes * j], sq4[t][lane8 + kLanes * j], kq);
            kq = row_sum(kq);
            if (lane8 == 0) skq[t] = kq;
            __syncthreads();
        }
        float4 k[J], q[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            k[j] = sk4[0][lane8 + kLanes * j];
            q[j] = sq4[0][lane8 + kLanes * j];
        }
#pragma unroll 2
        for (int t = 0; t < n; ++t) {
            const float a = sg[t], b = sb[t];
            float sk[R], sq[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float4 x = zero, y = zero;        // four sums each
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    x = make_float4(fmaf(s[r][j].x, k[j].x, x.x), fmaf(s[r][j].y, k[j].y, x.y), fmaf(s[r][j].z, k[j].z, x.z), fmaf(s[r][j].w, k[j].w, x.w));
                    y = make_float4(fmaf(s[r][j].x, q[j].x, y.x), fmaf(s[r][j].y, q[j].y, y.y), fmaf(s[r][j].z, q[j].z, y.z), fmaf(s[r][j].w, q[j].w, y.w));
                }
                sk[r] = (x.x + x.y) + (x.z + x.w);
                sq[r] = (y.x + y.y) + (y.z + y.w);
            }
            const int ahead = t + 1 < kTile ? t + 1 : t;
            float4 k1[J], q1[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                k1[j] = sk4[ahead][lane8 + kLanes * j];
                q1[j] = sq4[ahead][lane8 + kLanes * j];
            }
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    sk[r] += __shfl_xor_sync(0xffffffffu, sk[r], o);
                    sq[r] += __shfl_xor_sync(0xffffffffu, sq[r], o);
                }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int row = row_in + r * kRowSets;
                const float u = b * fmaf(-a, sk[r], sv[t][row]);
#pragma unroll
                for (int j = 0; j < J; ++j) s[r][j] = axpy4(u, k[j], scale4(a, s[r][j]));
                if (want_y) {
                    const float y = p.scale * fmaf(u, skq[t], a * sq[r]);
                    if (lane8 == 0 && row_base + row < p.dv)
                        store_any(p.y, p.y_dtype, ((t0 + t) * p.hv + head) * p.dv + row_base + row, y);
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j) k[j] = k1[j], q[j] = q1[j];
        }
    }
    if (p.states == nullptr) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = row_base + row_in + r * kRowSets, col = 4 * (lane8 + kLanes * j);
            if (row >= p.dv || col >= p.dk) continue;
            const int64_t at = ((seq * p.L_total + p.layer) * p.hv + head) * head_elems + static_cast<int64_t>(row) * p.dk + col;
            if (p.state_dtype == PRECOG_F32) store4(static_cast<float *>(p.states) + at, s[r][j]);
            else store4(static_cast<__nv_bfloat16 *>(p.states) + at, s[r][j]);
        }
}

template <typename T, int J, int R>
cudaError_t step_rows(const DeltaParams &p, cudaStream_t stream) {
    const int tiles = (p.dv + kRowSets * R - 1) / (kRowSets * R);
    delta_step_kernel<T, J, R><<<static_cast<unsigned>(p.n_seqs * p.hv * tiles), kThreads, 0, stream>>>(p, tiles);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T, int J, int R>
cudaError_t scan_rows(const DeltaParams &p, cudaStream_t stream) {
    const int tiles = (p.dv + kRowSets * R - 1) / (kRowSets * R);
    delta_token_scan_kernel<T, J, R><<<static_cast<unsigned>(p.n_seqs * p.hv * tiles), kThreads, 0, stream>>>(p, tiles);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launches(1);
    return e;
}

static_assert(kTile == kRowSets, "the tile's k.q take 8 lanes a token, and a thread fetches 2 R of v");

// Two rows a thread keep more of the states in flight (256 sequences x 16 heads of 128 x 128: 89 us,
// one row 98, four rows 93), unless that leaves an SM fewer than eight CTAs: then latency counts.
template <typename T, int J>
cudaError_t step_tiles(const DeltaParams &p, cudaStream_t stream) {
    return p.n_seqs * p.hv * ((p.dv + 2 * kRowSets - 1) / (2 * kRowSets)) >= 8LL * device_sm_count() ? step_rows<T, J, 2>(p, stream)
                                                                                                    : step_rows<T, J, 1>(p, stream);
}

template <typename T>
cudaError_t step_cols(const DeltaParams &p, cudaStream_t stream) {
    switch ((p.dk + 31) / 32) {
        case 1: return step_tiles<T, 1>(p, stream);
        case 2: return step_tiles<T, 2>(p, stream);
        case 3: return step_tiles<T, 3>(p, stream);
        default: return step_tiles<T, 4>(p, stream);
    }
}

// Two rows a thread share what they read of a token, where that leaves an SM eight CTAs (16 heads of
// 128 x 128, 64 tokens: 256 sequences 1407 us, one row a thread 1617; 32 sequences 188 and 208; 8
// sequences 72 and 57, one sequence 27 and 17).
template <typename T, int J>
cudaError_t scan_tiles(const DeltaParams &p, cudaStream_t stream) {
    return p.n_seqs * p.hv * ((p.dv + 2 * kRowSets - 1) / (2 * kRowSets)) >= 8LL * device_sm_count() ? scan_rows<T, J, 2>(p, stream)
                                                                                                    : scan_rows<T, J, 1>(p, stream);
}

template <typename T>
cudaError_t scan_cols(const DeltaParams &p, cudaStream_t stream) {
    switch ((p.dk + 31) / 32) {
        case 1: return scan_tiles<T, 1>(p, stream);
        case 2: return scan_tiles<T, 2>(p, stream);
        case 3: return scan_tiles<T, 3>(p, stream);
        default: return scan_tiles<T, 4>(p, stream);
    }
}

}  // namespace

cudaError_t launch_delta_step(const DeltaParams &p, cudaStream_t stream) {
    return p.in_dtype == PRECOG_F32 ? step_cols<float>(p, stream) : step_cols<__nv_bfloat16>(p, stream);
}

namespace {

// Whether the chunk kernel is the faster one, by what both measured (16 heads of 128 x 128 unless said):
//   1 sequence of 32 / 48 tokens    token 10.2 / 13.7 us  chunk 13.0 / 12.8
//   4 sequences of 16 / 24          token 10.3 / 14.7     chunk 13.8 / 13.7
//   16 of 12 / 16                   token 27.3 / 32.7     chunk 27.5 / 27.1
//   256 of 8 / 16                   token 257 / 405       chunk 370 / 365
//   64 of 40 / 48, 64 x 64          token 67 / 78         chunk 76 / 76
// A round of CTAs in chunks takes 13 us however few its tokens are. A token of the other kernel takes
// 0.25 us by its latency, or 6.2 ns a head of 128 x 128 where the SMs are full. Lengths lie on the
// device: the rule knows their mean, T_tot / n_seqs, and a batch whose one long sequence is hidden among
// short ones goes token by token (400 tokens among fifteen empty sequences, one head: 100 us by these
// figures, some 30 in chunks).
bool in_chunks(const DeltaParams &p) {
    if (p.in_dtype != PRECOG_BF16 || p.n_seqs <= 0) return false;
    const double heads = static_cast<double>(p.n_seqs) * p.hv, tokens = static_cast<double>(p.T_tot) / p.n_seqs;
    const double rounds = ceil(heads * ((p.dv + 127) / 128) / device_sm_count());
    const double token = fmax(0.25, 0.0062 * heads * p.dk * p.dv / (128 * 128));
    return 3.5 + tokens * token > 13 * rounds;
}

}  // namespace

size_t delta_scan_workspace_size(const DeltaParams &p) { return in_chunks(p) ? delta_chunk_workspace_size(p) : 0; }

cudaError_t launch_delta_scan(const DeltaParams &p, cudaStream_t stream) {
    if (in_chunks(p)) return launch_delta_chunk(p, stream);
    return p.in_dtype == PRECOG_F32 ? scan_cols<float>(p, stream) : scan_cols<__nv_bfloat16>(p, stream);
}

cudaError_t delta_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_delta_status); }

}  // namespace precog
