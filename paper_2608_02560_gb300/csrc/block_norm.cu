// The end of a block in one pass over its rows: skip, gate, norm, residual with its scale, the next block's norm.
//
//   a = x + skip u ;  a <- a silu(gate) [before the norm] ;  a <- a rsqrt(mean a^2 + eps) weight [of each group]
//   a <- a silu(gate) [after the norm] ;  without a residual: out = a
//   h = residual + scale a ;  residual_out = h ;  out = h rsqrt(mean h^2 + eps) out_weight
//
// A row (or, where groups are normed, a group of one) belongs to LANES lanes that hold ENTRIES entries each, in pieces of
// 16 bytes; what is read is read once, all of it before the first is used, and stays in registers as fp32 until it is
// written. Sums are fp32, in an order that depends on the row's length, the types and, for long bf16 rows beside an fp32
// residual, on whether the call has a skip or gate.
//
// Memory bounds it: 65,521 bf16 rows of 2048, norm, scaled fp32 residual, next norm (1.61 GB, 237 us at the measured copy
// rate): 232 us; rows of 4096 with skip and gate (2.15 GB, 316 us): 300, in groups of 64 to 512 304 to 315. What carries it
// is warps: the first kernel, one load after the other, took 461 and 577, all loads ahead 280 and 342, CTAs of four warps
// for 2048 (two pieces a lane instead of one) 237, registers for what a call has 300. Two pieces a lane are best at every
// length: one, or four, took 280 for 2048, and one 390 for groups. fp32 rows: 23,437 of 2048 112 us (32 bytes a lane in one
// piece 123), 5859 of 8192 113 to 125. Rows of 16,384 take 1.6 of the copy's time; with all of skip,
// gate and fp32 residual rows of 2048 1.05, of 4096 1.24, of 8192 and 16,384 1.7 and 1.6 (fp32 rows of 8192 1.4). Lanes go to the next power of two, which
// other widths pay for: bf16 rows of 1536, 2560, 5120 and 6144 take 1.1, 1.2, 1.3 and 1.2 of it.
// Two rows a CTA for one load of the weights took more registers than that saves; rows in turn with the next one's copies
// in shared memory took the L1 that the weights live in (1.4 to 2 times as long); a cluster of two CTAs a row took 491
// for the rows of 4096.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"
#include "vec8.cuh"

namespace precog {
namespace {

// Sum over the row's lanes (each use has its own shared words).
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *part, int in_row) {
#pragma unroll
    for (int o = (LANES < 32 ? LANES : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (LANES > 32) {
        if ((threadIdx.x & 31) == 0) part[in_row / 32] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < LANES / 32; ++i) v += part[i];
    }
    return v;
}

// fp32 weights of V entries, or 1
template <int V>
__device__ __forceinline__ void weights(const float *w, int e, float (&v)[V]) {
    if (w == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 1.f;
        return;
    }
    unpack(load_piece<V>(w + e), v);
}

// What a call may have; what it has not takes no registers, and so leaves them to more warps.
enum Form { kAll, kInside, kBetween };   // (inside a block: no residual; between two: no skip, no gate)
// CTAs an SM that the registers have to be enough for: 48 warps of kInside (rows of 4096 above: 32 warps 329 us, 40 304,
// 48 300; several rows a CTA spill there, 379 in groups of 256 where 40 take 304). Between blocks 40 warps would spill.
template <typename T, typename TR, Form FORM, int LANES, int ENTRIES>
constexpr int min_ctas() {
    constexpr int block = LANES > 128 ? LANES : 128;
    if (LANES > 512) return 1;
    if (sizeof(T) == 4 && LANES == 512 && ENTRIES == 16) return 2;   // (8192: 165 us with one, 113 with two, 178 with three)
    if (FORM == kInside) return (LANES <= 64 ? 1280 : 1536) / block;
    if (sizeof(T) == 4 && LANES == 512 && FORM == kBetween) return 3;
    if (sizeof(T) < sizeof(TR) && FORM == kAll && LANES <= 128) return 7;   // (72 registers, gate to fp32: 65,521 rows of 2048 276 us, with 80 289)
    return 1;
}

template <typename T, typename TR, Form FORM, int LANES, int ENTRIES>
__global__ void __launch_bounds__(LANES > 128 ? LANES : 128, min_ctas<T, TR, FORM, LANES, ENTRIES>()) block_norm_kernel(const BlockNormParams p, int64_t rows) {
    grid_dependency_wait();
    constexpr bool kRes = FORM != kInside, kSkipGate = FORM != kBetween;
    using Widest = std::conditional_t<kRes, TR, T>;   // of the outputs: what the gate has to be exact for
    // Entries in one piece: 16 bytes of a row. Of long bf16 rows beside an fp32 residual 8, so that a warp reads that and the
    // weights in whole lines (rows of 4096: 89 us where 16 bytes take 97, of 8192 102 and 115; of 2048 they are equal, a
    // single row 2.5 and 2.1).
    constexpr int V = sizeof(T) == 4 || (sizeof(TR) == 4 && FORM == kBetween && LANES >= 256) ? 4 : 8, CH = ENTRIES / V;
    constexpr int kBlock = LANES > 128 ? LANES : 128, kRows = kBlock / LANES;
    __shared__ float part[2][kRows][LANES > 32 ? LANES / 32 : 1];
    const int mine = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + mine;
    const bool live = row < rows;   // (all rows of a CTA meet at its barriers)
    const int64_t t = live ? (p.groups == 1 ? row : static_cast<unsigned>(row) / static_cast<unsigned>(p.groups)) : 0;   // (rows < 2^31)
    const int size = p.groups == 1 ? p.dim : p.dim / p.groups, first = live ? static_cast<int>(row - t * p.groups) * size : 0;
    // every load of the row before the first is used
    Piece<T, V> x[CH], u[CH], g[CH];
    Piece<TR, V> res[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * LANES + lane) * V;
        if (!live || e >= size) continue;
        x[c] = load_piece<V>(static_cast<const T *>(p.x) + t * p.x_stride + first + e);
        if (kSkipGate && p.skip) u[c] = load_piece<V>(static_cast<const T *>(p.skip_input) + t * p.skip_stride + first + e);
        if (kSkipGate && p.gate) g[c] = load_piece<V>(static_cast<const T *>(p.gate) + t * p.gate_stride + first + e);
        if (kRes && p.residual) res[c] = load_piece<V>(static_cast<const TR *>(p.residual) + t * p.residual_stride + first + e);
    }
    float v[CH][V], w[V];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * LANES + lane) * V;
        if (!live || e >= size) continue;
        unpack(x[c], v[c]);
        if (kSkipGate && p.skip) {
            float s[V];
            unpack(u[c], s);
            weights(p.skip, first + e, w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] = fmaf(w[i], s[i], v[c][i]);
        }
        if (kSkipGate && p.gate && p.gate_first) {
            float s[V];
            unpack(g[c], s);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= silu<T, Widest>(s[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sum = fmaf(v[c][i], v[c][i], sum);
    }
    float scale = 1.f;
    if (p.norm == PRECOG_NORM_RMS) scale = rsqrtf(row_sum<LANES>(sum, part[0][mine], lane) / static_cast<float>(size) + p.eps);
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * LANES + lane) * V;
        if (!live || e >= size) continue;
        if (p.norm == PRECOG_NORM_RMS) {
            weights(p.weight, first + e, w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= scale * w[i];
        }
        if (kSkipGate && p.gate && !p.gate_first) {
            float s[V];
            unpack(g[c], s);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= silu<T, Widest>(s[i]);
        }
        if (kRes && p.residual) {
            float r[V];
            unpack(res[c], r);
            weights(p.scale_weight, first + e, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[c][i] = fmaf(p.scale * w[i], v[c][i], r[i]);
                sum = fmaf(v[c][i], v[c][i], sum);
            }
            TR *out = static_cast<TR *>(p.residual_out) + t * p.residual_out_stride + first + e;
            store_piece(out, v[c]);
        }
    }
    if (p.out == nullptr) return;   // (for all threads or none)
    scale = kRes && p.residual ? rsqrtf(row_sum<LANES>(sum, part[1][mine], lane) / static_cast<float>(size) + p.eps) : 1.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * LANES + lane) * V;
        if (!live || e >= size) continue;
        if (kRes && p.residual) {
            weights(p.out_weight, first + e, w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= scale * w[i];
        }
        T *out = static_cast<T *>(p.out) + t * p.out_stride + first + e;
        store_piece(out, v[c]);
    }
}

template <typename T, typename TR, Form FORM, int LANES, int ENTRIES>
cudaError_t launch_form(const BlockNormParams &p, cudaStream_t stream) {
    constexpr int kBlock = LANES > 128 ? LANES : 128, kRows = kBlock / LANES;
    const int64_t rows = p.T * p.groups, blocks = (rows + kRows - 1) / kRows;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_dependent(block_norm_kernel<T, TR, FORM, LANES, ENTRIES>, dim3(static_cast<unsigned>(blocks)), dim3(kBlock), 0, stream, p, rows);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T, typename TR, int LANES, int ENTRIES>
cudaError_t launch_shape(const BlockNormParams &p, cudaStream_t stream) {
    if constexpr (sizeof(TR) == 4)   // (without a residual TR is float)
        if (!p.residual) return launch_form<T, TR, kInside, LANES, ENTRIES>(p, stream);
    if (!p.skip && !p.gate) return launch_form<T, TR, kBetween, LANES, ENTRIES>(p, stream);
    return launch_form<T, TR, kAll, LANES, ENTRIES>(p, stream);
}

template <typename T, typename TR>
cudaError_t launch_typed(const BlockNormParams &p, cudaStream_t stream) {
    const int size = p.dim / p.groups;
    constexpr int E = sizeof(T) == 2 ? 16 : 8;   // entries a lane
    if (size <= 32) return launch_shape<T, TR, 32 / E, E>(p, stream);
    if (size <= 64) return launch_shape<T, TR, 64 / E, E>(p, stream);
    if (size <= 128) return launch_shape<T, TR, 128 / E, E>(p, stream);
    if (size <= 256) return launch_shape<T, TR, 256 / E, E>(p, stream);
    if (size <= 512) return launch_shape<T, TR, 512 / E, E>(p, stream);
    if (size <= 1024) return launch_shape<T, TR, 1024 / E, E>(p, stream);
    if (size <= 2048) return launch_shape<T, TR, 2048 / E, E>(p, stream);
    if (size <= 4096) return launch_shape<T, TR, 4096 / E, E>(p, stream);
    if (size <= 8192) return launch_shape<T, TR, 512, 16>(p, stream);
    return launch_shape<T, TR, 1024, 16>(p, stream);
}

}  // namespace

cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t stream) {
    if (p.dtype == PRECOG_F32) return launch_typed<float, float>(p, stream);
    return p.residual_dtype == PRECOG_F32 ? launch_typed<__nv_bfloat16, float>(p, stream)
                                          : launch_typed<__nv_bfloat16, __nv_bfloat16>(p, stream);
}

}  // namespace precog
