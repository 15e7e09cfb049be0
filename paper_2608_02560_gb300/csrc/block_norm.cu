// The end of a block in one pass over its rows: skip, gate, norm, residual with its scale, the next block's norm.
//
//   a = x + skip u ;  a <- a silu(gate) [before the norm] ;  a <- a rsqrt(mean a^2 + eps) weight [of each group]
//   a <- a silu(gate) [after the norm] ;  without a residual: out = a
//   h = residual + scale a ;  residual_out = h ;  out = h rsqrt(mean h^2 + eps) out_weight
//
// A row (or, where groups are normed, a group of one) belongs to LANES lanes that hold 16 bytes of neighbouring entries
// CH times each; what is read is read once, all of it before the first is used, and stays in registers as fp32 until it
// is written. Sums are fp32, in an order that depends on the row's length and type alone.
//
// Memory bounds it: 65,521 bf16 rows of 2048, norm, scaled fp32 residual, next norm (1.61 GB, 237 us at the measured copy
// rate): 235.5 us; rows of 4096 with skip and gate (2.15 GB, 316 us): 338, in groups of 64 to 512 332 to 344. Twice 16
// bytes a lane are best at every length (us, rows of 2048: 128 lanes 237, 256 lanes with one piece 280, 64 with four 281;
// of 4096, gated: 256 lanes 340, 128 with four 386, 512 with one 392; groups of 64 to 256 with one 390): more bytes a
// thread on the way, fewer warps at a barrier. Four entries a lane in bf16, which would read the fp32 weights in whole
// lines, took 231 and 364; fp32 rows have them so (32 bytes a lane: 123 us where 16 take 113 for 23,437 rows of 2048).
// Beyond 4096 a row's barriers leave the CTA waiting (8192: 1.3 to 1.6 of the copy's time). Two rows a CTA for one load of
// the weights took more registers than that saves (278 and 412 us); rows in turn with the next one's copies in shared
// memory took the L1 that the weights live in (1.4 to 2 times as long); a cluster of two CTAs for a row of 4096 took 491.
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

template <typename T, typename TR, int LANES, int CH>
__global__ void __launch_bounds__(LANES > 128 ? LANES : 128) block_norm_kernel(const BlockNormParams p, int64_t rows) {
    grid_dependency_wait();
    constexpr int V = 16 / static_cast<int>(sizeof(T));   // entries of 16 bytes of a row
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
        if (p.skip) u[c] = load_piece<V>(static_cast<const T *>(p.skip_input) + t * p.skip_stride + first + e);
        if (p.gate) g[c] = load_piece<V>(static_cast<const T *>(p.gate) + t * p.gate_stride + first + e);
        if (p.residual) res[c] = load_piece<V>(static_cast<const TR *>(p.residual) + t * p.residual_stride + first + e);
    }
    float v[CH][V], w[V];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * LANES + lane) * V;
        if (!live || e >= size) continue;
        unpack(x[c], v[c]);
        if (p.skip) {
            float s[V];
            unpack(u[c], s);
            weights(p.skip, first + e, w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] = fmaf(w[i], s[i], v[c][i]);
        }
        if (p.gate && p.gate_first) {
            float s[V];
            unpack(g[c], s);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= silu<T>(s[i]);
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
        if (p.gate && !p.gate_first) {
            float s[V];
            unpack(g[c], s);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= silu<T>(s[i]);
        }
        if (p.residual) {
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
    scale = p.residual ? rsqrtf(row_sum<LANES>(sum, part[1][mine], lane) / static_cast<float>(size) + p.eps) : 1.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * LANES + lane) * V;
        if (!live || e >= size) continue;
        if (p.residual) {
            weights(p.out_weight, first + e, w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[c][i] *= scale * w[i];
        }
        T *out = static_cast<T *>(p.out) + t * p.out_stride + first + e;
        store_piece(out, v[c]);
    }
}

template <typename T, typename TR, int LANES, int CH>
cudaError_t launch_shape(const BlockNormParams &p, cudaStream_t stream) {
    constexpr int kBlock = LANES > 128 ? LANES : 128, kRows = kBlock / LANES;
    const int64_t rows = p.T * p.groups, blocks = (rows + kRows - 1) / kRows;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_dependent(block_norm_kernel<T, TR, LANES, CH>, dim3(static_cast<unsigned>(blocks)), dim3(kBlock), 0, stream, p, rows);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

template <typename T, typename TR>
cudaError_t launch_typed(const BlockNormParams &p, cudaStream_t stream) {
    const int size = p.dim / p.groups;
    constexpr bool kHalf = sizeof(T) == 2;
    if (size <= 32) return launch_shape<T, TR, kHalf ? 2 : 4, 2>(p, stream);
    if (size <= 64) return launch_shape<T, TR, kHalf ? 4 : 8, 2>(p, stream);
    if (size <= 128) return launch_shape<T, TR, kHalf ? 8 : 16, 2>(p, stream);
    if (size <= 256) return launch_shape<T, TR, kHalf ? 16 : 32, 2>(p, stream);
    if (size <= 512) return launch_shape<T, TR, kHalf ? 32 : 64, 2>(p, stream);
    if (size <= 1024) return launch_shape<T, TR, kHalf ? 64 : 128, 2>(p, stream);
    if (size <= 2048) return launch_shape<T, TR, kHalf ? 128 : 256, 2>(p, stream);
    if (size <= 4096) return launch_shape<T, TR, kHalf ? 256 : 512, 2>(p, stream);
    if (size <= 8192) return launch_shape<T, TR, 512, kHalf ? 2 : 4>(p, stream);
    return launch_shape<T, TR, 1024, kHalf ? 2 : 4>(p, stream);
}

}  // namespace

cudaError_t launch_block_norm(const BlockNormParams &p, cudaStream_t stream) {
    if (p.dtype == PRECOG_F32) return launch_typed<float, float>(p, stream);
    return p.residual_dtype == PRECOG_F32 ? launch_typed<__nv_bfloat16, float>(p, stream)
                                          : launch_typed<__nv_bfloat16, __nv_bfloat16>(p, stream);
}

}  // namespace precog
