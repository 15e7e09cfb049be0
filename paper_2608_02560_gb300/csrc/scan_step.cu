// One token of the diagonal selective scan for each row of a serving batch, on a table of fp32 states.
//
//   h <- exp(dt A) h + B x dt ;  y = (sum_n C h [its real part] + skip x) silu(gate)
//
// A channel's 16 states are four lanes' (four 16-byte pieces, complex ones eight), the readout's sum two
// shuffles. What bounds it is memory: a state is read once and written once.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"
#include "vec8.cuh"

namespace precog {
namespace {

__device__ uint32_t g_scan_step_status;

constexpr int kThreads = 256;
constexpr int kN = 16;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T> struct Raw4;
template <> struct Raw4<float> { using type = uint4; };
template <> struct Raw4<__nv_bfloat16> { using type = uint2; };
__device__ __forceinline__ void unpack4(const uint4 &q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x), v[1] = __uint_as_float(q.y), v[2] = __uint_as_float(q.z), v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack4(const uint2 &q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xffff0000u);
    v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xffff0000u);
}

// What a row brings: its pieces of the state, B and C, and the channel's x, dt and gate.
template <typename T, int W>
struct StepRow {
    float *state;   // nullptr: idle
    uint4 h[W];
    typename Raw4<T>::type B, C;
    T x, dt, gate;
};

// A CTA has 64 channels of one layer, whose A stays in registers, and the rows first, first + stride, ...: AHEAD of
// them are on their way while one is worked on, and their slots one round before.
template <typename T, bool COMPLEX, int AHEAD>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(const ScanStepParams p, unsigned channel_blocks, unsigned row_blocks) {
    grid_dependency_wait();
    constexpr int W = COMPLEX ? 2 : 1;   // 16-byte pieces of states a thread
    const unsigned rest = blockIdx.x / channel_blocks;
    const int64_t l = rest / row_blocks;
    const int first = static_cast<int>(rest % row_blocks), n = static_cast<int>(p.n), stride = static_cast<int>(row_blocks);
    const int d = static_cast<int>(blockIdx.x % channel_blocks) * (kThreads / 4) + threadIdx.x / 4, part = threadIdx.x % 4;
    const bool inside = d < p.D;   // (all lanes meet at the shuffles)
    const bool flag = threadIdx.x == 0 && blockIdx.x % channel_blocks == 0 && l == 0;
    auto slot_of = [&](int64_t i) -> int64_t { return i >= n ? -1 : p.slots ? p.slots[i] : i; };
    StepRow<T, W> row[AHEAD];
    int64_t slot[AHEAD];
    auto load = [&](StepRow<T, W> &v, int64_t i, int64_t s) {
        v.state = nullptr;
        if (s < 0 || s >= p.n_slots) {
            if (s != -1 && flag) atomicOr(&g_scan_step_status, PRECOG_DEV_BAD_INDEX);
        } else if (inside) {
            v.state = p.states + ((s * p.L_total + p.layer0 + l) * p.D + d) * (kN * W) + 4 * W * part;
#pragma unroll
            for (int k = 0; k < W; ++k) v.h[k] = reinterpret_cast<const uint4 *>(v.state)[k];
            const int64_t in = l * p.ls_xd + i * p.D + d, bc = l * p.ls_bc + i * kN + 4 * part;
            v.x = static_cast<const T *>(p.x)[in];
            v.dt = static_cast<const T *>(p.dt)[in];
            v.B = *reinterpret_cast<const typename Raw4<T>::type *>(static_cast<const T *>(p.B) + bc);
            v.C = *reinterpret_cast<const typename Raw4<T>::type *>(static_cast<const T *>(p.C) + bc);
            if (p.gate) v.gate = static_cast<const T *>(p.gate)[l * p.gate_layer_stride + i * p.gate_stride + d];
        }
    };
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) slot[r] = slot_of(first + static_cast<int64_t>(r) * stride);
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) load(row[r], first + static_cast<int64_t>(r) * stride, slot[r]);
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) slot[r] = slot_of(first + static_cast<int64_t>(AHEAD + r) * stride);
    float a[4 * W] = {}, skip = 0.f;
    if (inside) {
#pragma unroll
        for (int k = 0; k < W; ++k)
            unpack4(reinterpret_cast<const uint4 *>(p.A + (l * p.D + d) * (kN * W) + 4 * W * part)[k], *reinterpret_cast<float(*)[4]>(a + 4 * k));
        if (p.skip) skip = p.skip[l * p.D + d];
    }
    for (int64_t i0 = first; i0 < n; i0 += static_cast<int64_t>(AHEAD) * stride) {
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            const int64_t i = i0 + static_cast<int64_t>(r) * stride;
            if (i >= n) break;
            float *const state = row[r].state;
            float sum = 0.f, x = 0.f, gate = 0.f;
            if (state != nullptr) {
                float h[4 * W], B[4], C[4];
#pragma unroll
                for (int k = 0; k < W; ++k) unpack4(row[r].h[k], *reinterpret_cast<float(*)[4]>(h + 4 * k));
                unpack4(row[r].B, B);
                unpack4(row[r].C, C);
                x = to_f32(row[r].x);
                gate = p.gate ? to_f32(row[r].gate) : 0.f;
                const float dt = to_f32(row[r].dt), u = x * dt;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (COMPLEX) {
                        // the angle's product keeps its low half: phases of tens of turns would lose 2^-24 of themselves
                        const float angle = dt * a[2 * k + 1], low = fmaf(dt, a[2 * k + 1], -angle);
                        float sn, cs;
                        sincosf(angle, &sn, &cs);
                        const float sn1 = fmaf(low, cs, sn), cs1 = fmaf(-low, sn, cs), e = dt * a[2 * k] * kLog2e;
                        const float re = h[2 * k], im = h[2 * k + 1];
                        h[2 * k] = fma_exp2(fmaf(cs1, re, -sn1 * im), e, B[k] * u);
                        h[2 * k + 1] = fma_exp2(fmaf(cs1, im, sn1 * re), e, 0.f);
                        sum = fmaf(C[k], h[2 * k], sum);
                    } else {
                        h[k] = fma_exp2(h[k], dt * a[k] * kLog2e, B[k] * u);
                        sum = fmaf(C[k], h[k], sum);
                    }
                }
#pragma unroll
                for (int k = 0; k < W; ++k)
                    reinterpret_cast<float4 *>(state)[k] = make_float4(h[4 * k], h[4 * k + 1], h[4 * k + 2], h[4 * k + 3]);
            }
            const bool idle = state == nullptr;
            load(row[r], i + static_cast<int64_t>(AHEAD) * stride, slot[r]);
            slot[r] = slot_of(i + static_cast<int64_t>(2 * AHEAD) * stride);
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if (!inside || part != 0) continue;
            if (!idle) {
                if (p.skip) sum = fmaf(skip, x, sum);
                if (p.gate) sum *= silu<T>(gate);
            }
            const int64_t o = (l * p.n + i) * p.D + d;
            if (p.y_dtype == PRECOG_F32) static_cast<float *>(p.y)[o] = sum;
            else static_cast<__nv_bfloat16 *>(p.y)[o] = __float2bfloat16_rn(sum);
        }
    }
}

template <typename T, bool COMPLEX>
cudaError_t launch_typed(const ScanStepParams &p, cudaStream_t stream) {
    const int64_t columns = static_cast<int64_t>((p.D + kThreads / 4 - 1) / (kThreads / 4)) * p.n_layers;
    constexpr int kAhead = 2, kResident = 8;
    if (columns > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    auto go = [&](auto kernel, int64_t row_blocks) {
        if (row_blocks * columns > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
        return launch_dependent(kernel, dim3(static_cast<unsigned>(row_blocks * columns)), dim3(kThreads), 0, stream, p,
                                static_cast<unsigned>(columns / p.n_layers), static_cast<unsigned>(row_blocks));
    };
    const int64_t room = static_cast<int64_t>(device_sm_count()) * kResident * kAhead;
    if (columns * p.n <= room) return go(scan_step_kernel<T, COMPLEX, 1>, p.n);
    int64_t row_blocks = static_cast<int64_t>(device_sm_count()) * kResident / columns;
    row_blocks = row_blocks < 1 ? 1 : row_blocks;
    return go(scan_step_kernel<T, COMPLEX, kAhead>, row_blocks < p.n ? row_blocks : p.n);
}

}  // namespace

cudaError_t launch_scan_step(const ScanStepParams &p, cudaStream_t stream) {
    const bool f32 = p.in_dtype == PRECOG_F32;
    const cudaError_t e = p.complex ? (f32 ? launch_typed<float, true>(p, stream) : launch_typed<__nv_bfloat16, true>(p, stream))
                                    : (f32 ? launch_typed<float, false>(p, stream) : launch_typed<__nv_bfloat16, false>(p, stream));
    if (e == cudaSuccess) count_launches(1);
    return e;
}

cudaError_t scan_step_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_scan_step_status); }

}  // namespace precog
