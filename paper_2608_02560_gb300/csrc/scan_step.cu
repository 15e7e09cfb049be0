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

// four neighbouring elements as fp32
__device__ __forceinline__ void load4(const float *p, float (&v)[4]) {
    const float4 q = *reinterpret_cast<const float4 *>(p);
    v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16 *p, float (&v)[4]) {
    const uint2 q = *reinterpret_cast<const uint2 *>(p);
    v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xffff0000u);
    v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xffff0000u);
}

template <typename T, bool COMPLEX>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(const ScanStepParams p) {
    grid_dependency_wait();
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t per = static_cast<int64_t>(p.D) * 4;
    const int64_t pair = at / per;   // (layer, row)
    const bool live = pair < p.n_layers * p.n;
    const int rest = static_cast<int>(at - pair * per);
    const int d = rest / 4, part = rest % 4;
    const int64_t l = pair / p.n, i = pair - l * p.n;
    int64_t slot = -1;
    if (live) {
        slot = p.slots ? p.slots[i] : i;
        if (slot < -1 || slot >= p.n_slots) {
            if (rest == 0 && l == 0) atomicOr(&g_scan_step_status, PRECOG_DEV_BAD_INDEX);
            slot = -1;
        }
    }
    float sum = 0.f, x = 0.f;
    if (slot >= 0) {
        const int64_t in = l * p.ls_xd + i * p.D + d;
        x = to_f32(static_cast<const T *>(p.x)[in]);
        const float dt = to_f32(static_cast<const T *>(p.dt)[in]), u = x * dt;
        float B[4], C[4];
        const int64_t bc = l * p.ls_bc + i * kN + 4 * part;
        load4(static_cast<const T *>(p.B) + bc, B);
        load4(static_cast<const T *>(p.C) + bc, C);
        constexpr int W = COMPLEX ? 2 : 1;
        float *state = p.states + ((slot * p.L_total + p.layer0 + l) * p.D + d) * (kN * W) + 4 * W * part;
        const float *A = p.A + (l * p.D + d) * (kN * W) + 4 * W * part;
        float h[4 * W], a[4 * W];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            load4(state + 4 * k, *reinterpret_cast<float(*)[4]>(h + 4 * k));
            load4(A + 4 * k, *reinterpret_cast<float(*)[4]>(a + 4 * k));
        }
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
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (!live || part != 0) return;
    if (slot >= 0) {
        if (p.skip) sum = fmaf(p.skip[l * p.D + d], x, sum);
        if (p.gate) sum *= silu<T>(to_f32(static_cast<const T *>(p.gate)[l * p.gate_layer_stride + i * p.gate_stride + d]));
    }
    const int64_t o = (l * p.n + i) * p.D + d;
    if (p.y_dtype == PRECOG_F32) static_cast<float *>(p.y)[o] = sum;
    else static_cast<__nv_bfloat16 *>(p.y)[o] = __float2bfloat16_rn(sum);
}

}  // namespace

cudaError_t launch_scan_step(const ScanStepParams &p, cudaStream_t stream) {
    const int64_t blocks = (p.n_layers * p.n * p.D * 4 + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    auto go = [&](auto kernel) { return launch_dependent(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, p); };
    const bool f32 = p.in_dtype == PRECOG_F32;
    cudaError_t e;
    if (p.complex) e = f32 ? go(scan_step_kernel<float, true>) : go(scan_step_kernel<__nv_bfloat16, true>);
    else e = f32 ? go(scan_step_kernel<float, false>) : go(scan_step_kernel<__nv_bfloat16, false>);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

cudaError_t scan_step_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_scan_step_status); }

}  // namespace precog
