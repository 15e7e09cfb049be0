// One token of the diagonal selective scan for each row of a serving batch, on a table of fp32 states.
//
//   h <- exp(dt A) h + B x dt ;  y = (sum_n C h [its real part] + skip x) silu(gate)
//
// A channel's 16 states are four lanes'. What bounds it is memory: a state is read once and written once. 256 rows of 4096
// channels, bf16 with skip and gate (143 MB, 21.1 us at the measured copy rate): 27.0 us, of which the kernel's start and
// end are some four. With one channel for four lanes, 230 instructions for 16 bytes of state, it was 34 to 70 us.
#include "../../include/precog.h"
#include "internal.h"
#include "ptx.cuh"
#include "vec8.cuh"

namespace precog {
namespace {

__device__ uint32_t g_scan_step_status;

constexpr int kThreads = 128;
constexpr int kN = 16;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T>
__device__ __forceinline__ typename Raw4<T>::type raw4(const void *p, int64_t at) { return load4(static_cast<const T *>(p) + at); }

// The part of a launch that a warp works on: 32 channels of one layer, and every row_blocks-th row.
struct Share {
    int64_t layer;
    int first, d0;
    bool flag;   // one thread a row
};
__device__ __forceinline__ bool share_of(const ScanStepParams &p, unsigned channel_warps, unsigned row_blocks, int channels, Share &s) {
    const int64_t warp = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / 32;
    const int64_t rest = warp / channel_warps;
    s.d0 = static_cast<int>(warp % channel_warps) * channels;
    s.layer = rest / row_blocks;
    s.first = static_cast<int>(rest % row_blocks);
    s.flag = threadIdx.x % 32 == 0 && s.d0 == 0 && s.layer == 0;
    return s.layer < p.n_layers;
}
__device__ __forceinline__ int64_t slot_of(const ScanStepParams &p, int64_t i) { return i >= p.n ? -1 : p.slots ? p.slots[i] : i; }
__device__ __forceinline__ bool usable(const ScanStepParams &p, int64_t slot, bool flag) {
    if (slot >= 0 && slot < p.n_slots) return true;
    if (slot != -1 && flag) atomicOr(&g_scan_step_status, PRECOG_DEV_BAD_INDEX);
    return false;
}
// y times SiLU of a gate of type T, as exact as y is stored.
template <typename T>
__device__ __forceinline__ float gated(const ScanStepParams &p, float y, float gate) {
    return y * (p.y_dtype == PRECOG_F32 ? silu<T, float>(gate) : silu<T>(gate));
}
__device__ __forceinline__ void store_y(const ScanStepParams &p, int64_t at, float y) {
    if (p.y_dtype == PRECOG_F32) static_cast<float *>(p.y)[at] = y;
    else static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(y);
}

// What a row brings to a thread: four states (its quarter) of each of four neighbouring channels, its quarter of B
// and C, the channels' x and dt, and the gate of the channel whose y it writes.
template <typename T>
struct StepRow {
    float *state;   // nullptr: idle
    uint4 h[4];
    typename Raw4<T>::type B, C, x, dt;
    T gate;
};

// Real A. Four lanes have four channels: lane `part` states 4 part .. 4 part + 3 of each, so that x, dt, B and C are
// read and unpacked once for sixteen states, whose A stays in registers; and, of the readouts, channel `part`'s sum.
// Two rows are on their way while one is worked on, their slots a round before. (One row ahead in more warps: 28 to 29
// us for the case above; lanes with every eighth channel, for loads of 512 bytes in a piece: 28.2.)
template <typename T>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(const ScanStepParams p, unsigned channel_warps, unsigned row_blocks) {
    grid_dependency_wait();
    constexpr int kAhead = 2;
    Share share;
    if (!share_of(p, channel_warps, row_blocks, 32, share)) return;
    const int lane = threadIdx.x % 32, part = lane % 4, d = share.d0 + (lane & ~3);   // its channels d .. d + 3
    const bool inside = d < p.D;   // (D is a multiple of four; all lanes meet at the shuffles)
    const int64_t l = share.layer;
    StepRow<T> row[kAhead];
    int64_t slot[kAhead];
    auto load = [&](StepRow<T> &v, int64_t i, int64_t s) {
        v.state = nullptr;
        if (!usable(p, s, share.flag) || !inside) return;
        v.state = p.states + ((s * p.L_total + p.layer0 + l) * p.D + d) * kN + 4 * part;
#pragma unroll
        for (int c = 0; c < 4; ++c) v.h[c] = *reinterpret_cast<const uint4 *>(v.state + c * kN);
        const int64_t in = l * p.ls_xd + i * p.D + d, bc = l * p.ls_bc + i * kN + 4 * part;
        v.x = raw4<T>(p.x, in), v.dt = raw4<T>(p.dt, in);
        v.B = raw4<T>(p.B, bc), v.C = raw4<T>(p.C, bc);
        if (p.gate) v.gate = static_cast<const T *>(p.gate)[l * p.gate_layer_stride + i * p.gate_stride + d + part];
    };
#pragma unroll
    for (int r = 0; r < kAhead; ++r) slot[r] = slot_of(p, share.first + static_cast<int64_t>(r) * row_blocks);
#pragma unroll
    for (int r = 0; r < kAhead; ++r) load(row[r], share.first + static_cast<int64_t>(r) * row_blocks, slot[r]);
#pragma unroll
    for (int r = 0; r < kAhead; ++r) slot[r] = slot_of(p, share.first + static_cast<int64_t>(kAhead + r) * row_blocks);
    f2 a[4][2];        // log2(e) A
    float large[4];    // the largest of a channel's, in magnitude
    float skip = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        float v[4] = {};
        if (inside) unpack4(*reinterpret_cast<const uint4 *>(p.A + (l * p.D + d + c) * kN + 4 * part), v);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] *= kLog2e;
        a[c][0] = pack2(v[0], v[1]), a[c][1] = pack2(v[2], v[3]);
        large[c] = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
    }
    if (inside && p.skip) skip = p.skip[l * p.D + d + part];

    for (int64_t i0 = share.first; i0 < p.n; i0 += static_cast<int64_t>(kAhead) * row_blocks) {
#pragma unroll
        for (int r = 0; r < kAhead; ++r) {
            const int64_t i = i0 + static_cast<int64_t>(r) * row_blocks;
            if (i >= p.n) break;
            float *const state = row[r].state;
            float sum[4] = {}, x[4] = {};
            const float gate = state != nullptr && p.gate ? to_f32(row[r].gate) : 0.f;
            if (state != nullptr) {
                float dt[4], B[4], C[4];
                unpack4(row[r].x, x);
                unpack4(row[r].dt, dt);
                unpack4(row[r].B, B);
                unpack4(row[r].C, C);
                const f2 B2[2] = {pack2(B[0], B[1]), pack2(B[2], B[3])}, C2[2] = {pack2(C[0], C[1]), pack2(C[2], C[3])};
                // e^(dt A) can leave fp32 only where |dt A| is large; there a zero state must not meet an infinite factor
                const bool plain = fmaxf(fmaxf(fabsf(dt[0]) * large[0], fabsf(dt[1]) * large[1]),
                                         fmaxf(fabsf(dt[2]) * large[2], fabsf(dt[3]) * large[3])) <= kExp2Near;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float h[4];
                    unpack4(row[r].h[c], h);
                    const float u = x[c] * dt[c];
                    const f2 u2 = pack2(u, u), dt2 = pack2(dt[c], dt[c]);
                    f2 y2 = 0;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        f2 add = mul2(B2[k], u2), e = mul2(a[c][k], dt2), now;
                        float e0, e1;
                        unpack2(e, e0, e1);
                        if (plain) {
                            now = fma2(pack2(ex2(e0), ex2(e1)), pack2(h[2 * k], h[2 * k + 1]), add);
                        } else {
                            float b0, b1;
                            unpack2(add, b0, b1);
                            now = pack2(fma_exp2(h[2 * k], e0, b0), fma_exp2(h[2 * k + 1], e1, b1));
                        }
                        y2 = k == 0 ? mul2(C2[0], now) : fma2(C2[1], now, y2);
                        unpack2(now, h[2 * k], h[2 * k + 1]);
                    }
                    *reinterpret_cast<float4 *>(state + c * kN) = make_float4(h[0], h[1], h[2], h[3]);
                    float s0, s1;
                    unpack2(y2, s0, s1);
                    sum[c] = s0 + s1;
                }
            }
            load(row[r], i + static_cast<int64_t>(kAhead) * row_blocks, slot[r]);
            slot[r] = slot_of(p, i + static_cast<int64_t>(2 * kAhead) * row_blocks);
            // lane `part` keeps channel `part`'s sum: pairs of lanes exchange two channels, then one
            const bool odd = part & 1, high = part & 2;
            const float m0 = (odd ? sum[1] : sum[0]) + __shfl_xor_sync(0xffffffffu, odd ? sum[0] : sum[1], 1);
            const float m1 = (odd ? sum[3] : sum[2]) + __shfl_xor_sync(0xffffffffu, odd ? sum[2] : sum[3], 1);
            float y = (high ? m1 : m0) + __shfl_xor_sync(0xffffffffu, high ? m0 : m1, 2);
            if (!inside) continue;
            if (state != nullptr) {
                if (p.skip) y = fmaf(skip, high ? (odd ? x[3] : x[2]) : (odd ? x[1] : x[0]), y);
                if (p.gate) y = gated<T>(p, y, gate);
            }
            store_y(p, (l * p.n + i) * p.D + d + part, y);
        }
    }
}

// Complex A, states in pairs: four lanes have a channel, each four of its states. The sines take longer than the copies: 256
// rows of 4096 channels, bf16 with skip and gate (277 MB, 40.9 us at the measured copy rate): 60 us.
template <typename T>
__global__ void __launch_bounds__(kThreads) scan_step_complex_kernel(const ScanStepParams p, unsigned channel_warps, unsigned row_blocks) {
    grid_dependency_wait();
    Share share;
    if (!share_of(p, channel_warps, row_blocks, 8, share)) return;
    const int lane = threadIdx.x % 32, part = lane % 4, d = share.d0 + lane / 4;
    const bool inside = d < p.D;
    const int64_t l = share.layer;
    float a[8] = {}, skip = 0.f;
    if (inside) {
        const float *A = p.A + ((l * p.D + d) * kN + 4 * part) * 2;
        unpack4(reinterpret_cast<const uint4 *>(A)[0], *reinterpret_cast<float(*)[4]>(a));
        unpack4(reinterpret_cast<const uint4 *>(A)[1], *reinterpret_cast<float(*)[4]>(a + 4));
        if (p.skip) skip = p.skip[l * p.D + d];
    }
    for (int64_t i = share.first; i < p.n; i += row_blocks) {
        const int64_t slot = slot_of(p, i);
        const bool live = usable(p, slot, share.flag) && inside;
        float sum = 0.f, x = 0.f, gate = 0.f;
        if (live) {
            float *const state = p.states + (((slot * p.L_total + p.layer0 + l) * p.D + d) * kN + 4 * part) * 2;
            const int64_t in = l * p.ls_xd + i * p.D + d, bc = l * p.ls_bc + i * kN + 4 * part;
            const uint4 h0 = reinterpret_cast<const uint4 *>(state)[0], h1 = reinterpret_cast<const uint4 *>(state)[1];
            const auto rB = raw4<T>(p.B, bc), rC = raw4<T>(p.C, bc);
            x = to_f32(static_cast<const T *>(p.x)[in]);
            const float dt = to_f32(static_cast<const T *>(p.dt)[in]), u = x * dt;
            if (p.gate) gate = to_f32(static_cast<const T *>(p.gate)[l * p.gate_layer_stride + i * p.gate_stride + d]);
            float h[8], B[4], C[4];
            unpack4(h0, *reinterpret_cast<float(*)[4]>(h));
            unpack4(h1, *reinterpret_cast<float(*)[4]>(h + 4));
            unpack4(rB, B);
            unpack4(rC, C);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // the angle's product keeps its low half: phases of tens of turns would lose 2^-24 of themselves
                const float angle = dt * a[2 * k + 1], low = fmaf(dt, a[2 * k + 1], -angle);
                float sn, cs;
                sincosf(angle, &sn, &cs);
                const float sn1 = fmaf(low, cs, sn), cs1 = fmaf(-low, sn, cs), e = dt * a[2 * k] * kLog2e;
                const float re = h[2 * k], im = h[2 * k + 1];
                h[2 * k] = fma_exp2(fmaf(cs1, re, -sn1 * im), e, B[k] * u);
                h[2 * k + 1] = fma_exp2(fmaf(cs1, im, sn1 * re), e, 0.f);
                sum = fmaf(C[k], h[2 * k], sum);
            }
            reinterpret_cast<float4 *>(state)[0] = make_float4(h[0], h[1], h[2], h[3]);
            reinterpret_cast<float4 *>(state)[1] = make_float4(h[4], h[5], h[6], h[7]);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (!inside || part != 0) continue;
        if (live) {
            if (p.skip) sum = fmaf(skip, x, sum);
            if (p.gate) sum = gated<T>(p, sum, gate);
        }
        store_y(p, (l * p.n + i) * p.D + d, sum);
    }
}

// `channels` a warp; as many row blocks as make up to `warps` warps an SM: 12 are one round of the real kernel's (10 and 16:
// 30.5 and 33.1 us where 12 take 27.5, one layer of 4096 channels, 128 columns, which use 98 % of the round). The division is
// rounded down, so other calls use less of it, or begin a second one: 16 layers of 1312 channels (656 columns, 72 %) with 93
// rows take 55 us where the copy would 39, 8 layers of 4096 (1024 columns, 56 %) with 64 and 256 rows 66 of 42 and 250 of 169,
// 24 layers of 2560 (1920 columns, a second round of 96 warps) with 64 rows 130 of 79, 24 of 256 with 256 rows 40 of 32.
template <typename Kernel>
cudaError_t launch_kernel(Kernel kernel, const ScanStepParams &p, int channels, int warps, cudaStream_t stream) {
    const int64_t channel_warps = (p.D + channels - 1) / channels, columns = channel_warps * p.n_layers;
    int64_t row_blocks = static_cast<int64_t>(device_sm_count()) * warps / columns;
    row_blocks = row_blocks < 1 ? 1 : row_blocks > p.n ? p.n : row_blocks;
    const int64_t blocks = (columns * row_blocks * 32 + kThreads - 1) / kThreads;
    if (columns > 0x7fffffffLL || blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return launch_dependent(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, p,
                            static_cast<unsigned>(channel_warps), static_cast<unsigned>(row_blocks));
}

}  // namespace

cudaError_t launch_scan_step(const ScanStepParams &p, cudaStream_t stream) {
    const bool f32 = p.in_dtype == PRECOG_F32;
    cudaError_t e;
    if (p.complex) e = f32 ? launch_kernel(scan_step_complex_kernel<float>, p, 8, 128, stream)
                           : launch_kernel(scan_step_complex_kernel<__nv_bfloat16>, p, 8, 128, stream);
    else e = f32 ? launch_kernel(scan_step_kernel<float>, p, 32, 12, stream) : launch_kernel(scan_step_kernel<__nv_bfloat16>, p, 32, 12, stream);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

cudaError_t scan_step_status_word(uint32_t **word) { return cudaGetSymbolAddress(reinterpret_cast<void **>(word), g_scan_step_status); }

}  // namespace precog
