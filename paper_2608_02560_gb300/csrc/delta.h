// What the kernels of the gated delta rule share (delta.cu, delta_chunk.cu).
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "../../include/precog.h"
#include "internal.h"

namespace precog {

// The scan on the tensor cores: bf16 inputs, any lengths.
cudaError_t launch_delta_chunk(const DeltaParams &p, cudaStream_t stream);
size_t delta_chunk_workspace_size(const DeltaParams &p);

// Eight neighbouring numbers of a state in its storage type (`at` a multiple of 8).
__device__ __forceinline__ void delta_load8(const void *base, int dtype, int64_t at, float (&v)[8]) {
    if (dtype == PRECOG_F32) {   // whole 32-byte sectors where the address allows
        const float *s = static_cast<const float *>(base) + at;
        if ((reinterpret_cast<uintptr_t>(s) & 31u) == 0) {
            asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                         : "l"(s)
                         : "memory");
            return;
        }
        const float4 a = reinterpret_cast<const float4 *>(s)[0], b = reinterpret_cast<const float4 *>(s)[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(base) + at);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
__device__ __forceinline__ void delta_store8(void *base, int dtype, int64_t at, const float (&v)[8]) {
    if (dtype == PRECOG_F32) {
        float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(base) + at);
        if ((reinterpret_cast<uintptr_t>(d) & 31u) == 0) {
            asm volatile("st.global.v8.f32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                         "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "l"(d)
                         : "memory");
            return;
        }
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(base) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

}  // namespace precog
