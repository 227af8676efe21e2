// What the kernels of the projection share: the epilogue's arguments, the activations and their slopes, vector accesses.
#pragma once

#include <cuda_bf16.h>

#include "rglru_internal.h"
#include "sm100_ptx.cuh"

namespace rglru {

struct LinearEpilogue {
    const float *bias;      // [N] or null
    const void *residual;   // [M,N] io or null (may be y)
    void *y, *preact;       // [M,N] io; preact may be null
    int activation;
};

constexpr float SQRT_HALF = 0.70710678118654752440f, INV_SQRT_2PI = 0.39894228040143267794f;
// Phi(z); 0 for minus infinity, where z Phi(z) would be NaN, is dealt with by the callers
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * erfcf(-z * SQRT_HALF); }
__device__ __forceinline__ float sigmoid32(float z) { return 1.0f / (1.0f + expf(-z)); }
// GeLU and SiLU tend to 0 at minus infinity and their slopes to 0 and 1: what remains is 0 * inf, which arithmetic has as NaN
__device__ __forceinline__ float activate(float z, int kind) {
    if (kind == RGLRU_ACT_NONE) return z;
    if (z == -INFINITY) return 0.0f;
    return z * (kind == RGLRU_ACT_GELU ? normal_cdf(z) : sigmoid32(z));
}
__device__ __forceinline__ float activation_slope(float z, int kind) {
    if (kind == RGLRU_ACT_NONE) return 1.0f;
    if (isinf(z)) return z > 0.0f ? 1.0f : 0.0f;
    if (kind == RGLRU_ACT_GELU) return fmaf(z * INV_SQRT_2PI, expf(-0.5f * z * z), normal_cdf(z));
    const float s = sigmoid32(z);
    return s * fmaf(z, 1.0f - s, 1.0f);
}

template <typename IO, int VE> struct LinearVec {
    static __device__ __forceinline__ void load(const IO *p, float (&f)[VE]) {
        if constexpr (VE == 1) {
            if constexpr (sizeof(IO) == 4) f[0] = *p;
            else f[0] = __bfloat162float(*p);
        } else if constexpr (sizeof(IO) == 4) {
            const float4 v = *(const float4 *)p;
            f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
        } else {
            const uint4 v = *(const uint4 *)p;
            const float2 a = ptx::bf2x(v.x), b = ptx::bf2x(v.y), c = ptx::bf2x(v.z), d = ptx::bf2x(v.w);
            f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
        }
    }
    static __device__ __forceinline__ void store(IO *p, const float (&f)[VE]) {
        if constexpr (VE == 1) {
            if constexpr (sizeof(IO) == 4) *p = f[0];
            else *p = __float2bfloat16_rn(f[0]);
        } else if constexpr (sizeof(IO) == 4) {
            *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
        } else {
            *(uint4 *)p = make_uint4(ptx::pack_bf16(f[0], f[1]), ptx::pack_bf16(f[2], f[3]), ptx::pack_bf16(f[4], f[5]), ptx::pack_bf16(f[6], f[7]));
        }
    }
};

}  // namespace rglru
