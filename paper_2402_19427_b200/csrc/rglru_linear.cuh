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

// ---- the products on the tensor cores (rglru_sm100_linear.cu)
// out[m][n] = epilogue(sum_k A(m,k) B(n,k)).  An operand is a matrix in memory [rows][cols]; `turned`: K runs along its rows.
struct LinearOperand {
    const void *p;
    long long rows, cols;
    bool turned;
};
struct LinearProduct {
    LinearOperand a, b;
    long long M, N, K;
    int io;
    LinearEpilogue e;
};
// Whether the tensor cores serve the product better than the CUDA cores, and the scratch that it takes
bool sm100_linear_wanted(const LinearProduct &g);
size_t sm100_linear_bytes(const LinearProduct &g);
cudaError_t sm100_linear(const LinearProduct &g, void *scratch, uint32_t *status, cudaStream_t st);

// Activations and their slopes, to fp32's last places for fp32 io.  What goes to bf16 takes Phi from the rational approximation 7.1.26 of
// Abramowitz & Stegun (off by less than 7.5e-8) and the hardware's exponential and reciprocal: a third of the instructions, and the
// element-wise kernels and epilogues are bound by memory or the tensor cores again.  At the infinities GeLU and SiLU are 0 and
// infinity, their slopes 0 and 1, where their formulas have 0 * inf.
constexpr float SQRT_HALF = 0.70710678118654752440f, INV_SQRT_2PI = 0.39894228040143267794f, LOG2_E = 1.44269504088896340736f;
struct Normal { float tail, density; };   // Phi(-|z|) and exp(-z^2 / 2), for |z| held at 30
__device__ __forceinline__ Normal normal_tail(float z) {
    const float a = fabsf(z) > 30.0f ? 30.0f : fabsf(z);   // NaN stays
    const float t = ptx::rcp_approx(fmaf(a, 0.3275911f * SQRT_HALF, 1.0f));
    float p = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
    p = fmaf(p, t, 0.5f * 1.421413741f); p = fmaf(p, t, 0.5f * -0.284496736f); p = fmaf(p, t, 0.5f * 0.254829592f);
    const float e = ptx::ex2_approx(a * a * (-0.5f * LOG2_E));
    return {p * t * e, e};
}
template <bool FAST> __device__ __forceinline__ float sigmoid_of(float z) {
    if constexpr (FAST) return ptx::rcp_approx(1.0f + ptx::ex2_approx(-LOG2_E * z));
    else return 1.0f / (1.0f + expf(-z));
}
template <bool FAST> __device__ __forceinline__ float activate(float z, int kind) {
    if (kind == RGLRU_ACT_NONE) return z;
    if (kind == RGLRU_ACT_GELU) {
        if constexpr (FAST) {
            const float a = fabsf(z) > 30.0f ? 30.0f : fabsf(z);
            return fmaf(-a, normal_tail(z).tail, z > 0.0f ? z : 0.0f);
        } else {
            return z == -INFINITY ? 0.0f : z * (0.5f * erfcf(-z * SQRT_HALF));
        }
    }
    return z < -100.0f ? 0.0f : z * sigmoid_of<FAST>(z);
}
template <bool FAST> __device__ __forceinline__ float activation_slope(float z, int kind) {
    if (kind == RGLRU_ACT_NONE) return 1.0f;
    if (kind == RGLRU_ACT_GELU) {
        const float zc = z > 30.0f ? 30.0f : z < -30.0f ? -30.0f : z;
        if constexpr (FAST) {
            const Normal n = normal_tail(zc);
            return fmaf(zc * INV_SQRT_2PI, n.density, zc > 0.0f ? 1.0f - n.tail : n.tail);
        } else {
            return fmaf(zc * INV_SQRT_2PI, expf(-0.5f * zc * zc), 0.5f * erfcf(-zc * SQRT_HALF));
        }
    }
    const float zc = z > 100.0f ? 100.0f : z < -100.0f ? -100.0f : z, s = sigmoid_of<FAST>(zc);
    return s * fmaf(zc, 1.0f - s, 1.0f);
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
