// What the kernels of the projection share: the epilogue's arguments, the activations and their slopes, vector accesses.
#pragma once

#include <cuda_bf16.h>

#include <type_traits>

#include "rglru_internal.h"
#include "rglru_io.cuh"
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
    // Where the tensor cores' form of the operand lies (sm100_linear_packed_bytes of it) if two products share it, and whether it is there already
    void *packed = nullptr;
    bool ready = false;
};
struct LinearProduct {
    LinearOperand a, b;
    long long M, N, K;
    int io;
    LinearEpilogue e;
    uint32_t flags = 0;   // RGLRU_FLAG_* of the call
};
// The scratch that the product takes
size_t sm100_linear_bytes(const LinearProduct &g);
// what an operand takes besides, 0 if it is read where it lies
size_t sm100_linear_packed_bytes(const LinearOperand &o, int io);
cudaError_t sm100_linear(const LinearProduct &g, void *scratch, uint32_t *status, cudaStream_t st);

// Activations and their slopes, to fp32's last places for fp32 io.  What goes to bf16 takes the hardware's exponential and reciprocal and, for Phi(-a) =
// P(t) t exp(-a^2 / 2) with t = 1 / (1 + 0.291 a), a polynomial of our own: a third of the instructions, and the element-wise kernels and
// epilogues are bound by memory or the tensor cores again.  P is the solution of a linear program over a = 0 .. 13.5 (where bf16 ends) that
// holds Phi's error to 6e-8 of one and to 1e-4 of itself, a fortieth of the least half step of a bf16 result, whichever is less; in fp32 arithmetic 2e-7
// and 1e-4.  (The same form with Abramowitz & Stegun's 7.1.26, one term shorter, holds the first alone: GeLU was off by two steps of its
// result at -6.)  At the infinities GeLU and SiLU are 0 and infinity, their slopes 0 and 1, where their formulas have 0 * inf.
constexpr float SQRT_HALF = 0.70710678118654752440f, INV_SQRT_2PI = 0.39894228040143267794f, LOG2_E = 1.44269504088896340736f;
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) { return ptx::fma2(a, b, c); }
__device__ __forceinline__ float2 both_of(float x) { return make_float2(x, x); }
// Phi(-|z|) and exp(-z^2 / 2) of two values whose magnitudes a are held at 30 (numbers: one reciprocal serves both)
struct Normal { float2 tail, density; };
__device__ __forceinline__ Normal normal_tail(float2 a) {
    const float2 d = fma_pair(a, both_of(0.291f), both_of(1.0f));
    const float2 t = ptx::mul2(make_float2(d.y, d.x), both_of(ptx::rcp_approx(d.x * d.y)));
    float2 p = fma_pair(t, both_of(-0.0881677568f), both_of(0.27912575f));
    p = fma_pair(p, t, both_of(-0.0864556655f));
    p = fma_pair(p, t, both_of(0.176318154f));
    p = fma_pair(p, t, both_of(0.101991124f));
    p = fma_pair(p, t, both_of(0.117188342f));
    const float2 x = ptx::mul2(ptx::mul2(a, a), both_of(-0.5f * LOG2_E));
    const float2 e = make_float2(ptx::ex2_approx(x.x), ptx::ex2_approx(x.y));
    return {ptx::mul2(ptx::mul2(p, t), e), e};
}
__device__ __forceinline__ float held(float z, float most) {   // NaN stays
    float c;
    asm("{\n.reg .f32 t;\nmin.NaN.f32 t, %1, %2;\nmax.NaN.f32 %0, t, %3;\n}" : "=f"(c) : "f"(z), "f"(most), "f"(-most));
    return c;
}
__device__ __forceinline__ float2 magnitudes(float2 z) { return make_float2(fminf(fabsf(z.x), 30.0f), fminf(fabsf(z.y), 30.0f)); }   // 30 for NaN
// for bf16 results
__device__ __forceinline__ float2 activate_fast(float2 z, int kind) {
    if (kind == RGLRU_ACT_NONE) return z;
    if (kind == RGLRU_ACT_GELU) {
        const float2 a = magnitudes(z);
        return fma_pair(make_float2(-a.x, -a.y), normal_tail(a).tail, make_float2(z.x < 0.0f ? 0.0f : z.x, z.y < 0.0f ? 0.0f : z.y));   // (NaN passes)
    }
    const float2 s = make_float2(ptx::rcp_approx(1.0f + ptx::ex2_approx(-LOG2_E * z.x)), ptx::rcp_approx(1.0f + ptx::ex2_approx(-LOG2_E * z.y)));
    return make_float2(z.x < -100.0f ? 0.0f : z.x * s.x, z.y < -100.0f ? 0.0f : z.y * s.y);
}
__device__ __forceinline__ float2 slope_fast(float2 z, int kind) {
    if (kind == RGLRU_ACT_GELU) {
        const float2 c = make_float2(held(z.x, 30.0f), held(z.y, 30.0f));
        const Normal n = normal_tail(magnitudes(z));
        const float2 phi = make_float2(c.x > 0.0f ? 1.0f - n.tail.x : n.tail.x, c.y > 0.0f ? 1.0f - n.tail.y : n.tail.y);
        return fma_pair(ptx::mul2(c, both_of(INV_SQRT_2PI)), n.density, phi);
    }
    const float2 c = make_float2(held(z.x, 100.0f), held(z.y, 100.0f));
    const float2 s = make_float2(ptx::rcp_approx(1.0f + ptx::ex2_approx(-LOG2_E * c.x)), ptx::rcp_approx(1.0f + ptx::ex2_approx(-LOG2_E * c.y)));
    return ptx::mul2(s, fma_pair(c, make_float2(1.0f - s.x, 1.0f - s.y), both_of(1.0f)));
}
// for fp32 results; out of line, since the libraries' functions are long
static __device__ __noinline__ float activate_exact(float z, int kind) {
    if (kind == RGLRU_ACT_GELU) return z == -INFINITY ? 0.0f : z * (0.5f * erfcf(-z * SQRT_HALF));
    return z < -100.0f ? 0.0f : z / (1.0f + expf(-z));
}
static __device__ __noinline__ float slope_exact(float z, int kind) {
    if (kind == RGLRU_ACT_GELU) {
        const float c = held(z, 30.0f);
        return fmaf(c * INV_SQRT_2PI, expf(-0.5f * c * c), 0.5f * erfcf(-c * SQRT_HALF));
    }
    const float c = held(z, 100.0f), s = 1.0f / (1.0f + expf(-c));
    return s * fmaf(c, 1.0f - s, 1.0f);
}
template <bool FAST> __device__ __forceinline__ float activate(float z, int kind) {
    if (kind == RGLRU_ACT_NONE) return z;
    if constexpr (FAST) return activate_fast(make_float2(z, z), kind).x;
    else return activate_exact(z, kind);
}
template <bool FAST> __device__ __forceinline__ float activation_slope(float z, int kind) {
    if (kind == RGLRU_ACT_NONE) return 1.0f;
    if constexpr (FAST) return slope_fast(make_float2(z, z), kind).x;
    else return slope_exact(z, kind);
}

template <typename IO, int VE> struct LinearVec {
    using Raw = std::conditional_t<VE == 1, IO, uint4>;   // as it lies in memory
    static __device__ __forceinline__ void unpack(const Raw &v, float (&f)[VE]) {
        if constexpr (VE == 1) {
            f[0] = (float)v;
        } else if constexpr (sizeof(IO) == 4) {
            f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
        } else {
            const float2 a = ptx::bf2x(v.x), b = ptx::bf2x(v.y), c = ptx::bf2x(v.z), d = ptx::bf2x(v.w);
            f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
        }
    }
    static __device__ __forceinline__ void load(const IO *p, float (&f)[VE]) { unpack(*(const Raw *)p, f); }
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
