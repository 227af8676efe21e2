// Normalisation of rows (layer norm, or the mean square alone) and its gradients: extern "C" entry points and CUDA kernels.
//
//   forward   mu = mean(x), r = 1/sqrt(mean((x - mu)^2) + eps), y = (x - mu) r w + b
//   backward  xh = (x - mu) r, g = dy w:  dx = r (g - mean(g) - xh mean(g xh)),  dw = sum dy xh,  db = sum dy
//
// Both are bound by memory: 4 bytes an element forward, 6 backward (bf16).  A row is read once and stays in registers between the
// statistics and the result, so that the deviations are taken from the mean itself (no difference of large sums).  A group of threads owns a
// row: up to a warp of them for narrow rows, several rows a warp; a whole block for wide ones.  Groups walk rows with the next row's
// loads in flight and the weights in registers.
#include <cuda_bf16.h>

#include "rglru_internal.h"
#include "sm100_ptx.cuh"

namespace rglru {
namespace {

using namespace ptx;

struct NormArgs {
    long long rows;
    int N, G;            // G: threads a row (narrow rows: 8, 16 or 32; wide ones: the block)
    int center;
    float eps, inv_n;
    const void *x, *dy;
    const float *weight, *bias;
    const float *mean_in, *rstd_in;
    void *out;           // y or dx
    float *mean, *rstd;
    float *part;         // backward: [blocks][2][N] sums of dy xh and dy over a block's rows, or null
};

// VE neighbouring elements as they lie in memory
template <typename IO, int VE> struct Raw { uint32_t w[VE * sizeof(IO) / 4]; };
template <> struct Raw<__nv_bfloat16, 1> { uint16_t w; };

template <typename IO, int VE> __device__ __forceinline__ Raw<IO, VE> load_raw(const IO *p) {
    Raw<IO, VE> r;
    if constexpr (VE * sizeof(IO) == 16) {
        const uint4 v = *(const uint4 *)p;
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else if constexpr (sizeof(IO) == 4) {
        r.w[0] = *(const uint32_t *)p;
    } else {
        r.w = *(const uint16_t *)p;
    }
    return r;
}
template <typename IO, int VE> __device__ __forceinline__ void unpack(const Raw<IO, VE> &r, float (&f)[VE]) {
    if constexpr (sizeof(IO) == 4) {
#pragma unroll
        for (int e = 0; e < VE; ++e) f[e] = __uint_as_float(r.w[e]);
    } else if constexpr (VE == 1) {
        f[0] = __uint_as_float((uint32_t)r.w << 16);
    } else {
#pragma unroll
        for (int e = 0; e < VE; e += 2) { const f32x2 v = bf2x(r.w[e / 2]); f[e] = v.x; f[e + 1] = v.y; }
    }
}
template <typename IO, int VE> __device__ __forceinline__ void store_vec(IO *p, const float (&f)[VE]) {
    if constexpr (VE == 1) {
        if constexpr (sizeof(IO) == 4) *p = f[0];
        else *p = __float2bfloat16_rn(f[0]);
    } else if constexpr (sizeof(IO) == 4) {
        *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        *(uint4 *)p = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
}
template <int VE> __device__ __forceinline__ void load_f32(const float *p, float (&f)[VE]) {
#pragma unroll
    for (int e = 0; e < VE; e += (VE % 4 == 0 ? 4 : 1)) {
        if constexpr (VE % 4 == 0) { const float4 v = *(const float4 *)(p + e); f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w; }
        else f[e] = p[e];
    }
}

// Sums of K values over the group of threads that owns a row; every thread of the group gets them.  Wide groups go through
// shared memory, in two buffers used in turn, so that one barrier per call is enough.
template <bool WIDE, int K> struct GroupSum {
    float (*buf)[K][32];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[K], int G) {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            if (WIDE || o < G) {
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
            }
        }
        if constexpr (WIDE) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = G >> 5;
            float (&b)[K][32] = buf[turn];
            turn ^= 1;
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) b[k][warp] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = lane < warps ? b[k][lane] : 0.0f;
#pragma unroll
                for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
            }
        }
    }
};

// Rows of at most G V VE elements.  Thread t of a group holds the vectors t, t + G, ... of its row.
template <typename IO, int VE, int V, bool WIDE, int MAXT> __global__ void __launch_bounds__(MAXT) norm_kernel(NormArgs a) {
    __shared__ float red[2][1][32];
    dependency_wait();
    const int G = a.G, t = WIDE ? threadIdx.x : threadIdx.x & (G - 1);
    const long long group = WIDE ? blockIdx.x : ((long long)blockIdx.x * blockDim.x + threadIdx.x) / G;
    const long long groups = WIDE ? gridDim.x : (long long)gridDim.x * blockDim.x / G;
    GroupSum<WIDE, 1> sum{red};
    bool in[V];
    float w[V][VE], b[V][VE];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (t + v * G) * VE;
        in[v] = c < a.N;
#pragma unroll
        for (int e = 0; e < VE; ++e) { w[v][e] = 1.0f; b[v][e] = 0.0f; }
        if (in[v] && a.weight) load_f32<VE>(a.weight + c, w[v]);
        if (in[v] && a.bias) load_f32<VE>(a.bias + c, b[v]);
    }
    Raw<IO, VE> next[V] = {};
    auto fetch = [&](long long row) {
        const IO *p = (const IO *)a.x + row * a.N + t * VE;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (in[v]) next[v] = load_raw<IO, VE>(p + v * G * VE);
    };
    if (group < a.rows) fetch(group);
    // all lanes of a warp stay in the loop while one of its groups has a row, for the shuffles; a wide group's block leaves as one
    for (long long row = group; WIDE ? row < a.rows : __any_sync(0xffffffffu, row < a.rows); row += groups) {
        float f[V][VE];
#pragma unroll
        for (int v = 0; v < V; ++v) unpack<IO, VE>(next[v], f[v]);
        if (row + groups < a.rows) fetch(row + groups);
        float s[1] = {0.0f};
        if (a.center) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < VE; ++e) s[0] += in[v] ? f[v][e] : 0.0f;
            sum(s, G);
        }
        const float mu = s[0] * a.inv_n;
        s[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < VE; ++e) { f[v][e] -= mu; s[0] += in[v] ? f[v][e] * f[v][e] : 0.0f; }
        sum(s, G);
        const float r = 1.0f / sqrtf(s[0] * a.inv_n + a.eps);
        if (row < a.rows) {
            IO *p = (IO *)a.out + row * a.N + t * VE;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!in[v]) continue;
#pragma unroll
                for (int e = 0; e < VE; ++e) f[v][e] = fmaf(f[v][e] * r, w[v][e], b[v][e]);
                store_vec<IO, VE>(p + v * G * VE, f[v]);
            }
            if (t == 0) {
                if (a.mean) a.mean[row] = mu;
                if (a.rstd) a.rstd[row] = r;
            }
        }
    }
    dependency_trigger();
}

// The gradients, rows as above.  The column sums of a group's rows stay in registers and leave once, added over the block's groups.
template <typename IO, int VE, int V, bool WIDE, int MAXT> __global__ void __launch_bounds__(MAXT) norm_backward_kernel(NormArgs a) {
    __shared__ float red[2][2][32];
    extern __shared__ float cols[];   // narrow rows: [2][N] sums of the block
    dependency_wait();
    const int G = a.G, t = WIDE ? threadIdx.x : threadIdx.x & (G - 1);
    const long long group = WIDE ? blockIdx.x : ((long long)blockIdx.x * blockDim.x + threadIdx.x) / G;
    const long long groups = WIDE ? gridDim.x : (long long)gridDim.x * blockDim.x / G;
    GroupSum<WIDE, 2> sum{red};
    bool in[V];
    float w[V][VE], dw[V][VE] = {}, db[V][VE] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (t + v * G) * VE;
        in[v] = c < a.N;
#pragma unroll
        for (int e = 0; e < VE; ++e) w[v][e] = 1.0f;
        if (in[v] && a.weight) load_f32<VE>(a.weight + c, w[v]);
    }
    Raw<IO, VE> nx[V] = {}, ny[V] = {};
    float nmu = 0.0f, nr = 0.0f;
    auto fetch = [&](long long row) {
        const IO *px = (const IO *)a.x + row * a.N + t * VE, *py = (const IO *)a.dy + row * a.N + t * VE;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (in[v]) { nx[v] = load_raw<IO, VE>(px + v * G * VE); ny[v] = load_raw<IO, VE>(py + v * G * VE); }
        nmu = a.center ? a.mean_in[row] : 0.0f;
        nr = a.rstd_in[row];
    };
    if (group < a.rows) fetch(group);
    for (long long row = group; WIDE ? row < a.rows : __any_sync(0xffffffffu, row < a.rows); row += groups) {
        const bool live = row < a.rows;
        float h[V][VE], g[V][VE];
        const float mu = nmu, r = nr;
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            unpack<IO, VE>(nx[v], h[v]);
            unpack<IO, VE>(ny[v], g[v]);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                h[v][e] = (h[v][e] - mu) * r;
                if (live && in[v]) {
                    dw[v][e] = fmaf(g[v][e], h[v][e], dw[v][e]);
                    db[v][e] += g[v][e];
                }
                g[v][e] *= w[v][e];
                if (in[v]) { s[0] = fmaf(g[v][e], h[v][e], s[0]); s[1] += g[v][e]; }
            }
        }
        if (row + groups < a.rows) fetch(row + groups);
        sum(s, G);
        const float c2 = s[0] * a.inv_n, c1 = a.center ? s[1] * a.inv_n : 0.0f;
        if (live) {
            IO *p = (IO *)a.out + row * a.N + t * VE;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!in[v]) continue;
#pragma unroll
                for (int e = 0; e < VE; ++e) g[v][e] = r * (fmaf(-h[v][e], c2, g[v][e]) - c1);
                store_vec<IO, VE>(p + v * G * VE, g[v]);
            }
        }
    }
    dependency_trigger();
    if (a.part == nullptr) return;
    float *part = a.part + (size_t)blockIdx.x * 2 * a.N;
    if constexpr (WIDE) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (in[v])
#pragma unroll
                for (int e = 0; e < VE; ++e) { part[(t + v * G) * VE + e] = dw[v][e]; part[a.N + (t + v * G) * VE + e] = db[v][e]; }
    } else {
        // the groups of a warp by shuffles, the warps of a block one after the other, in a fixed order
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < VE; ++e)
                for (int o = G; o < 32; o <<= 1) {
                    dw[v][e] += __shfl_xor_sync(0xffffffffu, dw[v][e], o);
                    db[v][e] += __shfl_xor_sync(0xffffffffu, db[v][e], o);
                }
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        for (int k = 0; k < warps; ++k) {
            if (warp == k && lane < G) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (in[v])
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            const int c = (t + v * G) * VE + e;
                            const float p0 = k ? cols[c] : 0.0f, p1 = k ? cols[a.N + c] : 0.0f;
                            if (k < warps - 1) { cols[c] = p0 + dw[v][e]; cols[a.N + c] = p1 + db[v][e]; }
                            else { part[c] = p0 + dw[v][e]; part[a.N + c] = p1 + db[v][e]; }
                        }
            }
            __syncthreads();
        }
    }
}

// Rows that no block holds in registers: a block reads its row three times (the second and third time mostly out of L2).
template <typename IO> __device__ __forceinline__ float at(const void *p, long long i) {
    if constexpr (sizeof(IO) == 4) return ((const float *)p)[i];
    else return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
}
template <typename IO> __device__ __forceinline__ void put(void *p, long long i, float v) {
    const float f[1] = {v};
    store_vec<IO, 1>((IO *)p + i, f);
}
template <typename IO> __global__ void __launch_bounds__(1024) norm_long_kernel(NormArgs a) {
    __shared__ float red[2][1][32];
    dependency_wait();
    GroupSum<true, 1> sum{red};
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const long long base = row * a.N;
        float s[1] = {0.0f};
        if (a.center) {
            for (int c = threadIdx.x; c < a.N; c += 1024) s[0] += at<IO>(a.x, base + c);
            sum(s, 1024);
        }
        const float mu = s[0] * a.inv_n;
        s[0] = 0.0f;
        for (int c = threadIdx.x; c < a.N; c += 1024) { const float d = at<IO>(a.x, base + c) - mu; s[0] = fmaf(d, d, s[0]); }
        sum(s, 1024);
        const float r = 1.0f / sqrtf(s[0] * a.inv_n + a.eps);
        for (int c = threadIdx.x; c < a.N; c += 1024)
            put<IO>(a.out, base + c, fmaf((at<IO>(a.x, base + c) - mu) * r, a.weight ? a.weight[c] : 1.0f, a.bias ? a.bias[c] : 0.0f));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mu;
            if (a.rstd) a.rstd[row] = r;
        }
    }
    dependency_trigger();
}
template <typename IO> __global__ void __launch_bounds__(1024) norm_long_backward_kernel(NormArgs a) {
    __shared__ float red[2][2][32];
    dependency_wait();
    GroupSum<true, 2> sum{red};
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const long long base = row * a.N;
        const float mu = a.center ? a.mean_in[row] : 0.0f, r = a.rstd_in[row];
        float s[2] = {0.0f, 0.0f};
        for (int c = threadIdx.x; c < a.N; c += 1024) {
            const float g = at<IO>(a.dy, base + c) * (a.weight ? a.weight[c] : 1.0f);
            s[0] = fmaf(g, (at<IO>(a.x, base + c) - mu) * r, s[0]);
            s[1] += g;
        }
        sum(s, 1024);
        const float c2 = s[0] * a.inv_n, c1 = a.center ? s[1] * a.inv_n : 0.0f;
        for (int c = threadIdx.x; c < a.N; c += 1024) {
            const float g = at<IO>(a.dy, base + c) * (a.weight ? a.weight[c] : 1.0f);
            put<IO>(a.out, base + c, r * (fmaf(-(at<IO>(a.x, base + c) - mu) * r, c2, g) - c1));
        }
    }
    dependency_trigger();
}
// their column sums: a thread per column, blockIdx.y: a share of the rows
template <typename IO> __global__ void __launch_bounds__(256) norm_long_columns_kernel(NormArgs a) {
    dependency_wait();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < a.N) {
        float dw = 0.0f, db = 0.0f;
        for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
            const float g = at<IO>(a.dy, row * a.N + c);
            dw = fmaf(g, (at<IO>(a.x, row * a.N + c) - (a.center ? a.mean_in[row] : 0.0f)) * a.rstd_in[row], dw);
            db += g;
        }
        a.part[(size_t)blockIdx.y * 2 * a.N + c] = dw;
        a.part[(size_t)blockIdx.y * 2 * a.N + a.N + c] = db;
    }
    dependency_trigger();
}

// How a row is laid out over threads: elements a load (VE), loads a thread (V), threads (G); V == 0: the long kernels
struct Layout { int VE, V, G; bool wide; };
Layout norm_layout(int N, int io, bool backward) {
    const int ve = io == RGLRU_BF16 ? 8 : 4;
    if (N % ve == 0) {   // 16-byte accesses: every row starts on a 16-byte boundary
        const int n = N / ve;
        if (n <= 8) return {ve, 1, 8, false};
        if (n <= 16) return {ve, 2, 8, false};
        if (n <= 32) return {ve, 2, 16, false};
        if (n <= 64) return {ve, 2, 32, false};
        if (n <= (backward ? 1024 : 2048)) return {ve, 2, ceil_div((size_t)n, 64) * 32, true};   // the backward's column sums fit 512 threads' registers
        return {ve, 0, 1024, true};
    }
    if (N <= 64) return {1, 8, 8, false};
    if (N <= 128) return {1, 8, 16, false};
    if (N <= 256) return {1, 8, 32, false};
    if (N <= 8192) return {1, 8, ceil_div((size_t)N, 256) * 32, true};
    return {1, 0, 1024, true};
}

constexpr int NORM_SMS = 148;   // the block count is part of the workspace's size, so it does not depend on the device
constexpr int LONG_COLUMN_SPLITS = 32;
// Blocks of the backward: a block's column sums are 2 N floats of extra traffic each way
int backward_blocks(const rglru_norm_shape_t *s, const Layout &l) {
    if (l.V == 0) return (int)(s->rows < LONG_COLUMN_SPLITS ? s->rows : LONG_COLUMN_SPLITS);
    const int threads = l.wide ? l.G : 256;
    const long long need = l.wide ? s->rows : (s->rows + 256 / l.G - 1) / (256 / l.G);
    const int per_sm = threads >= 1024 ? 1 : 1024 / threads;
    const long long most = (long long)NORM_SMS * per_sm;
    return (int)(need < most ? need : most);
}

template <typename IO, int VE> cudaError_t launch_norm(const Layout &l, bool backward, unsigned blocks, const NormArgs &a, cudaStream_t st) {
    const dim3 grid(blocks), block(l.wide ? l.G : 256);
    const size_t smem = backward && !l.wide ? (size_t)2 * a.N * sizeof(float) : 0;
#define RGLRU_NORM(V, WIDE, MAXT)                                                                       \
    return backward ? launch_dependent(norm_backward_kernel<IO, VE, V, WIDE, MAXT>, grid, block, smem, st, a) \
                    : launch_dependent(norm_kernel<IO, VE, V, WIDE, MAXT>, grid, block, 0, st, a)
    if constexpr (VE == 1) {
        if (l.G > 512) { RGLRU_NORM(8, true, 1024); }
        if (l.wide) { RGLRU_NORM(8, true, 512); }
        RGLRU_NORM(8, false, 256);
    } else {
        if (l.G > 512) return launch_dependent(norm_kernel<IO, VE, 2, true, 1024>, grid, block, 0, st, a);   // forward only
        if (l.wide) { RGLRU_NORM(2, true, 512); }
        if (l.V == 1) { RGLRU_NORM(1, false, 256); }
        RGLRU_NORM(2, false, 256);
    }
#undef RGLRU_NORM
}
template <typename IO> cudaError_t launch_norm(const Layout &l, bool backward, unsigned blocks, const NormArgs &a, cudaStream_t st) {
    if (l.V == 0)
        return backward ? launch_dependent(norm_long_backward_kernel<IO>, dim3(blocks), dim3(1024), 0, st, a)
                        : launch_dependent(norm_long_kernel<IO>, dim3(blocks), dim3(1024), 0, st, a);
    return l.VE == 1 ? launch_norm<IO, 1>(l, backward, blocks, a, st) : launch_norm<IO, 16 / sizeof(IO)>(l, backward, blocks, a, st);
}

int32_t check_norm(const rglru_norm_shape_t *s) {
    if (s == nullptr) return RGLRU_ERR_NULL;
    if (s->rows <= 0 || s->N <= 0 || s->N > (1 << 30) || !(s->eps >= 0.0f) || s->rows > INT64_MAX / 16 / s->N) return RGLRU_ERR_SHAPE;
    if (s->io != RGLRU_F32 && s->io != RGLRU_BF16) return RGLRU_ERR_UNSUPPORTED;
    return RGLRU_OK;
}
NormArgs norm_args(const rglru_norm_shape_t *s, const Layout &l) {
    NormArgs a{};
    a.rows = s->rows; a.N = s->N; a.G = l.G; a.center = s->center != 0; a.eps = s->eps; a.inv_n = 1.0f / (float)s->N;
    return a;
}

}  // namespace
}  // namespace rglru

using namespace rglru;

extern "C" {

int32_t rglru_layer_norm(const rglru_norm_shape_t *s, const void *x, const float *weight, const float *bias, void *y, float *mean, float *rstd,
                         void *cuda_stream) {
    const int32_t rc = check_norm(s);
    if (rc != RGLRU_OK) return rc;
    if (!x || !y) return RGLRU_ERR_NULL;
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(weight, 16) || !aligned(bias, 16) || !aligned(mean, 16) || !aligned(rstd, 16)) return RGLRU_ERR_ALIGN;
    const size_t bytes = (size_t)s->rows * s->N * io_bytes(s->io);
    if (overlap(x, bytes, y, bytes)) return RGLRU_ERR_ALIAS;
    const Layout l = norm_layout(s->N, s->io, false);
    NormArgs a = norm_args(s, l);
    a.x = x; a.weight = weight; a.bias = bias; a.out = y; a.mean = mean; a.rstd = rstd;
    const int threads = l.wide ? l.G : 256;
    const long long need = l.wide ? s->rows : (s->rows + 256 / l.G - 1) / (256 / l.G), most = (long long)num_sms() * (2048 / threads);
    const unsigned blocks = (unsigned)(need < most ? need : most);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return call_status(s->io == RGLRU_F32 ? launch_norm<float>(l, false, blocks, a, st) : launch_norm<__nv_bfloat16>(l, false, blocks, a, st));
}

size_t rglru_layer_norm_workspace_bytes(const rglru_norm_shape_t *s) {
    if (check_norm(s) != RGLRU_OK) return 0;
    return up256((size_t)backward_blocks(s, norm_layout(s->N, s->io, true)) * 2 * s->N * sizeof(float));
}

int32_t rglru_layer_norm_backward(const rglru_norm_shape_t *s, const void *dy, const void *x, const float *mean, const float *rstd, const float *weight,
                                  void *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    const int32_t rc = check_norm(s);
    if (rc != RGLRU_OK) return rc;
    const bool sums = dweight || dbias;
    if (!dy || !x || !rstd || !dx || (s->center && !mean) || (sums && !workspace)) return RGLRU_ERR_NULL;
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(mean, 16) || !aligned(rstd, 16) || !aligned(weight, 16) || !aligned(dx, 16) || !aligned(dweight, 16) ||
        !aligned(dbias, 16) || !aligned(workspace, 256))
        return RGLRU_ERR_ALIGN;
    if (sums && workspace_bytes < rglru_layer_norm_workspace_bytes(s)) return RGLRU_ERR_WORKSPACE;
    const size_t bytes = (size_t)s->rows * s->N * io_bytes(s->io);
    if (overlap(dx, bytes, x, bytes) || overlap(dx, bytes, dy, bytes)) return RGLRU_ERR_ALIAS;
    const Layout l = norm_layout(s->N, s->io, true);
    NormArgs a = norm_args(s, l);
    a.x = x; a.dy = dy; a.weight = weight; a.mean_in = mean; a.rstd_in = rstd; a.out = dx;
    a.part = sums ? (float *)workspace : nullptr;
    const int blocks = backward_blocks(s, l);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool f32 = s->io == RGLRU_F32;
    const unsigned grid = l.V == 0 ? (unsigned)(s->rows < num_sms() ? s->rows : num_sms()) : (unsigned)blocks;
    cudaError_t e = f32 ? launch_norm<float>(l, true, grid, a, st) : launch_norm<__nv_bfloat16>(l, true, grid, a, st);
    if (e == cudaSuccess && sums && l.V == 0)
        e = launch_dependent(f32 ? norm_long_columns_kernel<float> : norm_long_columns_kernel<__nv_bfloat16>, dim3((s->N + 255) / 256, blocks), dim3(256), 0, st, a);
    if (e == cudaSuccess && sums) {
        ReduceJobs jobs{};
        add_reduce_job(jobs, a.part, blocks, (size_t)2 * s->N, dweight, s->N, dbias, s->N, nullptr, 0);
        e = run_reduce_jobs(jobs, st);
    }
    return call_status(e);
}

}  // extern "C"
