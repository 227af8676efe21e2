// Normalisation of rows (layer norm, or the mean square alone) and its gradients: extern "C" entry points and CUDA kernels.
//
//   forward   mu = mean(x), r = 1/sqrt(mean((x - mu)^2) + eps), y = (x - mu) r w + b
//   backward  xh = (x - mu) r, g = dy w:  dx = r (g - mean(g) - xh mean(g xh)),  dw = sum dy xh,  db = sum dy
//
// Both are bound by memory: 4 bytes an element forward, 6 backward (bf16).  A row is read once and stays in registers between the
// statistics and the result, so that the deviations are taken from the mean itself (no difference of large sums).  A group of threads owns a
// row: up to a warp of them for narrow rows, several rows a warp; a whole block for wide ones.  The
// backward's groups walk rows with the next row's loads in flight, the weights and the columns' sums in registers.
#include <cuda_bf16.h>

#include "rglru_internal.h"
#include "rglru_io.cuh"
#include "sm100_ptx.cuh"

namespace rglru {
namespace {

using namespace ptx;

struct NormArgs {
    long long rows;
    int N, G;            // G: threads a row (narrow rows: 4, 8, 16 or 32; wide ones: the block)
    int center;
    float eps, inv_n;
    const void *x, *dy;
    const float *weight, *bias;
    const float *mean_in, *rstd_in;
    void *out;           // y or dx
    float *mean, *rstd;
    float *part;         // backward: [blocks][2][N] sums of dy xh and dy over a block's rows, or null
};

// VE neighbouring elements as they lie in memory: 2, 4, 8 or 16 bytes
template <int BYTES> struct Word { using type = uint4; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<2> { using type = uint16_t; };
template <typename IO, int VE> using Raw = typename Word<VE * (int)sizeof(IO)>::type;

template <typename IO, int VE> __device__ __forceinline__ Raw<IO, VE> load_raw(const IO *p) { return *(const Raw<IO, VE> *)p; }
template <typename IO, int VE> __device__ __forceinline__ void unpack(const Raw<IO, VE> &r, float (&f)[VE]) {
    if constexpr (sizeof(r) == 2) {
        f[0] = __uint_as_float((uint32_t)r << 16);
    } else {
        constexpr int W = sizeof(r) / 4;
        uint32_t w[W];
        if constexpr (W == 1) w[0] = r;
        else if constexpr (W == 2) { w[0] = r.x; w[1] = r.y; }
        else { w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w; }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(IO) == 4) f[i] = __uint_as_float(w[i]);
            else { const f32x2 v = bf2x(w[i]); f[2 * i] = v.x; f[2 * i + 1] = v.y; }
        }
    }
}
template <typename IO, int VE> __device__ __forceinline__ void store_vec(IO *p, const float (&f)[VE]) {
    if constexpr (VE * sizeof(IO) == 2) {
        *p = __float2bfloat16_rn(f[0]);
    } else {
        constexpr int W = VE * sizeof(IO) / 4;
        uint32_t w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(IO) == 4) w[i] = __float_as_uint(f[i]);
            else w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
        }
        if constexpr (W == 1) *(uint32_t *)p = w[0];
        else if constexpr (W == 2) *(uint2 *)p = make_uint2(w[0], w[1]);
        else
#pragma unroll
            for (int i = 0; i < W; i += 4) *((uint4 *)p + i / 4) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
}
template <int VE> __device__ __forceinline__ void load_f32(const float *p, float (&f)[VE]) {
#pragma unroll
    for (int e = 0; e < VE; e += (VE % 4 == 0 ? 4 : VE)) {
        if constexpr (VE % 4 == 0) { const float4 v = *(const float4 *)(p + e); f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w; }
        else if constexpr (VE == 2) { const float2 v = *(const float2 *)p; f[0] = v.x; f[1] = v.y; }
        else f[e] = p[e];
    }
}

// Sums of K values over the group of threads that owns a row; every thread of the group gets them.  Wide groups leave their warps' sums in
// shared memory, in two buffers used in turn, so that one barrier a call is enough, and every thread adds those up.
template <bool WIDE, int K> struct GroupSum {
    float (*buf)[K][16];
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
            float (&b)[K][16] = buf[turn];
            turn ^= 1;
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) b[k][warp] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < 16; w += 4)
                    if (w < warps) {   // the places behind the last warp hold zeros
                        const float4 f = *(const float4 *)&b[k][w];
                        v[k] += (f.x + f.y) + (f.z + f.w);
                    }
            }
        }
    }
};

// A thread's share of a row as pairs: element e of vector v is half e & 1 of pair (v VE + e) / 2.  Vectors behind the row's end hold zeros and
// `in` is false for them; single values (VE == 1) share pairs two by two.  All arithmetic is on pairs: with one operation a value
// the kernels were bound by issuing instructions (22 a value forward, 37 backward, 60 to 75 % of all slots), not by memory.
template <int VE, int V> struct Share {
    static constexpr int PAIRS = VE * V / 2;
    bool in[V];
    __device__ __forceinline__ bool pair_in(int i) const { return VE == 1 ? in[2 * i] : in[2 * i / VE]; }
    // a pair with zeros in the place of what is behind the row's end (only single values can be half in)
    __device__ __forceinline__ f32x2 masked(int i, f32x2 x) const {
        if constexpr (VE == 1) return make_float2(in[2 * i] ? x.x : 0.0f, in[2 * i + 1] ? x.y : 0.0f);
        else return x;
    }
};
template <typename IO, int VE, int V> __device__ __forceinline__ void unpack_row(const Raw<IO, VE> (&raw)[V], f32x2 (&f)[VE * V / 2]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float t[VE];
        unpack<IO, VE>(raw[v], t);
#pragma unroll
        for (int e = 0; e < VE; ++e) (v * VE + e & 1 ? f[(v * VE + e) / 2].y : f[(v * VE + e) / 2].x) = t[e];
    }
}
template <int VE, int V> __device__ __forceinline__ void load_vectors(const float *p, const bool (&in)[V], int G, float otherwise, f32x2 (&f)[VE * V / 2]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float t[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) t[e] = otherwise;
        if (p && in[v]) load_f32<VE>(p + v * G * VE, t);
#pragma unroll
        for (int e = 0; e < VE; ++e) (v * VE + e & 1 ? f[(v * VE + e) / 2].y : f[(v * VE + e) / 2].x) = t[e];
    }
}
template <typename T, int VE, int V> __device__ __forceinline__ void store_vectors(T *p, const bool (&in)[V], int G, const f32x2 (&f)[VE * V / 2]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!in[v]) continue;
        float t[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) t[e] = v * VE + e & 1 ? f[(v * VE + e) / 2].y : f[(v * VE + e) / 2].x;
        store_vec<T, VE>(p + v * G * VE, t);
    }
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { return fma2(a, pack2(1.0f, 1.0f), b); }
__device__ __forceinline__ f32x2 both(float x) { return pack2(x, x); }

// Rows of at most G V VE elements.  Thread t of a group holds the vectors t, t + G, ... of its row, the weights of its columns, and its next
// row's vectors on their way.  327680 x 128 bf16: 30 us for 168 MB, 86 % of the copy rate; 16384 x 4096: 47 us for 268 MB.
template <typename IO, int VE, int V, bool WIDE, int MAXT> __global__ void __launch_bounds__(MAXT) norm_kernel(NormArgs a) {
    __shared__ __align__(16) float red[2][1][16];
    constexpr int PAIRS = VE * V / 2;
    if (WIDE && threadIdx.x < 32) red[threadIdx.x >> 4][0][threadIdx.x & 15] = 0.0f;
    dependency_wait();
    if (WIDE) __syncthreads();
    const int G = a.G, t = WIDE ? threadIdx.x : threadIdx.x & (G - 1);
    const long long groups = WIDE ? gridDim.x : (long long)gridDim.x * blockDim.x / G;
    GroupSum<WIDE, 1> sum{red};
    long long row = WIDE ? blockIdx.x : ((long long)blockIdx.x * blockDim.x + threadIdx.x) / G;
    Share<VE, V> mine;
#pragma unroll
    for (int v = 0; v < V; ++v) mine.in[v] = (t + v * G) * VE < a.N;
    f32x2 w[PAIRS], b[PAIRS];
    load_vectors<VE, V>(a.weight ? a.weight + t * VE : nullptr, mine.in, G, 1.0f, w);
    load_vectors<VE, V>(a.bias ? a.bias + t * VE : nullptr, mine.in, G, 0.0f, b);
    Raw<IO, VE> next[V] = {};
    auto fetch = [&](long long from) {
        const IO *px = (const IO *)a.x + from * a.N + t * VE;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (mine.in[v]) next[v] = load_raw<IO, VE>(px + v * G * VE);
    };
    if (row < a.rows) fetch(row);
    // all lanes of a warp stay in the loop while one of its groups has a row, for the shuffles; a wide group's block leaves as one
    for (; WIDE ? row < a.rows : __any_sync(0xffffffffu, row < a.rows); row += groups) {
        f32x2 f[PAIRS];
        unpack_row<IO, VE, V>(next, f);
        if (row + groups < a.rows) fetch(row + groups);
        float s[1] = {0.0f};
        f32x2 s2 = both(0.0f);
        if (a.center) {
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) s2 = add2(f[i], s2);
            s[0] = s2.x + s2.y;
            sum(s, G);
        }
        const float mu = s[0] * a.inv_n;
        s2 = both(0.0f);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            f[i] = add2(f[i], both(-mu));
            if (mine.pair_in(i)) { const f32x2 d = mine.masked(i, f[i]); s2 = fma2(d, d, s2); }
        }
        s[0] = s2.x + s2.y;
        sum(s, G);
        const float r = 1.0f / sqrtf(s[0] * a.inv_n + a.eps);
        if (row < a.rows) {
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) f[i] = fma2(mul2(f[i], both(r)), w[i], b[i]);
            store_vectors<IO, VE, V>((IO *)a.out + row * a.N + t * VE, mine.in, G, f);
            if (t == 0) {
                if (a.mean) a.mean[row] = mu;
                if (a.rstd) a.rstd[row] = r;
            }
        }
    }
    dependency_trigger();
}

// 16-byte copies into a part of shared memory that is the thread's own
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ uint4 own16(uint32_t src) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
    return v;
}
constexpr int AHEAD = 3;   // rows that a wide row's threads have on their way in shared memory (one in registers: 16384 x 4096 bf16 83 us instead of 72)

// The gradients, rows as above.  The column sums of a group's rows stay in registers and leave once, added over the block's groups.  16384 x 4096
// bf16: 76 us for 403 MB, 79 % of the copy rate; dx alone 71.
template <typename IO, int VE, int V, bool WIDE, int MAXT> __global__ void __launch_bounds__(MAXT) norm_backward_kernel(NormArgs a) {
    __shared__ __align__(16) float red[2][2][16];
    extern __shared__ __align__(16) float cols[];   // narrow rows: [2][N] sums of the block
    constexpr int PAIRS = VE * V / 2;
    if (WIDE && threadIdx.x < 32) { red[threadIdx.x >> 4][0][threadIdx.x & 15] = 0.0f; red[threadIdx.x >> 4][1][threadIdx.x & 15] = 0.0f; }
    dependency_wait();
    if (WIDE) __syncthreads();
    const int G = a.G, t = WIDE ? threadIdx.x : threadIdx.x & (G - 1);
    const long long group = WIDE ? blockIdx.x : ((long long)blockIdx.x * blockDim.x + threadIdx.x) / G;
    const long long groups = WIDE ? gridDim.x : (long long)gridDim.x * blockDim.x / G;
    GroupSum<WIDE, 2> sum{red};
    Share<VE, V> mine;
#pragma unroll
    for (int v = 0; v < V; ++v) mine.in[v] = (t + v * G) * VE < a.N;
    f32x2 w[PAIRS], dw[PAIRS], db[PAIRS];
    load_vectors<VE, V>(a.weight ? a.weight + t * VE : nullptr, mine.in, G, 1.0f, w);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) dw[i] = db[i] = both(0.0f);
    constexpr bool RING = WIDE && VE * sizeof(IO) == 16;
    Raw<IO, VE> nx[V] = {}, ny[V] = {};
    float nmu = 0.0f, nr = 0.0f;
    const uint32_t own = smem_u32(cols) + threadIdx.x * 16, row_bytes = blockDim.x * 16;
    auto fetch = [&](int slot, long long row) {
        const IO *px = (const IO *)a.x + row * a.N + t * VE, *py = (const IO *)a.dy + row * a.N + t * VE;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!mine.in[v] || row >= a.rows) continue;
            if constexpr (RING) {
                copy16(own + (slot * 2 * V + v) * row_bytes, px + v * G * VE);
                copy16(own + (slot * 2 * V + V + v) * row_bytes, py + v * G * VE);
            } else {
                nx[v] = load_raw<IO, VE>(px + v * G * VE);
                ny[v] = load_raw<IO, VE>(py + v * G * VE);
            }
        }
        if (RING) copies_begun();
    };
    auto fetch_statistics = [&](long long row) {
        if (row >= a.rows) return;
        nmu = a.center ? a.mean_in[row] : 0.0f;
        nr = a.rstd_in[row];
    };
#pragma unroll
    for (int k = 0; k < (RING ? AHEAD : 1); ++k) fetch(k, group + k * groups);
    fetch_statistics(group);
    int slot = 0;
    for (long long row = group; WIDE ? row < a.rows : __any_sync(0xffffffffu, row < a.rows); row += groups) {
        const bool live = row < a.rows;
        f32x2 h[PAIRS], g[PAIRS];
        const float mu = nmu, r = nr;
        if constexpr (RING) {
            copies_wait<AHEAD - 1>();
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (mine.in[v]) { nx[v] = own16(own + (slot * 2 * V + v) * row_bytes); ny[v] = own16(own + (slot * 2 * V + V + v) * row_bytes); }
        }
        unpack_row<IO, VE, V>(nx, h);
        unpack_row<IO, VE, V>(ny, g);   // zeros behind the row's end
        fetch(slot, row + (RING ? AHEAD : 1) * groups);
        slot = slot + 1 == AHEAD ? 0 : slot + 1;
        fetch_statistics(row + groups);
        f32x2 s0 = both(0.0f), s1 = both(0.0f);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            h[i] = mul2(add2(h[i], both(-mu)), both(r));
            if (live) {
                dw[i] = fma2(g[i], h[i], dw[i]);
                db[i] = add2(g[i], db[i]);
            }
            g[i] = mul2(g[i], w[i]);
            if (mine.pair_in(i)) s0 = fma2(g[i], mine.masked(i, h[i]), s0);   // behind the row's end h is -mu r, which may be infinite
            s1 = add2(g[i], s1);
        }
        float s[2] = {s0.x + s0.y, s1.x + s1.y};
        sum(s, G);
        const float c2 = s[0] * a.inv_n, c1 = a.center ? s[1] * a.inv_n : 0.0f;
        if (live) {
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) g[i] = mul2(add2(fma2(h[i], both(-c2), g[i]), both(-c1)), both(r));
            store_vectors<IO, VE, V>((IO *)a.out + row * a.N + t * VE, mine.in, G, g);
        }
    }
    dependency_trigger();
    if (a.part == nullptr) return;
    float *part = a.part + (size_t)blockIdx.x * 2 * a.N;
    if constexpr (WIDE) {
        store_vectors<float, VE, V>(part + t * VE, mine.in, G, dw);
        store_vectors<float, VE, V>(part + a.N + t * VE, mine.in, G, db);
    } else {
        // the groups of a warp by shuffles, the warps of a block one after the other, in a fixed order
#pragma unroll
        for (int i = 0; i < PAIRS; ++i)
            for (int o = G; o < 32; o <<= 1) {
                dw[i].x += __shfl_xor_sync(0xffffffffu, dw[i].x, o); dw[i].y += __shfl_xor_sync(0xffffffffu, dw[i].y, o);
                db[i].x += __shfl_xor_sync(0xffffffffu, db[i].x, o); db[i].y += __shfl_xor_sync(0xffffffffu, db[i].y, o);
            }
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        for (int k = 0; k < warps; ++k) {
            if (warp == k && lane < G) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (mine.in[v])
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            const int c = (t + v * G) * VE + e, i = v * VE + e;
                            const float x = i & 1 ? dw[i / 2].y : dw[i / 2].x, y = i & 1 ? db[i / 2].y : db[i / 2].x;
                            const float p0 = k ? cols[c] : 0.0f, p1 = k ? cols[a.N + c] : 0.0f;
                            if (k < warps - 1) { cols[c] = p0 + x; cols[a.N + c] = p1 + y; }
                            else { part[c] = p0 + x; part[a.N + c] = p1 + y; }
                        }
            }
            __syncthreads();
        }
    }
}

// dweight | dbias = the sums of the blocks' columns: a block of 32 warps for 32 columns, every warp a 32nd of the parts, added up in a fixed order
__global__ void __launch_bounds__(1024) norm_columns_kernel(const float *part, int parts, int N, float *dweight, float *dbias) {
    __shared__ __align__(16) float red[32][33];
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane, stride = 2ll * N;
    float s = 0.0f;
    if (c < stride) {
#pragma unroll 8
        for (int p = warp; p < parts; p += 32) s += part[p * stride + c];
    }
    red[warp][lane] = s;
    __syncthreads();
    s = red[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const long long col = (long long)blockIdx.x * 32 + warp;
    if (lane == 0 && col < stride) {
        float *const out = col < N ? dweight : dbias;
        if (out) out[col < N ? col : col - N] = s;
    }
    dependency_trigger();
}

// Rows that no block holds in registers (4096 x 16384 bf16 backward 520 us): a block reads its row three times (the second and third time mostly out of L2).
template <typename IO> __global__ void __launch_bounds__(512) norm_long_kernel(NormArgs a) {
    __shared__ __align__(16) float red[2][1][16];
    dependency_wait();
    GroupSum<true, 1> sum{red};
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const long long base = row * a.N;
        float s[1] = {0.0f};
        if (a.center) {
            for (int c = threadIdx.x; c < a.N; c += 512) s[0] += at<IO>(a.x, base + c);
            sum(s, 512);
        }
        const float mu = s[0] * a.inv_n;
        s[0] = 0.0f;
        for (int c = threadIdx.x; c < a.N; c += 512) { const float d = at<IO>(a.x, base + c) - mu; s[0] = fmaf(d, d, s[0]); }
        sum(s, 512);
        const float r = 1.0f / sqrtf(s[0] * a.inv_n + a.eps);
        for (int c = threadIdx.x; c < a.N; c += 512)
            put<IO>(a.out, base + c, fmaf((at<IO>(a.x, base + c) - mu) * r, a.weight ? a.weight[c] : 1.0f, a.bias ? a.bias[c] : 0.0f));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mu;
            if (a.rstd) a.rstd[row] = r;
        }
    }
    dependency_trigger();
}
template <typename IO> __global__ void __launch_bounds__(512) norm_long_backward_kernel(NormArgs a) {
    __shared__ __align__(16) float red[2][2][16];
    dependency_wait();
    GroupSum<true, 2> sum{red};
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const long long base = row * a.N;
        const float mu = a.center ? a.mean_in[row] : 0.0f, r = a.rstd_in[row];
        float s[2] = {0.0f, 0.0f};
        for (int c = threadIdx.x; c < a.N; c += 512) {
            const float g = at<IO>(a.dy, base + c) * (a.weight ? a.weight[c] : 1.0f);
            s[0] = fmaf(g, (at<IO>(a.x, base + c) - mu) * r, s[0]);
            s[1] += g;
        }
        sum(s, 512);
        const float c2 = s[0] * a.inv_n, c1 = a.center ? s[1] * a.inv_n : 0.0f;
        for (int c = threadIdx.x; c < a.N; c += 512) {
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
    int ve = io == RGLRU_BF16 ? 8 : 4;
    const int most = ve;
    while (N % ve) ve /= 2;   // every row starts at a multiple of the access
    const int n = N / ve;
    const int v = ve == most ? (n > 128 && !backward ? 4 : 2) : ve == 1 || ve * 4 == most ? 8 : 4;
    for (int g = 4; g <= 32; g *= 2)
        if (n <= g * v) return {ve, v, g, false};
    if (n <= v * 512) return {ve, v, ceil_div((size_t)n, 32 * v) * 32, true};
    return {ve, 0, 512, true};
}

constexpr int NORM_SMS = 148;   // the block count is part of the workspace's size, so it does not depend on the device
constexpr int LONG_COLUMN_SPLITS = 32;
// Blocks of the backward: a block's column sums are 2 N floats of extra traffic each way
int backward_blocks(const rglru_norm_shape_t *s, const Layout &l) {
    if (l.V == 0) return (int)(s->rows < LONG_COLUMN_SPLITS ? s->rows : LONG_COLUMN_SPLITS);
    const int threads = l.wide ? l.G : 256, most_threads = s->io == RGLRU_F32 ? 1024 : 512, resident = threads > most_threads / 2 ? 1 : most_threads / threads;
    const long long need = l.wide ? s->rows : (s->rows + 256 / l.G - 1) / (256 / l.G);
    const long long most = (long long)NORM_SMS * resident;
    return (int)(need < most ? need : most);
}

// Blocks walk rows, so there are as many as are resident at a time: more would run in a second round beside idle SMs
template <typename K> cudaError_t launch_resident(K kernel, long long need, int threads, const NormArgs &a, cudaStream_t st) {
    const int sms = num_sms();
    int per_sm = 1;
    if (need > sms) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, 0);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) per_sm = 1;
    }
    const long long most = (long long)sms * per_sm;
    return launch_dependent(kernel, dim3((unsigned)(need < most ? need : most)), dim3(threads), 0, st, a);
}
template <typename IO, int VE, int V> cudaError_t launch_forward(const Layout &l, const NormArgs &a, cudaStream_t st) {
    return l.wide ? launch_resident(norm_kernel<IO, VE, V, true, 512>, a.rows, l.G, a, st)
                  : launch_resident(norm_kernel<IO, VE, V, false, 256>, (a.rows + 256 / l.G - 1) / (256 / l.G), 256, a, st);
}
template <typename IO, int VE, int V> cudaError_t launch_backward(const Layout &l, unsigned blocks, const NormArgs &a, cudaStream_t st) {
    if (!l.wide) return launch_dependent(norm_backward_kernel<IO, VE, V, false, 256>, dim3(blocks), dim3(256), (size_t)2 * a.N * sizeof(float), st, a);
    size_t smem = 0;
    if constexpr (VE * sizeof(IO) == 16) {
        static PerDeviceOptIn opt;
        const cudaError_t e = opt.ensure(norm_backward_kernel<IO, VE, V, true, 512>, AHEAD * 2 * V * 16 * 512);
        if (e != cudaSuccess) return e;
        smem = (size_t)AHEAD * 2 * V * 16 * l.G;
    }
    return launch_dependent(norm_backward_kernel<IO, VE, V, true, 512>, dim3(blocks), dim3(l.G), smem, st, a);
}
template <typename IO> cudaError_t launch_norm(const Layout &l, bool backward, unsigned blocks, const NormArgs &a, cudaStream_t st) {
    constexpr int MOST = 16 / sizeof(IO);
    if (l.V == 0)
        return backward ? launch_dependent(norm_long_backward_kernel<IO>, dim3(blocks), dim3(512), 0, st, a)
                        : launch_resident(norm_long_kernel<IO>, a.rows, 512, a, st);
#define RGLRU_NORM(VE, V) return backward ? launch_backward<IO, VE, V>(l, blocks, a, st) : launch_forward<IO, VE, V>(l, a, st)
    if (l.VE == MOST) {
        if (l.V == 4) return launch_forward<IO, MOST, 4>(l, a, st);
        RGLRU_NORM(MOST, 2);
    }
    if constexpr (MOST == 8) {
        if (l.VE == 4) { RGLRU_NORM(4, 4); }
        if (l.VE == 2) { RGLRU_NORM(2, 8); }
    } else {
        if (l.VE == 2) { RGLRU_NORM(2, 4); }
    }
    RGLRU_NORM(1, 8);
#undef RGLRU_NORM
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
    const size_t vec = (size_t)s->N * sizeof(float), stat = (size_t)s->rows * sizeof(float);
    if (overlap(x, bytes, y, bytes) || overlap(y, bytes, weight, vec) || overlap(y, bytes, bias, vec) || overlap(y, bytes, mean, stat) || overlap(y, bytes, rstd, stat) ||
        overlap(mean, stat, rstd, stat))
        return RGLRU_ERR_ALIAS;
    for (const float *out : {mean, rstd})
        if (overlap(out, stat, x, bytes) || overlap(out, stat, weight, vec) || overlap(out, stat, bias, vec)) return RGLRU_ERR_ALIAS;
    const Layout l = norm_layout(s->N, s->io, false);
    NormArgs a = norm_args(s, l);
    a.x = x; a.weight = weight; a.bias = bias; a.out = y; a.mean = mean; a.rstd = rstd;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return call_status(s->io == RGLRU_F32 ? launch_norm<float>(l, false, 0, a, st) : launch_norm<__nv_bfloat16>(l, false, 0, a, st));
}

size_t rglru_layer_norm_workspace_bytes(const rglru_norm_shape_t *s) {
    if (check_norm(s) != RGLRU_OK) return 0;
    return WS_HEADER_BYTES + up256((size_t)backward_blocks(s, norm_layout(s->N, s->io, true)) * 2 * s->N * sizeof(float));
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
    const size_t vec = (size_t)s->N * sizeof(float), stat = (size_t)s->rows * sizeof(float);
    if (overlap(dx, bytes, x, bytes) || overlap(dx, bytes, dy, bytes) || (s->center && overlap(dx, bytes, mean, stat)) || overlap(dx, bytes, rstd, stat) ||
        overlap(dx, bytes, weight, vec) || overlap(dx, bytes, dweight, vec) || overlap(dx, bytes, dbias, vec) || overlap(dweight, vec, dbias, vec))
        return RGLRU_ERR_ALIAS;
    const Layout l = norm_layout(s->N, s->io, true);
    NormArgs a = norm_args(s, l);
    a.x = x; a.dy = dy; a.weight = weight; a.mean_in = mean; a.rstd_in = rstd; a.out = dx;
    a.part = sums ? (float *)((char *)workspace + WS_HEADER_BYTES) : nullptr;
    const int blocks = backward_blocks(s, l);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool f32 = s->io == RGLRU_F32;
    const unsigned grid = l.V == 0 ? (unsigned)(s->rows < num_sms() ? s->rows : num_sms()) : (unsigned)blocks;
    cudaError_t e = f32 ? launch_norm<float>(l, true, grid, a, st) : launch_norm<__nv_bfloat16>(l, true, grid, a, st);
    if (e == cudaSuccess && sums && l.V == 0)
        e = launch_dependent(f32 ? norm_long_columns_kernel<float> : norm_long_columns_kernel<__nv_bfloat16>, dim3((s->N + 255) / 256, blocks), dim3(256), 0, st, a);
    if (e == cudaSuccess && sums)
        e = launch_dependent(norm_columns_kernel, dim3((unsigned)((2ll * s->N + 31) / 32)), dim3(1024), 0, st, (const float *)a.part, blocks, (int)s->N, dweight, dbias);
    return call_status(e);
}

}  // extern "C"
