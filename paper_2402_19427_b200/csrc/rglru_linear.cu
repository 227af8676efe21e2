// Projection with bias, activation and residual in its epilogue, and its gradients: extern "C" entry points, the kernels for any
// shape and type on the CUDA cores, and the element-wise part of the backward.
//
//   forward   z = x W^T + b,  y = act(z) + residual
//   backward  dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum_rows dz
#include <cuda_bf16.h>

#include "rglru_linear.cuh"

namespace rglru {
namespace {

using namespace ptx;

// C[m][n] = sum_k A(m,k) B(n,k) in fp32 on the CUDA cores, 128 x 128 results a block, 8 x 8 a thread, K in steps of 16 through shared
// memory.  A(m,k) = a[m a_m + k a_k], B(n,k) = b[n b_n + k b_k]: the forward has K innermost in both, dx in A alone, dW in neither.
constexpr int GT = 128, GK = 16;
struct GenericGemm {
    const void *a, *b;
    long long a_m, a_k, b_n, b_k, M, N, K;
    LinearEpilogue e;
};
template <typename IO> __global__ void __launch_bounds__(256) generic_linear_kernel(GenericGemm g) {
    __shared__ __align__(16) float sa[GK][GT + 4], sb[GK][GT + 4];
    dependency_wait();
    const long long tiles_n = (g.N + GT - 1) / GT, m0 = blockIdx.x / tiles_n * GT, n0 = blockIdx.x % tiles_n * GT;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[8][8] = {};
    for (long long k0 = 0; k0 < g.K; k0 += GK) {
        // neighbouring threads read along whichever dimension is innermost in memory
#pragma unroll
        for (int i = 0; i < GT * GK / 256; ++i) {
            const int at_ = threadIdx.x + i * 256;
            const int ka = g.a_k == 1 ? at_ % GK : at_ / GT, ma = g.a_k == 1 ? at_ / GK : at_ % GT;
            sa[ka][ma] = m0 + ma < g.M && k0 + ka < g.K ? at<IO>(g.a, (m0 + ma) * g.a_m + (k0 + ka) * g.a_k) : 0.0f;
            const int kb = g.b_k == 1 ? at_ % GK : at_ / GT, nb = g.b_k == 1 ? at_ / GK : at_ % GT;
            sb[kb][nb] = n0 + nb < g.N && k0 + kb < g.K ? at<IO>(g.b, (n0 + nb) * g.b_n + (k0 + kb) * g.b_k) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < GK; ++k) {
            float a[8], b[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 va = *(const float4 *)&sa[k][h * 64 + ty * 4], vb = *(const float4 *)&sb[k][h * 64 + tx * 4];
                a[4 * h] = va.x; a[4 * h + 1] = va.y; a[4 * h + 2] = va.z; a[4 * h + 3] = va.w;
                b[4 * h] = vb.x; b[4 * h + 1] = vb.y; b[4 * h + 2] = vb.z; b[4 * h + 3] = vb.w;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
        }
        __syncthreads();
    }
    const LinearEpilogue &e = g.e;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const long long m = m0 + (i >> 2) * 64 + ty * 4 + (i & 3);
        if (m >= g.M) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const long long n = n0 + (j >> 2) * 64 + tx * 4 + (j & 3);
            if (n >= g.N) continue;
            const long long o = m * g.N + n;
            const float z = acc[i][j] + (e.bias ? e.bias[n] : 0.0f);
            if (e.preact) put<IO>(e.preact, o, z);
            const float y = activate<sizeof(IO) == 2>(z, e.activation) + (e.residual ? at<IO>(e.residual, o) : 0.0f);
            put<IO>(e.y, o, y);
        }
    }
    dependency_trigger();
}

// The forward of few rows (tokens): bound by reading the weights once.  A block takes four outputs and its warps share K, so that even a few
// hundred outputs fill the SMs; a lane reads 16 bytes of each of the four weight rows and, out of the first-level cache, of each row of x.
// Tensor cores would need the weights in shared memory first, the tokens padded and K split over the SMs by a launch of its own.
constexpr int FEW_OUT = 4;
template <typename IO, int VE, int MT> __global__ void __launch_bounds__(256) few_rows_kernel(GenericGemm g) {
    __shared__ __align__(16) float red[8][FEW_OUT * MT];
    using Vec = LinearVec<IO, VE>;
    constexpr int PAIRS = VE > 1 ? VE / 2 : 1;
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long n0 = (long long)blockIdx.x * FEW_OUT;
    float2 acc[FEW_OUT][MT] = {};   // even and odd columns
    auto pairs = [](const float (&f)[VE], float2 (&p)[PAIRS]) {
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) p[e] = make_float2(f[VE > 1 ? 2 * e : 0], VE > 1 ? f[2 * e + 1] : 0.0f);
    };
#pragma unroll 2
    for (long long k = (long long)threadIdx.x * VE; k < g.K; k += 256 * VE) {
        float2 w[FEW_OUT][PAIRS];
#pragma unroll
        for (int i = 0; i < FEW_OUT; ++i) {
            float f[VE];
            Vec::load((const IO *)g.b + (n0 + i < g.N ? n0 + i : n0) * g.K + k, f);
            pairs(f, w[i]);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m >= g.M) break;
            float f[VE];
            float2 x[PAIRS];
            Vec::load((const IO *)g.a + m * g.K + k, f);
            pairs(f, x);
#pragma unroll
            for (int i = 0; i < FEW_OUT; ++i)
#pragma unroll
                for (int e = 0; e < PAIRS; ++e) acc[i][m] = fma_pair(w[i][e], x[e], acc[i][m]);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < FEW_OUT; ++i) {
            float z = acc[i][m].x + acc[i][m].y;
#pragma unroll
            for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            if (lane == 0) red[warp][m * FEW_OUT + i] = z;
        }
    __syncthreads();
    const int t = threadIdx.x;
    const long long m = t / FEW_OUT, n = n0 + t % FEW_OUT;
    if (t < FEW_OUT * MT && m < g.M && n < g.N) {
        const LinearEpilogue &e = g.e;
        const long long o = m * g.N + n;
        float z = red[0][t];
#pragma unroll
        for (int i = 1; i < 8; ++i) z += red[i][t];
        z += e.bias ? e.bias[n] : 0.0f;
        if (e.preact) put<IO>(e.preact, o, z);
        put<IO>(e.y, o, activate<sizeof(IO) == 2>(z, e.activation) + (e.residual ? at<IO>(e.residual, o) : 0.0f));
    }
    dependency_trigger();
}
constexpr int FEW_ROWS = 8;
template <typename IO, int VE> cudaError_t few_rows(const GenericGemm &g, cudaStream_t st) {
    const dim3 grid((unsigned)((g.N + FEW_OUT - 1) / FEW_OUT));
    return launch_dependent(g.M == 1 ? few_rows_kernel<IO, VE, 1> : g.M == 2 ? few_rows_kernel<IO, VE, 2> : g.M <= 4 ? few_rows_kernel<IO, VE, 4> : few_rows_kernel<IO, VE, 8>,
                            grid, dim3(256), 0, st, g);
}
template <typename IO> cudaError_t few_rows(const GenericGemm &g, cudaStream_t st) {
    constexpr int MOST = 16 / sizeof(IO);
    return g.K % MOST == 0 ? few_rows<IO, MOST>(g, st) : few_rows<IO, 1>(g, st);
}

// dz = dy act'(z) in the io type (the type of both products' operands; a second bf16 plane would double them), and the sums of the unrounded dz over a block's rows.  A thread owns VE columns and walks rows.  16384 x 2560 with
// GeLU: 47 us for 252 MB, bound by the slope's instructions (72 % of the issue slots); the sums alone 19 us for 84 MB.
struct DzArgs {
    long long M;
    int N, rows;              // rows a block
    int activation;
    const void *dy, *preact;
    void *dz;                 // null: only the sums (no activation: dz is dy)
    float *part;              // [row blocks][N] or null
};
template <typename IO, int VE> __global__ void __launch_bounds__(256, 2) linear_dz_kernel(DzArgs a) {
    __shared__ __align__(16) float red[8][32 * VE];
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = (blockIdx.x * 32 + lane) * VE;
    const long long r0 = (long long)blockIdx.y * a.rows, r1 = min(a.M, r0 + a.rows);
    float s[VE] = {};
    if (c < a.N) {
        // Rows in batches, the next one's loads in flight while this one is computed
        constexpr int BATCH = 4;
        using Vec = LinearVec<IO, VE>;
        typename Vec::Raw gs[BATCH], zs[BATCH];
        auto load = [&](long long r) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (r + 8 * u >= r1) continue;
                const long long o = (r + 8 * u) * a.N + c;
                gs[u] = *(const typename Vec::Raw *)((const IO *)a.dy + o);
                if (a.activation != RGLRU_ACT_NONE) zs[u] = *(const typename Vec::Raw *)((const IO *)a.preact + o);
            }
        };
        long long r = r0 + warp;
        load(r);
#pragma unroll 1
        while (r < r1) {
            typename Vec::Raw gn[BATCH], zn[BATCH];
            const long long now = r;
#pragma unroll
            for (int u = 0; u < BATCH; ++u) { gn[u] = gs[u]; zn[u] = zs[u]; }
            load(r += 8 * BATCH);
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (now + 8 * u >= r1) continue;
                float g[VE];
                Vec::unpack(gn[u], g);
                if (a.activation != RGLRU_ACT_NONE) {
                    float z[VE];
                    Vec::unpack(zn[u], z);
                    if constexpr (sizeof(IO) == 2 && VE > 1) {
#pragma unroll
                        for (int e = 0; e < VE; e += 2) {
                            const float2 d = mul2(make_float2(g[e], g[e + 1]), slope_fast(make_float2(z[e], z[e + 1]), a.activation));
                            g[e] = d.x;
                            g[e + 1] = d.y;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < VE; ++e) g[e] *= activation_slope<sizeof(IO) == 2>(z[e], a.activation);
                    }
                    if (a.dz) Vec::store((IO *)a.dz + (now + 8 * u) * a.N + c, g);
                }
                if constexpr (VE > 1) {
#pragma unroll
                    for (int e = 0; e < VE; e += 2) {
                        const float2 t = fma_pair(make_float2(g[e], g[e + 1]), both_of(1.0f), make_float2(s[e], s[e + 1]));
                        s[e] = t.x; s[e + 1] = t.y;
                    }
                } else {
                    s[0] += g[0];
                }
            }
        }
    }
    dependency_trigger();
    if (a.part == nullptr) return;
#pragma unroll
    for (int e = 0; e < VE; ++e) red[warp][lane * VE + e] = s[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * VE; i += 256) {
        const int col = blockIdx.x * 32 * VE + i;
        if (col >= a.N) break;
        float t = red[0][i];
#pragma unroll
        for (int w = 1; w < 8; ++w) t += red[w][i];
        a.part[(size_t)blockIdx.y * a.N + col] = t;
    }
}

// Rows a block of linear_dz_kernel takes: about eight blocks an SM over the whole call, at least 64 rows (eight a warp), at most as many blocks
// as a grid has along y
int dz_rows(const rglru_linear_shape_t *s) {
    const long long cols = (s->N + 255) / 256, want = s->M * cols / (148 * 8), most = s->M / 32768 + 8 > 4096 ? s->M / 32768 + 8 : 4096;
    return (int)(want < 64 ? 64 : want > most ? most / 8 * 8 : (want + 7) / 8 * 8);
}
int dz_blocks(const rglru_linear_shape_t *s) { return ceil_div((size_t)s->M, dz_rows(s)); }

cudaError_t linear_dz(const rglru_linear_shape_t *s, const DzArgs &args, cudaStream_t st) {
    DzArgs a = args;
    a.rows = dz_rows(s);
    const bool f32 = s->io == RGLRU_F32, vec = s->N % (f32 ? 4 : 8) == 0;
    const dim3 grid(ceil_div(s->N, 32 * (vec ? (f32 ? 4 : 8) : 1)), dz_blocks(s));
    if (f32) return vec ? launch_dependent(linear_dz_kernel<float, 4>, grid, dim3(256), 0, st, a) : launch_dependent(linear_dz_kernel<float, 1>, grid, dim3(256), 0, st, a);
    return vec ? launch_dependent(linear_dz_kernel<__nv_bfloat16, 8>, grid, dim3(256), 0, st, a)
               : launch_dependent(linear_dz_kernel<__nv_bfloat16, 1>, grid, dim3(256), 0, st, a);
}

cudaError_t generic_gemm(const GenericGemm &g, int io, cudaStream_t st) {
    const long long blocks = (g.M + GT - 1) / GT * ((g.N + GT - 1) / GT);
    if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    return launch_dependent(io == RGLRU_F32 ? generic_linear_kernel<float> : generic_linear_kernel<__nv_bfloat16>, dim3((unsigned)blocks), dim3(256), 0, st, g);
}

// The three products of a call; buffers may be null where only sizes matter
LinearProduct forward_product(const rglru_linear_shape_t *s, const void *x, const void *weight, const LinearEpilogue &e) {
    return {{x, s->M, s->K, false}, {weight, s->N, s->K, false}, s->M, s->N, s->K, s->io, e};
}
LinearProduct dx_product(const rglru_linear_shape_t *s, const void *dz, const void *weight, void *dx) {
    return {{dz, s->M, s->N, false}, {weight, s->N, s->K, true}, s->M, s->K, s->N, s->io, {nullptr, nullptr, dx, nullptr, RGLRU_ACT_NONE}};
}
LinearProduct dw_product(const rglru_linear_shape_t *s, const void *dz, const void *x, void *dweight) {
    return {{dz, s->M, s->N, true}, {x, s->M, s->K, true}, s->N, s->K, s->M, s->io, {nullptr, nullptr, dweight, nullptr, RGLRU_ACT_NONE}};
}
bool forced_generic(const rglru_linear_shape_t *s) { return s->flags & RGLRU_FLAG_FORCE_GENERIC; }
// dz in the tensor cores' form
size_t dz_packed_bytes(const rglru_linear_shape_t *s) { return forced_generic(s) ? 0 : sm100_linear_packed_bytes({nullptr, s->M, s->N, false}, s->io); }
size_t product_bytes(const rglru_linear_shape_t *s, const LinearProduct &g) { return forced_generic(s) ? 0 : sm100_linear_bytes(g); }
// Up to eight rows of fp32 (8 x 2560 x 2560: 16 us, on the tensor cores 31), of bf16 while the products are few beside the weights' bytes: one row always (2560 x
// 2560 5.0 and 8.3 us), more up to 2^25 products (4 x 2560 x 2560 9.9 and 10.2, 6 rows 17 and 10; 8 x 512 x 1024 4.8 and 6.6)
bool is_few_rows(const rglru_linear_shape_t *s) {
    if (forced_generic(s) || s->M > FEW_ROWS) return false;
    return s->io == RGLRU_F32 || s->M == 1 || (double)s->M * s->K * s->N <= 1 << 25;
}
cudaError_t run_product(const rglru_linear_shape_t *s, const LinearProduct &g, void *scratch, void *workspace, cudaStream_t st) {
    if (!forced_generic(s)) {
        LinearProduct p = g;
        p.flags = s->flags;
        return sm100_linear(p, scratch, (uint32_t *)workspace, st);
    }
    auto by_row = [](const LinearOperand &o) { return o.turned ? 1ll : o.cols; };
    auto by_k = [](const LinearOperand &o) { return o.turned ? o.cols : 1ll; };
    return generic_gemm(GenericGemm{g.a.p, g.b.p, by_row(g.a), by_k(g.a), by_row(g.b), by_k(g.b), g.M, g.N, g.K, g.e}, g.io, st);
}

constexpr int MAX_COLUMNS = INT32_MAX - 1023;   // a block's last column, behind the row's end, still is an int
int32_t check_linear(const rglru_linear_shape_t *s) {
    if (s == nullptr) return RGLRU_ERR_NULL;
    if (s->M <= 0 || s->M > INT32_MAX || s->K <= 0 || s->N <= 0 || s->K > MAX_COLUMNS || s->N > MAX_COLUMNS) return RGLRU_ERR_SHAPE;
    if (s->io != RGLRU_F32 && s->io != RGLRU_BF16) return RGLRU_ERR_UNSUPPORTED;
    if (s->activation < RGLRU_ACT_NONE || s->activation > RGLRU_ACT_SILU) return RGLRU_ERR_UNSUPPORTED;
    return RGLRU_OK;
}

}  // namespace
}  // namespace rglru

using namespace rglru;

extern "C" {

size_t rglru_linear_workspace_bytes(const rglru_linear_shape_t *s, int32_t op) {
    if (check_linear(s) != RGLRU_OK || (op != RGLRU_OP_PREFILL && op != RGLRU_OP_BACKWARD)) return 0;
    if (op == RGLRU_OP_PREFILL && is_few_rows(s)) return WS_HEADER_BYTES;
    if (op == RGLRU_OP_PREFILL) return WS_HEADER_BYTES + product_bytes(s, forward_product(s, nullptr, nullptr, {}));
    size_t bytes = WS_HEADER_BYTES + up256((size_t)dz_blocks(s) * s->N * sizeof(float));
    if (s->activation != RGLRU_ACT_NONE) bytes += up256((size_t)s->M * s->N * io_bytes(s->io));
    LinearProduct gx = dx_product(s, nullptr, nullptr, nullptr), gw = dw_product(s, nullptr, nullptr, nullptr);
    gx.a.packed = gw.a.packed = &gx;   // in a place of its own, if anywhere
    const size_t dx = product_bytes(s, gx), dw = product_bytes(s, gw);
    return bytes + dz_packed_bytes(s) + (dx > dw ? dx : dw);   // one after the other; both read dz
}

int32_t rglru_linear(const rglru_linear_shape_t *s, const void *x, const void *weight, const float *bias, const void *residual, void *y, void *preact,
                     void *workspace, size_t workspace_bytes, void *cuda_stream) {
    const int32_t rc = check_linear(s);
    if (rc != RGLRU_OK) return rc;
    if (!x || !weight || !y || !workspace) return RGLRU_ERR_NULL;
    if (!aligned(x, 16) || !aligned(weight, 16) || !aligned(bias, 16) || !aligned(residual, 16) || !aligned(y, 16) || !aligned(preact, 16) ||
        !aligned(workspace, 256))
        return RGLRU_ERR_ALIGN;
    if (workspace_bytes < rglru_linear_workspace_bytes(s, RGLRU_OP_PREFILL)) return RGLRU_ERR_WORKSPACE;
    const size_t io = io_bytes(s->io), xb = (size_t)s->M * s->K * io, wb = (size_t)s->N * s->K * io, yb = (size_t)s->M * s->N * io, bb = (size_t)s->N * sizeof(float);
    if (overlap(y, yb, bias, bb) || overlap(preact, yb, bias, bb) || overlap(y, yb, x, xb) || overlap(y, yb, weight, wb) || (residual != y && overlap(y, yb, residual, yb)) || overlap(preact, yb, x, xb) ||
        overlap(preact, yb, weight, wb) || overlap(preact, yb, residual, yb) || overlap(preact, yb, y, yb))
        return RGLRU_ERR_ALIAS;
    const LinearProduct g = forward_product(s, x, weight, {bias, residual, y, preact, s->activation});
    if (is_few_rows(s)) {
        const GenericGemm f{x, weight, s->K, 1, s->K, 1, s->M, s->N, s->K, g.e};
        return call_status(s->io == RGLRU_F32 ? few_rows<float>(f, (cudaStream_t)cuda_stream) : few_rows<__nv_bfloat16>(f, (cudaStream_t)cuda_stream));
    }
    return call_status(run_product(s, g, (char *)workspace + WS_HEADER_BYTES, workspace, (cudaStream_t)cuda_stream));
}

int32_t rglru_linear_backward(const rglru_linear_shape_t *s, const void *dy, const void *x, const void *weight, const void *preact, void *dx, void *dweight,
                              float *dbias, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    const int32_t rc = check_linear(s);
    if (rc != RGLRU_OK) return rc;
    const bool act = s->activation != RGLRU_ACT_NONE;
    if (!dy || !workspace || (act && !preact) || (dx && !weight) || (dweight && !x)) return RGLRU_ERR_NULL;
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(weight, 16) || !aligned(preact, 16) || !aligned(dx, 16) || !aligned(dweight, 16) ||
        !aligned(dbias, 16) || !aligned(workspace, 256))
        return RGLRU_ERR_ALIGN;
    if (workspace_bytes < rglru_linear_workspace_bytes(s, RGLRU_OP_BACKWARD)) return RGLRU_ERR_WORKSPACE;
    const size_t io = io_bytes(s->io), xb = (size_t)s->M * s->K * io, wb = (size_t)s->N * s->K * io, yb = (size_t)s->M * s->N * io, bb = (size_t)s->N * 4;
    const void *const ins[4] = {dy, x, weight, act ? preact : nullptr};
    const size_t in_bytes[4] = {yb, xb, wb, yb};
    void *const outs[3] = {dx, dweight, dbias};
    const size_t out_bytes[3] = {xb, wb, bb};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j)
            if (overlap(outs[i], out_bytes[i], ins[j], in_bytes[j])) return RGLRU_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], out_bytes[i], outs[j], out_bytes[j])) return RGLRU_ERR_ALIAS;
    }
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    char *p = (char *)workspace + WS_HEADER_BYTES;
    float *part = (float *)p;
    p += up256((size_t)dz_blocks(s) * s->N * sizeof(float));
    const void *dz = act ? p : dy;
    char *scratch = p + (act ? up256((size_t)s->M * s->N * io_bytes(s->io)) : 0);
    cudaError_t e = cudaSuccess;
    if ((act && (dx || dweight)) || dbias) e = linear_dz(s, DzArgs{s->M, s->N, 0, s->activation, dy, preact, act && (dx || dweight) ? p : nullptr, dbias ? part : nullptr}, st);
    if (e == cudaSuccess && dbias) {
        ReduceJobs jobs{};
        add_reduce_job(jobs, part, dz_blocks(s), s->N, dbias, s->N, nullptr, 0, nullptr, 0);
        e = run_reduce_jobs(jobs, st);
    }
    LinearProduct gx = dx_product(s, dz, weight, dx), gw = dw_product(s, dz, x, dweight);
    const size_t packed = dz_packed_bytes(s);
    if (packed) {
        gx.a.packed = gw.a.packed = scratch;
        gw.a.ready = dx != nullptr;
        scratch += packed;
    }
    if (e == cudaSuccess && dx) e = run_product(s, gx, scratch, workspace, st);
    if (e == cudaSuccess && dweight) e = run_product(s, gw, scratch, workspace, st);
    return call_status(e);
}

}  // extern "C"
