// Linear attention with a decay for each head: extern "C" entry points, the kernel for any type and width on the CUDA cores, and the
// decode step.  rglru_linattn.cuh has the mathematics.
#include <cuda_bf16.h>

#include "rglru_linattn.cuh"
#include "sm100_ptx.cuh"

namespace rglru {
namespace {

using namespace ptx;

constexpr int MAX_WIDTH = 256;
constexpr int C = 32, SLICE = 64, GEN_THREADS = 256;   // tokens a chunk, columns of v a block

template <typename IO> __device__ __forceinline__ float at(const void *p, long long i) {
    if constexpr (sizeof(IO) == 4) return ((const float *)p)[i];
    else return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
}
template <typename IO> __device__ __forceinline__ void put(void *p, long long i, float v) {
    if constexpr (sizeof(IO) == 4) ((float *)p)[i] = v;
    else ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(v);
}
__host__ __device__ inline int padded_width(int dk) { return (dk + 3) / 4 * 4 + 4; }
inline size_t generic_smem(int dk) { return sizeof(float) * (2 * C * padded_width(dk) + C * SLICE + (size_t)dk * SLICE + C * (C + 1) + C + 1); }

// One block walks the chunks of a (sequence, head) for 64 columns of v, its part of the state in shared memory.  Everything is fp32.
template <typename IO> __global__ void __launch_bounds__(GEN_THREADS) generic_mix_kernel(const __grid_constant__ MixArgs a) {
    extern __shared__ float4 smem4[];
    dependency_wait();
    const MixRole &r = a.role[blockIdx.y];
    const int dk = r.dk, dv = r.dv, ld = padded_width(dk), slices = gridDim.x / (a.B * a.H), c0 = blockIdx.x % slices * SLICE;
    const int unit = blockIdx.x / slices, h = unit % a.H, b = unit / a.H, tid = threadIdx.x;
    if (c0 >= dv) return;
    float *Q = (float *)smem4, *K = Q + C * ld, *V = K + C * ld, *S = V + C * SLICE, *P = S + dk * SLICE, *pw = P + C * (C + 1);
    const long long mat = (long long)unit * dk * dv;
    if (tid <= C) pw[tid] = decay_power(a.log_decay[h], (float)tid);
    for (int i = tid; i < dk * SLICE; i += GEN_THREADS) {
        const int d = i / SLICE, e = c0 + i % SLICE;
        S[i] = r.s_in && e < dv ? r.s_in[mat + (r.turned ? (long long)e * dk + d : (long long)d * dv + e)] : 0.0f;
    }
    for (int i = tid; i < 2 * C * ld; i += GEN_THREADS) Q[i] = 0.0f;   // the padding behind dk as well
    const int ty = tid >> 4, tx = tid & 15;
    for (int t0 = 0; t0 < a.T; t0 += C) {
        const int n = min(C, a.T - t0);
        __syncthreads();
        for (int i = tid; i < C * dk; i += GEN_THREADS) {
            const int j = i / dk, d = i % dk, t = r.reverse ? a.T - 1 - (t0 + j) : t0 + j;
            const bool in = j < n;
            Q[j * ld + d] = in ? at<IO>(r.q.p, b * r.q.batch + t * r.q.token + (long long)h * dk + d) : 0.0f;
            K[j * ld + d] = in ? at<IO>(r.k.p, b * r.k.batch + t * r.k.token + (long long)h * dk + d) : 0.0f;
        }
        for (int i = tid; i < C * SLICE; i += GEN_THREADS) {
            const int j = i / SLICE, e = c0 + i % SLICE, t = r.reverse ? a.T - 1 - (t0 + j) : t0 + j;
            V[i] = j < n && e < dv ? at<IO>(r.v.p, b * r.v.batch + t * r.v.token + (long long)h * dv + e) : 0.0f;
        }
        __syncthreads();
        {   // P[i][j] = sp d^(i-j) q_i k_j for j <= i
            float p[2][2] = {};
            if (tx <= ty)
                for (int d = 0; d < dk; d += 4) {
                    const float4 q0 = *(const float4 *)&Q[(2 * ty) * ld + d], q1 = *(const float4 *)&Q[(2 * ty + 1) * ld + d];
                    const float4 k0 = *(const float4 *)&K[(2 * tx) * ld + d], k1 = *(const float4 *)&K[(2 * tx + 1) * ld + d];
                    p[0][0] += q0.x * k0.x + q0.y * k0.y + q0.z * k0.z + q0.w * k0.w;
                    p[0][1] += q0.x * k1.x + q0.y * k1.y + q0.z * k1.z + q0.w * k1.w;
                    p[1][0] += q1.x * k0.x + q1.y * k0.y + q1.z * k0.z + q1.w * k0.w;
                    p[1][1] += q1.x * k1.x + q1.y * k1.y + q1.z * k1.z + q1.w * k1.w;
                }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int i = 2 * ty + u, j = 2 * tx + w;
                    P[i * (C + 1) + j] = j <= i ? p[u][w] * (r.sp * pw[i - j]) : 0.0f;
                }
        }
        __syncthreads();
        {   // outputs of rows 2 ty, 2 ty + 1, four columns
            float near[2][4] = {}, far[2][4] = {};
            for (int d = 0; d < dk; ++d) {
                const float4 s = *(const float4 *)&S[d * SLICE + tx * 4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float q = Q[(2 * ty + u) * ld + d];
                    far[u][0] = fmaf(q, s.x, far[u][0]); far[u][1] = fmaf(q, s.y, far[u][1]);
                    far[u][2] = fmaf(q, s.z, far[u][2]); far[u][3] = fmaf(q, s.w, far[u][3]);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
                for (int j = 0; j <= 2 * ty + u; ++j) {   // later tokens are not touched: what they hold may be no number
                    const float4 v = *(const float4 *)&V[j * SLICE + tx * 4];
                    const float p = P[(2 * ty + u) * (C + 1) + j];
                    near[u][0] = fmaf(p, v.x, near[u][0]); near[u][1] = fmaf(p, v.y, near[u][1]);
                    near[u][2] = fmaf(p, v.z, near[u][2]); near[u][3] = fmaf(p, v.w, near[u][3]);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = 2 * ty + u, t = r.reverse ? a.T - 1 - (t0 + i) : t0 + i;
                if (i >= n) continue;
                const float w = r.si * pw[i + r.first];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c0 + tx * 4 + e < dv) put<IO>(r.o.p, b * r.o.batch + t * r.o.token + (long long)h * dv + c0 + tx * 4 + e, fmaf(w, far[u][e], near[u][e]));
            }
        }
        __syncthreads();
        for (int d0 = ty; d0 < dk; d0 += 64) {   // state rows d0, d0 + 16, d0 + 32, d0 + 48, four columns
            float s[4][4] = {};
            for (int j = 0; j < n; ++j) {
                const float4 v = *(const float4 *)&V[j * SLICE + tx * 4];
                const float w = r.su * pw[n - j - r.first];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float k = d0 + 16 * u < dk ? w * K[j * ld + d0 + 16 * u] : 0.0f;
                    s[u][0] = fmaf(k, v.x, s[u][0]); s[u][1] = fmaf(k, v.y, s[u][1]); s[u][2] = fmaf(k, v.z, s[u][2]); s[u][3] = fmaf(k, v.w, s[u][3]);
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (d0 + 16 * u >= dk) continue;
                float4 *p = (float4 *)&S[(d0 + 16 * u) * SLICE + tx * 4];
                const float4 o = *p;
                *p = make_float4(fmaf(pw[n], o.x, s[u][0]), fmaf(pw[n], o.y, s[u][1]), fmaf(pw[n], o.z, s[u][2]), fmaf(pw[n], o.w, s[u][3]));
            }
        }
    }
    __syncthreads();
    if (r.s_out)
        for (int i = tid; i < dk * SLICE; i += GEN_THREADS) {
            const int d = i / SLICE, e = c0 + i % SLICE;
            if (e < dv) r.s_out[mat + (long long)d * dv + e] = S[i];
        }
    dependency_trigger();
}

cudaError_t generic_mix(const MixArgs &a, int io, cudaStream_t st) {
    int dk = 0, dv = 0;
    for (int i = 0; i < a.roles; ++i) { dk = a.role[i].dk > dk ? a.role[i].dk : dk; dv = a.role[i].dv > dv ? a.role[i].dv : dv; }
    const long long blocks = (long long)a.B * a.H * ((dv + SLICE - 1) / SLICE);
    if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks, a.roles);
    static PerDeviceOptIn opt_f32, opt_bf16;
    const size_t most = generic_smem(MAX_WIDTH);
    cudaError_t e = io == RGLRU_F32 ? opt_f32.ensure(generic_mix_kernel<float>, (int)most) : opt_bf16.ensure(generic_mix_kernel<__nv_bfloat16>, (int)most);
    if (e != cudaSuccess) return e;
    return launch_dependent(io == RGLRU_F32 ? generic_mix_kernel<float> : generic_mix_kernel<__nv_bfloat16>, grid, dim3(GEN_THREADS), generic_smem(dk), st, a);
}

// ---- decode step: s = d s + k v^T, o = scale q s.  Bound by the state, read and written once.  A thread owns VE columns of every 256 / LPR-th
// row of its block's columns; the rows' shares of o are added through shared memory in a fixed order.
struct StepArgs {
    int H, dk, dv;
    float scale;
    const void *q, *k, *v;
    const float *log_decay;
    float *s;
    void *o;
};
template <typename IO, int VE, int LPR> __global__ void __launch_bounds__(256) mix_step_kernel(StepArgs a) {
    extern __shared__ float sm[];     // q, k [dk], then [256][VE] shares of o
    constexpr int RG = 256 / LPR, UNROLL = 8;
    dependency_wait();
    const int slices = (a.dv + LPR * VE - 1) / (LPR * VE), slice = blockIdx.x % slices;
    const long long unit = blockIdx.x / slices;
    const int h = (int)(unit % a.H), rg = threadIdx.x / LPR, c = (slice * LPR + threadIdx.x % LPR) * VE;
    const bool in = c < a.dv;
    float *q = sm, *k = sm + a.dk, *red = k + a.dk;
    for (int i = threadIdx.x; i < a.dk; i += 256) { q[i] = at<IO>(a.q, unit * a.dk + i); k[i] = at<IO>(a.k, unit * a.dk + i); }
    const float d = decay_power(a.log_decay[h], 1.0f);
    float v[VE] = {}, o[VE] = {};
    if (in)
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = at<IO>(a.v, unit * a.dv + c + e);
    float *s = a.s + unit * a.dk * (long long)a.dv + c;
    __syncthreads();
    if (in)
        for (int r0 = rg; r0 < a.dk; r0 += RG * UNROLL) {
            float x[UNROLL][VE];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int r = r0 + u * RG;
                if (r < a.dk) {
                    if constexpr (VE == 4) { const float4 f = *(const float4 *)(s + (long long)r * a.dv); x[u][0] = f.x; x[u][1] = f.y; x[u][2] = f.z; x[u][3] = f.w; }
                    else x[u][0] = s[(long long)r * a.dv];
                }
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int r = r0 + u * RG;
                if (r < a.dk) {
                    const float kr = k[r], qr = q[r];
#pragma unroll
                    for (int e = 0; e < VE; ++e) { x[u][e] = fmaf(d, x[u][e], kr * v[e]); o[e] = fmaf(qr, x[u][e], o[e]); }
                    if constexpr (VE == 4) *(float4 *)(s + (long long)r * a.dv) = make_float4(x[u][0], x[u][1], x[u][2], x[u][3]);
                    else s[(long long)r * a.dv] = x[u][0];
                }
            }
        }
    dependency_trigger();
#pragma unroll
    for (int e = 0; e < VE; ++e) red[(rg * LPR + threadIdx.x % LPR) * VE + e] = o[e];
    __syncthreads();
    for (int i = threadIdx.x; i < LPR * VE; i += 256) {
        const int col = slice * LPR * VE + i;
        if (col >= a.dv) break;
        float t = 0.0f;
        for (int g = 0; g < RG; ++g) t += red[g * LPR * VE + i];
        put<IO>(a.o, unit * a.dv + col, t * a.scale);
    }
}

int32_t check_mix(const rglru_linear_attention_shape_t *s, bool need_T) {
    if (s == nullptr) return RGLRU_ERR_NULL;
    if (s->B <= 0 || s->H <= 0 || s->dk <= 0 || s->dv <= 0 || (need_T && s->T <= 0) || !isfinite(s->scale)) return RGLRU_ERR_SHAPE;
    if (s->io != RGLRU_F32 && s->io != RGLRU_BF16) return RGLRU_ERR_UNSUPPORTED;
    if (need_T ? s->dk > MAX_WIDTH || s->dv > MAX_WIDTH : s->dk > 4096) return RGLRU_ERR_UNSUPPORTED;
    if ((long long)s->B * s->H > INT32_MAX / 4 || (need_T && s->T > (1 << 30))) return RGLRU_ERR_UNSUPPORTED;
    return RGLRU_OK;
}
// The tensor with its distances, or false if its tokens overlap one another
bool place(const void *p, const rglru_stride_t &st, const rglru_linear_attention_shape_t *s, int width, MixTensor &t, size_t &bytes) {
    const long long row = (long long)s->H * width, B = s->B, T = s->T;
    t.p = const_cast<void *>(p);
    t.token = st.token; t.batch = st.batch;
    if (t.token == 0 && t.batch == 0) { t.token = row; t.batch = row * T; }
    if (t.token < 0 || t.batch < 0 || t.token > (1ll << 40) || t.batch > (1ll << 40)) return false;
    const bool by_token = (T == 1 || t.token >= row) && (B == 1 || t.batch >= (T - 1) * t.token + row);
    const bool by_batch = (B == 1 || t.batch >= row) && (T == 1 || t.token >= (B - 1) * t.batch + row);
    bytes = ((size_t)(B - 1) * t.batch + (size_t)(T - 1) * t.token + row) * io_bytes(s->io);
    return by_token || by_batch;
}
const rglru_linear_attention_strides_t DENSE{};
size_t state_bytes(const rglru_linear_attention_shape_t *s) { return (size_t)s->B * s->H * s->dk * s->dv * sizeof(float); }
bool may_use_tensor_cores(const rglru_linear_attention_shape_t *s) {
    return !(s->flags & RGLRU_FLAG_FORCE_GENERIC) && s->io == RGLRU_BF16 && s->dk <= 128 && s->dv <= 128 && s->dk % 8 == 0 && s->dv % 8 == 0;
}
cudaError_t run_mix(const rglru_linear_attention_shape_t *s, MixArgs &a, void *workspace, cudaStream_t st) {
    if (!may_use_tensor_cores(s) || !sm100_mix_supported(a, s->io)) return generic_mix(a, s->io, st);
    char *scratch = (char *)workspace + WS_HEADER_BYTES;
    const size_t sums = sm100_mix_bytes(a.roles, s->B, s->T, s->H);
    if (sums && a.role[0].s_in && a.role[0].s_in == a.role[0].s_out) {   // blocks that share a sequence all read its s0
        float *copy = (float *)(scratch + up256(sums));
        const cudaError_t e = cudaMemcpyAsync(copy, a.role[0].s_in, state_bytes(s), cudaMemcpyDeviceToDevice, st);
        if (e != cudaSuccess) return e;
        a.role[0].s_in = copy;
    }
    return sm100_mix(a, scratch, st);
}

}  // namespace
}  // namespace rglru

using namespace rglru;

extern "C" {

size_t rglru_linear_attention_workspace_bytes(const rglru_linear_attention_shape_t *s, int32_t op) {
    if (op != RGLRU_OP_PREFILL && op != RGLRU_OP_BACKWARD) return 0;
    if (check_mix(s, true) != RGLRU_OK) return 0;
    // the copy of s0 is for a call that overwrites it (s_T == s0) while blocks read it
    const int roles = op == RGLRU_OP_PREFILL ? 1 : 3;
    size_t bytes = WS_HEADER_BYTES;
    const size_t sums = may_use_tensor_cores(s) ? sm100_mix_bytes(roles, s->B, s->T, s->H) : 0;
    if (sums) bytes += up256(sums) + (roles == 1 ? up256(state_bytes(s)) : 0);
    return bytes;
}

int32_t rglru_linear_attention_prefill(const rglru_linear_attention_shape_t *s, const rglru_linear_attention_strides_t *strides, const void *q, const void *k,
                                       const void *v, const float *log_decay, const float *s0, void *o, float *s_T, void *workspace, size_t workspace_bytes,
                                       void *cuda_stream) {
    const int32_t rc = check_mix(s, true);
    if (rc != RGLRU_OK) return rc;
    if (!q || !k || !v || !log_decay || !o || !s_T || !workspace) return RGLRU_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(log_decay, 16) || !aligned(s0, 16) || !aligned(o, 16) || !aligned(s_T, 16) ||
        !aligned(workspace, 256))
        return RGLRU_ERR_ALIGN;
    const rglru_linear_attention_strides_t &st = strides ? *strides : DENSE;
    MixArgs a{};
    MixRole &r = a.role[0];
    size_t nq, nk, nv, no;
    if (!place(q, st.q, s, s->dk, r.q, nq) || !place(k, st.k, s, s->dk, r.k, nk) || !place(v, st.v, s, s->dv, r.v, nv) || !place(o, st.o, s, s->dv, r.o, no))
        return RGLRU_ERR_SHAPE;
    if (workspace_bytes < rglru_linear_attention_workspace_bytes(s, RGLRU_OP_PREFILL)) return RGLRU_ERR_WORKSPACE;
    const size_t mat = (size_t)s->B * s->H * s->dk * s->dv * sizeof(float);
    if (overlap(o, no, q, nq) || overlap(o, no, k, nk) || overlap(o, no, v, nv) || overlap(o, no, s0, mat) || overlap(s_T, mat, q, nq) ||
        overlap(s_T, mat, k, nk) || overlap(s_T, mat, v, nv) || overlap(s_T, mat, o, no) || (s0 != s_T && overlap(s_T, mat, s0, mat)))
        return RGLRU_ERR_ALIAS;
    a.roles = 1; a.B = s->B; a.T = s->T; a.H = s->H; a.log_decay = log_decay; a.status = (uint32_t *)workspace;
    r.dk = s->dk; r.dv = s->dv; r.s_in = s0; r.s_out = s_T; r.first = 1; r.sp = r.si = s->scale; r.su = 1.0f;
    return call_status(run_mix(s, a, workspace, (cudaStream_t)cuda_stream));
}

int32_t rglru_linear_attention_decode_step(const rglru_linear_attention_shape_t *s, const void *q, const void *k, const void *v, const float *log_decay,
                                           float *state, void *o, void *cuda_stream) {
    const int32_t rc = check_mix(s, false);
    if (rc != RGLRU_OK) return rc;
    if (!q || !k || !v || !log_decay || !state || !o) return RGLRU_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(log_decay, 16) || !aligned(state, 16) || !aligned(o, 16)) return RGLRU_ERR_ALIGN;
    const long long units = (long long)s->B * s->H;
    const size_t io = io_bytes(s->io), nq = units * s->dk * io, nv = units * s->dv * io, ns = (size_t)units * s->dk * s->dv * sizeof(float);
    if (overlap(o, nv, q, nq) || overlap(o, nv, k, nq) || overlap(o, nv, v, nv) || overlap(o, nv, state, ns) || overlap(state, ns, q, nq) ||
        overlap(state, ns, k, nq) || overlap(state, ns, v, nv))
        return RGLRU_ERR_ALIAS;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool vec = s->dv % 4 == 0, f32 = s->io == RGLRU_F32;
    // blocks of 32 lanes' columns, or, while they do not fill the SMs, of 8
    const int ve = vec ? 4 : 1, wide = units * ((s->dv + 32 * ve - 1) / (32 * ve)) >= 2 * num_sms();
    const int lpr = wide ? 32 : 8;
    const size_t smem = sizeof(float) * (2 * (size_t)s->dk + 256 * ve);
    const long long blocks = units * ((s->dv + lpr * ve - 1) / (lpr * ve));
    if (blocks > 0x7FFFFFFFll) return RGLRU_ERR_UNSUPPORTED;
    const StepArgs a{s->H, s->dk, s->dv, s->scale, q, k, v, log_decay, state, o};
#define RGLRU_STEP(IO, VE) \
    launch_dependent(wide ? mix_step_kernel<IO, VE, 32> : mix_step_kernel<IO, VE, 8>, dim3((unsigned)blocks), dim3(256), smem, st, a)
    const cudaError_t e = f32 ? (vec ? RGLRU_STEP(float, 4) : RGLRU_STEP(float, 1)) : (vec ? RGLRU_STEP(__nv_bfloat16, 4) : RGLRU_STEP(__nv_bfloat16, 1));
#undef RGLRU_STEP
    return call_status(e);
}

int32_t rglru_linear_attention_backward(const rglru_linear_attention_shape_t *s, const rglru_linear_attention_strides_t *strides, const void *q, const void *k,
                                        const void *v, const float *log_decay, const float *s0, const void *dout, const float *ds_T, void *dq, void *dk,
                                        void *dv, float *ds0, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    const int32_t rc = check_mix(s, true);
    if (rc != RGLRU_OK) return rc;
    if (!q || !k || !v || !log_decay || !dout || !dq || !dk || !dv || !workspace) return RGLRU_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(log_decay, 16) || !aligned(s0, 16) || !aligned(dout, 16) || !aligned(ds_T, 16) ||
        !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16) || !aligned(ds0, 16) || !aligned(workspace, 256))
        return RGLRU_ERR_ALIGN;
    const rglru_linear_attention_strides_t &st = strides ? *strides : DENSE;
    MixTensor t[7];
    size_t n[9];
    if (!place(q, st.q, s, s->dk, t[0], n[0]) || !place(k, st.k, s, s->dk, t[1], n[1]) || !place(v, st.v, s, s->dv, t[2], n[2]) ||
        !place(dout, st.o, s, s->dv, t[3], n[3]) || !place(dq, st.dq, s, s->dk, t[4], n[4]) || !place(dk, st.dk, s, s->dk, t[5], n[5]) ||
        !place(dv, st.dv, s, s->dv, t[6], n[6]))
        return RGLRU_ERR_SHAPE;
    if (workspace_bytes < rglru_linear_attention_workspace_bytes(s, RGLRU_OP_BACKWARD)) return RGLRU_ERR_WORKSPACE;
    const size_t mat = (size_t)s->B * s->H * s->dk * s->dv * sizeof(float);
    const void *const ins[6] = {q, k, v, dout, s0, ds_T};
    const size_t in_bytes[6] = {n[0], n[1], n[2], n[3], mat, mat};
    void *const outs[4] = {dq, dk, dv, ds0};
    const size_t out_bytes[4] = {n[4], n[5], n[6], mat};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 6; ++j)
            if (overlap(outs[i], out_bytes[i], ins[j], in_bytes[j])) return RGLRU_ERR_ALIAS;
    // dq, dk and dv may lie side by side in one gradient of a projection, tokens interleaved; the same place twice is refused
    if (dq == dk || dq == dv || dk == dv || overlap(ds0, mat, dq, n[4]) || overlap(ds0, mat, dk, n[5]) || overlap(ds0, mat, dv, n[6])) return RGLRU_ERR_ALIAS;
    MixArgs a{};
    a.roles = 3; a.B = s->B; a.T = s->T; a.H = s->H; a.log_decay = log_decay; a.status = (uint32_t *)workspace;
    a.role[0] = MixRole{t[3], t[2], t[1], t[4], s->dv, s->dk, s0, nullptr, 1, 0, 1, s->scale, s->scale, 1.0f};
    a.role[1] = MixRole{t[2], t[3], t[0], t[5], s->dv, s->dk, ds_T, nullptr, 1, 1, 0, s->scale, 1.0f, s->scale};
    a.role[2] = MixRole{t[1], t[0], t[3], t[6], s->dk, s->dv, ds_T, ds0, 0, 1, 0, s->scale, 1.0f, s->scale};
    return call_status(run_mix(s, a, workspace, (cudaStream_t)cuda_stream));
}

}  // extern "C"
