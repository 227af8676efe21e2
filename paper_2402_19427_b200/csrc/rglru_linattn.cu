// Linear attention with a decay for each head: extern "C" entry points, the kernel for any type and width on the CUDA cores, and the
// decode step.  rglru_linattn.cuh has the mathematics.
#include <climits>

#include <cuda_bf16.h>

#include "rglru_io.cuh"
#include "rglru_linattn.cuh"
#include "sm100_ptx.cuh"

namespace rglru {
namespace {

using namespace ptx;

constexpr int MAX_WIDTH = 256;
constexpr int MAX_STEP_DK = 4096, MAX_STEP_DV = INT_MAX - 1023;   // of the token step: q and k in shared memory; a block's last column, behind the row's end, still is an int
constexpr int C = 32, GEN_THREADS = 256;   // tokens a chunk

// ---- any type and width: fp32 on the CUDA cores.
// A block walks chunks of 32 tokens of a (role, sequence, head) for 32 CB columns of v, its part of the state in shared memory.  A chunk is
//     far = q S,   P = q k^T (decayed, masked; over q's place),   out = P v + decay far,   S <- d^n S + (decayed k)^T v
// A warp has 32 columns: lane (rg, cg) owns four of them and every fourth row, so that an operand read by 16 bytes serves 16 products and
// comes without bank conflicts.  Bound by the CUDA cores' instructions (dk = dv = 128: some 16 thousand issue slots of each scheduler a chunk, 15 us of an
// SM's, 55 % of the slots taken), with two blocks an SM so that one's loads and barriers lie under the other's products: q, k, v, S take half
// the SM's shared memory to the byte, the powers of the decay lie in the padding of k's rows.  8 x 2048 tokens of 20 heads take 1.5 ms, heads of 256
// columns (one block an SM) 4 x 2048 tokens of 16 heads 3.2.
// Long sequences of few heads are cut into equal segments: a first launch leaves the sums of each (STATE_ONLY), and a segment's block starts
// from the state before it, folded in order (65536 tokens of 16 heads 4.0 ms, in one piece 25 ms).
struct GenericArgs {
    MixArgs m;
    int slices, segments, launched, seg_chunks, rows;   // launched: segments of this launch; rows: of a sum in `local`
    float *local;                                       // [role][sequence, head][slice][segment][rows][32 CB]
};
__host__ __device__ inline int padded_width(int dk) { return (dk + 3) / 4 * 4 + 4; }
constexpr int PLD = 36;   // distance of P's rows
inline size_t generic_smem(int dk, int cb) {
    const int ld = padded_width(dk), q = C * ld > C * PLD ? C * ld : C * PLD;
    return sizeof(float) * (size_t)(q + C * ld + C * 32 * cb + (ld - 4) * 32 * cb);
}
template <typename IO, int VEC> __device__ __forceinline__ float4 at4(const void *p, long long i) {
    if constexpr (VEC == 1) {
        return make_float4(at<IO>(p, i), 0.0f, 0.0f, 0.0f);
    } else if constexpr (sizeof(IO) == 4) {
        return *(const float4 *)((const float *)p + i);
    } else {
        const uint2 w = *(const uint2 *)((const __nv_bfloat16 *)p + i);
        const f32x2 a = bf2x(w.x), b = bf2x(w.y);
        return make_float4(a.x, a.y, b.x, b.y);
    }
}
// VEC: 4 where every width and distance is a multiple of 4
template <typename IO, int CB, int VEC, bool STATE_ONLY> __global__ void __launch_bounds__(GEN_THREADS, 2) generic_mix_kernel(const __grid_constant__ GenericArgs p) {
    constexpr int NC = 32 * CB;
    extern __shared__ float4 smem4[];
    dependency_wait();
    const MixArgs &a = p.m;
    const MixRole &r = a.role[blockIdx.y];
    const int seg = blockIdx.x % p.launched, column = blockIdx.x / p.launched, slice = column % p.slices, unit = column / p.slices;
    const int dk = r.dk, dv = r.dv, dk4 = (dk + 3) / 4 * 4, ld = dk4 + 4, c0 = slice * NC, h = unit % a.H, b = unit / a.H;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rg = lane >> 3, col = warp % CB * 32 + (lane & 7) * 4, group = warp / CB;
    if (c0 >= dv) return;
    float *Q = (float *)smem4, *K = Q + (C * ld > C * PLD ? C * ld : C * PLD), *V = K + C * ld, *S = V + C * NC, *P = Q;
    const float decay = a.log_decay[h], pw32 = decay_power(decay, 32.0f);
    auto pw = [&](int n) { return n == 32 ? pw32 : K[n * ld + dk4]; };
    const int chunks = (a.T + C - 1) / C, first = seg * p.seg_chunks, last = min(chunks, first + p.seg_chunks);
    const long long mat = (long long)unit * dk * dv, sums = (((long long)blockIdx.y * a.B * a.H + unit) * p.slices + slice) * p.segments;
    const float before = STATE_ONLY ? 0.0f : decay_power(decay, (float)(p.seg_chunks * C));
    for (int i = tid; i < dk4 * NC; i += GEN_THREADS) {
        const int d = i / NC, e = c0 + i % NC;
        float s = 0.0f;
        if (!STATE_ONLY) {
            if (r.s_in && d < dk && e < dv) s = r.s_in[mat + (r.turned ? (long long)e * dk + d : (long long)d * dv + e)];
            for (int g = 0; g < seg; ++g) s = fmaf(before, s, p.local[(sums + g) * p.rows * NC + i]);
        }
        S[i] = s;
    }
    for (int i = tid; i < C * 4; i += GEN_THREADS) K[i / 4 * ld + dk4 + i % 4] = decay_power(decay, (float)(i / 4));
    for (int c = first; c < last; ++c) {
        const int t0 = c * C, n = min(C, a.T - t0);
        __syncthreads();
        auto load = [&](const MixTensor &t, float *to, int width, int from, int wide, int distance) {   // columns from, from + 1, .. of 32 tokens, zeros behind them
            for (int d = lane * VEC; d < wide; d += 32 * VEC) {
                float4 x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int j = warp + 8 * u, token = r.reverse ? a.T - 1 - (t0 + j) : t0 + j;
                    x[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (j < n && from + d < width) x[u] = at4<IO, VEC>(t.p, b * t.batch + token * t.token + (long long)h * width + from + d);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float *at_row = to + (warp + 8 * u) * distance + d;
                    if constexpr (VEC == 4) *(float4 *)at_row = x[u];
                    else *at_row = x[u].x;
                }
            }
        };
        if (!STATE_ONLY) load(r.q, Q, dk, 0, dk4, ld);
        load(r.k, K, dk, 0, dk4, ld);
        load(r.v, V, dv, c0, NC, NC);
        __syncthreads();
        if (!STATE_ONLY) {
            const int row = group * 4 * CB + rg;   // and every fourth from there on
            float far[CB][4] = {};
#pragma unroll 2
            for (int d = 0; d < dk4; d += 4) {
                float4 s[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = *(const float4 *)&S[(d + e) * NC + col];
#pragma unroll
                for (int u = 0; u < CB; ++u) {
                    const float4 q = *(const float4 *)&Q[(row + 4 * u) * ld + d];
                    const float x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        far[u][0] = fmaf(x[e], s[e].x, far[u][0]); far[u][1] = fmaf(x[e], s[e].y, far[u][1]);
                        far[u][2] = fmaf(x[e], s[e].z, far[u][2]); far[u][3] = fmaf(x[e], s[e].w, far[u][3]);
                    }
                }
            }
            float x[4] = {};   // rows 4 warp .. + 3 of P, column lane
            for (int d = 0; d < dk4; d += 4) {
                const float4 k = *(const float4 *)&K[lane * ld + d];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float4 q = *(const float4 *)&Q[(4 * warp + u) * ld + d];
                    x[u] = fmaf(q.x, k.x, x[u]); x[u] = fmaf(q.y, k.y, x[u]); x[u] = fmaf(q.z, k.z, x[u]); x[u] = fmaf(q.w, k.w, x[u]);
                }
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = 4 * warp + u;
                P[i * PLD + lane] = lane <= i ? x[u] * (r.sp * pw(i - lane)) : 0.0f;
            }
            __syncthreads();
            float near[CB][4] = {};
            for (int j = 0; j < group * 4 * CB + 4 * CB; j += 4) {
                float4 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = *(const float4 *)&V[(j + e) * NC + col];
#pragma unroll
                for (int u = 0; u < CB; ++u) {
                    const float4 w = *(const float4 *)&P[(row + 4 * u) * PLD + j];
                    const float y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (j + e > row + 4 * u) continue;   // later tokens are not touched: what they hold may be no number
                        near[u][0] = fmaf(y[e], v[e].x, near[u][0]); near[u][1] = fmaf(y[e], v[e].y, near[u][1]);
                        near[u][2] = fmaf(y[e], v[e].z, near[u][2]); near[u][3] = fmaf(y[e], v[e].w, near[u][3]);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < CB; ++u) {
                const int i = row + 4 * u, token = r.reverse ? a.T - 1 - (t0 + i) : t0 + i;
                if (i >= n) continue;
                const float w = r.si * pw(i + r.first);
                const long long o = b * r.o.batch + token * r.o.token + (long long)h * dv + c0 + col;
                const float y[4] = {fmaf(w, far[u][0], near[u][0]), fmaf(w, far[u][1], near[u][1]), fmaf(w, far[u][2], near[u][2]), fmaf(w, far[u][3], near[u][3])};
                if (VEC == 4 && sizeof(IO) == 4 && c0 + col < dv) {
                    *(float4 *)((float *)r.o.p + o) = make_float4(y[0], y[1], y[2], y[3]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c0 + col + e < dv) put<IO>(r.o.p, o + e, y[e]);
                }
            }
        }
        if (!STATE_ONLY && c + 1 == last && !(last == chunks && r.s_out)) break;   // nobody reads the state behind
        const float f = pw(n);
        for (int tile = 0; tile < dk4; tile += 128) {   // rows tile + 16 CB group + 16 i + 4 rg + e
            const int row = tile + group * 16 * CB + rg * 4;
            f32x2 sum[CB][2][4] = {};   // pairs of rows, four columns
            for (int j = 0; j < n; ++j) {
                const float4 v = *(const float4 *)&V[j * NC + col];
                const float w = r.su * pw(n - j - r.first);
                const f32x2 x[4] = {pack2(w * v.x, w * v.x), pack2(w * v.y, w * v.y), pack2(w * v.z, w * v.z), pack2(w * v.w, w * v.w)};
#pragma unroll
                for (int i = 0; i < CB; ++i) {
                    if (row + 16 * i >= dk4) continue;
                    const float4 k = *(const float4 *)&K[j * ld + row + 16 * i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sum[i][0][e] = fma2(pack2(k.x, k.y), x[e], sum[i][0][e]);
                        sum[i][1][e] = fma2(pack2(k.z, k.w), x[e], sum[i][1][e]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < CB; ++i) {
                if (row + 16 * i >= dk4) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (row + 16 * i + e >= dk) continue;   // padding stays 0: out of an infinite v it would become NaN, and q's padding bring that into the outputs
                    float4 *at_row = (float4 *)&S[(row + 16 * i + e) * NC + col];
                    const float4 o = *at_row;
                    const f32x2 *z = sum[i][e / 2];
                    *at_row = e % 2 ? make_float4(fmaf(f, o.x, z[0].y), fmaf(f, o.y, z[1].y), fmaf(f, o.z, z[2].y), fmaf(f, o.w, z[3].y))
                                    : make_float4(fmaf(f, o.x, z[0].x), fmaf(f, o.y, z[1].x), fmaf(f, o.z, z[2].x), fmaf(f, o.w, z[3].x));
                }
            }
        }
    }
    __syncthreads();
    if (STATE_ONLY) {
        for (int i = tid; i < dk4 * NC; i += GEN_THREADS) p.local[(sums + seg) * p.rows * NC + i] = S[i];
    } else if (r.s_out && last == chunks) {
        for (int i = tid; i < dk * NC; i += GEN_THREADS) {
            const int d = i / NC, e = c0 + i % NC;
            if (e < dv) r.s_out[mat + (long long)d * dv + e] = S[i];
        }
    }
    dependency_trigger();
}

// What a call on the CUDA cores takes: blocks of 64 columns where no role has more or blocks of 128, cut, would still leave half the SMs idle; segments, as many as make two blocks an SM but no shorter
// than eight chunks (a segment's sums cost a third of its walk again)
struct GenericPlan {
    int cb, slices, segments, seg_chunks, rows;
    size_t local_bytes;
};
GenericPlan generic_plan(int roles, int B, int T, int H, int dk, int dv) {   // dk, dv: the largest of all roles
    GenericPlan p{};
    const long long units = (long long)roles * B * H, chunks = (T + C - 1) / C, most = chunks < 16 ? 1 : chunks / 8;
    p.cb = dv <= 64 || units * ((dv + 127) / 128) * most <= 74 ? 2 : 4;
    p.slices = (dv + 32 * p.cb - 1) / (32 * p.cb);
    p.rows = (dk + 3) / 4 * 4;
    const long long blocks = units * p.slices;
    long long want = 296 / blocks;
    if (want > most) want = most;
    p.segments = want < 2 ? 1 : (int)want;
    p.seg_chunks = (int)((chunks + p.segments - 1) / p.segments);
    p.segments = (int)((chunks + p.seg_chunks - 1) / p.seg_chunks);
    p.local_bytes = p.segments == 1 ? 0 : (size_t)blocks * p.segments * p.rows * 32 * p.cb * sizeof(float);
    return p;
}
template <typename IO, int CB, int VEC> cudaError_t run_generic(const GenericPlan &plan, GenericArgs &p, size_t smem, size_t most, cudaStream_t st) {
    static PerDeviceOptIn opt, opt_state;
    const long long columns = (long long)p.m.B * p.m.H * plan.slices;
    if (columns * plan.segments > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    cudaError_t e = opt.ensure(generic_mix_kernel<IO, CB, VEC, false>, (int)most);
    if (e == cudaSuccess && plan.segments > 1) {
        e = opt_state.ensure(generic_mix_kernel<IO, CB, VEC, true>, (int)most);
        p.launched = plan.segments - 1;   // nothing comes behind the last one
        if (e == cudaSuccess) e = launch_dependent(generic_mix_kernel<IO, CB, VEC, true>, dim3((unsigned)(columns * p.launched), p.m.roles), dim3(GEN_THREADS), smem, st, p);
    }
    p.launched = plan.segments;
    if (e == cudaSuccess) e = launch_dependent(generic_mix_kernel<IO, CB, VEC, false>, dim3((unsigned)(columns * p.launched), p.m.roles), dim3(GEN_THREADS), smem, st, p);
    return e;
}
cudaError_t generic_mix(const MixArgs &a, int io, float *local, cudaStream_t st) {
    int dk = 0, dv = 0;
    bool vec = true;
    for (int i = 0; i < a.roles; ++i) {
        const MixRole &r = a.role[i];
        dk = r.dk > dk ? r.dk : dk; dv = r.dv > dv ? r.dv : dv;
        vec = vec && r.dk % 4 == 0 && r.dv % 4 == 0;
        for (const MixTensor *t : {&r.q, &r.k, &r.v, &r.o}) vec = vec && (a.T == 1 || t->token % 4 == 0) && (a.B == 1 || t->batch % 4 == 0);
    }
    const GenericPlan plan = generic_plan(a.roles, a.B, a.T, a.H, dk, dv);
    GenericArgs p{a, plan.slices, plan.segments, 0, plan.seg_chunks, plan.rows, local};
    const size_t smem = generic_smem(dk, plan.cb), most = generic_smem(MAX_WIDTH, plan.cb);
#define RGLRU_GENERIC(IO) \
    (plan.cb == 2 ? (vec ? run_generic<IO, 2, 4>(plan, p, smem, most, st) : run_generic<IO, 2, 1>(plan, p, smem, most, st)) \
                  : (vec ? run_generic<IO, 4, 4>(plan, p, smem, most, st) : run_generic<IO, 4, 1>(plan, p, smem, most, st)))
    return io == RGLRU_F32 ? RGLRU_GENERIC(float) : RGLRU_GENERIC(__nv_bfloat16);
#undef RGLRU_GENERIC
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
    extern __shared__ __align__(16) float sm[];     // q, k [dk], then [256][VE] shares of o
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
    if (need_T ? s->dk > MAX_WIDTH || s->dv > MAX_WIDTH : s->dk > MAX_STEP_DK || s->dv > MAX_STEP_DV) return RGLRU_ERR_UNSUPPORTED;
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
// Whether two tensors of which each token's row is `row_a` and `row_b` elements long keep clear of one another: apart, or side by side in the same rows
bool clear_of(const MixTensor &a, size_t a_bytes, long long row_a, const MixTensor &b, size_t b_bytes, long long row_b, const rglru_linear_attention_shape_t *s) {
    if (!overlap(a.p, a_bytes, b.p, b_bytes)) return true;
    if ((uintptr_t)a.p > (uintptr_t)b.p) return clear_of(b, b_bytes, row_b, a, a_bytes, row_a, s);
    if ((s->T > 1 && a.token != b.token) || (s->B > 1 && a.batch != b.batch)) return false;
    const long long token = s->T > 1 ? a.token : LLONG_MAX, batch = s->B > 1 ? a.batch : LLONG_MAX;
    const long long inner = token < batch ? token : batch, outer = token < batch ? batch : token, rows = token < batch ? s->T : s->B;   // rows: of a run `inner` apart
    const long long off = (long long)(((uintptr_t)b.p - (uintptr_t)a.p) / io_bytes(s->io));
    if (off < row_a || off > inner - row_b) return false;
    return outer == LLONG_MAX || (rows - 1) * inner + off + row_b <= outer;   // b's last row ends before a's next run
}
const rglru_linear_attention_strides_t DENSE{};
size_t state_bytes(const rglru_linear_attention_shape_t *s) { return (size_t)s->B * s->H * s->dk * s->dv * sizeof(float); }
bool may_use_tensor_cores(const rglru_linear_attention_shape_t *s) {
    return !(s->flags & RGLRU_FLAG_FORCE_GENERIC) && s->io == RGLRU_BF16 && s->dk <= 128 && s->dv <= 128 && s->dk % 8 == 0 && s->dv % 8 == 0;
}
// Sums of stretches of cut sequences, by either kernel: a call's strides decide between them, its size must do for both
size_t sums_bytes(const rglru_linear_attention_shape_t *s, int roles) {
    const int wide = s->dk > s->dv ? s->dk : s->dv;
    const size_t generic = roles == 1 ? generic_plan(1, s->B, s->T, s->H, s->dk, s->dv).local_bytes : generic_plan(roles, s->B, s->T, s->H, wide, wide).local_bytes;
    const size_t tensor = may_use_tensor_cores(s) ? sm100_mix_bytes(roles, s->B, s->T, s->H) : 0;
    return generic > tensor ? generic : tensor;
}
cudaError_t run_mix(const rglru_linear_attention_shape_t *s, MixArgs &a, void *workspace, cudaStream_t st) {
    char *scratch = (char *)workspace + WS_HEADER_BYTES;
    const size_t sums = sums_bytes(s, a.roles);
    if (sums && a.role[0].s_in && a.role[0].s_in == a.role[0].s_out) {   // blocks that share a sequence all read its s0
        float *copy = (float *)(scratch + up256(sums));
        const cudaError_t e = cudaMemcpyAsync(copy, a.role[0].s_in, state_bytes(s), cudaMemcpyDeviceToDevice, st);
        if (e != cudaSuccess) return e;
        a.role[0].s_in = copy;
    }
    return may_use_tensor_cores(s) && sm100_mix_supported(a, s->io) ? sm100_mix(a, s->flags, scratch, st) : generic_mix(a, s->io, (float *)scratch, st);
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
    const size_t sums = sums_bytes(s, roles);
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
    const size_t mat = state_bytes(s), nd = (size_t)s->H * sizeof(float);
    if (overlap(o, no, log_decay, nd) || overlap(s_T, mat, log_decay, nd) || overlap(o, no, q, nq) || overlap(o, no, k, nk) || overlap(o, no, v, nv) || overlap(o, no, s0, mat) || overlap(s_T, mat, q, nq) ||
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
    const size_t io = io_bytes(s->io), nq = units * s->dk * io, nv = units * s->dv * io, ns = state_bytes(s), nd = (size_t)s->H * sizeof(float);
    if (overlap(o, nv, log_decay, nd) || overlap(state, ns, log_decay, nd) || overlap(o, nv, q, nq) || overlap(o, nv, k, nq) || overlap(o, nv, v, nv) || overlap(o, nv, state, ns) || overlap(state, ns, q, nq) ||
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
    size_t n[7];
    if (!place(q, st.q, s, s->dk, t[0], n[0]) || !place(k, st.k, s, s->dk, t[1], n[1]) || !place(v, st.v, s, s->dv, t[2], n[2]) ||
        !place(dout, st.o, s, s->dv, t[3], n[3]) || !place(dq, st.dq, s, s->dk, t[4], n[4]) || !place(dk, st.dk, s, s->dk, t[5], n[5]) ||
        !place(dv, st.dv, s, s->dv, t[6], n[6]))
        return RGLRU_ERR_SHAPE;
    if (workspace_bytes < rglru_linear_attention_workspace_bytes(s, RGLRU_OP_BACKWARD)) return RGLRU_ERR_WORKSPACE;
    const size_t mat = state_bytes(s);
    const void *const ins[7] = {q, k, v, dout, s0, ds_T, log_decay};
    const size_t in_bytes[7] = {n[0], n[1], n[2], n[3], mat, mat, (size_t)s->H * sizeof(float)};
    void *const outs[4] = {dq, dk, dv, ds0};
    const size_t out_bytes[4] = {n[4], n[5], n[6], mat};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 7; ++j)
            if (overlap(outs[i], out_bytes[i], ins[j], in_bytes[j])) return RGLRU_ERR_ALIAS;
    // dq, dk and dv may lie side by side in one gradient of a projection, tokens interleaved
    const long long rk = (long long)s->H * s->dk, rv = (long long)s->H * s->dv;
    if (!clear_of(t[4], n[4], rk, t[5], n[5], rk, s) || !clear_of(t[4], n[4], rk, t[6], n[6], rv, s) || !clear_of(t[5], n[5], rk, t[6], n[6], rv, s) || overlap(ds0, mat, dq, n[4]) || overlap(ds0, mat, dk, n[5]) || overlap(ds0, mat, dv, n[6])) return RGLRU_ERR_ALIAS;
    MixArgs a{};
    a.roles = 3; a.B = s->B; a.T = s->T; a.H = s->H; a.log_decay = log_decay; a.status = (uint32_t *)workspace;
    a.role[0] = MixRole{t[3], t[2], t[1], t[4], s->dv, s->dk, s0, nullptr, 1, 0, 1, s->scale, s->scale, 1.0f};
    a.role[1] = MixRole{t[2], t[3], t[0], t[5], s->dv, s->dk, ds_T, nullptr, 1, 1, 0, s->scale, 1.0f, s->scale};
    a.role[2] = MixRole{t[1], t[0], t[3], t[6], s->dk, s->dv, ds_T, ds0, 0, 1, 0, s->scale, 1.0f, s->scale};
    return call_status(run_mix(s, a, workspace, (cudaStream_t)cuda_stream));
}

}  // extern "C"
