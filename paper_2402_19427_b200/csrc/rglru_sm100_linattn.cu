// Linear attention with a decay for each head on tcgen05 tensor cores (bf16 io, widths up to 128; rglru_linattn.cuh has the mathematics).
//
// A block walks chunks of 128 tokens of a (role, sequence, head).  A chunk is four products with fp32 accumulators in tensor memory,
//     scores  P = q k^T                       [128 tokens x 128 tokens]
//     far     X = q S                         S: the state before the chunk, rounded to bf16 for this product alone
//     state   U = (decayed k)^T v             [dk x dv]
//     near    Y = (decayed, masked P) v
// and out = Y + decay X, S <- d^n S + U.  The state itself stays in fp32 registers from chunk to chunk.  It is an output of the call and
// has to be as exact as fp32 sums are, so the decayed k enters U as three bf16 values that add up to it; P and S enter once.
//
// Bound by memory: a chunk of 128 x 128 moves 128 KB, 3.0 us of an SM's share of the measured copy rate; the products take 1.7 us.  One block
// an SM: 224 KB of q, k, v, the planes of k and S.  Each tile is requested again as soon as its last reader is done: q after the
// far product, k after the scores and planes, v at the chunk's end.  Warps: four turn P into the operand of the near product (in tensor memory,
// over the scores) and write the outputs, eight make the planes and keep the state, one copies, one issues.
//
// Blocks share the chunks of all (role, sequence, head) evenly, in order; a block that begins inside a sequence takes the state before it
// from the sums that a first launch (planes and state product only) leaves for the stretches in front of it.
#include <cuda.h>
#include <cuda_bf16.h>

#include "rglru_linattn.cuh"
#include "sm100_ptx.cuh"

namespace rglru {
namespace {

using namespace ptx;

constexpr int CH = 128;                          // tokens a chunk
constexpr int P_WARPS = 4, S_WARPS = 8, THREADS = (P_WARPS + S_WARPS + 2) * 32;
constexpr uint32_t BLOCK = 128 * 128;            // 128 rows of 64 bf16
constexpr uint32_t SM_Q = 0, SM_K = 2 * BLOCK, SM_V = 4 * BLOCK, SM_PLANES = 6 * BLOCK, SM_S = 12 * BLOCK, SM_BAR = 14 * BLOCK;
enum { QF, KF, VF, QE, KE, VE, SC, PR, PL, VK, DSF, SR, OF, OE, TB, NBAR };
constexpr uint32_t SM_TMEM = SM_BAR + NBAR * 8, SM_TAB = SM_TMEM + 16, SM_BAD = SM_TAB + (32 + CH) * 4,
                   SM_TOTAL = SM_BAD + 3 * 132, SM_ALLOC = SM_TOTAL + 1024;
static_assert(SM_ALLOC <= 232448, "shared memory of a block");
constexpr uint32_t TM_P = 0, TM_Y = 128, TM_X = 256, TM_U = 384;   // tensor-memory columns
constexpr int WALKERS = 148;                     // the plan, and with it the workspace, does not depend on the device

struct WalkArgs {
    alignas(64) CUtensorMap tm[3][3];            // q, k, v of each role: [B][T][H][width]
    MixArgs m;
    int units, chunks;                           // (role, sequence, head), chunks of each
    int walkers;
    float *local;                                // [walkers][32][128][4] sums of stretches, or null: no sequence is cut
    unsigned long long spin_ns;
};
// chunks [first, last) of the walk that block w takes, counted over all units
__device__ __forceinline__ long long share(const WalkArgs &p, int w) { return (long long)p.units * p.chunks * w / p.walkers; }

struct Step {
    int role, b, h, chunk, n, t0;                // t0: the tile's first token in memory (negative where a reversed walk ends)
};
__device__ __forceinline__ Step step_at(const WalkArgs &p, long long g) {
    Step s;
    const int unit = (int)(g / p.chunks), bh = p.m.B * p.m.H;
    s.chunk = (int)(g % p.chunks);
    s.role = unit / bh;
    s.b = unit % bh / p.m.H;
    s.h = unit % p.m.H;
    s.n = min(CH, p.m.T - s.chunk * CH);
    s.t0 = p.m.role[s.role].reverse ? p.m.T - (s.chunk + 1) * CH : s.chunk * CH;
    return s;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ bool has_no_number(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// The values of a 16-byte piece of v that are no numbers become 0 in shared memory: a product would carry them into rows of tokens
// before theirs, as 0 * NaN.  Byte c of `bad` holds the first token (in walking order) from which on column c is NaN, 255: none.
__device__ __noinline__ void mend_piece(uint32_t addr, int column, uint32_t token, uint32_t *bad) {
    uint4 v = lds128(addr);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    for (int e = 0; e < 8; ++e) {
        const uint32_t half = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFFu;
        if ((half & 0x7F80u) != 0x7F80u) continue;
        w[e / 2] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        uint32_t *word = bad + (column + e) / 4;
        const int shift = (column + e) % 4 * 8;
        uint32_t old = *(volatile uint32_t *)word;
        while ((old >> shift & 255u) > token) {
            const uint32_t seen = atomicCAS(word, old, (old & ~(255u << shift)) | token << shift);
            if (seen == old) break;
            old = seen;
        }
    }
    sts128(addr, make_uint4(w[0], w[1], w[2], w[3]));
    *(volatile uint32_t *)(bad + 32) = 1u;
}

// STATE_ONLY: the sums U of a block's last stretch, for the blocks that go on in the same sequence
template <bool STATE_ONLY> __global__ void __launch_bounds__(THREADS, 1) mix_walk_kernel(const __grid_constant__ WalkArgs p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw), base = (raw_addr + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw_addr);
    auto BAR = [&](int i) { return base + SM_BAR + 8u * i; };
    uint32_t *tmem_base_s = (uint32_t *)(smem + SM_TMEM);
    volatile int *abort_flag = (volatile int *)(tmem_base_s + 1);
    float *tab = (float *)(smem + SM_TAB);
    uint32_t *bad_base = (uint32_t *)(smem + SM_BAD);   // [3][33] words, by the step: a byte for each column, and whether there is any
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned long long spin = p.spin_ns;

    if (tid == 0) {
        const int count[NBAR] = {1, 1, 1, 1, STATE_ONLY ? S_WARPS : S_WARPS + 1, 1, 1, P_WARPS, S_WARPS, S_WARPS, 1, S_WARPS, 1, P_WARPS, P_WARPS};
        for (int i = 0; i < NBAR; ++i) mbar_init(BAR(i), count[i]);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 3 * 33) bad_base[tid] = tid % 33 == 32 ? 0u : 0xFFFFFFFFu;
    if (warp == P_WARPS + S_WARPS + 1) { tmem_alloc(smem_u32(tmem_base_s), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_base_s;
    bool ok = true;
    dependency_wait();

    const long long last = share(p, blockIdx.x + 1);
    long long first = share(p, blockIdx.x);
    if (STATE_ONLY) {
        const long long begin = last / p.chunks * p.chunks;   // the unit that the share ends in
        first = begin > first ? begin : first;                // nothing to do if it ends with a unit: first == last
    }
    const int steps = (int)(last - first);

    if (warp == P_WARPS + S_WARPS) {
        // ---- copies
        if (lane == 0) {
            for (int s = 0; s < steps && ok; ++s) {
                const Step st = step_at(p, first + s);
                const MixRole &r = p.m.role[st.role];
                const int kb = r.dk > 64 ? 2 : 1, vb = r.dv > 64 ? 2 : 1;
                const uint32_t before = (s & 1) ^ 1;
                if (!STATE_ONLY) {
                    ok = mbar_wait(BAR(QE), before, spin, abort_flag);
                    if (!ok) break;
                    mbar_expect_tx(BAR(QF), kb * BLOCK);
                    for (int j = 0; j < kb; ++j) tma_load_4d(base + SM_Q + j * BLOCK, &p.tm[st.role][0], j * 64, st.h, st.t0, st.b, BAR(QF));
                }
                ok = mbar_wait(BAR(KE), before, spin, abort_flag);
                if (!ok) break;
                mbar_expect_tx(BAR(KF), kb * BLOCK);
                for (int j = 0; j < kb; ++j) tma_load_4d(base + SM_K + j * BLOCK, &p.tm[st.role][1], j * 64, st.h, st.t0, st.b, BAR(KF));
                ok = mbar_wait(BAR(VE), before, spin, abort_flag);
                if (!ok) break;
                mbar_expect_tx(BAR(VF), vb * BLOCK);
                for (int j = 0; j < vb; ++j) tma_load_4d(base + SM_V + j * BLOCK, &p.tm[st.role][2], j * 64, st.h, st.t0, st.b, BAR(VF));
            }
            if (!ok) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
        }
    } else if (warp == P_WARPS + S_WARPS + 1) {
        // ---- products
        if (lane == 0) {
            for (int s = 0; s < steps && ok; ++s) {
                const Step st = step_at(p, first + s);
                const MixRole &r = p.m.role[st.role];
                const int ks = r.dk > 64 ? 8 : 4;
                const uint32_t ph = s & 1, nv = r.dv > 64 ? 128 : 64;
                const uint32_t id_p = make_idesc(128, 128), id_b = make_idesc(128, nv) | (1u << 16), id_ab = id_b | (1u << 15);
                auto wait = [&](int bar, uint32_t parity) { ok = ok && mbar_wait(BAR(bar), parity, spin, abort_flag); };
                if (!STATE_ONLY) {
                    wait(QF, ph); wait(KF, ph);
                    if (!ok) break;
                    tc_fence_after();
                    for (int k = 0; k < ks; ++k) {
                        const uint32_t off = (k >> 2) * BLOCK + (k & 3) * 32;
                        mma_ss(tmem + TM_P, make_desc_sw128(base + SM_Q + off), make_desc_sw128(base + SM_K + off), id_p, k != 0);
                    }
                    tc_commit(BAR(SC));
                    tc_commit(BAR(KE));
                    wait(SR, ph); wait(OE, ph ^ 1);
                    if (!ok) break;
                    tc_fence_after();
                    for (int k = 0; k < ks; ++k)   // S as it lies: a row of 64 columns of v, 128 rows a block
                        mma_ss(tmem + TM_X, make_desc_sw128(base + SM_Q + (k >> 2) * BLOCK + (k & 3) * 32), make_desc_sw128_mn(base + SM_S + k * 2048, BLOCK), id_b, k != 0);
                    tc_commit(BAR(QE));
                } else {
                    wait(SR, ph);
                    if (!ok) break;
                }
                wait(PL, ph); wait(VK, ph);
                if (!ok) break;
                tc_fence_after();
                for (int pl = 2; pl >= 0; --pl)   // the smallest first
                    for (int k = 0; k < 8; ++k)
                        mma_ss(tmem + TM_U, make_desc_sw128_mn(base + SM_PLANES + pl * 2 * BLOCK + k * 2048, BLOCK), make_desc_sw128_mn(base + SM_V + k * 2048, BLOCK), id_ab,
                               (pl != 2) | (k != 0));
                tc_commit(BAR(DSF));
                if (!STATE_ONLY) {
                    wait(PR, ph);
                    if (!ok) break;
                    tc_fence_after();
                    for (int k = 0; k < 8; ++k)
                        mma_ts(tmem + TM_Y, tmem + TM_P + k * 8, make_desc_sw128_mn(base + SM_V + k * 2048, BLOCK), id_b, k != 0);
                    tc_commit(BAR(OF));
                }
                tc_commit(BAR(VE));
            }
            if (!ok) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
        }
    } else if (warp < P_WARPS) {
        // ---- scores to weights, outputs: a thread has a row (a token)
        if (!STATE_ONLY) {
            const int row = warp * 32 + lane;
            const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
            int unit = -1, tables = 0;
            for (int s = 0; s < steps && ok; ++s) {
                const Step st = step_at(p, first + s);
                const MixRole &r = p.m.role[st.role];
                const uint32_t ph = s & 1;
                const int now = (st.role * p.m.B + st.b) * p.m.H + st.h;
                if (now != unit) {   // tab[32 + e] = sp decay^e; e < 0 is looked at in the pieces on the diagonal, but not used
                    // (the old table has been read: the last outputs waited for all four warps' weights)
                    for (int i = tid; i < 32 + CH; i += P_WARPS * 32) tab[i] = i < 32 ? 0.0f : r.sp * decay_power(p.m.log_decay[st.h], (float)(i - 32));
                    __syncwarp();
                    if (lane == 0) mbar_arrive(BAR(TB));
                    ok = warp_wait(BAR(TB), tables++ & 1, spin, abort_flag);
                    if (!ok) break;
                    unit = now;
                }
                ok = warp_wait(BAR(SC), ph, spin, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const int own = r.reverse ? P_WARPS - 1 - warp : warp;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    const int cw = r.reverse ? 3 - c : c;   // the 32 columns' place in walking order
                    f32x2 x[8];
                    uint32_t w[16];
                    if (cw > own) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = 0u;
                    } else {
                        f32x2 v[16];
                        tmem_ld32(lanes + TM_P + c * 32, v);
                        tmem_ld_wait();
                        const float *t = tab + 32 + (r.reverse ? c * 32 - row : row - c * 32);
                        if (cw == own) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) {   // chosen, not multiplied by 0: what is masked may be no number
                                const float w0 = r.reverse ? t[2 * j] : t[-2 * j], w1 = r.reverse ? t[2 * j + 1] : t[-2 * j - 1];
                                const int e0 = r.reverse ? c * 32 + 2 * j - row : row - c * 32 - 2 * j, e1 = r.reverse ? e0 + 1 : e0 - 1;
                                w[j] = pack_bf16(e0 >= 0 ? v[j].x * w0 : 0.0f, e1 >= 0 ? v[j].y * w1 : 0.0f);
                            }
                        } else if (r.reverse) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[j].x * t[2 * j], v[j].y * t[2 * j + 1]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[j].x * t[-2 * j], v[j].y * t[-2 * j - 1]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
                    // A forward walk overwrites columns that it has read; a reversed one as well: piece c ends at column 16 c + 15
                    tmem_st16(lanes + TM_P + c * 16, x);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(BAR(PR));

                ok = warp_wait(BAR(OF), ph, spin, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const int t = st.t0 + row, i = r.reverse ? CH - 1 - row : row;
                const bool live = t >= 0 && t < p.m.T;
                const float far = r.si * decay_power(p.m.log_decay[st.h], (float)(i + r.first));
                const uint8_t *bad = (const uint8_t *)(bad_base + s % 3 * 33);
                const bool any_bad = *(volatile const uint32_t *)(bad + 128) != 0;
                __nv_bfloat16 *out = (__nv_bfloat16 *)r.o.p + st.b * r.o.batch + t * r.o.token + (long long)st.h * r.dv;
#pragma unroll 1
                for (int c = 0; c < r.dv; c += 32) {
                    f32x2 y[16], x[16];
                    tmem_ld32(lanes + TM_Y + c, y);
                    tmem_ld32(lanes + TM_X + c, x);
                    tmem_ld_wait();
                    if (c + 32 >= r.dv && !any_bad) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(BAR(OE));
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) y[j] = fma2(x[j], pack2(far, far), y[j]);
                    if (any_bad) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            if (i >= bad[c + 2 * j]) y[j].x = __int_as_float(0x7FC00000);
                            if (i >= bad[c + 2 * j + 1]) y[j].y = __int_as_float(0x7FC00000);
                        }
                    }
                    if (live) {
#pragma unroll
                        for (int h = 0; h < 4; ++h)
                            if (c + 8 * h < r.dv)
                                *(uint4 *)(out + c + 8 * h) = make_uint4(pack_bf16(y[4 * h].x, y[4 * h].y), pack_bf16(y[4 * h + 1].x, y[4 * h + 1].y),
                                                                        pack_bf16(y[4 * h + 2].x, y[4 * h + 2].y), pack_bf16(y[4 * h + 3].x, y[4 * h + 3].y));
                    }
                }
                if (any_bad) {   // the list is read to its end before it may be cleared
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(BAR(OE));
                }
            }
            if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
        }
    } else {
        // ---- planes of the decayed k, and the state: a thread has row d of S and 64 columns
        const int st_tid = tid - P_WARPS * 32, q = warp & 3, e0 = (warp - P_WARPS) / 4 * 64, d = q * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
        float S[64];
        auto init_state = [&](const Step &st, long long g) {
            const MixRole &r = p.m.role[st.role];
            const long long mat = (long long)(st.b * p.m.H + st.h) * r.dk * r.dv;
            const float *src = STATE_ONLY ? nullptr : r.s_in;
#pragma unroll
            for (int j = 0; j < 64; ++j) S[j] = 0.0f;
            if (src && d < r.dk) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (e0 + j < r.dv) S[j] = src[mat + (r.turned ? (long long)(e0 + j) * r.dk + d : (long long)d * r.dv + e0 + j)];
            }
            if (!STATE_ONLY && st.chunk != 0) {   // the stretches in front of this one, block by block
                const long long begin = g - st.chunk;
                int w = (int)(begin * p.walkers / ((long long)p.units * p.chunks));
                while (share(p, w + 1) <= begin) ++w;
                for (; w < (int)blockIdx.x; ++w) {
                    const long long from = share(p, w) > begin ? share(p, w) : begin, to = share(p, w + 1);
                    const float f = decay_power(p.m.log_decay[st.h], (float)((to - from) * CH));
                    const float4 *l = (const float4 *)p.local + ((size_t)w * 32 + e0 / 4) * 128 + d;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float4 v = l[j * 128];
                        S[4 * j] = fmaf(f, S[4 * j], v.x); S[4 * j + 1] = fmaf(f, S[4 * j + 1], v.y);
                        S[4 * j + 2] = fmaf(f, S[4 * j + 2], v.z); S[4 * j + 3] = fmaf(f, S[4 * j + 3], v.w);
                    }
                }
            }
        };
        // S to shared memory for the far product: rows of 64 columns, 16-byte pieces swizzled as a tiled copy would have them
        auto hand_over = [&]() {
            if (!STATE_ONLY) {
                const uint32_t row = base + SM_S + (e0 / 64) * BLOCK + d * 128;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    sts128(row + ((j ^ (d & 7)) << 4), make_uint4(pack_bf16(S[8 * j], S[8 * j + 1]), pack_bf16(S[8 * j + 2], S[8 * j + 3]),
                                                                 pack_bf16(S[8 * j + 4], S[8 * j + 5]), pack_bf16(S[8 * j + 6], S[8 * j + 7])));
                fence_async_smem();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(SR));
        };
        int unit = -1, n_tokens = 0;
        float w[4] = {}, f = 0.0f;   // weights of this thread's rows of k, st_tid / 8 + 32 i; the state's
        if (steps > 0) {
            init_state(step_at(p, first), first);
            hand_over();
        }
        for (int s = 0; s < steps && ok; ++s) {
            const Step st = step_at(p, first + s);
            const MixRole &r = p.m.role[st.role];
            const uint32_t ph = s & 1;
            const int now = (st.role * p.m.B + st.b) * p.m.H + st.h;
            uint32_t *bad = bad_base + s % 3 * 33;
            if (now != unit || st.n != n_tokens) {
                const float ld = p.m.log_decay[st.h];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = (st_tid >> 3) + 32 * i, j = r.reverse ? CH - 1 - row : row;
                    w[i] = j < st.n ? decay_power(ld, (float)(st.n - j - r.first)) : 0.0f;
                }
                f = decay_power(ld, (float)st.n);
                unit = now;
                n_tokens = st.n;
            }
            ok = warp_wait(BAR(KF), ph, spin, abort_flag);
            if (!ok) break;
            const int blocks = r.dk > 64 ? 2 : 1;
#pragma unroll 1
            for (int b = 0; b < blocks; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = b * (int)(BLOCK / 16) + k * S_WARPS * 32 + st_tid;
                const uint4 v = lds128(base + SM_K + i * 16);
                const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                uint32_t hi[4], mid[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x2 x = mul2(bf2x(in[e]), pack2(w[k], w[k]));
                    hi[e] = pack_bf16(x.x, x.y);
                    const f32x2 h = bf2x(hi[e]), y = make_float2(x.x - h.x, x.y - h.y);
                    mid[e] = pack_bf16(y.x, y.y);
                    const f32x2 m = bf2x(mid[e]);
                    lo[e] = pack_bf16(y.x - m.x, y.y - m.y);
                }
                const uint32_t dst = base + SM_PLANES + i * 16;
                sts128(dst, make_uint4(hi[0], hi[1], hi[2], hi[3]));
                sts128(dst + 2 * BLOCK, make_uint4(mid[0], mid[1], mid[2], mid[3]));
                sts128(dst + 4 * BLOCK, make_uint4(lo[0], lo[1], lo[2], lo[3]));
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) { mbar_arrive(BAR(PL)); mbar_arrive(BAR(KE)); }
            ok = warp_wait(BAR(VF), ph, spin, abort_flag);
            if (!ok) break;
            const int vpieces = (r.dv > 64 ? 2 : 1) * (int)(BLOCK / 16);
#pragma unroll 4
            for (int i = st_tid; i < vpieces; i += S_WARPS * 32) {
                const uint4 v = lds128(base + SM_V + i * 16);
                if (has_no_number(v.x) || has_no_number(v.y) || has_no_number(v.z) || has_no_number(v.w)) {
                    const int row = (i >> 3) & 127, column = (i >> 10) * 64 + ((i & 7) ^ (row & 7)) * 8;
                    mend_piece(base + SM_V + i * 16, column, (uint32_t)(r.reverse ? CH - 1 - row : row), bad);
                    fence_async_smem();
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(VK));

            ok = warp_wait(BAR(DSF), ph, spin, abort_flag);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
                f32x2 u[16];
                if (e0 + c < r.dv) {
                    tmem_ld32(lanes + TM_U + e0 + c, u);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) { S[c + 2 * j] = fmaf(f, S[c + 2 * j], r.su * u[j].x); S[c + 2 * j + 1] = fmaf(f, S[c + 2 * j + 1], r.su * u[j].y); }
                }
            }
            if (*(volatile uint32_t *)(bad + 32)) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (((const uint8_t *)bad)[e0 + j] != 255) S[j] = __int_as_float(0x7FC00000);
            }
            // The list of the step before this one has been read: the outputs by OE and the states by SR, which this state product waited
            // for.  It serves again in two steps, whose state product waits for this warp's SR.
            if (warp == P_WARPS && s > 0) {
                uint32_t *old = bad_base + (s - 1) % 3 * 33;
                if (*(volatile uint32_t *)(old + 32)) {
                    old[lane] = 0xFFFFFFFFu;
                    __syncwarp();
                    if (lane == 0) old[32] = 0u;
                }
            }
            if (!STATE_ONLY && st.chunk == p.chunks - 1 && r.s_out && d < r.dk) {
                float *dst = r.s_out + (long long)(st.b * p.m.H + st.h) * r.dk * r.dv + (long long)d * r.dv + e0;
#pragma unroll
                for (int j = 0; j < 64; j += 4)
                    if (e0 + j < r.dv) *(float4 *)(dst + j) = make_float4(S[j], S[j + 1], S[j + 2], S[j + 3]);
            }
            if (s + 1 < steps) {
                if (st.chunk == p.chunks - 1) init_state(step_at(p, first + s + 1), first + s + 1);
                if (!STATE_ONLY) ok = warp_wait(BAR(QE), ph, spin, abort_flag);   // the far product has read S
                if (!ok) break;
                hand_over();
            }
        }
        if (STATE_ONLY && steps > 0 && ok) {
            float4 *l = (float4 *)p.local + ((size_t)blockIdx.x * 32 + e0 / 4) * 128 + d;
#pragma unroll
            for (int j = 0; j < 16; ++j) l[j * 128] = make_float4(S[4 * j], S[4 * j + 1], S[4 * j + 2], S[4 * j + 3]);
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
    }
    dependency_trigger();
    if (*abort_flag) {   // let copies and MMAs in flight land before shared and tensor memory are given back
        const uint64_t tw = gtimer();
        while (gtimer() - tw < 50000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == P_WARPS + S_WARPS + 1) tmem_dealloc(tmem, 512);
}

// Blocks: one a (role, sequence, head) while that is as fast, else 148 with equal shares.  In chunks: a block's own, and for cut
// sequences half of its last stretch again (state only) and some four for the second launch and the states read.
int plan_walkers(int roles, int B, int T, int H) {
    const long long units = (long long)roles * B * H, chunks = (T + CH - 1) / CH, all = units * chunks;
    const long long whole = (units + WALKERS - 1) / WALKERS * chunks;
    const long long share = (all + WALKERS - 1) / WALKERS, cut = share + (share < chunks ? share : chunks / 2) / 2 + 4;
    return whole <= cut || all < WALKERS ? (int)units : WALKERS;
}

}  // namespace

bool sm100_mix_supported(const MixArgs &a, int io) {
    if (io != RGLRU_BF16) return false;
    for (int i = 0; i < a.roles; ++i) {
        const MixRole &r = a.role[i];
        if (r.dk > 128 || r.dv > 128 || r.dk % 8 || r.dv % 8) return false;
        for (const MixTensor *t : {&r.q, &r.k, &r.v, &r.o})
            if ((a.T > 1 && t->token % 8) || (a.B > 1 && t->batch % 8)) return false;
    }
    return true;
}

size_t sm100_mix_bytes(int roles, int B, int T, int H) {
    const int w = plan_walkers(roles, B, T, H);
    return w == roles * B * H ? 0 : (size_t)w * 128 * 128 * sizeof(float);
}

cudaError_t sm100_mix(const MixArgs &a, void *scratch, cudaStream_t st) {
    WalkArgs p{};
    p.m = a;
    p.units = a.roles * a.B * a.H;
    p.chunks = (a.T + CH - 1) / CH;
    p.walkers = plan_walkers(a.roles, a.B, a.T, a.H);
    const bool cut = p.walkers != p.units;
    p.local = cut ? (float *)scratch : nullptr;
    p.spin_ns = g_spin_limit_ns;
    for (int i = 0; i < a.roles; ++i) {
        const MixRole &r = a.role[i];
        const MixTensor *t[3] = {&r.q, &r.k, &r.v};
        for (int j = 0; j < 3; ++j) {
            const uint64_t w = j < 2 ? r.dk : r.dv;
            // an axis of one element has no distance: any valid one
            const uint64_t token = a.T > 1 ? t[j]->token : w * a.H, batch = a.B > 1 ? t[j]->batch : w * a.H;
            const uint64_t dims[4] = {w, (uint64_t)a.H, (uint64_t)a.T, (uint64_t)a.B}, strides[3] = {w * 2, token * 2, batch * 2};
            const uint32_t box[4] = {64, 1, CH, 1};
            if (!encode_map16_4d(&p.tm[i][j], t[j]->p, dims, strides, box, true)) return cudaErrorNotSupported;
        }
    }
    static PerDeviceOptIn opt_main, opt_state;
    cudaError_t e = opt_main.ensure(mix_walk_kernel<false>, (int)SM_ALLOC);
    if (e == cudaSuccess && cut) e = opt_state.ensure(mix_walk_kernel<true>, (int)SM_ALLOC);
    if (e == cudaSuccess && cut) e = launch_dependent(mix_walk_kernel<true>, dim3(p.walkers), dim3(THREADS), SM_ALLOC, st, p);
    if (e == cudaSuccess) e = launch_dependent(mix_walk_kernel<false>, dim3(p.walkers), dim3(THREADS), SM_ALLOC, st, p);
    return e;
}

}  // namespace rglru
