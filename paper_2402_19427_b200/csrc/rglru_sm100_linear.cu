// The products of the projection on tcgen05 tensor cores: out[m][n] = epilogue(sum_k A(m,k) B(n,k)), for the forward (both operands with K
// innermost), dx (B along its rows) and dW (both along their rows).
//
// A cluster of two CTAs shares a tile of 256 x NT results (cta_group::2): each holds 128 rows of A and NT/2 rows of B of a 64-wide K block
// in shared memory, so that an operand byte is fetched from L2 once for 256 rows, and its 128 rows of the accumulator in tensor memory, in
// two buffers: the epilogue of one tile runs beside the products of the next.  Products of few tokens have the weights as A and the
// tokens as B (a tile of 256 outputs and 32 to 128 tokens), and K split over the SMs: they are bound by reading the weights.
//
// 16384 x 2560 x 2560 in bf16 takes 143 us (1500 TFLOP/s, the tensor pipe 89 % busy), with GeLU and the pre-activation 159; dx 143, dW 148; dW of 131072 rows 1201.  Narrow
// tiles are bound by their copies out of L2, 52 to 55 bytes a cycle and SM.
//
// fp32 operands are sums of three bf16 values; six of the nine products of those reach fp32's accuracy (what is left out is at
// most 2^-24 of a term).  The tensor core adds up by cutting off, so an accumulator takes 256 terms and the epilogue's warps add up what it
// held in registers.  Infinite operands are infinite in one product only: the first plane appears twice, once with zeros in
// the place of what is not finite, so that inf * w is what it is for w and not what the planes of w make of it.
#include <cuda.h>
#include <cuda_bf16.h>

#include "rglru_linear.cuh"

namespace rglru {
namespace {

using namespace ptx;

constexpr int THREADS = 352;              // a warp for A's copies, one for the products, one for B's copies, eight for the epilogue
constexpr uint32_t A_BYTES = 128 * 128, RING = 7 * 2 * A_BYTES;   // a CTA's 128 rows of a K block of 64 bf16; all stages
constexpr int MAX_STAGES = 12;            // a stage is A_BYTES and 64 NT bytes of B: 7 of NT = 256, 12 of NT = 32
constexpr uint32_t MN_BLOCK = 64 * 128;   // one copy of 64 K rows x 64 values of an operand turned
constexpr uint32_t TURN = 2 * A_BYTES;   // the ring's last bytes where rows start at any byte: 4 KB for each of the epilogue's warps to turn results in
constexpr uint32_t SMEM_BAR = RING;
constexpr uint32_t SMEM_TOTAL = SMEM_BAR + (2 * MAX_STAGES + 4) * 8 + 16, SMEM_ALLOC = SMEM_TOTAL + 1024;
constexpr int PAIRS = 74;                 // the plan, and with it the workspace, does not depend on the device
constexpr int PLANES = 4, PRODUCTS = 6;   // fp32: nearest, the same with zeros for what is not finite, second, third
__device__ constexpr uint8_t PLANE_A[PRODUCTS] = {3, 1, 2, 2, 1, 0}, PLANE_B[PRODUCTS] = {1, 3, 2, 1, 2, 0};

struct GemmArgs {
    alignas(64) CUtensorMap tm_a, tm_b;   // [planes][rows][cols]
    int a_turned, b_turned, split_planes; // split_planes: six products of planes instead of one
    int M, N, NT, nx, ny;                 // tiles: nx along M, ny along N
    int kblocks, vblocks;                 // vblocks: K blocks over all products
    int stages;
    int whole, splits, per_split;         // tiles whose K is one pair's work; of the others each is split
    long long out_m, out_n;               // distances between results along M and N
    int wide;                             // bytes a thread may store at once along N (32, 16, or 0: one value)
    LinearEpilogue e;
    float *part;                          // [tile - whole][split][256 x NT] fp32, along the results' innermost dimension
    float *carry;                         // [CTA][NT][128] fp32: what a tile's earlier accumulators held (bf16, long K), or null
    uint32_t *status;
    unsigned long long spin_ns;
    int b_never_comes;                    // test hook of the waits' limits
};

template <typename IO> __device__ __forceinline__ void finish_one(const LinearEpilogue &e, long long o, float z) {
    if (e.preact) put<IO>(e.preact, o, z);
    put<IO>(e.y, o, activate<sizeof(IO) == 2>(z, e.activation) + (e.residual ? at<IO>(e.residual, o) : 0.0f));
}
// 32 neighbouring results of row m, v, to their place: a thread has a row, and writes whole sectors of it
template <typename IO> __device__ __forceinline__ void finish_row(const GemmArgs &p, long long m, int n0, float *v) {
    const long long o = m * p.out_m + n0;
    const LinearEpilogue &e = p.e;
    auto store_f32 = [&](float *dst) {
#pragma unroll
        for (int j = 0; j < 8; ++j) *(float4 *)(dst + 4 * j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    };
    if (n0 + 32 > p.N) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (n0 + j >= p.N) continue;
            finish_one<IO>(e, o + j, v[j] + (e.bias ? e.bias[n0 + j] : 0.0f));
        }
        return;
    }
    if (e.bias) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float4 b = *(const float4 *)(e.bias + n0 + 4 * j);
            v[4 * j] += b.x; v[4 * j + 1] += b.y; v[4 * j + 2] += b.z; v[4 * j + 3] += b.w;
        }
    }
    auto store = [&](void *to) {
        if constexpr (sizeof(IO) == 4) {
            store_f32((float *)to + o);
        } else {
            __nv_bfloat16 *dst = (__nv_bfloat16 *)to + o;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = pack_bf16(v[16 * h + 2 * j], v[16 * h + 2 * j + 1]);
                if (p.wide == 32) {
                    st_global_v8(dst + 16 * h, w);
                } else {
                    *(uint4 *)(dst + 16 * h) = make_uint4(w[0], w[1], w[2], w[3]);
                    *(uint4 *)(dst + 16 * h + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
        }
    };
    if (e.preact) store(e.preact);
    if (e.activation != RGLRU_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            if constexpr (sizeof(IO) == 2) {
                const float2 y = activate_fast(make_float2(v[j], v[j + 1]), e.activation);
                v[j] = y.x; v[j + 1] = y.y;
            } else {
                v[j] = activate<false>(v[j], e.activation); v[j + 1] = activate<false>(v[j + 1], e.activation);
            }
        }
    }
    if (e.residual) {
        constexpr int VE = 16 / sizeof(IO);
#pragma unroll
        for (int j = 0; j < 32; j += VE) {
            float r[VE];
            LinearVec<IO, VE>::load((const IO *)e.residual + o + j, r);
#pragma unroll
            for (int i = 0; i < VE; ++i) v[j + i] += r[i];
        }
    }
    store(e.y);
}
// The warp's 32 x 32 results where rows start at any byte: turned in shared memory, so that lanes write side by side (a thread's row in pieces of one
// value took 100 us where this takes 31: 4097 x 1001 to 1531)
template <typename IO> __device__ __forceinline__ void finish_turned(const GemmArgs &p, long long m0, int n0, int lane, const float *v, float *turn) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 32; ++j) turn[lane * 32 + (j ^ lane)] = v[j];
    __syncwarp();
    const int n = n0 + lane;
    if (n >= p.N) return;
    const float b = p.e.bias ? p.e.bias[n] : 0.0f;
    const int rows = (int)min(32ll, p.M - m0);
#pragma unroll 4
    for (int i = 0; i < rows; ++i) finish_one<IO>(p.e, (m0 + i) * p.out_m + n, turn[i * 32 + (lane ^ i)] + b);
}
// 32 results of row m where neighbouring rows are neighbours in memory (tokens along N): lanes write side by side
template <typename IO> __device__ __forceinline__ void finish_column(const GemmArgs &p, long long m, int n0, const float *v) {
    const float b = p.e.bias ? p.e.bias[m] : 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (n0 + j >= p.N) continue;
        const long long o = m + (n0 + j) * p.out_n;
        finish_one<IO>(p.e, o, v[j] + b);
    }
}

// The tensor core cuts off what does not fit the sum so far, so an accumulator takes a limited number of terms.  fp32 io: it is emptied into registers every
// DRAIN_BLOCKS K blocks (NT <= 128).  bf16: 16384 terms (some 2^-13 of the sum at worst, a sixteenth of the result's own half step), then its sum goes
// on in fp32 in the block's place in `carry`, which a thread writes and reads back alone: 128 KB a CTA, out of L2, every 256 K blocks (131072 rows of 2560 x 2560: 1430 TFLOP/s, 16384 rows 1450).
constexpr int DRAIN_BLOCKS = 4, LONG_BLOCKS = 256;
template <typename IO> __global__ void __launch_bounds__(THREADS, 1) linear_gemm_kernel(const __grid_constant__ GemmArgs p) {
    constexpr bool DRAIN = sizeof(IO) == 4;
    constexpr int TAKE = DRAIN ? DRAIN_BLOCKS : LONG_BLOCKS;   // K blocks of an accumulator
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw), base = (raw_addr + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw_addr);
    const uint32_t bar0 = base + SMEM_BAR;
    auto BAR_FULL = [&](int s) { return bar0 + 8u * s; };
    auto BAR_EMPTY = [&](int s) { return bar0 + 8u * (MAX_STAGES + s); };
    auto BAR_ACCFULL = [&](int a) { return bar0 + 8u * (2 * MAX_STAGES + a); };
    auto BAR_ACCEMPTY = [&](int a) { return bar0 + 8u * (2 * MAX_STAGES + 2 + a); };
    uint32_t *tmem_base_s = (uint32_t *)(smem + SMEM_BAR + (2 * MAX_STAGES + 4) * 8);
    volatile int *abort_flag = (volatile int *)(tmem_base_s + 1);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    const unsigned long long spin = p.spin_ns;
    const int ntiles = p.whole + (p.nx * p.ny - p.whole) * p.splits, pair = blockIdx.x >> 1, npairs = gridDim.x >> 1, stages = p.stages;
    const uint32_t stage_bytes = A_BYTES + (uint32_t)p.NT * 64u;

    if (tid == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(BAR_FULL(s), 1); mbar_init(BAR_EMPTY(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(BAR_ACCFULL(a), 1); mbar_init(BAR_ACCEMPTY(a), 16); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) { tmem_alloc2(smem_u32(tmem_base_s), 512); tmem_relinquish2(); }
    if (warp == 0 && lane == 0) { prefetch_tensormap(&p.tm_a); prefetch_tensormap(&p.tm_b); }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = *tmem_base_s;
    bool ok = true;
    dependency_wait();

    // unit of work -> (m, n, K blocks); n fastest, so that the pairs at work at a time share rows of A
    struct Tile { int m, n, v0, v1, part; };
    auto tile_at = [&](int t) {
        if (t < p.whole) return Tile{t / p.ny * 256, t % p.ny * p.NT, 0, p.vblocks, -1};
        const int u = t - p.whole, s = u % p.splits, xy = p.whole + u / p.splits;
        return Tile{xy / p.ny * 256, xy % p.ny * p.NT, s * p.per_split, min(p.vblocks, (s + 1) * p.per_split), p.splits > 1 ? u : -1};
    };

    if (warp == 0 || warp == 2) {
        // (a copy takes its thread some 120 cycles: one thread for both operands would be slower than the products of a narrow tile)
        if (elect_one() && !(warp == 2 && p.b_never_comes)) {
            int s = 0;   // stage of the ring, and its turn
            uint32_t turn = 0;
            const int brows = p.NT / 2;
            const uint32_t tx = 2 * (A_BYTES + (uint32_t)brows * 128u);   // both CTAs' bytes
            for (int t = pair; t < ntiles && ok; t += npairs) {
                const Tile tl = tile_at(t);
                const int ma = tl.m + (int)rank * 128, nb = tl.n + (int)rank * brows;
                for (int v = tl.v0; v < tl.v1; ++v) {
                    ok = mbar_wait_spin(BAR_EMPTY(s), turn ^ 1, spin, abort_flag);
                    if (!ok) break;
                    if (warp == 0 && rank == 0) mbar_expect_tx(BAR_FULL(s), tx);
                    const int prod = p.split_planes ? v / p.kblocks : 0, k0 = (v - prod * p.kblocks) * 64;
                    const int pa = p.split_planes ? PLANE_A[prod] : 0, pb = p.split_planes ? PLANE_B[prod] : 0;
                    const uint32_t a_dst = base + s * stage_bytes, b_dst = a_dst + A_BYTES;
                    if (warp == 0) {
                        tma_load_3d_pair(a_dst, &p.tm_a, p.a_turned ? ma : k0, p.a_turned ? k0 : ma, pa, BAR_FULL(s));
                        if (p.a_turned) tma_load_3d_pair(a_dst + MN_BLOCK, &p.tm_a, ma + 64, k0, pa, BAR_FULL(s));
                    } else {
                        tma_load_3d_pair(b_dst, &p.tm_b, p.b_turned ? nb : k0, p.b_turned ? k0 : nb, pb, BAR_FULL(s));
                        if (p.b_turned && brows > 64) tma_load_3d_pair(b_dst + MN_BLOCK, &p.tm_b, nb + 64, k0, pb, BAR_FULL(s));
                    }
                    if (++s == stages) { s = 0; turn ^= 1; }
                }
            }
            if (!ok) { *abort_flag = 1; atomicExch(p.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = make_idesc(256, p.NT) | (uint32_t)p.a_turned << 15 | (uint32_t)p.b_turned << 16;
            // 16 of K an instruction: 32 bytes along a row, or 16 rows (descriptors count in units of 16 bytes)
            const uint64_t a0 = p.a_turned ? make_desc_sw128_mn(base, MN_BLOCK) : make_desc_sw128(base), a_step = p.a_turned ? 128 : 2;
            const uint64_t b0 = p.b_turned ? make_desc_sw128_mn(base + A_BYTES, MN_BLOCK) : make_desc_sw128(base + A_BYTES), b_step = p.b_turned ? 128 : 2;
            int s = 0, it = 0;   // it: accumulators begun
            uint32_t turn = 0;
            for (int t = pair; t < ntiles && ok; t += npairs) {
                const Tile tl = tile_at(t);
                for (int v = tl.v0; v < tl.v1 && ok; ++v) {
                    const int within = (v - tl.v0) % TAKE, acc = it & 1;
                    if (within == 0) ok = mbar_wait_spin(BAR_ACCEMPTY(acc), ((it >> 1) & 1) ^ 1, spin, abort_flag);
                    ok = ok && mbar_wait_spin(BAR_FULL(s), turn, spin, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t at = (uint64_t)s * (stage_bytes / 16), da = a0 + at, db = b0 + at;
                    const uint32_t d = tmem + acc * 256;
                    mma_ss2(d, da, db, idesc, within != 0);
#pragma unroll
                    for (int k = 1; k < 4; ++k) mma_ss2(d, da + k * a_step, db + k * b_step, idesc, 1);
                    tc_commit2(BAR_EMPTY(s), 3);
                    if (v + 1 == tl.v1 || within + 1 == TAKE) { tc_commit2(BAR_ACCFULL(acc), 3); ++it; }
                    if (++s == stages) { s = 0; turn ^= 1; }
                }
            }
            if (!ok) { *abort_flag = 1; atomicExch(p.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
        }
    } else {
        const int q = warp & 3, half = (warp - 3) >> 2;   // tensor-memory lanes 32 q .. + 31, every other 32 columns
        int it = 0;
        for (int t = pair; t < ntiles && ok; t += npairs) {
            const Tile tl = tile_at(t);
            const long long m = tl.m + (long long)rank * 128 + q * 32 + lane;
            const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
            auto finish = [&](int n0, float *v) {
                if (n0 >= p.N) return;
                if (tl.part < 0 && p.out_n == 1 && !p.wide) {
                    finish_turned<IO>(p, m - lane, n0, lane, v, (float *)(smem + RING - TURN) + (warp - 3) * 1024);
                    return;
                }
                if (m >= p.M) return;
                if (tl.part >= 0) {   // partial sums: whole tiles, in the order that the results have
                    const int row = (int)(m - tl.m), col = n0 - tl.n;
                    float *to = p.part + (size_t)tl.part * 256 * p.NT;
                    if (p.out_n == 1) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) *(float4 *)(to + row * p.NT + col + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) to[(col + j) * 256 + row] = v[j];
                    }
                } else if (p.out_n == 1) {
                    finish_row<IO>(p, m, n0, v);
                } else {
                    finish_column<IO>(p, m, n0, v);
                }
            };
            if constexpr (DRAIN) {
                float sum[2][32] = {};
                for (int v = tl.v0; v < tl.v1 && ok; v += DRAIN_BLOCKS, ++it) {
                    const int acc = it & 1;
                    ok = warp_wait_cl(BAR_ACCFULL(acc), (it >> 1) & 1, spin, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (half * 32 + j * 64 >= p.NT) continue;
                        f32x2 x[16];
                        tmem_ld32(lanes + acc * 256 + half * 32 + j * 64, x);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) { sum[j][2 * i] += x[i].x; sum[j][2 * i + 1] += x[i].y; }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_at(BAR_ACCEMPTY(acc), 0);
                }
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (half * 32 + j * 64 < p.NT) finish(tl.n + half * 32 + j * 64, sum[j]);
            } else {
                float *carry = p.carry + (size_t)blockIdx.x * p.NT * 128 + q * 32 + lane;
                for (int v0 = tl.v0; v0 < tl.v1 && ok; v0 += TAKE, ++it) {
                    const int acc = it & 1;
                    ok = warp_wait_cl(BAR_ACCFULL(acc), (it >> 1) & 1, spin, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = half * 32; c < p.NT; c += 64) {
                        f32x2 x[16];
                        __syncwarp();   // lanes part at rows that do not exist below, and tensor memory is read by whole warps
                        tmem_ld32(lanes + acc * 256 + c, x);
                        tmem_ld_wait();
                        float v[32];
#pragma unroll
                        for (int i = 0; i < 16; ++i) { v[2 * i] = x[i].x; v[2 * i + 1] = x[i].y; }
                        if (v0 != tl.v0) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] += carry[(c + j) * 128];
                        }
                        if (v0 + TAKE < tl.v1) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) carry[(c + j) * 128] = v[j];
                        } else {
                            finish(tl.n + c, v);
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_at(BAR_ACCEMPTY(acc), 0);
                }
                if (!ok) break;
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
    }
    __syncwarp();   // an elected thread and its warp: what follows is for whole warps
    dependency_trigger();
    if (*abort_flag) {   // let copies and MMAs in flight land before shared and tensor memory are given back
        const uint64_t tw = gtimer();
        while (gtimer() - tw < 50000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();   // the pair's products read this CTA's shared memory, and its barriers are arrived on from the other
    cluster_wait();
    if (warp == 1) tmem_dealloc2(tmem, 512);
}

// Sums over the splits of K in a fixed order, and the epilogue, of the tiles that are split.  A thread has four neighbours of a tile.
struct FinishArgs {
    int M, N, NT, ny, whole, splits;
    long long out_m, out_n;
    const float *part;
    LinearEpilogue e;
};
template <typename IO> __global__ void __launch_bounds__(256) linear_finish_kernel(FinishArgs a) {
    dependency_wait();
    const int quads = 64 * a.NT, quad = (blockIdx.x % (quads / 256)) * 256 + threadIdx.x;
    const int tile = blockIdx.x / (quads / 256), xy = a.whole + tile, inner = a.out_n == 1 ? a.NT : 256;
    const int at = quad * 4, i = at / inner, j = at % inner;   // j along the results' innermost dimension
    const int m = xy / a.ny * 256 + (a.out_n == 1 ? i : j), n = xy % a.ny * a.NT + (a.out_n == 1 ? j : i);
    if (m < a.M && n < a.N) {
        const float *p = a.part + (size_t)tile * a.splits * 256 * a.NT + at;
        float z[4] = {};
        for (int s = 0; s < a.splits; ++s, p += 256 * a.NT) {
            const float4 v = *(const float4 *)p;
            z[0] += v.x; z[1] += v.y; z[2] += v.z; z[3] += v.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int me = m + (a.out_n == 1 ? 0 : e), ne = n + (a.out_n == 1 ? e : 0);
            if (me < a.M && ne < a.N) finish_one<IO>(a.e, me * a.out_m + ne * a.out_n, z[e] + (a.e.bias ? a.e.bias[a.out_n == 1 ? ne : me] : 0.0f));
        }
    }
    dependency_trigger();
}

// An operand as the tensor copies want it, rows at multiples of 16 bytes: a copy of a bf16 matrix, or the planes of an fp32 one
struct PackArgs {
    const void *in;
    __nv_bfloat16 *out;
    long long rows, plane;
    int cols, ld;
};
template <typename IO> __global__ void __launch_bounds__(256) linear_pack_kernel(PackArgs a) {
    dependency_wait();
    const int groups = a.ld / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / groups;
    const int c = (int)(i % groups) * 8;
    if (row < a.rows) {
        float v[8];
        if constexpr (sizeof(IO) == 4) {
            const float *p = (const float *)a.in + row * a.cols + c;
            if (a.cols % 4 == 0 && c + 8 <= a.cols) {
                const float4 x = *(const float4 *)p, y = *(const float4 *)(p + 4);
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? p[e] : 0.0f;
            }
        } else {
            const __nv_bfloat16 *p = (const __nv_bfloat16 *)a.in + row * a.cols + c;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? __bfloat162float(p[e]) : 0.0f;
        }
        __nv_bfloat16 *out = a.out + row * a.ld + c;
        auto put8 = [&](int plane, const float (&f)[8]) {
            *(uint4 *)(out + plane * a.plane) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        };
        if constexpr (sizeof(IO) == 2) {
            put8(0, v);
        } else {
            float h[8], h0[8], m[8], l[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool finite = fabsf(v[e]) <= 3.402823466e38f;
                h[e] = __bfloat162float(__float2bfloat16_rn(v[e]));
                if (finite && fabsf(h[e]) > 3.402823466e38f) h[e] = copysignf(3.3895313892515355e38f, v[e]);   // the largest bf16
                h0[e] = finite ? h[e] : 0.0f;
                const float r = finite ? v[e] - h[e] : 0.0f;
                m[e] = __bfloat162float(__float2bfloat16_rn(r));
                l[e] = r - m[e];
            }
            put8(0, h); put8(1, h0); put8(2, m); put8(3, l);
        }
    }
    dependency_trigger();
}

// ---- plan
struct Plan {
    bool swapped, pack_a, pack_b;   // swapped: the caller's B is the kernel's A
    int NT, nx, ny, kblocks, vblocks, whole, splits, per_split;
    size_t a_bytes, b_bytes, part_bytes, carry_bytes;
};
inline bool f32(const LinearProduct &g) { return g.io == RGLRU_F32; }
size_t packed_bytes(const LinearOperand &o, bool is_f32) {
    if (!is_f32 && o.cols % 8 == 0) return 0;
    return up256((size_t)(is_f32 ? PLANES : 1) * o.rows * ((o.cols + 7) / 8 * 8) * 2);
}
Plan make_plan(const LinearProduct &g) {
    Plan p{};
    p.swapped = g.M <= 128 && g.N > g.M;
    const long long M = p.swapped ? g.N : g.M, N = p.swapped ? g.M : g.N;
    const LinearOperand &a = p.swapped ? g.b : g.a, &b = p.swapped ? g.a : g.b;
    p.kblocks = (int)((g.K + 63) / 64);
    p.vblocks = p.kblocks * (f32(g) ? PRODUCTS : 1);
    // Whole rounds of pairs take a tile each; the tiles of the last, partly filled round are split along K over all pairs.  The tile width and
    // the splits are those that take the busiest pair the fewest cycles: a K block costs what its copies out of L2 do (measured: 590
    // cycles of NT = 256, 470 of 128), a tile some 200 more, a split its partial results' way to memory and back and another launch.
    double best = 0;
    for (int nt : {256, 128, 64, 32}) {
        if ((f32(g) && nt > 128) || (b.turned && nt < 128)) continue;   // registers of the sums; copies 64 values wide
        const long long nx = (M + 255) / 256, ny = (N + nt - 1) / nt, tiles = nx * ny, whole = tiles / PAIRS * PAIRS, rest = tiles - whole;
        const double block = 350 + 0.94 * nt;
        for (int s = 1; s <= 32 && s <= p.vblocks; ++s) {
            const int per = (p.vblocks + s - 1) / s;
            if ((p.vblocks + per - 1) / per != s || (rest == 0 && s > 1)) continue;
            double cost = (double)(whole / PAIRS) * (p.vblocks * block + 200) + (double)((rest * s + PAIRS - 1) / PAIRS) * (per * block + 200);
            if (s > 1) cost += 3000 + (double)rest * s * 256 * nt * 8 / 2000;
            if (best == 0 || cost < best) {
                best = cost;
                p.NT = nt; p.nx = (int)nx; p.ny = (int)ny; p.whole = (int)(s > 1 ? whole : tiles); p.splits = s; p.per_split = per;
            }
        }
    }
    p.pack_a = packed_bytes(a, f32(g)) != 0;
    p.pack_b = packed_bytes(b, f32(g)) != 0;
    p.a_bytes = a.packed ? 0 : packed_bytes(a, f32(g));
    p.b_bytes = b.packed ? 0 : packed_bytes(b, f32(g));
    p.part_bytes = (size_t)((long long)p.nx * p.ny - p.whole) * p.splits * 256 * p.NT * sizeof(float);
    const int longest = p.whole ? p.vblocks : p.per_split;
    p.carry_bytes = f32(g) || longest <= LONG_BLOCKS ? 0 : (size_t)2 * PAIRS * 128 * p.NT * sizeof(float);
    return p;
}

// The operand's map, after packing it into `at` where its rows do not start at multiples of 16 bytes or it is fp32
cudaError_t place(const LinearOperand &o, int io, bool pack, void *at, int box_rows, CUtensorMap *tm, cudaStream_t st) {
    const long long ld = (o.cols + 7) / 8 * 8;
    const int planes = pack && io == RGLRU_F32 ? PLANES : 1;
    if (pack && o.packed) at = o.packed;
    if (pack && !o.ready) {
        PackArgs a{o.p, (__nv_bfloat16 *)at, o.rows, o.rows * ld, (int)o.cols, (int)ld};
        const long long blocks = (o.rows * (ld / 8) + 255) / 256;
        if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
        const cudaError_t e = launch_dependent(io == RGLRU_F32 ? linear_pack_kernel<float> : linear_pack_kernel<__nv_bfloat16>, dim3((unsigned)blocks), dim3(256), 0, st, a);
        if (e != cudaSuccess) return e;
    }
    const uint64_t dims[3] = {(uint64_t)o.cols, (uint64_t)o.rows, (uint64_t)planes}, strides[2] = {(uint64_t)ld * 2, (uint64_t)(o.rows * ld) * 2};
    const uint32_t box[3] = {64, (uint32_t)(o.turned ? 64 : box_rows), 1};
    return encode_map16_3d(tm, pack ? at : o.p, dims, strides, box, true) ? cudaSuccess : cudaErrorNotSupported;
}

struct Device {
    std::mutex mutex;
    int pairs[64] = {};
    // pairs that fit on the device at a time, after the opt-in to the shared memory that they use
    cudaError_t get(int *out) {
        int dev = -1;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
        std::lock_guard<std::mutex> lock(mutex);
        if (pairs[dev] == 0) {
            if ((e = cudaFuncSetAttribute(linear_gemm_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_ALLOC)) != cudaSuccess) return e;
            if ((e = cudaFuncSetAttribute(linear_gemm_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_ALLOC)) != cudaSuccess) return e;
            cudaLaunchConfig_t q{};
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim = {2, 1, 1};
            q.gridDim = dim3(num_sms() & ~1); q.blockDim = dim3(THREADS); q.dynamicSmemBytes = SMEM_ALLOC; q.attrs = attr; q.numAttrs = 1;
            int n = 0;
            pairs[dev] = cudaOccupancyMaxActiveClusters(&n, linear_gemm_kernel<__nv_bfloat16>, &q) == cudaSuccess && n > 0 ? n : num_sms() / 2;
            (void)cudaGetLastError();
        }
        *out = pairs[dev];
        return cudaSuccess;
    }
} g_device;

}  // namespace

size_t sm100_linear_packed_bytes(const LinearOperand &o, int io) { return packed_bytes(o, io == RGLRU_F32); }

size_t sm100_linear_bytes(const LinearProduct &g) {
    const Plan p = make_plan(g);
    return p.a_bytes + p.b_bytes + p.part_bytes + p.carry_bytes;
}

cudaError_t sm100_linear(const LinearProduct &g, void *scratch, uint32_t *status, cudaStream_t st) {
    const Plan p = make_plan(g);
    int pairs = 0;
    cudaError_t e = g_device.get(&pairs);
    if (e != cudaSuccess) return e;
    GemmArgs a{};
    const LinearOperand &oa = p.swapped ? g.b : g.a, &ob = p.swapped ? g.a : g.b;
    char *at = (char *)scratch;
    if ((e = place(oa, g.io, p.pack_a, at, 128, &a.tm_a, st)) != cudaSuccess) return e;
    if ((e = place(ob, g.io, p.pack_b, at + p.a_bytes, p.NT / 2, &a.tm_b, st)) != cudaSuccess) return e;
    a.a_turned = oa.turned; a.b_turned = ob.turned; a.split_planes = f32(g);
    a.M = (int)(p.swapped ? g.N : g.M); a.N = (int)(p.swapped ? g.M : g.N);
    a.NT = p.NT; a.nx = p.nx; a.ny = p.ny;
    a.kblocks = p.kblocks; a.vblocks = p.vblocks; a.whole = p.whole; a.splits = p.splits; a.per_split = p.per_split;
    a.out_m = p.swapped ? 1 : g.N; a.out_n = p.swapped ? g.N : 1;
    a.e = g.e;
    a.part = (float *)(at + p.a_bytes + p.b_bytes);
    if (p.carry_bytes) {
        a.carry = (float *)(at + p.a_bytes + p.b_bytes + p.part_bytes);
        if (pairs > PAIRS) pairs = PAIRS;   // as many as have a place there
    }
    const int per16 = 16 / (int)io_bytes(g.io);
    a.wide = g.N % per16 != 0 ? 0 : g.N % (2 * per16) == 0 && aligned(g.e.y, 32) && aligned(g.e.preact, 32) ? 32 : 16;
    a.stages = (int)((a.out_n == 1 && !a.wide ? RING - TURN : RING) / (A_BYTES + (uint32_t)p.NT * 64u));
    a.status = status; a.spin_ns = g_spin_limit_ns; a.b_never_comes = (g.flags & RGLRU_FLAG_TEST_CARRY_NEVER_ARRIVES) != 0;
    const long long split = (long long)p.nx * p.ny - p.whole, tiles = p.whole + split * p.splits;
    if (tiles > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {2, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2 * (unsigned)(tiles < pairs ? tiles : pairs)); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = SMEM_ALLOC; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = 2;
    e = f32(g) ? cudaLaunchKernelEx(&cfg, linear_gemm_kernel<float>, a) : cudaLaunchKernelEx(&cfg, linear_gemm_kernel<__nv_bfloat16>, a);
    if (e != cudaSuccess || split == 0) return e;
    const FinishArgs f{a.M, a.N, p.NT, p.ny, p.whole, p.splits, a.out_m, a.out_n, a.part, g.e};
    return launch_dependent(f32(g) ? linear_finish_kernel<float> : linear_finish_kernel<__nv_bfloat16>, dim3((unsigned)(split * (p.NT / 4))), dim3(256), 0, st, f);
}

}  // namespace rglru
