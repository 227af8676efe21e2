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
// A chunk of 128 x 128 moves 128 KB, 3.0 us of an SM's share of the measured copy rate; its 48 matrix instructions take 64 cycles each, 1.6 us.  It takes
// 4.4 to 4.6 us with all SMs at work: the way from one state product to the next (the state's update, the planes of the next k, its
// scores, each handed on through a barrier some 300 to 500 cycles after it is ready) is what bounds it, not one of its resources (41 % of the issue
// slots, 45 % of the shared-memory pipe).  One block an SM: 224 KB of q, k and v (twice), S and planes.  A tile is requested again as soon as its last
// reader is done: q after the far product, k and v after the state product.  Warps: four look through v and turn P into the operand of
// the near product (in tensor memory, over the scores), four write the outputs, eight keep the state, eight make the planes, one copies, one issues.
// Outputs go from registers to memory, 32 bytes a thread: staged in shared memory for a tiled copy they held v's place for
// another 4000 cycles a chunk.
//
// Each block walks as many whole (role, sequence, head) as there are for all, and an equal stretch of the chunks of those left over.  The state in front
// of a stretch comes from two small launches: one leaves the sums of every stretch's last sequence (planes and state product only, 2.3 us a
// chunk), one folds them in order.
#include <cuda.h>
#include <cuda_bf16.h>

#include "rglru_linattn.cuh"
#include "sm100_ptx.cuh"

namespace rglru {
namespace {

using namespace ptx;

constexpr int CH = 128;                          // tokens a chunk
// Warpgroups of four: weights, outputs, state (two), planes (two), copies and products.  896 threads start with 72 registers each;
// 2 x 80 + 2 x 112 + 2 x 40 + 40 are the same 504.
constexpr int P_WARPS = 4, O_WARPS = 4, S_WARPS = 8, K_WARPS = 8, S_FIRST = P_WARPS + O_WARPS, K_FIRST = S_FIRST + S_WARPS;
constexpr int COPY_WARP = K_FIRST + K_WARPS, MMA_WARP = COPY_WARP + 1, THREADS = (COPY_WARP + 4) * 32;
constexpr uint32_t BLOCK = 128 * 128;            // 128 rows of 64 bf16
// The planes of the decayed k are made 32 tokens (a piece) at a time.  The first plane takes the place of the k it is made from; the others
// of pieces 0 and 1 have slots of their own, those of pieces 2 and 3 lie in S's place, which is free from the far product to the next S.
constexpr int PIECES = 4;
constexpr uint32_t PLANE = 2 * 32 * 128, SLOT = 2 * PLANE;   // 32 tokens of 2 x 64 values
constexpr uint32_t TILE = 2 * BLOCK;
constexpr uint32_t SM_Q = 0, SM_K = TILE, SM_V = SM_K + 2 * TILE, SM_S = SM_V + 2 * TILE, SM_PLANES = SM_S + TILE, SM_BAR = SM_PLANES + 2 * SLOT;
__host__ __device__ constexpr uint32_t slot_at(int piece) { return piece < 2 ? SM_PLANES + piece * SLOT : SM_S + (piece - 2) * SLOT; }
static_assert(2 * SLOT <= TILE, "slots in S's place");
enum { QF, QE, SC, PR, DSF, UR, SR, OE, KF, VF = KF + 2, VK = VF + 2, KVE = VK + 2, PLE = KVE + 2, PLF = PLE + 1, NBAR = PLF + PIECES };   // two of each for the two tiles of k and v
constexpr uint32_t SM_TMEM = SM_BAR + (NBAR + 1) / 2 * 16, SM_BAD = SM_TMEM + 16,
                   SM_STEPS = (SM_BAD + 8 * 132 + 15) / 16 * 16, SM_TOTAL = SM_STEPS + 64, SM_ALLOC = SM_TOTAL + 1024;
static_assert(SM_ALLOC <= 232448, "shared memory of a block");
constexpr uint32_t TM_P = 0, TM_Y = 128, TM_X = 256, TM_U = 384;   // tensor-memory columns
constexpr int WALKERS = 148;                     // the plan, and with it the workspace, does not depend on the device

struct WalkArgs {
    alignas(64) CUtensorMap tm[3][3];            // q, k, v of each role: [B][T][H][width]
    MixArgs m;
    int nothing_comes, chunks;                   // test hook of the waits' limits; chunks of a (role, sequence, head)
    int walkers, rounds, rest;                   // blocks; units that each takes whole, and units left over, which are cut over all blocks
    int whole_steps;                             // rounds times chunks
    float *local, *starts;                       // [walkers][32][128][4] sums of stretches, and the states in front of them; null: no sequence is cut
    unsigned long long spin_ns;
};
// the first chunk of block w's stretch of the units left over, counted over those
__device__ __forceinline__ long long share(const WalkArgs &p, int w) { return (long long)p.rest * p.chunks * w / p.walkers; }
__device__ __forceinline__ long long left_over(const WalkArgs &p) { return (long long)p.rounds * p.walkers * p.chunks; }   // their first chunk, over all units

// One chunk of the walk; next() goes on to the one behind it
struct Step {
    int role, b, h, chunk, n, t0;                // t0: the tile's first token in memory (negative where a reversed walk ends)
    bool fresh;                                  // another (role, sequence, head) than the step before
    __device__ __forceinline__ void tokens(const WalkArgs &p) {
        n = min(CH, p.m.T - chunk * CH);
        t0 = p.m.role[role].reverse ? p.m.T - (chunk + 1) * CH : chunk * CH;
    }
    __device__ __forceinline__ Step() {}
    __device__ __forceinline__ Step(const WalkArgs &p, long long g) : Step(p, (int)(g / p.chunks), (int)(g % p.chunks)) {}   // chunk g of all
    __device__ __forceinline__ Step(const WalkArgs &p, int unit, int in) {
        const int bh = p.m.B * p.m.H;
        chunk = in;
        role = unit / bh;
        b = unit % bh / p.m.H;
        h = unit % p.m.H;
        fresh = true;
        if (role < p.m.roles) tokens(p);         // not behind the last chunk of the call
    }
    __device__ __forceinline__ void next(const WalkArgs &p) {
        fresh = ++chunk == p.chunks;
        if (fresh) {
            chunk = 0;
            if (++h == p.m.H) { h = 0; if (++b == p.m.B) { b = 0; ++role; } }
            if (role == p.m.roles) return;
        }
        tokens(p);
    }
};
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
// A step that was left in shared memory: the divisions behind it are done once a block
__device__ __forceinline__ Step step_at(uint32_t a) {
    const uint4 x = lds128(a), y = lds128(a + 16);
    Step st;
    st.role = (int)x.x; st.b = (int)x.y; st.h = (int)x.z; st.chunk = (int)x.w; st.n = (int)y.x; st.t0 = (int)y.y;
    st.fresh = true;
    return st;
}
__device__ __forceinline__ void leave_step(int *to, const Step &st) { to[0] = st.role; to[1] = st.b; to[2] = st.h; to[3] = st.chunk; to[4] = st.n; to[5] = st.t0; }
// What a block walks: whole units or a stretch; whole units and then a stretch (held to code of its own: two tests and a load a step cost 3 %); a
// stretch for its sums alone
enum { ONE, BOTH, SUMS };
// The step behind the first `done`: whole units first, then the stretch
template <int MODE> __device__ __forceinline__ void advance(Step &st, const WalkArgs &p, int done, uint32_t stretch) {
    if (MODE == BOTH && done == p.whole_steps) st = step_at(stretch);
    else st.next(p);
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ __nv_bfloat162 larger(__nv_bfloat162 top, uint32_t w) { return __hmax2_nan(top, __habs2(*(const __nv_bfloat162 *)&w)); }
// Bits 15 and 31 of the result: whether the two bf16 of w are infinite or NaN (all bits of the exponent set)
__device__ __forceinline__ uint32_t no_numbers(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }

// the upper 16 bits of two fp32 values: cut to bf16
__device__ __forceinline__ uint32_t upper_halves(f32x2 x) { return __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632); }
// The values of a 16-byte piece of v that are no numbers become 0 in shared memory: a product would carry them into rows of tokens
// before theirs, as 0 * NaN.  Byte c of `bad` holds the first token (in walking order) from which on column c is NaN, 255: none.
__device__ __forceinline__ void mend_piece(uint32_t addr, int column, uint32_t token, uint32_t *bad) {
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

__device__ __forceinline__ void load_tile(const WalkArgs &p, int which, const Step &st, int width, uint32_t to, uint32_t bar) {
    const int blocks = width > 64 ? 2 : 1;
    mbar_expect_tx(bar, blocks * BLOCK);
    for (int j = 0; j < blocks; ++j) tma_load_4d(to + j * BLOCK, &p.tm[st.role][which], j * 64, st.h, st.t0, st.b, bar);
}

// STATE_ONLY: the sums U of a block's last stretch, for the blocks that go on in the same sequence
template <int MODE> __global__ void __launch_bounds__(THREADS, 1) mix_walk_kernel(const __grid_constant__ WalkArgs p) {
    constexpr bool STATE_ONLY = MODE == SUMS;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw), base = (raw_addr + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw_addr);
    auto BAR = [&](int i) { return base + SM_BAR + 8u * i; };
    uint32_t *tmem_base_s = (uint32_t *)(smem + SM_TMEM);
    volatile int *abort_flag = (volatile int *)(tmem_base_s + 1);
    uint32_t *bad_base = (uint32_t *)(smem + SM_BAD);   // [8][33] words, by the step: a byte for each column, and whether there is any
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned long long spin = p.spin_ns;

    if (tid == 0) {
        for (int i = 0; i < NBAR; ++i) {
            const bool by_four = i == PR || i == OE || i == VK || i == VK + 1;
            mbar_init(BAR(i), by_four ? 4 : i == SR || i == UR ? S_WARPS : i >= PLF ? K_WARPS : 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 32) {   // the block's first step and its number of steps, and its stretch
        int *at = (int *)(smem + SM_STEPS);
        if (MODE != SUMS && p.rest == 0) {
            leave_step(at, Step(p, (int)blockIdx.x * p.rounds, 0));
            at[6] = p.whole_steps;
        } else {
            long long from = share(p, blockIdx.x);
            const long long to = share(p, blockIdx.x + 1), begin = to / p.chunks * p.chunks;   // begin: of the unit that the stretch ends in
            if (MODE == SUMS && begin > from) from = begin;   // nothing to do if it ends with a unit
            const Step stretch(p, left_over(p) + from);
            leave_step(at, MODE == BOTH ? Step(p, (int)blockIdx.x * p.rounds, 0) : stretch);
            leave_step(at + 8, stretch);
            at[6] = (MODE == BOTH ? p.whole_steps : 0) + (int)(to - from);
        }
    }
    if (tid < 8 * 33) bad_base[tid] = tid % 33 == 32 ? 0u : 0xFFFFFFFFu;
    if (warp == MMA_WARP) { tmem_alloc(smem_u32(tmem_base_s), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_base_s;
    bool ok = true;
    dependency_wait();

    const int steps = *(volatile int *)(smem + SM_STEPS + 24);

    // (each warpgroup takes its registers in its own branch: behind a join, all code would get by with the fewest)
    if (warp >= COPY_WARP) {
        reg_dec<40>();   // once for all four warps: a warpgroup executes the same setmaxnreg together
        if (warp == COPY_WARP) {
            // ---- copies: k and v one chunk ahead of q
            if (elect_one() && !p.nothing_comes) {
                auto wait = [&](int bar, uint32_t parity) { ok = ok && mbar_wait_spin(BAR(bar), parity, spin, abort_flag); return ok; };
                Step st = step_at(base + SM_STEPS), ahead = st;
                auto load_kv = [&](int s) {
                    const MixRole &r = p.m.role[ahead.role];
                    const int k = s & 1;
                    if (!wait(KVE + k, (s >> 1 & 1) ^ 1)) return;
                    load_tile(p, 1, ahead, r.dk, base + SM_K + k * TILE, BAR(KF + k));
                    load_tile(p, 2, ahead, r.dv, base + SM_V + k * TILE, BAR(VF + k));
                    advance<MODE>(ahead, p, s + 1, base + SM_STEPS + 32);
                };
                if (steps > 0) load_kv(0);
                for (int s = 0; s < steps && ok; ++s, advance<MODE>(st, p, s, base + SM_STEPS + 32)) {
                    if (!STATE_ONLY && wait(QE, (s & 1) ^ 1)) load_tile(p, 0, st, p.m.role[st.role].dk, base + SM_Q, BAR(QF));
                    if (ok && s + 1 < steps) load_kv(s + 1);
                }
                if (!ok) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
            }
        } else if (warp == MMA_WARP) {
            // ---- products
            // Waits never suspend the thread: what it waits for is tens of cycles away, waking up takes hundreds.
            if (elect_one()) {
                auto wait = [&](int bar, uint32_t parity) { ok = ok && mbar_wait_spin(BAR(bar), parity, spin, abort_flag); };
                // Descriptors are counted on from step to step (16 bytes are one unit of their address field): held for all steps at once they
                // would not fit this warpgroup's registers.
                auto kmajor = [&](uint32_t at) { return make_desc_sw128(base + at); };
                auto turned = [&](uint32_t at, uint32_t block) { return make_desc_sw128_mn(base + at, block); };
                auto scores = [&](int s, const MixRole &r) {
                    wait(QF, s & 1); wait(KF + (s & 1), s >> 1 & 1);
                    if (!ok) return;
                    tc_fence_after();
                    const uint32_t id = make_idesc(128, 128);
    #pragma unroll 1
                    for (int b = 0; b * 64 < r.dk; ++b) {
                        const uint64_t q = kmajor(SM_Q + b * BLOCK), k = kmajor(SM_K + (s & 1) * TILE + b * BLOCK);
    #pragma unroll
                        for (int i = 0; i < 4; ++i) mma_ss(tmem + TM_P, q + 2 * i, k + 2 * i, id, b | i);
                    }
                    tc_commit(BAR(SC));
                };
                Step st = step_at(base + SM_STEPS);
                if (!STATE_ONLY && steps > 0) scores(0, p.m.role[st.role]);
    #pragma unroll 1
                for (int s = 0; s < steps && ok; ++s) {
                    const MixRole &r = p.m.role[st.role];
                    const uint32_t ph = s & 1, nv = r.dv > 64 ? 128 : 64, id_b = make_idesc(128, nv) | (1u << 16), id_ab = id_b | (1u << 15);
                    const uint32_t v_at = SM_V + (s & 1) * TILE;
                    uint64_t v = turned(v_at, BLOCK);
                    auto piece = [&](int pc) {
                        wait(PLF + pc, ph);
                        if (!ok) return;
                        tc_fence_after();
                        const uint64_t first_plane = turned(SM_K + (s & 1) * TILE + pc * 4096, BLOCK), others = turned(slot_at(pc), PLANE / 2);
    #pragma unroll
                        for (int k = 0; k < 2; ++k) mma_ss(tmem + TM_U, others + PLANE / 16 + k * 128, v + k * 128, id_ab, pc | k);   // the smallest first
    #pragma unroll
                        for (int k = 0; k < 2; ++k) mma_ss(tmem + TM_U, others + k * 128, v + k * 128, id_ab, 1);
    #pragma unroll
                        for (int k = 0; k < 2; ++k) mma_ss(tmem + TM_U, first_plane + k * 128, v + k * 128, id_ab, 1);
                        v += 256;
                    };
                    wait(VK + (s & 1), s >> 1 & 1);
                    wait(UR, ph ^ 1);
    #pragma unroll 1
                    for (int pc = 0; pc < PIECES; ++pc) {
                        if (!STATE_ONLY && pc == 1) {
                            wait(SR, ph);
                            wait(OE, ph ^ 1);   // the last outputs have been read
                            if (!ok) break;
                            tc_fence_after();
                            uint64_t rows = turned(SM_S, BLOCK);   // S as it lies: rows of 64 columns of v
    #pragma unroll 1
                            for (int b = 0; b * 64 < r.dk; ++b, rows += 4 * 128) {
                                const uint64_t q = kmajor(SM_Q + b * BLOCK);
    #pragma unroll
                                for (int i = 0; i < 4; ++i) mma_ss(tmem + TM_X, q + 2 * i, rows + 128 * i, id_b, b | i);
                            }
                            tc_commit(BAR(QE));
                        }
                        if (pc == 2) tc_commit(BAR(PLE));   // the first two slots have been read
                        if (!STATE_ONLY && pc == 2) {
                            wait(PR, ph);
                            if (!ok) break;
                            tc_fence_after();
                            uint64_t rows = turned(v_at, BLOCK);
    #pragma unroll 4
                            for (int k = 0; k < 8; ++k, rows += 128) mma_ts(tmem + TM_Y, tmem + TM_P + k * 8, rows, id_b, k);
                        }
                        piece(pc);
                        if (!ok) break;
                    }
                    if (!ok) break;
                    tc_commit(BAR(DSF));   // all of the step's products
                    tc_commit(BAR(KVE + (s & 1)));
                    advance<MODE>(st, p, s + 1, base + SM_STEPS + 32);
                    if (!STATE_ONLY && s + 1 < steps) scores(s + 1, p.m.role[st.role]);
                }
                if (!ok) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
            }
        }
    } else if (warp < P_WARPS) {
        reg_inc<80>();
        // ---- what is no number in v; scores to weights: a thread has a row (a token)
        auto look_through = [&](int s, const Step &st) {
            const MixRole &r = p.m.role[st.role];
            const uint32_t tile = base + SM_V + (s & 1) * TILE;
            ok = warp_wait_held(BAR(VF + (s & 1)), s >> 1 & 1, spin, abort_flag);
            if (!ok) return;
            const int rounds = r.dv > 64 ? 16 : 8;
            __nv_bfloat162 top[4] = {};   // the largest magnitudes, NaN above all
#pragma unroll 8
            for (int k = 0; k < rounds; ++k) {
                const uint4 v = lds128(tile + (k * P_WARPS * 32 + tid) * 16);
                top[0] = larger(top[0], v.x); top[1] = larger(top[1], v.y); top[2] = larger(top[2], v.z); top[3] = larger(top[3], v.w);
            }
            uint32_t found = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) found |= no_numbers(*(const uint32_t *)&top[k]);
            if (found & 0x80008000u) {
                for (int k = 0; k < rounds; ++k) {
                    const int at = k * P_WARPS * 32 + tid, vrow = (at >> 3) & 127, column = (at >> 10) * 64 + ((at & 7) ^ (vrow & 7)) * 8;
                    mend_piece(tile + at * 16, column, (uint32_t)(r.reverse ? CH - 1 - vrow : vrow), bad_base + (s & 7) * 33);
                }
                fence_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(VK + (s & 1)));
        };
        const int row = warp * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        float ld = 0.0f, d1 = 0.0f;
        Step st = step_at(base + SM_STEPS), ahead = st;
        if (steps > 0) look_through(0, ahead);
        for (int s = 0; s < steps && ok; ++s, advance<MODE>(st, p, s, base + SM_STEPS + 32)) {
            advance<MODE>(ahead, p, s + 1, base + SM_STEPS + 32);
            if (STATE_ONLY) {
                if (s + 1 < steps) look_through(s + 1, ahead);
                continue;
            }
            const MixRole &r = p.m.role[st.role];
            const uint32_t ph = s & 1;
            const bool reverse = r.reverse;
            if (st.fresh) {
                ld = p.m.log_decay[st.h];
                d1 = decay_power(ld, 1.0f);
            }
            ok = warp_wait_held(BAR(SC), ph, spin, abort_flag);
            if (!ok) break;
            tc_fence_after();
            // Weights by multiplication, column after column away from the diagonal (so that they run into 0 and not out of infinity); a table
            // in shared memory would compete with the products' operands for its bandwidth.
            const int own = reverse ? 3 - warp : warp;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                const int cw = reverse ? 3 - c : c;   // the 32 columns' place in walking order
                uint32_t w[16];
                f32x2 v[16];
                if (cw <= own) tmem_ld32(lanes + TM_P + c * 32, v);
                if (cw > own) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = 0u;
                } else {
                    if (cw == own) {   // chosen, not multiplied by 0: what is masked may be no number
                        tmem_ld_wait();
                        float run = r.sp;
                        if (reverse) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const float a = 2 * j > lane ? run * d1 : run, b = 2 * j + 1 > lane ? a * d1 : a;
                                w[j] = pack_bf16(2 * j >= lane ? v[j].x * a : 0.0f, 2 * j + 1 >= lane ? v[j].y * b : 0.0f);
                                run = b;
                            }
                        } else {
#pragma unroll
                            for (int j = 15; j >= 0; --j) {
                                const float b = 2 * j + 1 < lane ? run * d1 : run, a = 2 * j < lane ? b * d1 : b;
                                w[j] = pack_bf16(2 * j <= lane ? v[j].x * a : 0.0f, 2 * j + 1 <= lane ? v[j].y * b : 0.0f);
                                run = a;
                            }
                        }
                    } else {
                        const float e = r.sp * decay_power(ld, (float)(reverse ? c * 32 - row : row - c * 32 - 31));
                        f32x2 run = reverse ? pack2(e, e * d1) : pack2(e * d1, e);
                        const f32x2 step = pack2(d1 * d1, d1 * d1);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const f32x2 x = mul2(reverse ? v[k] : v[15 - k], run);
                            const uint32_t both = pack_bf16(x.x, x.y);
                            if (reverse) w[k] = both;
                            else w[15 - k] = both;
                            run = mul2(run, step);
                        }
                    }
                }
                f32x2 x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
                // over columns that have been read: piece c ends at column 16 c + 15
                tmem_st16(lanes + TM_P + c * 16, x);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(PR));
            if (s + 1 < steps) look_through(s + 1, ahead);
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
    } else if (warp < P_WARPS + O_WARPS) {
        reg_inc<80>();
        // ---- outputs: a thread has a row (a token)
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        float far = 0.0f;
        Step st = step_at(base + SM_STEPS);
        for (int s = 0; !STATE_ONLY && s < steps && ok; ++s, advance<MODE>(st, p, s, base + SM_STEPS + 32)) {
            const MixRole &r = p.m.role[st.role];
            const uint32_t ph = s & 1;
            const int i = r.reverse ? CH - 1 - row : row;
            if (st.fresh) far = r.si * decay_power(p.m.log_decay[st.h], (float)(i + r.first));
            ok = warp_wait_held(BAR(DSF), ph, spin, abort_flag);
            if (!ok) break;
            tc_fence_after();
            const uint8_t *bad = (const uint8_t *)(bad_base + (s & 7) * 33);
            const bool any_bad = *(volatile const uint32_t *)(bad + 128) != 0;
            const int t = st.t0 + row;
            const bool there = t >= 0 && t < p.m.T;
            __nv_bfloat16 *to = (__nv_bfloat16 *)r.o.p + st.b * r.o.batch + t * r.o.token + (long long)st.h * r.dv;
            const bool wide = r.dv % 16 == 0 && (((size_t)r.o.p | (size_t)(r.o.token * 2) | (size_t)(r.o.batch * 2)) & 31) == 0;
#pragma unroll 1
            for (int c = 0; c < r.dv; c += 16) {
                f32x2 y[8], x[8];
                __syncwarp();   // lanes part at a ragged chunk's stores below, and tensor memory is read by whole warps
                tmem_ld16(lanes + TM_Y + c, y);
                tmem_ld16(lanes + TM_X + c, x);
                tmem_ld_wait();
                if (c + 16 >= r.dv) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(BAR(OE));
                }
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = fma2(x[j], pack2(far, far), y[j]);
                    w[j] = pack_bf16(y[j].x, y[j].y);
                }
                if (any_bad) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (i >= bad[c + 2 * j]) w[j] = w[j] & 0xFFFF0000u | 0x7FC0u;
                        if (i >= bad[c + 2 * j + 1]) w[j] = w[j] & 0x0000FFFFu | 0x7FC00000u;
                    }
                }
                if (there) {
                    if (wide) {
                        st_global_v8(to + c, w);
                    } else {
                        *(uint4 *)(to + c) = make_uint4(w[0], w[1], w[2], w[3]);
                        if (c + 8 < r.dv) *(uint4 *)(to + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
    } else if (warp < K_FIRST) {
        reg_inc<112>();
        // ---- the state: a thread has row d of S and 64 columns
        const int q = warp & 3, e0 = (warp - S_FIRST) / 4 * 64, d = q * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
        f32x2 S2[32];
        auto at = [&](int j) -> float & { return j & 1 ? S2[j / 2].y : S2[j / 2].x; };
        auto init_state = [&](const Step &st) {
            const MixRole &r = p.m.role[st.role];
            const long long mat = (long long)(st.b * p.m.H + st.h) * r.dk * r.dv;
            const float *src = STATE_ONLY ? nullptr : r.s_in;
            if (!STATE_ONLY && st.chunk != 0) {   // inside a sequence: the state was left there
                const float4 *l = (const float4 *)p.starts + ((size_t)blockIdx.x * 32 + e0 / 4) * 128 + d;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float4 v = l[j * 128];
                    S2[2 * j] = pack2(v.x, v.y);
                    S2[2 * j + 1] = pack2(v.z, v.w);
                }
                return;
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) S2[j] = pack2(0.0f, 0.0f);
            if (src && d < r.dk) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (e0 + j < r.dv) at(j) = src[mat + (r.turned ? (long long)(e0 + j) * r.dk + d : (long long)d * r.dv + e0 + j)];
            }
        };
        // S to shared memory for the far product: rows of 64 columns, 16-byte pieces swizzled as a tiled copy would have them; sixteen
        // columns at a time
        const uint32_t s_row = base + SM_S + (e0 / 64) * BLOCK + d * 128;
        auto put16 = [&](int c) {
#pragma unroll
            for (int j = c / 8; j < c / 8 + 2; ++j)
                sts128(s_row + ((j ^ (d & 7)) << 4), make_uint4(pack_bf16(S2[4 * j].x, S2[4 * j].y), pack_bf16(S2[4 * j + 1].x, S2[4 * j + 1].y),
                                                               pack_bf16(S2[4 * j + 2].x, S2[4 * j + 2].y), pack_bf16(S2[4 * j + 3].x, S2[4 * j + 3].y)));
        };
        auto handed_over = [&]() {
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(SR));
        };
        float ld = 0.0f;
        Step st = step_at(base + SM_STEPS);
#pragma unroll 1
        for (int s = 0; s < steps && ok; ++s, advance<MODE>(st, p, s, base + SM_STEPS + 32)) {
            const MixRole &r = p.m.role[st.role];
            const uint32_t ph = s & 1;
            uint32_t *bad = bad_base + (s & 7) * 33;
            if (st.fresh) {
                ld = p.m.log_decay[st.h];
                init_state(st);
                if (!STATE_ONLY) {
#pragma unroll
                    for (int c = 0; c < 64; c += 16) put16(c);
                    handed_over();
                }
            }
            const float f = decay_power(ld, (float)st.n), su = r.su;
            const bool last_chunk = st.chunk == p.chunks - 1;
            const int columns = r.dv - e0;
            ok = warp_wait_held(BAR(DSF), ph, spin, abort_flag);
            if (!ok) break;
            tc_fence_after();
            // The state product is done, and with it the far product and the products out of the second slot: S may be overwritten
            f32x2 u[2][8];
            tmem_ld16(lanes + TM_U + e0, u[0]);
#pragma unroll
            for (int c = 0; c < 64; c += 16) {
                tmem_ld_wait();
                if (c + 16 < 64) tmem_ld16(lanes + TM_U + e0 + c + 16, u[c / 16 + 1 & 1]);
                if (c < columns) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) S2[c / 2 + j] = fma2(pack2(f, f), S2[c / 2 + j], mul2(pack2(su, su), u[c / 16 & 1][j]));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(UR));
            if (*(volatile uint32_t *)(bad + 32)) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (((const uint8_t *)bad)[e0 + j] != 255) at(j) = __int_as_float(0x7FC00000);
            }
            if (!STATE_ONLY && !last_chunk) {
#pragma unroll
                for (int c = 0; c < 64; c += 16) put16(c);
                handed_over();
            }
            // The list of two steps ago has been read: by the outputs before they let the last step's go on, by the states before their SR.
            // It serves again in six steps, long after products that wait for this warp's SR.
            if (warp == S_FIRST && s > 1) {
                uint32_t *old = bad_base + (s - 2 & 7) * 33;
                if (*(volatile uint32_t *)(old + 32)) {
                    old[lane] = 0xFFFFFFFFu;
                    __syncwarp();
                    if (lane == 0) old[32] = 0u;
                }
            }
            if (!STATE_ONLY && last_chunk && r.s_out && d < r.dk) {
                float *dst = r.s_out + (long long)(st.b * p.m.H + st.h) * r.dk * r.dv + (long long)d * r.dv + e0;
#pragma unroll
                for (int j = 0; j < 64; j += 4)
                    if (e0 + j < r.dv) *(float4 *)(dst + j) = make_float4(S2[j / 2].x, S2[j / 2].y, S2[j / 2 + 1].x, S2[j / 2 + 1].y);
            }
        }
        if (STATE_ONLY && steps > 0 && ok) {
            float4 *l = (float4 *)p.local + ((size_t)blockIdx.x * 32 + e0 / 4) * 128 + d;
#pragma unroll
            for (int j = 0; j < 16; ++j) l[j * 128] = make_float4(S2[2 * j].x, S2[2 * j].y, S2[2 * j + 1].x, S2[2 * j + 1].y);
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
    } else {
        reg_dec<40>();
        // ---- planes of the decayed k
        const int k_tid = tid - K_FIRST * 32;
        float weight = 0.0f;
        int n_tokens = 0;
        Step st = step_at(base + SM_STEPS);
#pragma unroll 1
        for (int s = 0; s < steps && ok; ++s, advance<MODE>(st, p, s, base + SM_STEPS + 32)) {
            const MixRole &r = p.m.role[st.role];
            const uint32_t ph = s & 1;
            if (st.fresh || st.n != n_tokens) {   // lane (8 i + m) of a warp: the weight decay^(n - j - first) of the warp's row i + 16 m
                const int row = (k_tid >> 3 & 15) + 16 * (lane & 7), j = r.reverse ? CH - 1 - row : row;
                weight = j < st.n ? decay_power(p.m.log_decay[st.h], (float)(st.n - j - r.first)) : 0.0f;
                n_tokens = st.n;
            }
            ok = warp_wait_held(BAR(KF + ph), s >> 1 & 1, spin, abort_flag);
            if (!ok) break;
            // A thread has the same 16 bytes of two rows, 16 apart; the first 128 threads have columns 0 to 63 of k
            const bool mine = k_tid < 128 || r.dk > 64;
            const uint32_t src = base + SM_K + ph * TILE + (k_tid >> 7) * BLOCK + (k_tid & 127) * 16;
            const uint32_t dst = base + (k_tid >> 7) * (PLANE / 2) + (k_tid & 127) * 16;
#pragma unroll 1
            for (int pc = 0; pc < PIECES; ++pc) {
                const float w0 = __shfl_sync(0xffffffffu, weight, (lane & 24) + 2 * pc), w1 = __shfl_sync(0xffffffffu, weight, (lane & 24) + 2 * pc + 1);
                uint32_t v[8] = {}, hi[8], mid[8], lo[8];
                if (mine) {
                    const uint4 v0 = lds128(src + pc * 4096), v1 = lds128(src + pc * 4096 + 2048);
                    v[0] = v0.x; v[1] = v0.y; v[2] = v0.z; v[3] = v0.w; v[4] = v1.x; v[5] = v1.y; v[6] = v1.z; v[7] = v1.w;
                }
                // cut, not rounded: 24 bits are three times eight, so the three add up to the product exactly
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const f32x2 minus = pack2(-1.0f, -1.0f);
                    f32x2 x = mul2(bf2x(v[i]), i < 4 ? pack2(w0, w0) : pack2(w1, w1));
                    hi[i] = upper_halves(x);
                    x = fma2(bf2x(hi[i]), minus, x);
                    mid[i] = upper_halves(x);
                    x = fma2(bf2x(mid[i]), minus, x);
                    lo[i] = upper_halves(x);
                }
                // The last state product has read the slots, the scores k, and the far product S
                if (pc == 0) {
                    ok = warp_wait_held(BAR(PLE), ph ^ 1, spin, abort_flag);
                    if (!STATE_ONLY) ok = ok && warp_wait_held(BAR(SC), ph, spin, abort_flag);
                } else if (pc == 2) {
                    ok = STATE_ONLY ? warp_wait_held(BAR(DSF), ph ^ 1, spin, abort_flag) : warp_wait_held(BAR(QE), ph, spin, abort_flag);
                }
                if (!ok) break;
                if (mine) {
                    const uint32_t to = dst + slot_at(pc);
#pragma unroll
                    for (int i = 0; i < 8; i += 4) {
                        sts128(src + pc * 4096 + i * 512, make_uint4(hi[i], hi[i + 1], hi[i + 2], hi[i + 3]));
                        sts128(to + i * 512, make_uint4(mid[i], mid[i + 1], mid[i + 2], mid[i + 3]));
                        sts128(to + i * 512 + PLANE, make_uint4(lo[i], lo[i + 1], lo[i + 2], lo[i + 3]));
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(BAR(PLF + pc));
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.m.status, STATUS_MAGIC | (uint32_t)RGLRU_ERR_TIMEOUT); }
    }
    __syncwarp();   // an elected thread and its warp: what follows is for whole warps
    dependency_trigger();
    if (*abort_flag) {   // let copies and MMAs in flight land before shared and tensor memory are given back
        const uint64_t tw = gtimer();
        while (gtimer() - tw < 50000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MMA_WARP) tmem_dealloc(tmem, 512);
}

// From the sums of stretches to the states in front of them, sequence by sequence: a thread has four columns of a row, the sums of eight stretches on
// their way.
__global__ void __launch_bounds__(256) mix_fold_kernel(const __grid_constant__ WalkArgs p) {
    dependency_wait();
    const int unit = blockIdx.x / 16, item = blockIdx.x % 16 * 256 + threadIdx.x, d = item % 128, e0 = item / 128 * 4;
    const long long begin = (long long)unit * p.chunks, end = begin + p.chunks;
    const Step st(p, left_over(p) + begin);
    const MixRole &r = p.m.role[st.role];
    const float ld = p.m.log_decay[st.h];
    float s[4] = {};
    if (r.s_in && d < r.dk) {
        const float *src = r.s_in + (long long)(st.b * p.m.H + st.h) * r.dk * r.dv;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e0 + j < r.dv) s[j] = src[r.turned ? (long long)(e0 + j) * r.dk + d : (long long)d * r.dv + e0 + j];
    }
    int w = (int)(begin * p.walkers / ((long long)p.rest * p.chunks));
    while (share(p, w + 1) <= begin) ++w;
    const size_t at = (size_t)(item / 128) * 128 + d;
    for (; w < p.walkers && share(p, w) < end; w += 8) {
        float4 sums[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (w + k < p.walkers && share(p, w + k + 1) < end) sums[k] = ((const float4 *)p.local)[(size_t)(w + k) * 4096 + at];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (w + k >= p.walkers) break;
            const long long from = share(p, w + k), to = share(p, w + k + 1);
            if (from >= end || from == to) continue;   // (with fewer chunks than blocks some have none, and leave no sums)
            if (from > begin) ((float4 *)p.starts)[(size_t)(w + k) * 4096 + at] = make_float4(s[0], s[1], s[2], s[3]);
            if (to < end) {
                const float f = decay_power(ld, (float)((to - (from > begin ? from : begin)) * CH));
                s[0] = fmaf(f, s[0], sums[k].x); s[1] = fmaf(f, s[1], sums[k].y); s[2] = fmaf(f, s[2], sums[k].z); s[3] = fmaf(f, s[3], sums[k].w);
            }
        }
    }
    dependency_trigger();
}

// Blocks: one a (role, sequence, head) while that is as fast, else 148: each takes as many whole ones as there are for all, and an equal stretch of the
// rest.  In chunks: a block's own, and for stretches half of theirs again (sums only) and some six for two more launches and the states read.
// (Stretches of everything, in one order, cost sums of half a sequence a block: 8 x 2048 tokens of 20 heads took 139 us.)
struct WalkPlan { int walkers, rounds, rest; };
WalkPlan walk_plan(int roles, int B, int T, int H) {
    const long long units = (long long)roles * B * H, chunks = (T + CH - 1) / CH;
    const long long rounds = units / WALKERS, rest = units % WALKERS, share = (rest * chunks + WALKERS - 1) / WALKERS;
    const long long whole = (rounds + (rest != 0)) * chunks, cut = rounds * chunks + share + share / 2 + 6;
    if (whole <= cut || units * chunks < WALKERS) return {(int)units, 1, 0};
    return {WALKERS, (int)rounds, (int)rest};
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
    const WalkPlan w = walk_plan(roles, B, T, H);
    return w.rest == 0 ? 0 : (size_t)w.walkers * 128 * 128 * 2 * sizeof(float);
}

cudaError_t sm100_mix(const MixArgs &a, uint32_t flags, void *scratch, cudaStream_t st) {
    WalkArgs p{};
    p.m = a;
    p.nothing_comes = (flags & RGLRU_FLAG_TEST_CARRY_NEVER_ARRIVES) != 0;
    p.chunks = (a.T + CH - 1) / CH;
    const WalkPlan plan = walk_plan(a.roles, a.B, a.T, a.H);
    p.walkers = plan.walkers; p.rounds = plan.rounds; p.rest = plan.rest;
    const bool cut = p.rest != 0;
    p.whole_steps = p.rounds * p.chunks;
    p.local = cut ? (float *)scratch : nullptr;
    p.starts = cut ? p.local + (size_t)p.walkers * 128 * 128 : nullptr;
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
    static PerDeviceOptIn opt_one, opt_both, opt_sums;
    const bool both = cut && p.rounds != 0;
    cudaError_t e = both ? opt_both.ensure(mix_walk_kernel<BOTH>, (int)SM_ALLOC) : opt_one.ensure(mix_walk_kernel<ONE>, (int)SM_ALLOC);
    if (e == cudaSuccess && cut) e = opt_sums.ensure(mix_walk_kernel<SUMS>, (int)SM_ALLOC);
    if (e == cudaSuccess && cut) e = launch_dependent(mix_walk_kernel<SUMS>, dim3(p.walkers), dim3(THREADS), SM_ALLOC, st, p);
    if (e == cudaSuccess && cut) e = launch_dependent(mix_fold_kernel, dim3(16 * p.rest), dim3(256), 0, st, p);
    if (e == cudaSuccess) e = launch_dependent(both ? mix_walk_kernel<BOTH> : mix_walk_kernel<ONE>, dim3(p.walkers), dim3(THREADS), SM_ALLOC, st, p);
    return e;
}

}  // namespace rglru
