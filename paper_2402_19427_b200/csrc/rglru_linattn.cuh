// Linear attention with a decay for each head: what its kernels share.
//
// Forward and backward are the same walk.  With (q, k, v, S) standing for one of four sets of tensors, over tokens in walking order
//     out_i = sp sum_{j <= i} d^(i-j) (q_i k_j) v_j + si d^(i+first) q_i S_in,   S_out = d^n S_in + su sum_j d^(n-j-first) k_j v_j^T
//   output   (q, k, v),   S0,             first 1, sp = si = scale, su = 1
//   dq       (do, v, k),  S0 transposed,  first 1, sp = si = scale, su = 1
//   dk       (v, do, q),  dS_T transposed, last token first, first 0, sp = su = scale, si = 1
//   dv       (k, q, do),  dS_T,           last token first, first 0, sp = su = scale, si = 1;  its S_out is dS0
// The tokens of a chunk go through matrix products, the state goes from chunk to chunk.
#pragma once

#include "rglru_internal.h"

namespace rglru {

struct MixTensor {
    void *p;
    long long token, batch;   // distances in elements
};
struct MixRole {
    MixTensor q, k, v, o;
    int dk, dv;               // widths of q and k, and of v and o
    const float *s_in;        // [B,H,dk,dv], transposed [B,H,dv,dk] if turned, or null
    float *s_out;             // [B,H,dk,dv] or null
    int turned, reverse, first;
    float sp, si, su;
};
struct MixArgs {
    MixRole role[3];
    int roles, B, T, H;
    const float *log_decay;
    uint32_t *status;
};

// ---- tensor cores (rglru_sm100_linattn.cu): bf16 io, widths that are multiples of 8 up to 128, distances that are multiples of 8
bool sm100_mix_supported(const MixArgs &a, int io);
size_t sm100_mix_bytes(int roles, int B, int T, int H);
cudaError_t sm100_mix(const MixArgs &a, uint32_t flags, void *scratch, cudaStream_t st);

// decay^n; n = 0 is 1 whatever the decay (log_decay may be minus infinity).  Powers beyond fp32's range are held at its largest number: what has grown out
// of the range still comes out infinite, but a state that is 0 stays 0 (inf * 0 is NaN).
__device__ __forceinline__ float decay_power(float log_decay, float n) {
    const float e = n == 0.0f ? 1.0f : expf(log_decay * n);
    return e > 3.402823466e38f ? 3.402823466e38f : e;
}

}  // namespace rglru
