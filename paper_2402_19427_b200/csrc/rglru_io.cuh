// One element of an io tensor (fp32 or bf16), as fp32
#pragma once

#include <cuda_bf16.h>

namespace rglru {

template <typename IO> __device__ __forceinline__ float at(const void *p, long long i) {
    if constexpr (sizeof(IO) == 4) return ((const float *)p)[i];
    else return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
}
template <typename IO> __device__ __forceinline__ void put(void *p, long long i, float v) {
    if constexpr (sizeof(IO) == 4) ((float *)p)[i] = v;
    else ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(v);
}

}  // namespace rglru
