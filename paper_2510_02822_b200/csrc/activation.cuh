// Activation functions of the operators between the quantized layers, in fp32.
#pragma once
#include <stdint.h>

#include "flexiq.h"

namespace flexiq {

inline bool act_known(int act) { return act >= FLEXIQ_ACT_NONE && act <= FLEXIQ_ACT_SILU; }

// Negative infinity times a zero would be a NaN where the functions have the limit 0; every finite v below -1e30 gives 0 as well.
template <int ACT> __device__ __forceinline__ float activate(float v)
{
    if (ACT == FLEXIQ_ACT_RELU) return v < 0.f ? 0.f : v;   // a NaN stays
    if (ACT == FLEXIQ_ACT_GELU) {
        const float x = v < -1e30f ? -1e30f : v;
        return __fmul_rn(x, __fmul_rn(0.5f, erfcf(__fmul_rn(x, -0.70710678f))));
    }
    if (ACT == FLEXIQ_ACT_GELU_TANH) {   // (1 + tanh u) / 2 = 1 / (1 + exp(-2u))
        const float x = v < -1e10f ? -1e10f : v;   // (its cube has to stay finite)
        const float u2 = __fmul_rn(__fmul_rn(x, 1.5957691f), __fmaf_rn(__fmul_rn(0.044715f, x), x, 1.0f));
        return __fdiv_rn(x, __fadd_rn(1.0f, expf(-u2)));
    }
    if (ACT == FLEXIQ_ACT_SILU) {
        const float x = v < -1e30f ? -1e30f : v;
        return __fdiv_rn(x, __fadd_rn(1.0f, expf(-x)));
    }
    return v;
}

template <int ACT, int N> __device__ __forceinline__ void activate_all(float *v)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activate<ACT>(v[i]);
}
// `act` is the same for the whole launch: one uniform branch for N values
template <int N> __device__ __forceinline__ void activate_n(int act, float *v)
{
    switch (act) {
        case FLEXIQ_ACT_RELU: activate_all<FLEXIQ_ACT_RELU, N>(v); break;
        case FLEXIQ_ACT_GELU: activate_all<FLEXIQ_ACT_GELU, N>(v); break;
        case FLEXIQ_ACT_GELU_TANH: activate_all<FLEXIQ_ACT_GELU_TANH, N>(v); break;
        case FLEXIQ_ACT_SILU: activate_all<FLEXIQ_ACT_SILU, N>(v); break;
        default: break;
    }
}

}  // namespace flexiq
