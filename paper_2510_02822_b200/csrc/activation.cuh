// Activation functions of the operators between the quantized layers, in fp32, two values at a time.
//
// The epilogue of a GEMM evaluates one for every output, and at short K it has about as many issue slots as the mainloop has MMA cycles (a
// 128 x 256 tile at K = 768: 4400 cycles, 64 values a thread and four warps a scheduler, so 17 slots a value), hence forms of few instructions and packed arithmetic (fma.rn.f32x2).
//
// All three are v F(v) with F(v) + F(-v) = 1, so that v F(v) = max(v, 0) - a F(-a) with a = |v|, and F(-a) is evaluated where it is small:
//   GELU       F(-a) = Phi(-a) = 2^q(a):  log2 Phi(-a) is nearly a parabola, and a polynomial of degree 6 weighted by F gives F to 1.5e-7
//   tanh form  the same with log2 of 1 / (1 + exp(2 sqrt(2/pi) (a + 0.044715 a^3))), degree 8: 1.5e-7
//   SiLU       e / (1 + e), e = 2^(-a log2 e); two values share a reciprocal, 1/x = y / (xy): the special-function unit serves 4 lanes a
//              cycle and scheduler
// (The polynomials were fitted by Lawson's reweighted least squares, and go on down to below -126, where the exponential is 0, up to the bound
// put on a.)  With the exponential's 2^-22, F and 2^-23 around the quotient, F is off by at most 2.8e-7 and the result, rounded
// once, by less than the 2^-21 |v| that is promised; far out on the negative side the error falls with F.
// A first form, v times a clipped odd polynomial of 13 coefficients, took 10.5 instructions a value and this one takes 6.5 (ViT-B fc1 with GELU
// over 12,608 rows 41.4 -> 36.4 us, in the kernel of that time, which could add a residual too; 31.4 now).
//
// The bound on a (min drops a NaN, and an infinity becomes a number whose F is 0) keeps one value of a pair from
// spoiling the other and gives infinities their limits; max.NaN passes a NaN on.
#pragma once
#include <stdint.h>

#include "flexiq.h"

namespace flexiq {

inline bool act_known(int act) { return act >= FLEXIQ_ACT_NONE && act <= FLEXIQ_ACT_SILU; }

// two fp32 values in one 64-bit register pair
typedef unsigned long long pair_t;
__device__ __forceinline__ pair_t pair(float a, float b)
{
    pair_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ void unpair(pair_t p, float *a, float *b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(p)); }
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c)
{
    pair_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b)
{
    pair_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b)
{
    pair_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float exp2_approx(float a)
{
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(a));
    return d;
}
__device__ __forceinline__ float rcp_approx(float a)
{
    float d;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(a));
    return d;
}

// log2 F(x) for -bound <= x <= 0
template <int ACT> struct LogTail;
template <> struct LogTail<FLEXIQ_ACT_GELU> {
    static constexpr float bound = 16.0f;
    static constexpr int degree = 6;
    static __device__ __forceinline__ constexpr float c(int k)
    {
        constexpr float v[] = {-0.9999997019767761f, 1.1511220932006836f, -0.4590602517127991f, 0.052965421229600906f, 0.007754434831440449f, 0.000658615434076637f,
                               1.9176322894054465e-05f};
        return v[k];
    }
};
template <> struct LogTail<FLEXIQ_ACT_GELU_TANH> {
    static constexpr float bound = 10.0f;
    static constexpr int degree = 8;
    static __device__ __forceinline__ constexpr float c(int k)
    {
        constexpr float v[] = {-1.000000238418579f, 1.1510820388793945f, -0.45948898792266846f, 0.050299640744924545f, 0.005195413716137409f, -0.0026956943329423666f,
                               -0.001993067329749465f, -0.0003464187029749155f, -1.8559790987637825e-05f};
        return v[k];
    }
};

template <int ACT> __device__ __forceinline__ void activate2(float &a, float &b)
{
    const float ma = max_nan(a, 0.f), mb = max_nan(b, 0.f);
    if constexpr (ACT == FLEXIQ_ACT_RELU) {
        a = ma;
        b = mb;
    } else if constexpr (ACT == FLEXIQ_ACT_SILU) {
        const pair_t x = pair(fmaxf(-fabsf(a), -100.f), fmaxf(-fabsf(b), -100.f));
        float za, zb, da, db;
        unpair(mul2(x, pair(1.4426950409f, 1.4426950409f)), &za, &zb);
        const pair_t e = pair(exp2_approx(za), exp2_approx(zb));
        unpair(add2(e, pair(1.f, 1.f)), &da, &db);
        const float r = rcp_approx(__fmul_rn(da, db));
        // (products one by one: a pair in another order, or of one value twice, has to be moved together first)
        unpair(fma2(mul2(x, e), pair(__fmul_rn(r, db), __fmul_rn(r, da)), pair(ma, mb)), &a, &b);
    } else {
        typedef LogTail<ACT> F;
        const pair_t x = pair(fmaxf(-fabsf(a), -F::bound), fmaxf(-fabsf(b), -F::bound));
        pair_t q = pair(F::c(F::degree), F::c(F::degree));
#pragma unroll
        for (int k = F::degree - 1; k >= 0; --k) q = fma2(q, x, pair(F::c(k), F::c(k)));
        float qa, qb;
        unpair(q, &qa, &qb);
        unpair(fma2(x, pair(exp2_approx(qa), exp2_approx(qb)), pair(ma, mb)), &a, &b);
    }
}

template <int ACT, int N> __device__ __forceinline__ void activate_all(pair_t *v)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float a, b;
        unpair(v[i], &a, &b);
        activate2<ACT>(a, b);
        v[i] = pair(a, b);
    }
}
// N pairs.  `act` is the same for the whole launch: one uniform branch
template <int N> __device__ __forceinline__ void activate_n(int act, pair_t *v)
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
