// Group normalisation of channels-last tensors with an activation, into a floating-point tensor or a layer's slab.
//
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c]),   mean and var over an image's positions and a group's channels
//
// The variance is the mean square of the deviations from the mean (two passes over the data), not the difference of two sums, which loses
// everything where the mean is large against the deviation; the rounding error left in the mean, known from the sum of the deviations, is
// taken out of both.  Both are summed in 64 bits: thousands of values a thread in a row are too many for 32.
#include "flexiq_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sm100_ptx.cuh"
#include "eq1_quantize.cuh"
#include "activation.cuh"

namespace flexiq {

constexpr int kNormThreads = 256;

// Where the results go: Y, or the slab of a layer.
struct NormOut {
    void *Y;
    int y_dtype;              // FLEXIQ_DTYPE_I8: the slab
    const int32_t *ent;       // [C/16] where an original chunk of 16 channels lies in the slab | its group's position << 24
    int K_lo;
    QuotientPlan quot;
    float q_scale;
};
struct NormArgs {
    const void *X;
    long long Nb, P;
    int C, groups, x_dtype, act;
    const float *gamma, *beta;
    float eps;
    NormOut out;
};

__device__ __forceinline__ float load_as_f32(const void *p, size_t i, int dtype)
{
    if (dtype == FLEXIQ_DTYPE_F32) return static_cast<const float *>(p)[i];
    if (dtype == FLEXIQ_DTYPE_F16) return __half2float(static_cast<const __half *>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ int quantize_one(const NormOut &o, float v, int c, int *at)
{
    const int ent = o.ent[c >> 4], pos = (ent & 0xffffff) * 16;
    float lo = -128.f, hi = 127.f;
    int mask = -1;
    if (pos < o.K_lo) {
        const int s = ent >> 24;
        hi = (float)(8 << s) - 1.f;
        lo = -(float)(8 << s);
        mask = -1 << s;
    }
    *at = pos + (c & 15);
    float t;
    if (o.quot.form == kQuotTwoTerm) t = TwoTerm::clip(TwoTerm{o.quot.r_hi, o.quot.r_lo}(v), lo, hi);
    else t = Divider::clip(make_divider(o.q_scale)(v), lo, hi);
    return __float2int_rn(t) & mask;
}

__device__ __forceinline__ void store_one(const NormOut &o, size_t row, int C, int c, float v)
{
    const size_t i = row * C + c;
    if (o.y_dtype == FLEXIQ_DTYPE_F32) static_cast<float *>(o.Y)[i] = v;
    else if (o.y_dtype == FLEXIQ_DTYPE_F16) static_cast<__half *>(o.Y)[i] = __float2half_rn(v);
    else if (o.y_dtype == FLEXIQ_DTYPE_BF16) static_cast<__nv_bfloat16 *>(o.Y)[i] = __float2bfloat16_rn(v);
    else {
        int at;
        const int q = quantize_one(o, v, c, &at);
        static_cast<int8_t *>(o.Y)[row * C + at] = (int8_t)q;
    }
}

__device__ __forceinline__ double block_sum(double v, double *s)   // s: one value a warp
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
    for (int i = 0; i < (int)blockDim.x / 32; ++i) t += s[i];
    return t;
}

// One block per image and group.
__global__ void __launch_bounds__(kNormThreads) group_norm_kernel(const NormArgs a)
{
    __shared__ double s[kNormThreads / 32];
    ptx::pdl_wait();
    const int cpg = a.C / a.groups;
    const long long n = a.P * cpg;
    for (long long unit = blockIdx.x; unit < a.Nb * a.groups; unit += gridDim.x) {
        const long long img = unit / a.groups;
        const int c0 = (int)(unit - img * a.groups) * cpg;
        const size_t row0 = (size_t)img * a.P;
        double sum = 0.0;
        for (long long i = threadIdx.x; i < n; i += blockDim.x) sum += load_as_f32(a.X, (row0 + i / cpg) * a.C + c0 + i % cpg, a.x_dtype);
        const float mean = (float)(block_sum(sum, s) / (double)n);
        double dev = 0.0, sq = 0.0;
        for (long long i = threadIdx.x; i < n; i += blockDim.x) {
            const float d = load_as_f32(a.X, (row0 + i / cpg) * a.C + c0 + i % cpg, a.x_dtype) - mean;
            dev += d;
            sq += (double)d * d;
        }
        const float off = (float)(block_sum(dev, s) / (double)n);   // the mean's rounding error
        const float var = fmaxf((float)(block_sum(sq, s) / (double)n) - off * off, 0.f);
        const float rstd = 1.0f / sqrtf(var + a.eps);
        for (long long i = threadIdx.x; i < n; i += blockDim.x) {
            const int c = c0 + (int)(i % cpg);
            const size_t row = row0 + i / cpg;
            const float d = load_as_f32(a.X, row * a.C + c, a.x_dtype) - mean;
            const float scale = rstd * (a.gamma ? a.gamma[c] : 1.f);
            store_one(a.out, row, a.C, c, activate_one(a.act, fmaf(d, scale, fmaf(-off, scale, a.beta ? a.beta[c] : 0.f))));
        }
    }
}

static int check_shape(int x_dtype, int64_t Nb, int64_t P, int C, int groups)
{
    if (x_dtype != FLEXIQ_DTYPE_F32 && x_dtype != FLEXIQ_DTYPE_F16 && x_dtype != FLEXIQ_DTYPE_BF16)
        return set_error(FLEXIQ_ERR_INVALID_ARG, "x_dtype %d is not F32, F16 or BF16", x_dtype);
    if (Nb < 0 || P < 0) return set_error(FLEXIQ_ERR_INVALID_ARG, "bad shape: Nb = %lld, P = %lld", (long long)Nb, (long long)P);
    if (C <= 0 || groups <= 0 || C % groups) return set_error(FLEXIQ_ERR_INVALID_ARG, "C = %d is not a positive multiple of groups = %d", C, groups);
    int64_t rows, values;
    if (__builtin_mul_overflow(Nb, P, &rows) || __builtin_mul_overflow(rows, (int64_t)C * 4, &values))
        return set_error(FLEXIQ_ERR_INVALID_ARG, "Nb * P * C does not fit 64 bits");
    return FLEXIQ_OK;
}
static int check_norm(const void *X, int x_dtype, int64_t Nb, int64_t P, int C, int groups, const float *gamma, const float *beta, float eps, int act, const void *Y)
{
    if (int rc = check_shape(x_dtype, Nb, P, C, groups)) return rc;
    if (!act_known(act)) return set_error(FLEXIQ_ERR_INVALID_ARG, "unknown act %d", act);
    if (!(eps > 0.0f) || eps > 3.0e38f) return set_error(FLEXIQ_ERR_INVALID_ARG, "eps %g must be positive", (double)eps);
    if (Nb == 0 || P == 0) return FLEXIQ_OK;
    if (!X || !Y) return set_error(FLEXIQ_ERR_INVALID_ARG, "the input or the output is NULL");
    if ((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(Y) | reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(beta)) & 15)
        return set_error(FLEXIQ_ERR_INVALID_ARG, "X_dev, the output, gamma_dev and beta_dev must be 16-byte aligned");
    return FLEXIQ_OK;
}

static int run_norm(const NormArgs &a, void *scratch, cudaStream_t st)
{
    const long long units = a.Nb * a.groups;
    FLEXIQ_CUDA_TRY(launch_pdl(group_norm_kernel, (unsigned)(units < 65536 ? units : 65536), kNormThreads, 0, st, a));
    return FLEXIQ_OK;
}

}  // namespace flexiq

using namespace flexiq;

extern "C" int flexiq_group_norm_scratch(int x_dtype, int64_t Nb, int64_t P, int C, int groups, int64_t *bytes_out)
{
    if (!bytes_out) return set_error(FLEXIQ_ERR_INVALID_ARG, "bytes_out is NULL");
    if (int rc = check_shape(x_dtype, Nb, P, C, groups)) return rc;
    *bytes_out = 0;
    return FLEXIQ_OK;
}

extern "C" int flexiq_group_norm(const void *X_dev, int x_dtype, int64_t Nb, int64_t P, int C, int groups, const float *gamma_dev,
                                 const float *beta_dev, float eps, int act, int y_dtype, void *Y_dev, void *scratch_dev, void *stream)
{
    if (y_dtype != FLEXIQ_DTYPE_F32 && y_dtype != FLEXIQ_DTYPE_F16 && y_dtype != FLEXIQ_DTYPE_BF16)
        return set_error(FLEXIQ_ERR_INVALID_ARG, "y_dtype %d is not F32, F16 or BF16", y_dtype);
    int rc = check_norm(X_dev, x_dtype, Nb, P, C, groups, gamma_dev, beta_dev, eps, act, Y_dev);
    if (rc) return rc;
    if (X_dev == Y_dev && x_dtype != y_dtype && Nb && P) return set_error(FLEXIQ_ERR_INVALID_ARG, "Y_dev is X_dev, which needs the same type");
    if (Nb == 0 || P == 0) return FLEXIQ_OK;
    if ((rc = check_device_sm100())) return rc;
    NormArgs a{};
    a.X = X_dev; a.Nb = Nb; a.P = P; a.C = C; a.groups = groups; a.x_dtype = x_dtype; a.act = act;
    a.gamma = gamma_dev; a.beta = beta_dev; a.eps = eps;
    a.out.Y = Y_dev; a.out.y_dtype = y_dtype;
    return run_norm(a, scratch_dev, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int flexiq_group_norm_to_slab(flexiq_layer_t layer, const void *X_dev, int x_dtype, int64_t Nb, int64_t P, int groups,
                                         const float *gamma_dev, const float *beta_dev, float eps, int act, float x_scale,
                                         uint8_t *X4_dev, void *scratch_dev, void *stream)
{
    Layer *L = as_layer(layer);
    if (!L) return set_error(FLEXIQ_ERR_INVALID_ARG, "not a live flexiq layer handle");
    if (L->lowbit_path != FLEXIQ_LOWBIT_MASKED_I8) return set_error(FLEXIQ_ERR_UNSUPPORTED, "the layer must use the masked low-bit path");
    if (!(x_scale > 0.0f)) return set_error(FLEXIQ_ERR_INVALID_ARG, "x_scale %g must be positive", (double)x_scale);
    int rc = check_norm(X_dev, x_dtype, Nb, P, L->C, groups, gamma_dev, beta_dev, eps, act, X4_dev);
    if (rc) return rc;
    if (Nb == 0 || P == 0) return FLEXIQ_OK;
    if (static_cast<const void *>(X4_dev) == X_dev) return set_error(FLEXIQ_ERR_INVALID_ARG, "the slab cannot be X_dev");
    if ((rc = check_device_sm100())) return rc;
    if ((rc = check_layer_device(L))) return rc;
    NormArgs a{};
    a.X = X_dev; a.Nb = Nb; a.P = P; a.C = L->C; a.groups = groups; a.x_dtype = x_dtype; a.act = act;
    a.gamma = gamma_dev; a.beta = beta_dev; a.eps = eps;
    a.out.Y = X4_dev; a.out.y_dtype = FLEXIQ_DTYPE_I8;
    a.out.ent = L->chunk_ent; a.out.K_lo = L->K_lo;
    a.out.quot = quotient_plan(L, x_scale, FLEXIQ_DTYPE_F32);
    a.out.q_scale = x_scale;
    if ((rc = run_norm(a, scratch_dev, reinterpret_cast<cudaStream_t>(stream)))) return rc;
    record_slab(L, X4_dev, L->K_lo);
    return FLEXIQ_OK;
}
