// Group normalisation of channels-last tensors with an activation, into a floating-point tensor or a layer's slab.
//
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c]),   mean and var over an image's positions and a group's channels
//
// Bound by memory: every input byte is to be read once and every output byte written once.  Three ways, by what fits where:
//   rows   one position per image (layer normalisation): a warp holds a group in registers
//   held   an image's block of channels (whole groups, 128 bytes a position where that is enough) is held in the registers of a block, or of a
//          cluster of up to eight, between the statistics and their use; the blocks of a cluster exchange their groups' statistics
//          through distributed shared memory
//   twice  larger images: the statistics of pieces of an image go to scratch memory, and a second kernel reads the input again, in
//          the reverse order, so that what the L2 cache still holds of it comes first
//
// Statistics.  The variance is a mean square of deviations, never a difference of two sums, which would lose everything where the mean
// is large against the deviation.  A thread takes the mean and the sum of squared deviations M2 of its own values (at most 128, in registers, two
// passes); those are joined in a fixed order by
//   mean = ref + sum n_i (mean_i - ref) / n,   M2 = sum M2_i + n_i (mean_i - mean)^2          (ref: one of the means)
// over the threads, the cluster's blocks or the pieces.  No sum is longer than some sixty roundings, and results do not depend on timing.
#include "flexiq_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "sm100_ptx.cuh"
#include "eq1_quantize.cuh"
#include "activation.cuh"
#include "norm_plan.h"

namespace flexiq {


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
    int C, groups, act;
    const float *gamma, *beta;
    float eps;
    NormOut out;
    // the plan
    int cpg;                  // channels per group
    int gpb, nch;             // groups of a channel block, and its 16-byte (scalar form: one-value) pieces per position
    int cpt;                  // pieces of a position a thread has where there are more than threads, else 1
    int lanes;                // positions side by side in a block
    int cluster;              // blocks per image and channel block ("held"), or pieces of the image ("twice")
    long long span;           // positions of one of them
    float2 *stats;            // "twice": [image][group][piece] mean, M2
};

__device__ __forceinline__ uint4 load_piece(const void *p)
{
    uint4 u;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
    return u;
}

// VEC values in a row as they are: a 16-byte piece, or one value
template <int DT, int VEC> struct Piece {
    static constexpr int kBytes = DT == FLEXIQ_DTYPE_F32 ? 4 : 2;
    typename std::conditional<VEC == 1, float, uint4>::type raw;
    __device__ __forceinline__ void load(const void *X, size_t i)
    {
        const char *p = static_cast<const char *>(X) + i * kBytes;
        if constexpr (VEC == 1) {
            if (DT == FLEXIQ_DTYPE_F32) raw = *reinterpret_cast<const float *>(p);
            else if (DT == FLEXIQ_DTYPE_F16) raw = __half2float(*reinterpret_cast<const __half *>(p));
            else raw = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p));
        } else {
            raw = load_piece(p);
        }
    }
    __device__ __forceinline__ void widen(float *x) const
    {
        if constexpr (VEC == 1) x[0] = raw;
        else {
#pragma unroll
            for (int k = 0; k < VEC / 4; ++k) widen4<DT>(&raw, k, x + 4 * k);
        }
    }
};
template <int DT> struct FullVec { static constexpr int v = DT == FLEXIQ_DTYPE_F32 ? 4 : 8; };

// int8 of N values for slab chunk entry `ent`
template <int N> __device__ __forceinline__ void quantize_values(const NormOut &o, int ent, const float *v, unsigned *words)
{
    float lo = -128.f, hi = 127.f;
    unsigned mask = 0xffffffffu;
    if ((ent & 0xffffff) * 16 < o.K_lo) {
        const int s = ent >> 24;
        hi = (float)(8 << s) - 1.f;
        lo = -(float)(8 << s);
        mask = ((0xffu << s) & 0xffu) * 0x01010101u;
    }
    float t[N < 4 ? 4 : N] = {};
    if (o.quot.form == kQuotTwoTerm) {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = TwoTerm::clip(TwoTerm{o.quot.r_hi, o.quot.r_lo}(v[i]), lo, hi);
    } else {
        const Divider div = make_divider(o.q_scale);
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = Divider::clip(div(v[i]), lo, hi);
    }
#pragma unroll
    for (int i = 0; i < (N + 3) / 4; ++i) words[i] = quant4(t[4 * i], t[4 * i + 1], t[4 * i + 2], t[4 * i + 3]) & mask;
}
__device__ __forceinline__ unsigned pack_f16(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned *>(&h);
}
__device__ __forceinline__ unsigned pack_bf16(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned *>(&h);
}

// What a thread keeps of its channels: y = (x - mean) scale + beta.  (x scale + b with the mean in b would round b, by up to 2^-24 |mean| scale: a constant
// image came out 4e-5 off its beta.)  MANY: the channels belong to several groups, with a mean each.
template <int VEC, bool MANY> struct Affine {
    float minus[MANY ? VEC : 1], scale[VEC], beta[VEC];
    int ent;                  // the slab's entry of their chunk
    // of channels c .. and their groups' (mean, 1 / deviation)
    __device__ __forceinline__ void set(const NormArgs &n, int c, const float2 *stat)
    {
        if constexpr (VEC == 1) {
            scale[0] = n.gamma ? n.gamma[c] : 1.f;
            beta[0] = n.beta ? n.beta[c] : 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i) {
                const float4 g = n.gamma ? reinterpret_cast<const float4 *>(n.gamma + c)[i] : make_float4(1.f, 1.f, 1.f, 1.f);
                const float4 h = n.beta ? reinterpret_cast<const float4 *>(n.beta + c)[i] : make_float4(0.f, 0.f, 0.f, 0.f);
                scale[4 * i] = g.x; scale[4 * i + 1] = g.y; scale[4 * i + 2] = g.z; scale[4 * i + 3] = g.w;
                beta[4 * i] = h.x; beta[4 * i + 1] = h.y; beta[4 * i + 2] = h.z; beta[4 * i + 3] = h.w;
            }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) scale[i] = __fmul_rn(scale[i], stat[MANY ? i : 0].y);
#pragma unroll
        for (int i = 0; i < (MANY ? VEC : 1); ++i) minus[i] = -stat[i].x;
        ent = n.out.y_dtype == FLEXIQ_DTYPE_I8 ? n.out.ent[c >> 4] : 0;
    }
};
// VEC values at channel c of a row, normalised and activated, to where they go
template <int VEC, bool MANY> __device__ __forceinline__ void finish_values(const NormArgs &n, size_t row, int c, const float *x, const Affine<VEC, MANY> &f)
{
    const NormOut &o = n.out;
    const int ent = f.ent;
    float y[VEC];
    if constexpr (VEC == 1) {
        y[0] = activate_one(n.act, __fmaf_rn(__fadd_rn(x[0], f.minus[0]), f.scale[0], f.beta[0]));
        const size_t i = row * n.C + c;
        if (o.y_dtype == FLEXIQ_DTYPE_F32) static_cast<float *>(o.Y)[i] = y[0];
        else if (o.y_dtype == FLEXIQ_DTYPE_F16) static_cast<__half *>(o.Y)[i] = __float2half_rn(y[0]);
        else if (o.y_dtype == FLEXIQ_DTYPE_BF16) static_cast<__nv_bfloat16 *>(o.Y)[i] = __float2bfloat16_rn(y[0]);
        else {
            unsigned w;
            quantize_values<1>(o, ent, y, &w);
            static_cast<int8_t *>(o.Y)[row * n.C + (ent & 0xffffff) * 16 + (c & 15)] = (int8_t)w;
        }
    } else {
        pair_t t[VEC / 2];
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i)
            t[i] = fma2(add2(pair(x[2 * i], x[2 * i + 1]), pair(f.minus[MANY ? 2 * i : 0], f.minus[MANY ? 2 * i + 1 : 0])),
                        pair(f.scale[2 * i], f.scale[2 * i + 1]), pair(f.beta[2 * i], f.beta[2 * i + 1]));
        activate_n<VEC / 2>(n.act, t);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) unpair(t[i], &y[2 * i], &y[2 * i + 1]);
        if (o.y_dtype == FLEXIQ_DTYPE_F32) {
            float4 *to = reinterpret_cast<float4 *>(static_cast<float *>(o.Y) + row * n.C + c);
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i) to[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        } else if (o.y_dtype != FLEXIQ_DTYPE_I8) {
            unsigned w[VEC / 2];
            if (o.y_dtype == FLEXIQ_DTYPE_F16) {
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) w[i] = pack_f16(y[2 * i], y[2 * i + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) w[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
            }
            void *to = static_cast<char *>(o.Y) + (row * n.C + c) * 2;
            if constexpr (VEC == 8) *static_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            else *static_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        } else {
            unsigned w[VEC / 4];
            quantize_values<VEC>(o, ent, y, w);
            void *to = static_cast<char *>(o.Y) + row * n.C + (ent & 0xffffff) * 16 + (c & 15);
            if constexpr (VEC == 8) *static_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
            else *static_cast<unsigned *>(to) = w[0];
        }
    }
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float deviation_inverse(float M2, float n, float eps) { return __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(M2, n), eps))); }

// Mean and M2 of one run of values: tile by tile, joined as above
struct Moments {
    float n, mean, M2;
    __device__ __forceinline__ void join(float nb, float mb, float Mb)
    {
        const float all = n + nb, d = mb - mean, share = n > 0.f ? __fdiv_rn(nb, all) : 1.f;
        mean = __fmaf_rn(d, share, mean);
        M2 = __fadd_rn(M2, __fmaf_rn(__fmul_rn(d, d), __fmul_rn(n, share), Mb));
        n = all;
    }
};

// Sums and then squared deviations of the values of NV pieces, `valid` bit by bit; MANY: each channel of the piece apart.  Returns the pieces counted.
template <int DT, int VEC, int NV, bool MANY>
__device__ __forceinline__ int piece_moments(const Piece<DT, VEC> *v, unsigned valid, float *mean, float *M2)
{
    constexpr int S = MANY ? VEC : 1;
    const int cnt = __popc(valid);
    float s[S] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (valid >> j & 1) {
            float x[VEC];
            v[j].widen(x);
            if (MANY) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[i % S] += x[i];
            } else {
#pragma unroll
                for (int w = VEC / 2; w; w >>= 1)
#pragma unroll
                    for (int i = 0; i < w; ++i) x[i] += x[i + w];
                s[0] += x[0];
            }
        }
    const float count = (float)(cnt ? cnt * (MANY ? 1 : VEC) : 1);   // (divided by, not multiplied by an inverse: the mean of equal values is that value)
#pragma unroll
    for (int i = 0; i < S; ++i) { mean[i] = __fdiv_rn(s[i], count); M2[i] = 0.f; }
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (valid >> j & 1) {
            float x[VEC];
            v[j].widen(x);
            if (MANY) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) { const float d = x[i] - mean[i % S]; M2[i % S] = __fmaf_rn(d, d, M2[i % S]); }
            } else {
                float q = 0.f;
#pragma unroll
                for (int i = 0; i < VEC; ++i) { const float d = x[i] - mean[0]; q = __fmaf_rn(d, d, q); }
                M2[0] += q;
            }
        }
    return cnt;
}

// What the threads of a block found -> their groups' moments in gstat[0 .. gpb): a warp per group over the entries of its threads (its channels').
template <int VEC, bool MANY>
__device__ __forceinline__ void block_moments(const NormArgs &a, float *red_mean, float *red_M2, const float *red_n, Moments *gstat)
{
    constexpr int S = MANY ? VEC : 1;
    __syncthreads();
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const int pitch = a.cpt > 1 ? (int)blockDim.x : a.nch * S, each = a.cpt > 1 ? (int)blockDim.x : (MANY ? a.cpg : a.cpg / VEC);   // entries of a position, and of a group among them
    for (int g = threadIdx.x >> 5; g < a.gpb; g += warps) {
        const int total = a.lanes * each, first = g * each;
        const float ref = red_mean[first];
        float n = 0.f, d = 0.f;
        for (int i = lane; i < total; i += 32) {
            const int row = i / each, e = row * pitch + first + (i - row * each);
            const float w = red_n[MANY ? e / S : e];
            n += w;
            d = __fmaf_rn(w, red_mean[e] - ref, d);
        }
        n = warp_sum(n);
        d = warp_sum(d);
        const float mean = n > 0.f ? ref + __fdiv_rn(d, n) : 0.f;
        float M2 = 0.f;
        for (int i = lane; i < total; i += 32) {
            const int row = i / each, e = row * pitch + first + (i - row * each);
            const float w = red_n[MANY ? e / S : e], q = red_mean[e] - mean;
            if (w > 0.f) M2 += __fmaf_rn(w * q, q, red_M2[e]);
        }
        M2 = warp_sum(M2);
        if (lane == 0) gstat[g] = Moments{n, mean, M2};
    }
    __syncthreads();
}

// Which pieces a thread has: piece j of its positions
struct Pieces {
    int col, pl;        // its column and position side by side; cpt > 1: its first column, position 0
    bool live;
    __device__ __forceinline__ Pieces(const NormArgs &a)
    {
        const int t = threadIdx.x;
        if (a.cpt > 1) { pl = 0; col = t; live = true; }
        else { pl = t / a.nch; col = t - pl * a.nch; live = pl < a.lanes; }
    }
    // (position, column) of the thread's piece j, walked in order
    struct Walk {
        int p, c, k;
    };
    __device__ __forceinline__ Walk begin() const { return Walk{pl, col, 0}; }
    __device__ __forceinline__ void next(const NormArgs &a, Walk &w) const
    {
        if (a.cpt > 1) {
            w.c += blockDim.x;
            if (++w.k == a.cpt) { w.k = 0; w.c = col; ++w.p; }
        } else {
            w.p += a.lanes;
        }
    }
};

// (mean, 1 / deviation) of the channels of column `col` (MANY: of each)
template <int VEC, bool MANY> __device__ __forceinline__ void column_stats(const NormArgs &a, int col, const float2 *fin, float2 *stat)
{
    int g = col * VEC / a.cpg, left = a.cpg - (col * VEC - g * a.cpg);
    stat[0] = fin[g];
#pragma unroll
    for (int i = 1; i < (MANY ? VEC : 1); ++i) {
        if (--left == 0) { left = a.cpg; ++g; }
        stat[i] = fin[g];
    }
}

// "held": block rank `blockIdx.x % cluster` of an image's channel block
template <int DT, int VEC, int NV, bool MANY>
__global__ void __launch_bounds__(kNormThreads, NV <= 4 ? 4 : 2) group_norm_held_kernel(const NormArgs a)
{
    constexpr int S = MANY ? VEC : 1;
    __shared__ float red_mean[kNormThreads * S], red_M2[kNormThreads * S], red_n[kNormThreads];
    __shared__ Moments gstat[kMaxGroups];
    __shared__ float2 fin[kMaxGroups];
    const int blocks = a.groups / a.gpb;                       // channel blocks
    const unsigned unit = blockIdx.x / (unsigned)a.cluster;
    const int rank = (int)(blockIdx.x - unit * (unsigned)a.cluster);
    const long long img = unit / (unsigned)blocks;
    const int c0 = (int)(unit - (unsigned)img * (unsigned)blocks) * a.gpb * a.cpg;
    const long long p0 = rank * a.span, left = a.P - p0;
    const int mine = (int)(left < 0 ? 0 : left < a.span ? left : a.span);
    const size_t row0 = (size_t)img * a.P + p0;
    const Pieces who(a);
    ptx::pdl_wait();
    Piece<DT, VEC> v[NV];
    unsigned valid = 0;
    {
        Pieces::Walk w = who.begin();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (who.live && w.p < mine && w.c < a.nch) {
                v[j].load(a.X, (row0 + w.p) * a.C + c0 + w.c * VEC);
                valid |= 1u << j;
            }
            who.next(a, w);
        }
    }
    float mean[S], M2[S];
    const int cnt = piece_moments<DT, VEC, NV, MANY>(v, valid, mean, M2);
#pragma unroll
    for (int i = 0; i < S; ++i) { red_mean[threadIdx.x * S + i] = mean[i]; red_M2[threadIdx.x * S + i] = M2[i]; }
    red_n[threadIdx.x] = (float)(cnt * (MANY ? 1 : VEC));
    block_moments<VEC, MANY>(a, red_mean, red_M2, red_n, gstat);
    if (a.cluster > 1) {
        ptx::cluster_sync_all();
        for (int g = threadIdx.x; g < a.gpb; g += blockDim.x) {
            float n[kNormCluster], m[kNormCluster], q[kNormCluster];
#pragma unroll
            for (int r = 0; r < kNormCluster; ++r) {
                n[r] = m[r] = q[r] = 0.f;
                if (r < a.cluster) {
                    const uint32_t at = ptx::mapa(ptx::smem_u32(&gstat[g]), (uint32_t)r);
                    n[r] = __uint_as_float(ptx::ld_shared_cluster(at));
                    m[r] = __uint_as_float(ptx::ld_shared_cluster(at + 4));
                    q[r] = __uint_as_float(ptx::ld_shared_cluster(at + 8));
                }
            }
            float all = 0.f, d = 0.f, M = 0.f;
#pragma unroll
            for (int r = 0; r < kNormCluster; ++r) { all += n[r]; d = __fmaf_rn(n[r], m[r] - m[0], d); }
            const float centre = m[0] + __fdiv_rn(d, all);
#pragma unroll
            for (int r = 0; r < kNormCluster; ++r) { const float o = m[r] - centre; if (n[r] > 0.f) M += __fmaf_rn(n[r] * o, o, q[r]); }
            fin[g] = make_float2(centre, deviation_inverse(M, all, a.eps));
        }
    } else {
        for (int g = threadIdx.x; g < a.gpb; g += blockDim.x) fin[g] = make_float2(gstat[g].mean, deviation_inverse(gstat[g].M2, gstat[g].n, a.eps));
    }
    ptx::pdl_launch_dependents();
    __syncthreads();
    if (a.cluster > 1) ptx::cluster_arrive();                  // this block has read what it needs of the others
    if (valid) {
        float2 stat[MANY ? VEC : 1];
        Affine<VEC, MANY> f;
        Pieces::Walk w = who.begin();
        auto column = [&]() {
            column_stats<VEC, MANY>(a, a.cpt > 1 ? 0 : w.c, fin, stat);   // (cpt > 1: one group)
            f.set(a, c0 + w.c * VEC, stat);
        };
        column();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (valid >> j & 1) {
                if (a.cpt > 1 && j) column();
                float x[VEC];
                v[j].widen(x);
                finish_values(a, row0 + w.p, c0 + w.c * VEC, x, f);
            }
            who.next(a, w);
        }
    }
    __syncwarp();
    if (a.cluster > 1) ptx::cluster_wait();                    // the others have read what they need of this one
}

// "twice", the first: moments of a piece of an image's channel block
template <int DT, int VEC, bool MANY>
__global__ void __launch_bounds__(kNormThreads, 2) group_norm_stats_kernel(const NormArgs a)
{
    constexpr int S = MANY ? VEC : 1, NV = 8;
    __shared__ float red_mean[kNormThreads * S], red_M2[kNormThreads * S], red_n[kNormThreads];
    __shared__ Moments gstat[kMaxGroups];
    const int blocks = a.groups / a.gpb;
    const unsigned unit = blockIdx.x / (unsigned)a.cluster;
    const int piece = (int)(blockIdx.x - unit * (unsigned)a.cluster);
    const long long img = unit / (unsigned)blocks;
    const int block = (int)(unit - (unsigned)img * (unsigned)blocks), c0 = block * a.gpb * a.cpg;
    const long long p0 = piece * a.span, left = a.P - p0, mine = left < 0 ? 0 : left < a.span ? left : a.span;
    const size_t row0 = (size_t)img * a.P + p0;
    const Pieces who(a);
    ptx::pdl_wait();
    Moments sum[S];
#pragma unroll
    for (int i = 0; i < S; ++i) sum[i] = Moments{0.f, 0.f, 0.f};
    const int tile = a.cpt > 1 ? 1 : a.lanes * NV;             // positions a step (cpt > 1: NV of a position's pieces a step)
    for (long long base = 0; base < mine; base += tile) {
        for (int k0 = 0; k0 < a.cpt; k0 += NV) {
            Piece<DT, VEC> v[NV];
            unsigned valid = 0;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const long long p = base + (a.cpt > 1 ? 0 : who.pl + j * a.lanes);
                const int c = a.cpt > 1 ? who.col + (k0 + j) * (int)blockDim.x : who.col;
                if (who.live && p < mine && c < a.nch) {
                    v[j].load(a.X, (row0 + p) * a.C + c0 + c * VEC);
                    valid |= 1u << j;
                }
            }
            float mean[S], M2[S];
            const float n = (float)(piece_moments<DT, VEC, NV, MANY>(v, valid, mean, M2) * (MANY ? 1 : VEC));
#pragma unroll
            for (int i = 0; i < S; ++i) sum[i].join(n, mean[i], M2[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < S; ++i) { red_mean[threadIdx.x * S + i] = sum[i].mean; red_M2[threadIdx.x * S + i] = sum[i].M2; }
    red_n[threadIdx.x] = sum[0].n;
    ptx::pdl_launch_dependents();
    block_moments<VEC, MANY>(a, red_mean, red_M2, red_n, gstat);
    for (int g = threadIdx.x; g < a.gpb; g += blockDim.x)
        a.stats[((size_t)img * a.groups + block * a.gpb + g) * a.cluster + piece] = make_float2(gstat[g].mean, gstat[g].M2);
}

// "twice", the second: the pieces' moments joined, and the values.  Blocks in reverse order: what was read last is in the L2 cache.
template <int DT, int VEC, bool MANY>
__global__ void __launch_bounds__(kNormThreads, 4) group_norm_apply_kernel(const NormArgs a)
{
    constexpr int NV = 4;
    __shared__ float2 fin[kMaxGroups];
    const int blocks = a.groups / a.gpb;
    const unsigned id = gridDim.x - 1 - blockIdx.x, unit = id / (unsigned)a.cluster;
    const int piece = (int)(id - unit * (unsigned)a.cluster);
    const long long img = unit / (unsigned)blocks;
    const int block = (int)(unit - (unsigned)img * (unsigned)blocks), c0 = block * a.gpb * a.cpg;
    const long long p0 = piece * a.span, left = a.P - p0, mine = left < 0 ? 0 : left < a.span ? left : a.span;
    const size_t row0 = (size_t)img * a.P + p0;
    const Pieces who(a);
    const int lane = threadIdx.x & 31;
    ptx::pdl_wait();
    for (int g = threadIdx.x >> 5; g < a.gpb; g += (int)blockDim.x >> 5) {
        const float2 *from = a.stats + ((size_t)img * a.groups + block * a.gpb + g) * a.cluster;
        const float ref = from[0].x;
        float n[kNormSplits / 32], m[kNormSplits / 32], q[kNormSplits / 32], all = 0.f, d = 0.f, M2 = 0.f;
#pragma unroll
        for (int k = 0; k < kNormSplits / 32; ++k) {
            const int i = lane + 32 * k;
            n[k] = m[k] = q[k] = 0.f;
            if (i < a.cluster) {
                const long long rest = a.P - i * a.span, has = rest < 0 ? 0 : rest < a.span ? rest : a.span;
                const float2 s = from[i];
                n[k] = (float)(has * a.cpg);
                m[k] = s.x;
                q[k] = s.y;
            }
            all += n[k];
            if (n[k] > 0.f) d = __fmaf_rn(n[k], m[k] - ref, d);
        }
        all = warp_sum(all);
        const float centre = ref + __fdiv_rn(warp_sum(d), all);
#pragma unroll
        for (int k = 0; k < kNormSplits / 32; ++k) { const float o = m[k] - centre; if (n[k] > 0.f) M2 += __fmaf_rn(n[k] * o, o, q[k]); }
        M2 = warp_sum(M2);
        if (lane == 0) fin[g] = make_float2(centre, deviation_inverse(M2, all, a.eps));
    }
    __syncthreads();
    ptx::pdl_launch_dependents();
    float2 stat[MANY ? VEC : 1];
    Affine<VEC, MANY> f;
    auto column = [&](int c) {
        column_stats<VEC, MANY>(a, a.cpt > 1 ? 0 : c, fin, stat);
        f.set(a, c0 + c * VEC, stat);
    };
    if (a.cpt > 1) {
        for (long long p = 0; p < mine; ++p)
            for (int c = who.col; c < a.nch; c += blockDim.x) {
                Piece<DT, VEC> v;
                v.load(a.X, (row0 + p) * a.C + c0 + c * VEC);
                column(c);
                float x[VEC];
                v.widen(x);
                finish_values(a, row0 + p, c0 + c * VEC, x, f);
            }
        return;
    }
    if (!who.live) return;
    column(who.col);
    const int c = c0 + who.col * VEC;
    for (long long base = who.pl; base < mine; base += (long long)a.lanes * NV) {
        Piece<DT, VEC> v[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (base + j * a.lanes < mine) v[j].load(a.X, (row0 + base + j * a.lanes) * a.C + c);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (base + j * a.lanes < mine) {
                float x[VEC];
                v[j].widen(x);
                finish_values(a, row0 + base + j * a.lanes, c, x, f);
            }
    }
}

// "rows": one position per image.  A warp takes a group at a time (its cpg values are contiguous) and has the next one's values on the way.
template <int DT, int VEC, int NV>
__global__ void __launch_bounds__(kNormThreads, NV <= 4 ? 4 : 2) group_norm_rows_kernel(const NormArgs a)
{
    const int lane = threadIdx.x & 31;
    const long long total = a.Nb * a.groups, step = (long long)gridDim.x * (blockDim.x >> 5);
    long long seg = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    ptx::pdl_wait();
    Piece<DT, VEC> next[NV], v[NV];
    auto request = [&](long long s) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + 32 * j < a.nch) next[j].load(a.X, (size_t)s * a.cpg + (lane + 32 * j) * VEC);
    };
    if (seg < total) request(seg);
    for (; seg < total; seg += step) {
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = next[j];
        if (seg + step < total) request(seg + step);
        else ptx::pdl_launch_dependents();
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + 32 * j < a.nch) {
                float x[VEC];
                v[j].widen(x);
#pragma unroll
                for (int w = VEC / 2; w; w >>= 1)
#pragma unroll
                    for (int i = 0; i < w; ++i) x[i] += x[i + w];
                s += x[0];
            }
        const float mean = __fdiv_rn(warp_sum(s), (float)a.cpg);
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + 32 * j < a.nch) {
                float x[VEC];
                v[j].widen(x);
#pragma unroll
                for (int i = 0; i < VEC; ++i) { const float d = x[i] - mean; q = __fmaf_rn(d, d, q); }
            }
        const float rstd = deviation_inverse(warp_sum(q), (float)a.cpg, a.eps);
        const long long row = a.groups == 1 ? seg : seg / a.groups;
        const int c0 = a.groups == 1 ? 0 : (int)(seg - row * a.groups) * a.cpg;
        const float2 stat = make_float2(mean, rstd);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (lane + 32 * j < a.nch) {
                const int c = c0 + (lane + 32 * j) * VEC;
                float x[VEC];
                Affine<VEC, false> f;
                v[j].widen(x);
                f.set(a, c, &stat);
                finish_values(a, (size_t)row, c, x, f);
            }
    }
}

// ------------------------------------------------------------------------------------ host side
template <int DT, int VEC, int NV, bool MANY> static int launch_held(const NormArgs &a, const NormPlan &p, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.Nb * (a.groups / a.gpb) * a.cluster), 1, 1);
    cfg.blockDim = dim3((unsigned)p.threads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.cluster > 1 ? 2 : 1;
    FLEXIQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, group_norm_held_kernel<DT, VEC, NV, MANY>, a));
    return FLEXIQ_OK;
}
template <int DT, int VEC, bool MANY> static int launch_held_nv(const NormArgs &a, const NormPlan &p, cudaStream_t st)
{
    switch (p.nv) {
        case 1: return launch_held<DT, VEC, 1, MANY>(a, p, st);
        case 2: return launch_held<DT, VEC, 2, MANY>(a, p, st);
        case 4: return launch_held<DT, VEC, 4, MANY>(a, p, st);
        case 8: return launch_held<DT, VEC, 8, MANY>(a, p, st);
        default: return launch_held<DT, VEC, 16, MANY>(a, p, st);
    }
}
template <int DT, int VEC, bool MANY> static int launch_twice(const NormArgs &a, const NormPlan &p, cudaStream_t st)
{
    const unsigned grid = (unsigned)(a.Nb * (a.groups / a.gpb) * a.cluster);
    FLEXIQ_CUDA_TRY(launch_pdl(group_norm_stats_kernel<DT, VEC, MANY>, grid, (unsigned)p.threads, 0, st, a));
    FLEXIQ_CUDA_TRY(launch_pdl(group_norm_apply_kernel<DT, VEC, MANY>, grid, (unsigned)p.threads, 0, st, a));
    return FLEXIQ_OK;
}
template <int DT, int VEC> static int launch_norm_rows(const NormArgs &a, const NormPlan &p, int sms, cudaStream_t st)
{
    // few rows: as many blocks as there are; many: four blocks of eight warps an SM, each walking over rows
    const long long total = a.Nb * a.groups;
    const unsigned threads = total < 8ll * sms ? 64 : kNormThreads;
    long long blocks = ceil_div(total, threads / 32);
    const long long most = 4ll * sms;
    if (blocks > most && threads == kNormThreads) blocks = most;
    auto go = [&](auto kernel) -> int { FLEXIQ_CUDA_TRY(launch_pdl(kernel, (unsigned)blocks, threads, 0, st, a)); return FLEXIQ_OK; };
    switch (p.nv) {
        case 1: return go(group_norm_rows_kernel<DT, VEC, 1>);
        case 2: return go(group_norm_rows_kernel<DT, VEC, 2>);
        case 3: return go(group_norm_rows_kernel<DT, VEC, 3>);
        case 4: return go(group_norm_rows_kernel<DT, VEC, 4>);
        case 5: case 6: return go(group_norm_rows_kernel<DT, VEC, 6>);
        default: return go(group_norm_rows_kernel<DT, VEC, 8>);
    }
}
template <int DT> static int launch_norm(const NormArgs &a, const NormPlan &p, int sms, cudaStream_t st)
{
    constexpr int V = FullVec<DT>::v;
    if (p.kind == kNormRows) return p.vec == 1 ? launch_norm_rows<DT, 1>(a, p, sms, st) : launch_norm_rows<DT, V>(a, p, sms, st);
    if (p.kind == kNormHeld) return p.vec == 1 ? launch_held_nv<DT, 1, false>(a, p, st) : p.many ? launch_held_nv<DT, V, true>(a, p, st) : launch_held_nv<DT, V, false>(a, p, st);
    return p.vec == 1 ? launch_twice<DT, 1, false>(a, p, st) : p.many ? launch_twice<DT, V, true>(a, p, st) : launch_twice<DT, V, false>(a, p, st);
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

// SMs of the device the plan is for: the current one (148 where there is none to ask)
static int plan_sms()
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 148; }
    const int n = device_sm_count(dev);
    return n > 0 ? n : 148;
}
static long long scratch_bytes(const NormPlan &p, long long Nb, int groups) { return p.kind == kNormTwice ? Nb * groups * p.cluster * (long long)sizeof(float2) : 0; }

static int run_norm(NormArgs &a, int x_dtype, void *scratch, cudaStream_t st)
{
    const int sms = plan_sms();
    const NormPlan p = plan_norm(x_dtype, a.Nb, a.P, a.C, a.groups, sms);
    if (p.kind != kNormRows && a.Nb * (a.groups / p.gpb) * (long long)p.cluster > 0x7fffffffll)
        return set_error(FLEXIQ_ERR_UNSUPPORTED, "too many images and groups for one launch");
    if (p.kind == kNormTwice && (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 15)))
        return set_error(FLEXIQ_ERR_INVALID_ARG, "scratch_dev is NULL or not 16-byte aligned: this shape needs %lld bytes", scratch_bytes(p, a.Nb, a.groups));
    a.cpg = a.C / a.groups;
    a.gpb = p.gpb; a.nch = p.nch; a.cpt = p.cpt; a.lanes = p.lanes; a.cluster = p.cluster; a.span = p.span;
    a.stats = static_cast<float2 *>(scratch);
    switch (x_dtype) {
        case FLEXIQ_DTYPE_F32: return launch_norm<FLEXIQ_DTYPE_F32>(a, p, sms, st);
        case FLEXIQ_DTYPE_F16: return launch_norm<FLEXIQ_DTYPE_F16>(a, p, sms, st);
        default: return launch_norm<FLEXIQ_DTYPE_BF16>(a, p, sms, st);
    }
}

}  // namespace flexiq

using namespace flexiq;

extern "C" int flexiq_group_norm_scratch(int x_dtype, int64_t Nb, int64_t P, int C, int groups, int64_t *bytes_out)
{
    if (!bytes_out) return set_error(FLEXIQ_ERR_INVALID_ARG, "bytes_out is NULL");
    if (int rc = check_shape(x_dtype, Nb, P, C, groups)) return rc;
    *bytes_out = Nb == 0 || P == 0 ? 0 : scratch_bytes(plan_norm(x_dtype, Nb, P, C, groups, plan_sms()), Nb, groups);
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
    a.X = X_dev; a.Nb = Nb; a.P = P; a.C = C; a.groups = groups; a.act = act;
    a.gamma = gamma_dev; a.beta = beta_dev; a.eps = eps;
    a.out.Y = Y_dev; a.out.y_dtype = y_dtype;
    return run_norm(a, x_dtype, scratch_dev, reinterpret_cast<cudaStream_t>(stream));
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
    a.X = X_dev; a.Nb = Nb; a.P = P; a.C = L->C; a.groups = groups; a.act = act;
    a.gamma = gamma_dev; a.beta = beta_dev; a.eps = eps;
    a.out.Y = X4_dev; a.out.y_dtype = FLEXIQ_DTYPE_I8;
    a.out.ent = L->chunk_ent; a.out.K_lo = L->K_lo;
    a.out.quot = quotient_plan(L, x_scale, FLEXIQ_DTYPE_F32);
    a.out.q_scale = x_scale;
    if ((rc = run_norm(a, x_dtype, scratch_dev, reinterpret_cast<cudaStream_t>(stream)))) return rc;
    record_slab(L, X4_dev, L->K_lo);
    return FLEXIQ_OK;
}
