// Group normalisation of channels-last tensors with an activation, into a floating-point tensor or a layer's slab.
//
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c]),   mean and var over an image's positions and a group's channels
//
// Bound by memory: every input byte is to be read once and every output byte written once.  Three ways, by what fits where:
//   rows   one position per image (layer normalisation): a warp, or four, holds a group in registers
//   held   an image's block of channels (whole groups; norm_plan.h says how many) is held in the shared memory of a block, or of a
//          cluster of up to four, between the statistics and their use; the blocks of a cluster exchange their groups' statistics
//          through distributed shared memory
//   twice  larger images: the statistics of pieces of an image go to scratch memory, and a second kernel reads the input again, in
//          the reverse order, so that what the L2 cache still holds of it comes first
//
// Statistics.  The variance is a mean square of deviations, never a difference of two sums, which would lose everything where the mean
// is large against the deviation.  A thread takes the mean and the sum of squared deviations M2 of its own values (two passes over what it holds, 64
// pieces at most; one about the first ones' mean where it holds nothing, 256 pieces at a time); those are joined in a fixed order by
//   m = sum n_i mean_i / n,   q_i = mean_i - m,   mean = m + sum n_i q_i / n,   M2 = sum M2_i + n_i q_i^2
// over the threads, the cluster's blocks or the pieces.  (The second sum takes out what the first has rounded.  The first is not taken from one of
// the means: where that one holds an outlier, its rounding would be the error.)  No sum is longer than some sixty roundings, and
// one more for every 256 pieces that a thread of "twice" has; results do not depend on timing.
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
    int cluster_log;          // "held": its logarithm; "twice": that of the blocks whose statistics are joined in a cluster
    int joined;               // "twice": what that leaves of each image
    long long span;           // positions of one of them
    unsigned by_nch, by_lanes, by_cpg;   // 2^32 / those, rounded up: quotients of less than 2^16 by a multiplication
    int cuts;                 // "twice": the second kernel's own pieces, and positions of one
    long long cut_span;
    float2 *stats;            // "twice": [image][group][piece] mean, M2
};

// VEC values in a row as they are: a 16-byte piece, or one value widened
template <int DT, int VEC> struct Piece {
    static constexpr int kBytes = DT == FLEXIQ_DTYPE_F32 ? 4 : 2, kPairs = VEC == 1 ? 1 : VEC / 2;
    typedef typename std::conditional<VEC == 1, float, uint4>::type Raw;
    Raw raw;
    __device__ __forceinline__ void load(const char *p)
    {
        if constexpr (VEC == 1) {
            if (DT == FLEXIQ_DTYPE_F32) raw = *reinterpret_cast<const float *>(p);
            else if (DT == FLEXIQ_DTYPE_F16) raw = __half2float(*reinterpret_cast<const __half *>(p));
            else raw = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p));
        } else {
            asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w) : "l"(p) : "memory");
        }
    }
    // in pairs of fp32 (a single value: with a zero beside it)
    __device__ __forceinline__ void widen(pair_t *x) const
    {
        if constexpr (VEC == 1) x[0] = pair(raw, 0.f);
        else if constexpr (DT == FLEXIQ_DTYPE_F32) {
            x[0] = pair(__uint_as_float(raw.x), __uint_as_float(raw.y));
            x[1] = pair(__uint_as_float(raw.z), __uint_as_float(raw.w));
        } else {
            const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (DT == FLEXIQ_DTYPE_F16) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                    x[i] = pair(f.x, f.y);
                } else {   // bf16: the 16 bits are the top half of an fp32
                    x[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
                }
            }
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

// gamma and beta of VEC channels from c on
template <int VEC> __device__ __forceinline__ void load_affine(const NormArgs &n, int c, pair_t *gamma, pair_t *beta)
{
    if constexpr (VEC == 1) {
        gamma[0] = pair(n.gamma ? n.gamma[c] : 1.f, 1.f);
        beta[0] = pair(n.beta ? n.beta[c] : 0.f, 0.f);
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
            const float4 g = n.gamma ? reinterpret_cast<const float4 *>(n.gamma + c)[i] : make_float4(1.f, 1.f, 1.f, 1.f);
            const float4 h = n.beta ? reinterpret_cast<const float4 *>(n.beta + c)[i] : make_float4(0.f, 0.f, 0.f, 0.f);
            gamma[2 * i] = pair(g.x, g.y); gamma[2 * i + 1] = pair(g.z, g.w);
            beta[2 * i] = pair(h.x, h.y); beta[2 * i + 1] = pair(h.z, h.w);
        }
    }
}
// What a thread keeps of its channels: y = (x - mean) scale + beta.  (x scale + b with the mean in b would round b, by up to 2^-24 |mean| scale: a constant
// image came out 4e-5 off its beta.)  MANY: the channels belong to several groups, with a mean each.
template <int VEC, bool MANY> struct Affine {
    static constexpr int kPairs = VEC == 1 ? 1 : VEC / 2;
    pair_t minus[MANY ? kPairs : 1], scale[kPairs], beta[kPairs];
    // of channels c .. and their groups' (mean, 1 / deviation)
    __device__ __forceinline__ void set(const NormArgs &n, int c, const float2 *stat)
    {
        load_affine<VEC>(n, c, scale, beta);
        finish(stat);
    }
    __device__ __forceinline__ void finish(const float2 *stat)   // (what load_affine has put here goes with `stat`)
    {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) scale[i] = mul2(scale[i], pair(stat[MANY ? 2 * i : 0].y, stat[MANY ? 2 * i + 1 : 0].y));
#pragma unroll
        for (int i = 0; i < (MANY ? kPairs : 1); ++i) minus[i] = pair(-stat[MANY ? 2 * i : 0].x, -stat[MANY ? 2 * i + 1 : 0].x);
    }
};
__device__ __forceinline__ int out_bytes(const NormOut &o) { return o.y_dtype == FLEXIQ_DTYPE_F32 ? 4 : o.y_dtype == FLEXIQ_DTYPE_I8 ? 1 : 2; }
// Where channel c of a row lies in the output, against where it would in the original order
__device__ __forceinline__ int slab_shift(const NormOut &o, int c, int *ent)
{
    if (o.y_dtype != FLEXIQ_DTYPE_I8) return 0;
    *ent = o.ent[c >> 4];
    return (*ent & 0xffffff) * 16 + (c & 15) - c;
}
// N pieces of normalised values, activated, to at(j) where live(j); ent(j): the slab's entry of their chunk.  One branch for all of them on the
// activation, and on the output's type.
template <int VEC, int N, class Live, class At, class Ent>
__device__ __forceinline__ void store_pieces(const NormArgs &n, pair_t (*t)[VEC == 1 ? 1 : VEC / 2], Live live, At at, Ent ent)
{
    const NormOut &o = n.out;
    constexpr int kPairs = VEC == 1 ? 1 : VEC / 2;
    activate_n<N * kPairs>(n.act, &t[0][0]);
    auto each = [&](auto store) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (live(j)) {
                float y[2 * kPairs];
#pragma unroll
                for (int k = 0; k < kPairs; ++k) unpair(t[j][k], &y[2 * k], &y[2 * k + 1]);
                store(j, static_cast<char *>(at(j)), y);
            }
    };
    if (o.y_dtype == FLEXIQ_DTYPE_F32)
        each([](int, char *to, const float *y) {
            if constexpr (VEC == 1) *reinterpret_cast<float *>(to) = y[0];
            else {
#pragma unroll
                for (int k = 0; k < VEC / 4; ++k) reinterpret_cast<float4 *>(to)[k] = make_float4(y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]);
            }
        });
    else if (o.y_dtype == FLEXIQ_DTYPE_F16)
        each([](int, char *to, const float *y) {
            if constexpr (VEC == 1) *reinterpret_cast<__half *>(to) = __float2half_rn(y[0]);
            else if constexpr (VEC == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(pack_f16(y[0], y[1]), pack_f16(y[2], y[3]));
            else *reinterpret_cast<uint4 *>(to) = make_uint4(pack_f16(y[0], y[1]), pack_f16(y[2], y[3]), pack_f16(y[4], y[5]), pack_f16(y[6], y[7]));
        });
    else if (o.y_dtype == FLEXIQ_DTYPE_BF16)
        each([](int, char *to, const float *y) {
            if constexpr (VEC == 1) *reinterpret_cast<__nv_bfloat16 *>(to) = __float2bfloat16_rn(y[0]);
            else if constexpr (VEC == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            else *reinterpret_cast<uint4 *>(to) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        });
    else
        each([&](int j, char *to, const float *y) {
            unsigned w[(VEC + 3) / 4];
            quantize_values<VEC>(o, ent(j), y, w);
            if constexpr (VEC == 1) *to = (char)w[0];
            else if constexpr (VEC == 4) *reinterpret_cast<unsigned *>(to) = w[0];
            else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        });
}
template <int VEC, bool MANY> __device__ __forceinline__ void normalise(pair_t *x, const Affine<VEC, MANY> &f)
{
#pragma unroll
    for (int i = 0; i < Affine<VEC, MANY>::kPairs; ++i) x[i] = fma2(add2(x[i], f.minus[MANY ? i : 0]), f.scale[i], f.beta[i]);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
// over `width` lanes (a power of two) side by side
__device__ __forceinline__ float part_sum(float v, int width)
{
    for (int d = width >> 1; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float both(pair_t p)
{
    float a, b;
    unpair(p, &a, &b);
    return a + b;
}
template <int N> __device__ __forceinline__ float fold(const pair_t *p)
{
    float s = both(p[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) s += both(p[i]);
    return s;
}
// (two units in the last place at most)
__device__ __forceinline__ float deviation_inverse(float M2, float n, float eps) { return rsqrtf(__fadd_rn(__fdividef(M2, n), eps)); }

__device__ __forceinline__ int quotient(int n, unsigned inverse) { return inverse ? (int)__umulhi((unsigned)n, inverse) : n; }   // (0 stands for 2^32: by one)

struct Moments { float n, mean, M2; };
// s / n, one rounding off at most and exact where it can be (the mean of equal values is that value): a product corrected by its remainder
__device__ __forceinline__ pair_t divide(pair_t s, pair_t minus_n, pair_t inverse)
{
    const pair_t m = mul2(s, inverse);
    return fma2(fma2(m, minus_n, s), inverse, m);
}
__device__ __forceinline__ float divide(float s, float n, float inverse)
{
    const float m = __fmul_rn(s, inverse);
    return __fmaf_rn(__fmaf_rn(-m, n, s), inverse, m);
}
// Sums of pairs per channel -> means, of each channel (MANY) or of all
template <int VEC, bool MANY> __device__ __forceinline__ void means_of(const pair_t *s, int pieces, float *mean)
{
    const float n = (float)(pieces ? pieces * (MANY ? 1 : VEC) : 1), inverse = __frcp_rn(n);
    constexpr int kPairs = VEC == 1 ? 1 : VEC / 2;
    if (MANY) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) unpair(divide(s[i], pair(-n, -n), pair(inverse, inverse)), &mean[(2 * i) % VEC], &mean[(2 * i + 1) % VEC]);
    } else {
        mean[0] = divide(fold<kPairs>(s), n, inverse);
    }
}
template <int VEC, bool MANY> __device__ __forceinline__ void minus_means(const float *mean, pair_t *m)
{
#pragma unroll
    for (int i = 0; i < (MANY ? VEC / 2 : 1); ++i) m[i] = pair(-mean[MANY ? 2 * i : 0], VEC == 1 ? 0.f : -mean[MANY ? 2 * i + 1 : 0]);
}
template <int VEC, bool MANY> __device__ __forceinline__ void squares_of(const pair_t *q, float *M2)
{
    constexpr int kPairs = VEC == 1 ? 1 : VEC / 2;
    if (MANY) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) unpair(q[i], &M2[(2 * i) % VEC], &M2[(2 * i + 1) % VEC]);
    } else {
        M2[0] = fold<kPairs>(q);
    }
}

__device__ unsigned int g_norm_status = 0;

// A thread's moments as entries, [entry][thread], and its number of pieces.  One, where a piece's channels are of one group; MANY: one for each of the groups it has a part of, in order,
// from the channels' own (K the first one's mean, s and ss the sums of the others' distances from it and of their squares).
template <int VEC, bool MANY, int T>
__device__ __forceinline__ void put_moments(const NormArgs &a, int col, const float *mean, const float *M2, float pieces, float *red_mean, float *red_M2, float *red_n)
{
    const int t = threadIdx.x;
    red_n[t] = pieces;
    if (!MANY) {
        red_mean[t] = mean[0];
        red_M2[t] = M2[0];
        return;
    }
    int left = a.cpg - (col * VEC - quotient(col * VEC, a.by_cpg) * a.cpg), at = t;
    float K = mean[0], s = 0.f, ss = 0.f, M = 0.f, c = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float d = mean[i] - K;
        s += d;
        ss = __fmaf_rn(d, d, ss);
        M += M2[i];
        c += 1.f;
        if (--left == 0 || i == VEC - 1) {
            const float away = __fdividef(s, c);
            red_mean[at] = K + away;
            red_M2[at] = pieces > 0.f ? __fmaf_rn(pieces, fmaxf(__fmaf_rn(-s, away, ss), 0.f), M) : 0.f;
            at += T;
            left = a.cpg;
            if (i + 1 < VEC) { K = mean[(i + 1) % VEC]; s = ss = M = c = 0.f; }
        }
    }
}
// The threads' entries -> their groups' moments in gstat[0 .. gpb): some lanes per group over the columns that hold a part of it, at every position.
template <int VEC, bool MANY, int T>
__device__ __forceinline__ void block_moments(const NormArgs &a, const float *red_mean, const float *red_M2, const float *red_n, Moments *gstat)
{
    __syncthreads();
    int width_log = 5;                                // lanes per group: fewer where there are more groups than warps
    while (width_log > 2 && (T >> width_log) < a.gpb) --width_log;
    const int width = 1 << width_log, sub = threadIdx.x & (width - 1), step = T >> width_log;
    const int pitch = a.cpt > 1 ? T : a.nch;          // threads of a position
    for (int g0 = 0; g0 < a.gpb; g0 += step) {        // (all lanes stay: the sums need them)
        const int g = g0 + (int)(threadIdx.x >> width_log);
        const bool live = g < a.gpb;
        int col0 = 0, cols;                           // its columns
        if (a.cpt > 1) cols = T;
        else if (!MANY) { cols = a.cpg / VEC; col0 = g * cols; }
        else { col0 = g * a.cpg / VEC; cols = ((g + 1) * a.cpg - 1) / VEC - col0 + 1; }
        // the lane's entries: (position row, column in), `width` further each time
        const unsigned by_cols = cols > 1 ? 0xffffffffu / (unsigned)cols + 1u : 0u;
        const int jump = quotient(width, by_cols), rest = width - jump * cols, row0 = quotient(sub, by_cols), in0 = sub - row0 * cols, rows = live ? a.lanes : 0;
        auto over = [&](auto take) {
            for (int row = row0, in = in0; row < rows;) {
                const int col = col0 + in, t = row * pitch + col;
                if (MANY) {                               // the entry, and how many of the piece's channels it has
                    const int c0 = col * VEC, lo = g * a.cpg, from = c0 > lo ? c0 : lo, to = c0 + VEC < lo + a.cpg ? c0 + VEC : lo + a.cpg;
                    take(t + (g - quotient(c0, a.by_cpg)) * T, red_n[t] * (float)(to - from));
                } else {
                    take(t, red_n[t] * (float)VEC);
                }
                row += jump;
                in += rest;
                if (in >= cols) { in -= cols; ++row; }
            }
        };
        float n = 0.f, d = 0.f, M2 = 0.f, c = 0.f;
        over([&](int e, float w) {
            n += w;
            d = __fmaf_rn(w, red_mean[e], d);
        });
        n = part_sum(n, width);
        d = part_sum(d, width);
        const float mean = n > 0.f ? __fdiv_rn(d, n) : 0.f;
        over([&](int e, float w) {
            const float q = red_mean[e] - mean, wq = w * q;
            c += wq;
            M2 += __fmaf_rn(wq, q, red_M2[e]);             // (a thread without values: all zero)
        });
        M2 = part_sum(M2, width);
        c = part_sum(c, width);
        if (sub == 0 && live) gstat[g] = Moments{n, n > 0.f ? mean + __fdividef(c, n) : 0.f, M2};
    }
    __syncthreads();
}

// A thread's pieces: its column and its position among those side by side; cpt > 1: its first column, at every position
struct Place {
    int col, pl, cols;        // cols: columns of a position that are its own (cpt > 1)
    bool live;
    __device__ __forceinline__ Place(const NormArgs &a)
    {
        const int t = threadIdx.x;
        if (a.cpt > 1) { pl = 0; col = t; cols = (a.nch - t + (int)blockDim.x - 1) / (int)blockDim.x; live = t < a.nch; }
        else { pl = quotient(t, a.by_nch); col = t - pl * a.nch; cols = 1; live = pl < a.lanes; }
    }
    // its pieces among `positions` (fewer than 2^16: by a multiplication)
    __device__ __forceinline__ int count(const NormArgs &a, int positions) const
    {
        if (!live || positions <= pl) return 0;
        if (a.cpt > 1) return positions * cols;
        const int n = positions - pl + a.lanes - 1;
        return n < 65536 ? quotient(n, a.by_lanes) : n / a.lanes;
    }
};

// (mean, 1 / deviation) of the channels of column `col` (MANY: of each)
template <int VEC, bool MANY> __device__ __forceinline__ void column_stats(const NormArgs &a, int col, const float2 *fin, float2 *stat)
{
    int g = quotient(col * VEC, a.by_cpg), left = a.cpg - (col * VEC - g * a.cpg);
    stat[0] = fin[g];
#pragma unroll
    for (int i = 1; i < (MANY ? VEC : 1); ++i) {
        if (--left == 0) { left = a.cpg; ++g; }
        stat[i] = fin[g];
    }
}

// A thread's pieces through shared memory, NV at a time and DEPTH - 1 batches ahead: its own slots, [batch][piece][thread], so it waits for no one else.
template <int DT, int VEC, int NV, int DEPTH> struct PieceRing {
    typedef Piece<DT, VEC> P;
    typename P::Raw *hold;
    const char *from;
    size_t apart;             // bytes from one piece to the next
    int left;                 // pieces not asked for yet
    int slot;                 // (the first piece's place)
    static constexpr int T = kNormThreads, kBatch = NV * T;
    __device__ __forceinline__ PieceRing(void *smem, const char *from_, size_t apart_, int cnt_)
        : hold(static_cast<typename P::Raw *>(smem) + threadIdx.x), from(from_), apart(apart_), left(cnt_), slot(0)
    {
        for (int k = 0; k < DEPTH - 1; ++k) ask(k * kBatch);
    }
    __device__ __forceinline__ void one(int at)
    {
        if constexpr (VEC == 1) {
            P v;
            v.load(from);
            hold[at] = v.raw;
        } else {
            ptx::cp_async_16(ptx::smem_u32(&hold[at]), from);
        }
        from += apart;
    }
    __device__ __forceinline__ void ask(int to)           // (an empty batch of copies where there is nothing left)
    {
        if (left >= NV) {
#pragma unroll
            for (int j = 0; j < NV; ++j) one(to + j * T);
            left -= NV;
        } else {
            for (int at = to; left > 0; --left, at += T) one(at);
        }
        ptx::cp_async_commit();
    }
    // the next batch is here; the one DEPTH - 1 behind it is asked for (into the slots read last)
    __device__ __forceinline__ void turn()
    {
        ask(slot == 0 ? (DEPTH - 1) * kBatch : slot - kBatch);
        ptx::cp_async_wait_but<DEPTH - 1>();
    }
    __device__ __forceinline__ P piece(int j) const
    {
        P v;
        v.raw = hold[slot + j * T];
        return v;
    }
    __device__ __forceinline__ void done()
    {
        slot = slot == (DEPTH - 1) * kBatch ? 0 : slot + kBatch;
    }
};

// Of `bytes` that the blocks of the cluster will write: this block's barrier stands, and the others learn that it does (cluster_wait).
__device__ __forceinline__ void announce(uint64_t *arrived, unsigned bytes)
{
    if (threadIdx.x == 0) {
        ptx::mbar_init(arrived, 1);
        ptx::fence_mbar_init();
        ptx::mbar_expect_tx(arrived, bytes);
    }
    __syncthreads();
    ptx::cluster_arrive();
}
__device__ __forceinline__ void wait_arrived(uint64_t *arrived)   // bounded: about two seconds
{
    bool here = ptx::mbar_try_wait(arrived, 0);
    for (uint32_t i = 0; i < (1u << 21) && !here; ++i) here = ptx::mbar_try_wait_hint_s(ptx::smem_u32(arrived), 0, 1000u);   // (parked for a microsecond at most)
    if (!here) atomicMax(&g_norm_status, 0x401u);
}
// k parts side by side in the lanes, this lane's with n of the `all` values
__device__ __forceinline__ Moments join_cluster(float2 s, float n, float all, int k)
{
    const float centre = __fdiv_rn(part_sum(__fmul_rn(n, s.x), k), all), o = s.x - centre, no = n * o;
    const float M = part_sum(__fmaf_rn(no, o, s.y), k), c = part_sum(no, k);
    return Moments{all, centre + __fdividef(c, all), M};
}

// "held": block rank `blockIdx.x % cluster` of an image's channel block.  A thread's pieces lie in shared memory, [piece][thread]: in registers
// the loops over them had to be unrolled, and fetching some thousands of instructions once each cost more than the memory.
template <int DT, int VEC, bool MANY, int T>
__global__ void __launch_bounds__(T, 1024 / T) group_norm_held_kernel(const NormArgs a)
{
    constexpr int S = MANY ? VEC : 1, kPairs = VEC == 1 ? 1 : VEC / 2, kNext = T * (VEC == 1 ? 4 : 16);
    typedef Piece<DT, VEC> P;
    extern __shared__ __align__(16) uint8_t hold_bytes[];
    __shared__ float red_mean[T * S], red_M2[T * S], red_n[T];
    __shared__ Moments gstat[kMaxGroups];
    __shared__ float2 fin[kMaxGroups], inbox[kNormCluster][kMaxGroups];
    __shared__ uint64_t arrived;
    // The blocks of a cluster write their groups' moments into one another's shared memory.  First each has to know that the others have begun
    // and their barriers stand: that is waited for below, while the data comes.  (Reading them from the others between two
    // barriers of the cluster: 32 x 196 x 256 fp16 6.5 us, 5.3 so.)
    if (a.cluster_log) announce(&arrived, (unsigned)(a.gpb << a.cluster_log) * 8u);
    // block (image and rank in the cluster, channel block)
    const int rank = (int)(blockIdx.x & ((1u << a.cluster_log) - 1u));
    const long long img = blockIdx.x >> a.cluster_log;
    const int c0 = (int)blockIdx.y * a.gpb * a.cpg;
    const long long p0 = rank * a.span, left = a.P - p0;
    const int mine = (int)(left < 0 ? 0 : left < a.span ? left : a.span);
    const Place who(a);
    const int cnt = who.count(a, mine);
    // element of piece j: one position after another (cpt > 1: its columns of a position first)
    const size_t e0 = ((size_t)img * a.P + p0 + who.pl) * a.C + c0 + (size_t)who.col * VEC;
    const size_t step = (size_t)a.lanes * a.C;
    const bool wide = a.cpt > 1;
    auto element = [&](int j) { return e0 + (size_t)(j / who.cols) * a.C + (size_t)(j % who.cols) * T * VEC; };   // (wide)
    uint8_t *const hold = hold_bytes + threadIdx.x * (VEC == 1 ? 4 : 16);
    ptx::pdl_wait();
    {
        const char *from = static_cast<const char *>(a.X) + e0 * P::kBytes;
        const size_t next = step * P::kBytes;
        uint8_t *to = hold;
#pragma unroll 4
        for (int j = 0; j < cnt; ++j) {
            if (wide) from = static_cast<const char *>(a.X) + element(j) * P::kBytes;
            if constexpr (VEC == 1) {
                P v;
                v.load(from);
                *reinterpret_cast<float *>(to) = v.raw;
            } else {
                ptx::cp_async_16(ptx::smem_u32(to), from);
            }
            from += next;
            to += kNext;
        }
        ptx::cp_async_wait();                                  // (each thread reads what it asked for itself)
    }
    auto piece = [&](const uint8_t *at, pair_t *x) {
        P v;
        v.raw = *reinterpret_cast<const typename P::Raw *>(at);
        v.widen(x);
    };
    float mean[S], M2[S];
    {
        pair_t s[kPairs] = {}, m[MANY ? kPairs : 1];
        const uint8_t *at = hold;
#pragma unroll 4
        for (int j = 0; j < cnt; ++j, at += kNext) {
            pair_t x[kPairs];
            piece(at, x);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) s[i] = add2(s[i], x[i]);
        }
        means_of<VEC, MANY>(s, cnt, mean);
        minus_means<VEC, MANY>(mean, m);
        pair_t q[kPairs] = {};
        at = hold;
#pragma unroll 4
        for (int j = 0; j < cnt; ++j, at += kNext) {
            pair_t x[kPairs];
            piece(at, x);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) { x[i] = add2(x[i], m[MANY ? i : 0]); q[i] = fma2(x[i], x[i], q[i]); }
        }
        squares_of<VEC, MANY>(q, M2);
    }
    // the channels' own numbers, asked for ahead of the exchange
    Affine<VEC, MANY> f;
    int ent = 0, shift = 0;
    const int c_own = c0 + who.col * VEC;
    if (!wide && cnt) {
        load_affine<VEC>(a, c_own, f.scale, f.beta);
        shift = slab_shift(a.out, c_own, &ent);
    }
    put_moments<VEC, MANY, T>(a, who.col, mean, M2, (float)cnt, red_mean, red_M2, red_n);
    block_moments<VEC, MANY, T>(a, red_mean, red_M2, red_n, gstat);
    if (a.cluster_log) {
        // a thread per group and block of the cluster, those of a group side by side
        const int k = 1 << a.cluster_log, per = T >> a.cluster_log, r = threadIdx.x & (k - 1);
        ptx::cluster_wait();
        const uint32_t bar = ptx::mapa(ptx::smem_u32(&arrived), (uint32_t)r);
        for (int g = (int)(threadIdx.x >> a.cluster_log); g < a.gpb; g += per)
            ptx::st_async_64(ptx::mapa(ptx::smem_u32(&inbox[rank][g]), (uint32_t)r), gstat[g].mean, gstat[g].M2, bar);
        wait_arrived(&arrived);
        const long long other = a.P - r * a.span;              // positions of block r
        const float n = (float)((other < 0 ? 0 : other < a.span ? (int)other : (int)a.span) * a.cpg), all = (float)(a.P * a.cpg);
        for (int g0 = 0; g0 < a.gpb; g0 += per) {              // (all lanes stay: the sums need them)
            const int g = g0 + (int)(threadIdx.x >> a.cluster_log);
            const Moments m = join_cluster(inbox[r][g < a.gpb ? g : 0], n, all, k);
            if (r == 0 && g < a.gpb) fin[g] = make_float2(m.mean, deviation_inverse(m.M2, all, a.eps));
        }
    } else {
        for (int g = threadIdx.x; g < a.gpb; g += T) fin[g] = make_float2(gstat[g].mean, deviation_inverse(gstat[g].M2, gstat[g].n, a.eps));
    }
    ptx::pdl_launch_dependents();
    __syncthreads();
    if (cnt) {
        float2 stat[S];
        const int ob = out_bytes(a.out);
        column_stats<VEC, MANY>(a, wide ? 0 : who.col, fin, stat);   // (wide: one group)
        const uint8_t *at = hold;
        if (!wide) {
            constexpr int NV = 2;
            f.finish(stat);
            char *to = static_cast<char *>(a.out.Y) + (e0 + shift) * ob;
            const size_t far = step * ob;
            auto batch = [&](auto whole, int n) {              // (what is not there is not stored)
                pair_t x[NV][kPairs];
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (decltype(whole)::value || j < n) piece(at + j * kNext, x[j]);
                    else {
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) x[j][i] = pair(0.f, 0.f);
                    }
#pragma unroll
                for (int j = 0; j < NV; ++j) normalise<VEC, MANY>(x[j], f);
                store_pieces<VEC, NV>(a, x, [&](int j) { return decltype(whole)::value || j < n; }, [&](int) { char *const here = to; to += far; return here; }, [&](int) { return ent; });
                at += NV * kNext;
            };
            int j = 0;
#pragma unroll 1
            for (; j + NV <= cnt; j += NV) batch(std::true_type{}, NV);
            if (j < cnt) batch(std::false_type{}, cnt - j);
        } else {
#pragma unroll 1
            for (int j = 0; j < cnt; ++j, at += kNext) {
                const int c = c0 + (who.col + (j % who.cols) * T) * VEC;
                f.set(a, c, stat);
                char *to = static_cast<char *>(a.out.Y) + (element(j) + slab_shift(a.out, c, &ent)) * ob;
                pair_t x[1][kPairs];
                piece(at, x[0]);
                normalise<VEC, MANY>(x[0], f);
                store_pieces<VEC, 1>(a, x, [](int) { return true; }, [&](int) { return to; }, [&](int) { return ent; });
            }
        }
    }
}

constexpr int kStatsPieces = 8, kStatsDepth = 2, kApplyPieces = 4, kApplyDepth = 3;
constexpr int kStatsRun = 32;     // batches whose sums are taken about one K
// "twice", the first: moments of a piece of an image's channel block
template <int DT, int VEC, bool MANY>
__global__ void __launch_bounds__(kNormThreads, 2) group_norm_stats_kernel(const NormArgs a)
{
    constexpr int S = MANY ? VEC : 1, kPairs = VEC == 1 ? 1 : VEC / 2, NV = kStatsPieces;
    typedef Piece<DT, VEC> P;
    extern __shared__ __align__(16) uint8_t hold_bytes[];
    __shared__ float red_mean[kNormThreads * S], red_M2[kNormThreads * S], red_n[kNormThreads];
    __shared__ Moments gstat[kMaxGroups];
    // block (image and piece, channel block)
    const long long img = blockIdx.x / (unsigned)a.cluster;
    const int part = (int)(blockIdx.x - (unsigned)img * (unsigned)a.cluster), block = (int)blockIdx.y, c0 = block * a.gpb * a.cpg;
    __shared__ float2 inbox[kNormCluster][kMaxGroups];
    __shared__ uint64_t arrived;
    if (a.cluster_log) announce(&arrived, (unsigned)(a.gpb << a.cluster_log) * 8u);
    const long long p0 = part * a.span, left = a.P - p0;
    const int mine = (int)(left < 0 ? 0 : left < a.span ? left : a.span);
    const Place who(a);
    const size_t e0 = ((size_t)img * a.P + p0 + who.pl) * a.C + c0 + (size_t)who.col * VEC;
    const bool wide = a.cpt > 1;
    const int cnt = who.count(a, mine);
    const size_t step = (size_t)a.lanes * a.C * P::kBytes;
    ptx::pdl_wait();
    // One pass: sums of x - K and of its square, K the mean of the first NV pieces of a run of kStatsRun batches.  Their squares' sum is at most
    // 1 + n / NV^2 = 5 times (n pieces) what is left of it when the mean is taken out, however far one of the first values lies, since that one is
    // among them; four batches are summed apart before they are added to the rest of the run.  A run that more pieces follow is closed: its moments
    // join those of the runs before it, which lie in the thread's own places of the block's arrays.  (One K for all of a thread's pieces, 4096 of
    // them with an outlier in front: the variance off by 420 units of 2^-24, 5 so; none of the measured shapes has a second run.)
    const char *from = static_cast<const char *>(a.X) + e0 * P::kBytes;
    pair_t K[MANY ? kPairs : 1], S1[kPairs] = {}, S2[kPairs] = {};
    float shift[S] = {};
    int batches = 0;
    pair_t s[kPairs] = {}, q[kPairs] = {};
    const int own = threadIdx.x;
    // the open run's moments, of `pieces`; those together with the closed runs'
    auto run_moments = [&](int pieces, float *mean, float *M2) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) { S1[i] = add2(S1[i], s[i]); S2[i] = add2(S2[i], q[i]); }
        float off[S];
        means_of<VEC, MANY>(S1, pieces, off);
        squares_of<VEC, MANY>(S2, M2);
        const float n = (float)(pieces * (MANY ? 1 : VEC));
#pragma unroll
        for (int i = 0; i < S; ++i) {
            mean[i] = shift[i] + off[i];
            M2[i] = fmaxf(__fmaf_rn(-n * off[i], off[i], M2[i]), 0.f);   // (an infinite sum of squares stays one: the product is not rounded)
            if (off[i] != off[i]) M2[i] = off[i];
        }
    };
    auto join_runs = [&](int pieces, float *mean, float *M2) {
        const float before = red_n[own], part = __fdividef((float)pieces, before + (float)pieces), n = before * part * (MANY ? 1.f : (float)VEC);
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const float d = mean[i] - red_mean[i * kNormThreads + own];
            mean[i] = __fmaf_rn(d, part, red_mean[i * kNormThreads + own]);
            M2[i] = __fmaf_rn(d * n, d, M2[i] + red_M2[i * kNormThreads + own]);
        }
    };
    auto close_run = [&] {
        constexpr int kPieces = kStatsRun * NV;
        float mean[S], M2[S];
        run_moments(kPieces, mean, M2);
        if (batches > kStatsRun) join_runs(kPieces, mean, M2);
#pragma unroll
        for (int i = 0; i < S; ++i) { red_mean[i * kNormThreads + own] = mean[i]; red_M2[i * kNormThreads + own] = M2[i]; }
        red_n[own] = (float)(batches * NV);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) S1[i] = S2[i] = s[i] = q[i] = pair(0.f, 0.f);
    };
    auto tile = [&](auto piece, int pieces, auto all) {      // `all`: every piece of the tile is there
        if (batches % kStatsRun == 0) {
            if (batches) close_run();
            pair_t t[kPairs] = {};
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (decltype(all)::value || j < pieces) {
                    pair_t x[kPairs];
                    piece(j).widen(x);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) t[i] = add2(t[i], x[i]);
                }
            means_of<VEC, MANY>(t, pieces, shift);
            minus_means<VEC, MANY>(shift, K);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (decltype(all)::value || j < pieces) {
                pair_t x[kPairs];
                piece(j).widen(x);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) { x[i] = add2(x[i], K[MANY ? i : 0]); s[i] = add2(s[i], x[i]); q[i] = fma2(x[i], x[i], q[i]); }
            }
        if ((++batches & 3) == 0) {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) { S1[i] = add2(S1[i], s[i]); S2[i] = add2(S2[i], q[i]); s[i] = q[i] = pair(0.f, 0.f); }
        }
    };
    if (!wide) {
        PieceRing<DT, VEC, NV, kStatsDepth> ring(hold_bytes, from, step, cnt);
        auto piece = [&](int j) { return ring.piece(j); };
        int todo = cnt;
        for (; todo >= NV; todo -= NV) {
            ring.turn();
            tile(piece, NV, std::true_type{});
            ring.done();
        }
        if (todo) {
            ring.turn();
            tile(piece, todo, std::false_type{});
        }
    } else {
        for (int j0 = 0; j0 < cnt; j0 += NV) {
            P v[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int p = (j0 + j) / who.cols;
                if (j0 + j < cnt) v[j].load(from + ((size_t)p * a.C + (size_t)(j0 + j - p * who.cols) * blockDim.x * VEC) * P::kBytes);
            }
            tile([&](int j) { return v[j]; }, cnt - j0 < NV ? cnt - j0 : NV, std::false_type{});
        }
    }
    float mean[S], M2[S];
    {
        const int closed = cnt ? (batches - 1) / kStatsRun * (kStatsRun * NV) : 0;   // pieces
        run_moments(cnt - closed, mean, M2);
        if (closed) join_runs(cnt - closed, mean, M2);
    }
    ptx::pdl_launch_dependents();
    put_moments<VEC, MANY, kNormThreads>(a, who.col, mean, M2, (float)cnt, red_mean, red_M2, red_n);
    block_moments<VEC, MANY, kNormThreads>(a, red_mean, red_M2, red_n, gstat);
    float2 *const to = a.stats + ((size_t)img * a.groups + block * a.gpb) * a.joined + (part >> a.cluster_log);
    if (a.cluster_log) {
        // the first block of the cluster joins what the others write into its shared memory
        const int k = 1 << a.cluster_log, rank = part & (k - 1), r = threadIdx.x & (k - 1), per = kNormThreads >> a.cluster_log;
        ptx::cluster_wait();
        const uint32_t bar = ptx::mapa(ptx::smem_u32(&arrived), 0);
        for (int g = threadIdx.x; g < a.gpb; g += kNormThreads) ptx::st_async_64(ptx::mapa(ptx::smem_u32(&inbox[rank][g]), 0), gstat[g].mean, gstat[g].M2, bar);
        if (rank) return;
        wait_arrived(&arrived);
        const long long other = a.P - (part + r) * a.span, here = a.P - part * a.span;
        const float n = (float)((other < 0 ? 0 : other < a.span ? other : a.span) * a.cpg), all = (float)((here < a.span << a.cluster_log ? here : a.span << a.cluster_log) * a.cpg);
        for (int g0 = 0; g0 < a.gpb; g0 += per) {              // (all lanes stay: the sums need them)
            const int g = g0 + (int)(threadIdx.x >> a.cluster_log);
            const Moments m = join_cluster(inbox[r][g < a.gpb ? g : 0], n, all, k);
            // (nothing to be joined, which no plan asks for, would be 0 / 0, a NaN that the entry's weight of zero does not take away)
            if (r == 0 && g < a.gpb) to[(size_t)g * a.joined] = all > 0.f ? make_float2(m.mean, m.M2) : make_float2(0.f, 0.f);
        }
    } else {
        for (int g = threadIdx.x; g < a.gpb; g += kNormThreads) to[(size_t)g * a.joined] = make_float2(gstat[g].mean, gstat[g].M2);
    }
}

// "twice", the second: the pieces' moments joined, and the values.  Blocks in reverse order: what was read last is in the L2 cache.
template <int DT, int VEC, bool MANY>
__global__ void __launch_bounds__(kNormThreads, 3) group_norm_apply_kernel(const NormArgs a)
{
    constexpr int S = MANY ? VEC : 1, kPairs = VEC == 1 ? 1 : VEC / 2, NV = kApplyPieces;
    typedef Piece<DT, VEC> P;
    extern __shared__ __align__(16) uint8_t hold_bytes[];
    __shared__ float2 fin[kMaxGroups];
    const unsigned id = gridDim.x - 1 - blockIdx.x;
    const long long img = id / (unsigned)a.cuts;
    const int part = (int)(id - (unsigned)img * (unsigned)a.cuts), block = (int)(gridDim.y - 1 - blockIdx.y), c0 = block * a.gpb * a.cpg;
    const long long p0 = part * a.cut_span, left = a.P - p0;
    const int mine = (int)(left < 0 ? 0 : left < a.cut_span ? left : a.cut_span);
    const Place who(a);
    const int cnt = who.count(a, mine);
    // The first values are asked for at once: the statistics' kernel writes none of X, and every block of it had waited for what ran before when it
    // let this one begin.
    const size_t e = ((size_t)img * a.P + p0 + who.pl) * a.C + c0 + (size_t)who.col * VEC;
    const char *from = static_cast<const char *>(a.X) + e * P::kBytes;
    const size_t bytes = (size_t)a.lanes * a.C * P::kBytes;
    PieceRing<DT, VEC, NV, kApplyDepth> ring(hold_bytes, from, bytes, a.cpt > 1 ? 0 : cnt);
    ptx::pdl_wait();
    {
        const long long span = a.span << a.cluster_log;        // positions of an entry
        const float all = (float)(a.P * a.cpg), each = (float)(span * a.cpg);
        // 8 to 32 lanes a group: as many as let the block take all its groups at once (a warp for each, one after another, was 2 us slower with 32)
        int k = 8;
        while (k < 32 && a.gpb * k * 2 <= kNormThreads) k *= 2;
        const int r = threadIdx.x & (k - 1);
        auto weight = [&](int i) {                             // values of entry i
            const long long rest = a.P - i * span;
            return rest >= span ? each : rest > 0 ? (float)(rest * a.cpg) : 0.f;
        };
        for (int g0 = 0; g0 < a.gpb; g0 += kNormThreads / k) { // (all lanes stay: the sums need them)
            const int g = g0 + (int)threadIdx.x / k;
            const float2 *at = a.stats + ((size_t)img * a.groups + block * a.gpb + (g < a.gpb ? g : 0)) * a.joined;
            float d = 0.f, M2 = 0.f, c = 0.f;
#pragma unroll 8
            for (int i = r; i < a.joined; i += k) d = __fmaf_rn(weight(i), at[i].x, d);
            const float centre = __fdiv_rn(part_sum(d, k), all);
#pragma unroll 8
            for (int i = r; i < a.joined; i += k) {
                const float2 s = at[i];
                const float q = s.x - centre, wq = weight(i) * q;
                c += wq;
                M2 += __fmaf_rn(wq, q, s.y);
            }
            M2 = part_sum(M2, k);
            c = part_sum(c, k);
            if (r == 0 && g < a.gpb) fin[g] = make_float2(centre + __fdividef(c, all), deviation_inverse(M2, all, a.eps));
        }
    }
    __syncthreads();
    ptx::pdl_launch_dependents();
    if (cnt == 0) return;
    float2 stat[S];
    Affine<VEC, MANY> f;
    int ent = 0;
    column_stats<VEC, MANY>(a, a.cpt > 1 ? 0 : who.col, fin, stat);
    const int ob = out_bytes(a.out);
    if (a.cpt > 1) {
        for (int j = 0; j < cnt; ++j) {
            const int p = j / who.cols, k = (j - p * who.cols) * (int)blockDim.x, c = c0 + (who.col + k) * VEC;
            const size_t off = (size_t)p * a.C + (size_t)k * VEC;
            P v;
            v.load(from + off * P::kBytes);
            f.set(a, c, stat);
            char *to = static_cast<char *>(a.out.Y) + (e + off + slab_shift(a.out, c, &ent)) * ob;
            pair_t x[1][kPairs];
            v.widen(x[0]);
            normalise<VEC, MANY>(x[0], f);
            store_pieces<VEC, 1>(a, x, [](int) { return true; }, [&](int) { return to; }, [&](int) { return ent; });
        }
        return;
    }
    const int c = c0 + who.col * VEC;
    f.set(a, c, stat);
    char *to = static_cast<char *>(a.out.Y) + (e + slab_shift(a.out, c, &ent)) * ob;
    const size_t far = (size_t)a.lanes * a.C * ob;
    auto batch = [&](auto whole, int n) {                  // (what is not there is not stored)
        ring.turn();
        pair_t x[NV][kPairs];
#pragma unroll
        for (int j = 0; j < NV; ++j) ring.piece(j).widen(x[j]);
        ring.done();
#pragma unroll
        for (int j = 0; j < NV; ++j) normalise<VEC, MANY>(x[j], f);
        store_pieces<VEC, NV>(a, x, [&](int j) { return decltype(whole)::value || j < n; }, [&](int) { char *const here = to; to += far; return here; }, [&](int) { return ent; });
    };
    int todo = cnt;
    for (; todo >= NV; todo -= NV) batch(std::true_type{}, NV);
    if (todo) batch(std::false_type{}, todo);
}

// "rows": one position per image.  A warp takes a group at a time (its cpg values are contiguous) and has the next kRowDepth - 1 on the way, in shared
// memory of its own; gamma and beta stay in registers where it meets the same channels again (one group, or a stride of whole rows).  NV is the
// number of a lane's pieces exactly, so that only the last may be missing: with a test on every piece a third of the instructions were branches.
// Long groups are taken by WARPS warps together, which exchange their sums.
constexpr int kRowDepth = 4;
template <int DT, int VEC, int NV, int WARPS>
__global__ void __launch_bounds__(kNormThreads, NV == 1 ? 3 : 2) group_norm_rows_kernel(const NormArgs a)
{
    constexpr int kPairs = VEC == 1 ? 1 : VEC / 2, kLanes = 32 * WARPS, kSlot = NV * kLanes * (VEC == 1 ? 4 : 16), kTeams = kNormThreads / kLanes;
    constexpr bool kKeep = NV * VEC <= 32;
    typedef Piece<DT, VEC> P;
    extern __shared__ __align__(16) uint8_t hold_bytes[];
    __shared__ float part[2][kTeams][WARPS];
    const int lane = (int)threadIdx.x % kLanes, team = (int)threadIdx.x / kLanes, teams = (int)blockDim.x / kLanes;
    const int total = (int)(a.Nb * a.groups), step = (int)gridDim.x * teams;   // (the host takes no more than 2^30 of them)
    int seg = (int)blockIdx.x * teams + team;
    const bool last = lane + kLanes * (NV - 1) < a.nch;
    // over the team's lanes; `which`: the two sums of a group, whose places are free again by the next one's
    auto sum = [&](float v, int which) {
        v = warp_sum(v);
        if constexpr (WARPS > 1) {
            if ((threadIdx.x & 31) == 0) part[which][team][lane >> 5] = v;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(kLanes) : "memory");
            v = part[which][team][0];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) v += part[which][team][w];
        }
        return v;
    };
    ptx::pdl_wait();
    if (seg >= total) return;
    // [team][group][piece][lane]
    uint8_t *const hold = hold_bytes + team * (kRowDepth * kSlot) + lane * (VEC == 1 ? 4 : 16);
    const char *from = static_cast<const char *>(a.X) + ((size_t)seg * a.cpg + lane * VEC) * P::kBytes;
    const size_t stride = (size_t)step * a.cpg * P::kBytes;
    auto request = [&](bool there, int slot) {             // (an empty batch of copies where there is no such group)
        if (there) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < NV - 1 || last) {
                    uint8_t *const to = hold + slot + j * kLanes * (VEC == 1 ? 4 : 16);
                    if constexpr (VEC == 1) {
                        P v;
                        v.load(from + j * kLanes * VEC * P::kBytes);
                        *reinterpret_cast<float *>(to) = v.raw;
                    } else {
                        ptx::cp_async_16(ptx::smem_u32(to), from + j * kLanes * VEC * P::kBytes);
                    }
                }
        }
        ptx::cp_async_commit();
        from += stride;
    };
    int ahead = seg, slot = 0;
#pragma unroll
    for (int k = 0; k < kRowDepth - 1; ++k, ahead = ahead < total - step ? ahead + step : total) request(ahead < total, k * kSlot);
    pair_t gamma[kKeep ? NV : 1][kPairs], beta[kKeep ? NV : 1][kPairs];
    int shift[NV], ent[NV], held = -1;
#pragma unroll
    for (int j = 0; j < NV; ++j) shift[j] = ent[j] = 0;
    const int ob = out_bytes(a.out), next_piece = kLanes * VEC * ob;
    char *to = static_cast<char *>(a.out.Y) + ((size_t)seg * a.cpg + lane * VEC) * ob;
    const size_t far = (size_t)step * a.cpg * ob;
    const float count = (float)a.cpg, inverse = __frcp_rn(count);
    for (;;) {
        request(ahead < total, slot == 0 ? (kRowDepth - 1) * kSlot : slot - kSlot);
        if (ahead < total) ahead = ahead < total - step ? ahead + step : total;
        ptx::cp_async_wait_but<kRowDepth - 1>();           // (each lane reads what it asked for itself)
        pair_t x[NV][kPairs], s[kPairs];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < NV - 1 || last) {
                P v;
                v.raw = *reinterpret_cast<const typename P::Raw *>(hold + slot + j * kLanes * (VEC == 1 ? 4 : 16));
                v.widen(x[j]);
            } else {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) x[j][i] = pair(0.f, 0.f);
            }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            s[i] = x[0][i];
#pragma unroll
            for (int j = 1; j < NV; ++j) s[i] = add2(s[i], x[j][i]);
        }
        slot = slot == (kRowDepth - 1) * kSlot ? 0 : slot + kSlot;
        const float mean = divide(sum(fold<kPairs>(s), 0), count, inverse);
        const pair_t minus = pair(-mean, VEC == 1 ? 0.f : -mean), minus_last = last ? minus : pair(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                x[j][i] = add2(x[j][i], j < NV - 1 ? minus : minus_last);
                s[i] = j == 0 ? mul2(x[j][i], x[j][i]) : fma2(x[j][i], x[j][i], s[i]);
            }
        }
        const int g = a.groups == 1 ? 0 : seg % a.groups;
        if (g != held) {
            held = g;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j < NV - 1 || last) {
                    const int c = g * a.cpg + (lane + kLanes * j) * VEC;
                    if (kKeep) load_affine<VEC>(a, c, gamma[kKeep ? j : 0], beta[kKeep ? j : 0]);
                    shift[j] = slab_shift(a.out, c, &ent[j]);
                }
        }
        const float rstd = deviation_inverse(sum(fold<kPairs>(s), 1), count, a.eps);
        const pair_t r = pair(rstd, rstd);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!kKeep && (j < NV - 1 || last)) load_affine<VEC>(a, g * a.cpg + (lane + kLanes * j) * VEC, gamma[0], beta[0]);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) x[j][i] = fma2(x[j][i], mul2(gamma[kKeep ? j : 0][i], r), beta[kKeep ? j : 0][i]);
        }
        store_pieces<VEC, NV>(a, x, [&](int j) { return j < NV - 1 || last; }, [&](int j) { return to + (j * next_piece + shift[j]); }, [&](int j) { return ent[j]; });
        if (seg >= total - step) break;
        seg += step;
        to += far;
    }
    ptx::pdl_launch_dependents();
}

// ------------------------------------------------------------------------------------ host side
// Dynamic shared memory beyond the default, once per kernel and device whatever the size asked for later.
template <class K> static int allow_smem(K kernel, bool (&done)[64], int bytes)
{
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 64 && done[dev]) return FLEXIQ_OK;
    FLEXIQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (dev < 64) done[dev] = true;
    return FLEXIQ_OK;
}
static void set_attributes(cudaLaunchAttribute *attr, unsigned cluster)
{
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
}
// Clusters go to as few SMs as hold their blocks, which leaves others idle.  Where the machine has room for all of them with one block to an SM, or with two,
// they ask for so much shared memory that no SM takes more: fp16, 32 groups, 32 x 784 x 256 (32 clusters of four) 8.6 us, 9.3 without; 33 x 1000 x 64 in 16
// groups 7.0 and 8.5.  The room is asked for, since parts of the machine whose SMs the cluster's size does not divide leave some free: one cluster
// more than there is room for waits for another's end (36 x 1053 x 64, 36 of them, 14.1 us so and 10.2 with two blocks to an SM).
template <class K> static int spread_clusters(K kernel, cudaLaunchConfig_t &cfg, int cluster_log)
{
    struct Room { int own; int clusters[2][2]; };            // [log of the size - 1][blocks to an SM - 1], 0: not asked yet
    static Room rooms[64] = {};                              // (per kernel and device; written twice at worst)
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 64) return FLEXIQ_OK;
    Room &room = rooms[dev];
    const long long clusters = (long long)cfg.gridDim.x * cfg.gridDim.y >> cluster_log;
    for (int share = 1; share <= 2; ++share) {
        int &most = room.clusters[cluster_log - 1][share - 1];
        if (!most) {
            cudaFuncAttributes f;
            FLEXIQ_CUDA_TRY(cudaFuncGetAttributes(&f, kernel));
            room.own = (int)f.sharedSizeBytes;
            cudaLaunchConfig_t ask = cfg;
            ask.dynamicSmemBytes = apart_smem(share, room.own);
            FLEXIQ_CUDA_TRY(cudaOccupancyMaxActiveClusters(&most, kernel, &ask));
        }
        const int apart = apart_smem(share, room.own);
        if ((int)cfg.dynamicSmemBytes >= apart) return FLEXIQ_OK;
        if (clusters <= most) {
            cfg.dynamicSmemBytes = apart;
            return FLEXIQ_OK;
        }
    }
    return FLEXIQ_OK;
}
template <int DT, int VEC, bool MANY, int T> static int launch_held_threads(const NormArgs &a, const NormPlan &p, int sms, cudaStream_t st)
{
    static bool done[64] = {};
    if (int rc = allow_smem(group_norm_held_kernel<DT, VEC, MANY, T>, done, kSmemSM / 2)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.Nb << a.cluster_log), (unsigned)(a.groups / a.gpb), 1);
    cfg.blockDim = dim3((unsigned)T, 1, 1);
    cfg.dynamicSmemBytes = p.nv * T * (VEC == 1 ? 4 : 16);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    set_attributes(attr, 1u << a.cluster_log);
    cfg.attrs = attr;
    cfg.numAttrs = a.cluster_log ? 2 : 1;
    if (a.cluster_log)
        if (int rc = spread_clusters(group_norm_held_kernel<DT, VEC, MANY, T>, cfg, a.cluster_log)) return rc;
    FLEXIQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, group_norm_held_kernel<DT, VEC, MANY, T>, a));
    return FLEXIQ_OK;
}
template <int DT, int VEC, bool MANY> static int launch_held(const NormArgs &a, const NormPlan &p, int sms, cudaStream_t st)
{
    switch (p.threads) {
        case 64: return launch_held_threads<DT, VEC, MANY, 64>(a, p, sms, st);
        case 128: return launch_held_threads<DT, VEC, MANY, 128>(a, p, sms, st);
        case 256: return launch_held_threads<DT, VEC, MANY, 256>(a, p, sms, st);
        default: return launch_held_threads<DT, VEC, MANY, 512>(a, p, sms, st);
    }
}
template <int DT, int VEC, bool MANY> static int launch_twice(const NormArgs &a, const NormPlan &p, cudaStream_t st)
{
    const unsigned blocks = (unsigned)(a.groups / a.gpb);
    constexpr int kStats = kNormThreads * kStatsPieces * kStatsDepth * (VEC == 1 ? 4 : 16), kApply = kNormThreads * kApplyPieces * kApplyDepth * (VEC == 1 ? 4 : 16);
    static bool done[2][64] = {};
    if (int rc = allow_smem(group_norm_stats_kernel<DT, VEC, MANY>, done[0], kStats)) return rc;
    if (int rc = allow_smem(group_norm_apply_kernel<DT, VEC, MANY>, done[1], kApply)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.Nb * a.cluster), blocks, 1);
    cfg.blockDim = dim3((unsigned)p.threads, 1, 1);
    cfg.dynamicSmemBytes = kStats;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    set_attributes(attr, 1u << a.cluster_log);
    cfg.attrs = attr;
    cfg.numAttrs = a.cluster_log ? 2 : 1;
    FLEXIQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, group_norm_stats_kernel<DT, VEC, MANY>, a));
    FLEXIQ_CUDA_TRY(launch_pdl(group_norm_apply_kernel<DT, VEC, MANY>, dim3((unsigned)(a.Nb * a.cuts), blocks, 1), (unsigned)p.threads, kApply, st, a));
    return FLEXIQ_OK;
}
template <int DT, int VEC, int NV, int WARPS> static int launch_rows_nv(const NormArgs &a, int sms, cudaStream_t st)
{
    // few rows: as many blocks as there are; many: as many blocks of eight warps as an SM holds, each team of warps walking over rows
    const long long total = a.Nb * a.groups;
    const unsigned threads = total < 8ll * sms ? (WARPS > 2 ? 32 * WARPS : 64) : kNormThreads;
    long long blocks = ceil_div(total, threads / (32 * WARPS));
    const long long most = (NV == 1 ? 3ll : 2ll) * sms;
    if (blocks > most && threads == kNormThreads) blocks = most;
    constexpr int kRow = kRowDepth * NV * (VEC == 1 ? 4 : 16);   // a thread's slots
    static bool done[64] = {};
    if (int rc = allow_smem(group_norm_rows_kernel<DT, VEC, NV, WARPS>, done, kNormThreads * kRow)) return rc;
    FLEXIQ_CUDA_TRY(launch_pdl(group_norm_rows_kernel<DT, VEC, NV, WARPS>, (unsigned)blocks, threads, (size_t)threads * kRow, st, a));
    return FLEXIQ_OK;
}
template <int DT, int VEC> static int launch_norm_rows(const NormArgs &a, const NormPlan &p, int sms, cudaStream_t st)
{
    if constexpr (VEC > 1) {
        if (p.warps > 1) switch (p.nv) {
            case 3: return launch_rows_nv<DT, VEC, 3, kRowWarps>(a, sms, st);
            case 4: return launch_rows_nv<DT, VEC, 4, kRowWarps>(a, sms, st);
            case 5: return launch_rows_nv<DT, VEC, 5, kRowWarps>(a, sms, st);
            case 6: return launch_rows_nv<DT, VEC, 6, kRowWarps>(a, sms, st);
            case 7: return launch_rows_nv<DT, VEC, 7, kRowWarps>(a, sms, st);
            default: return launch_rows_nv<DT, VEC, 8, kRowWarps>(a, sms, st);
        }
    }
    switch (p.nv) {
        case 1: return launch_rows_nv<DT, VEC, 1, 1>(a, sms, st);
        case 2: return launch_rows_nv<DT, VEC, 2, 1>(a, sms, st);
        case 3: return launch_rows_nv<DT, VEC, 3, 1>(a, sms, st);
        case 4: return launch_rows_nv<DT, VEC, 4, 1>(a, sms, st);
        case 5: return launch_rows_nv<DT, VEC, 5, 1>(a, sms, st);
        case 6: return launch_rows_nv<DT, VEC, 6, 1>(a, sms, st);
        case 7: return launch_rows_nv<DT, VEC, 7, 1>(a, sms, st);
        default: return launch_rows_nv<DT, VEC, 8, 1>(a, sms, st);
    }
}
template <int DT> static int launch_norm(const NormArgs &a, const NormPlan &p, int sms, cudaStream_t st)
{
    constexpr int V = FullVec<DT>::v;
    if (p.kind == kNormRows) return p.vec == 1 ? launch_norm_rows<DT, 1>(a, p, sms, st) : launch_norm_rows<DT, V>(a, p, sms, st);
    if (p.kind == kNormHeld) return p.vec == 1 ? launch_held<DT, 1, false>(a, p, sms, st) : p.many ? launch_held<DT, V, true>(a, p, sms, st) : launch_held<DT, V, false>(a, p, sms, st);
    return p.vec == 1 ? launch_twice<DT, 1, false>(a, p, st) : p.many ? launch_twice<DT, V, true>(a, p, st) : launch_twice<DT, V, false>(a, p, st);
}

unsigned norm_status()
{
    unsigned word = 0;
    const unsigned zero = 0;
    if (cudaMemcpyFromSymbol(&word, g_norm_status, sizeof(word)) != cudaSuccess) return 0;   // the caller's own read reports it
    if (word) cudaMemcpyToSymbol(g_norm_status, &zero, sizeof(zero));
    return word;
}

static long long value_bytes(int dtype) { return dtype == FLEXIQ_DTYPE_F32 ? 4 : 2; }
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
static long long scratch_bytes(const NormPlan &p, long long Nb, int groups) { return p.kind == kNormTwice ? Nb * groups * (p.cluster >> p.cluster_log) * (long long)sizeof(float2) : 0; }

static int run_norm(NormArgs &a, int x_dtype, void *scratch, cudaStream_t st)
{
    const int sms = plan_sms();
    const NormPlan p = plan_norm(x_dtype, a.Nb, a.P, a.C, a.groups, sms);
    if ((p.kind == kNormRows ? a.Nb * a.groups : a.Nb * (long long)(p.cluster > p.cuts ? p.cluster : p.cuts)) > 0x40000000ll || (p.kind != kNormRows && a.groups / p.gpb > 65535))
        return set_error(FLEXIQ_ERR_UNSUPPORTED, "too many images and groups for one launch");
    if (p.kind == kNormTwice && (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 15)))
        return set_error(FLEXIQ_ERR_INVALID_ARG, "scratch_dev is NULL or not 16-byte aligned: this shape needs %lld bytes", scratch_bytes(p, a.Nb, a.groups));
    a.cpg = a.C / a.groups;
    a.gpb = p.gpb; a.nch = p.nch; a.cpt = p.cpt; a.lanes = p.lanes; a.cluster = p.cluster; a.span = p.span; a.cuts = p.cuts; a.cut_span = p.cut_span;
    a.stats = static_cast<float2 *>(scratch);
    a.cluster_log = p.cluster_log; a.joined = p.cluster >> p.cluster_log;
    auto inverse = [](int d) { return d > 1 ? (unsigned)((0x100000000ull + d - 1) / d) : 0u; };   // (exact for numerators below 2^16 and such d)
    a.by_nch = inverse(p.nch); a.by_lanes = inverse(p.lanes); a.by_cpg = inverse(a.cpg);
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
    if (Nb == 0 || P == 0) return FLEXIQ_OK;
    if (X_dev == Y_dev && x_dtype != y_dtype) return set_error(FLEXIQ_ERR_INVALID_ARG, "Y_dev is X_dev, which needs the same type");
    if (X_dev != Y_dev && share_memory(X_dev, Nb * P * C * value_bytes(x_dtype), Y_dev, Nb * P * C * value_bytes(y_dtype)))
        return set_error(FLEXIQ_ERR_INVALID_ARG, "X_dev and Y_dev overlap and are not the same");
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
    if (share_memory(X_dev, Nb * P * L->C * value_bytes(x_dtype), X4_dev, Nb * P * L->C)) return set_error(FLEXIQ_ERR_INVALID_ARG, "X_dev and the slab overlap");
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
