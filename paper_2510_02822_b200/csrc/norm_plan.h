// How a group normalisation is cut up for its shape (host only; flexiq_norm.cu has the kernels).
#pragma once
#include "flexiq.h"

namespace flexiq {

constexpr int kNormThreads = 256;
constexpr int kRowWarps = 4;           // warps that take a long row together
constexpr int kNormHold = 65536;        // bytes a block holds ("held")
constexpr int kNormCluster = 4;        // blocks of a cluster at most ("held")
constexpr int kNormEntries = 160;      // statistics of an image's group that "twice" leaves for its second kernel, at most
constexpr int kNormSplits = 2 * kNormEntries;   // pieces of an image's channel block at most ("twice")
constexpr int kNormCuts = 512;          // and for the second kernel
constexpr int kMaxGroups = 128;        // groups of a channel block at most

enum NormKind { kNormRows, kNormHeld, kNormTwice };
struct NormPlan { NormKind kind; int vec, nv, warps, threads, gpb, nch, cpt, lanes, cluster, cluster_log, cuts; long long span, cut_span; bool many; };

inline int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
inline int round_up_pow2(long long v) { int p = 1; while (p < v) p <<= 1; return p; }

// (a function of the shape alone, so that the scratch size can be asked for)
inline NormPlan plan_norm(int x_dtype, long long Nb, long long P, int C, int groups, int sms)
{
    const int bytes = x_dtype == FLEXIQ_DTYPE_F32 ? 4 : 2, full = 16 / bytes, cpg = C / groups;
    NormPlan p{};
    p.cpt = 1;
    if (P == 1) {
        const int vec = cpg % full == 0 ? full : 1, pieces = cpg / vec;
        p.warps = pieces <= 256 ? 1 : kRowWarps;
        p.nv = (int)ceil_div(pieces, 32 * p.warps);
        if (p.nv <= 8 && (vec > 1 || p.warps == 1)) {
            p.kind = kNormRows; p.vec = vec; p.nch = pieces;
            return p;
        }
    }
    // the smallest block of whole groups and whole pieces, then more groups
    const int base_groups = C % full == 0 ? full / gcd(cpg, full) : 1;
    const long long base_pieces = (long long)base_groups * cpg / full;
    p.vec = C % full == 0 && (base_pieces <= kNormThreads || cpg % full == 0) ? full : 1;
    const int unit_groups = p.vec == 1 ? 1 : base_groups, units = groups / unit_groups;
    auto shape = [&](int m) {   // m of the smallest blocks together
        p.gpb = unit_groups * m;
        p.nch = (int)((long long)p.gpb * cpg / p.vec);
        p.many = p.vec > 1 && cpg % p.vec != 0;
        p.cpt = (int)ceil_div(p.nch, kNormThreads);
    };
    auto run = [&](int w) { return (long long)unit_groups * w * cpg * bytes; };   // bytes of a position that a block takes
    // Positions a block holds: 64 KB of pieces (two blocks an SM), eight a thread of 512 (a piece of the scalar form is shorter, but as long to work on).
    auto capacity = [&](int w) {
        const long long nch = (long long)unit_groups * w * cpg / p.vec;
        return nch > kNormThreads ? 16 / ceil_div(nch, kNormThreads) : 512 / nch * 8;
    };
    const bool one_wave = Nb * P * C * bytes <= 2ll * sms * kNormHold;
    // Runs of 128 bytes at least, and of short images so many channels that a block's own work (sums over its threads, the joining) is spread over
    // 32 KB: 1024 x 49 x 512 fp16 in 32 groups 24.6 us, 40.7 in runs of 128 bytes; 4096 x 16 x 256 in 8 groups 21 and 31.
    int m = 1;
    while (m < units && (run(m) < 128 || run(m) * P < kNormHold / 2) && unit_groups * m < kMaxGroups / 2) {
        int next = m + 1;
        while (units % next) ++next;
        if ((long long)unit_groups * next * cpg / p.vec > kNormThreads || unit_groups * next > kMaxGroups || (run(m) >= 128 && capacity(next) < P)) break;
        m = next;
    }
    for (int w = m; w >= 1; --w) {
        if (units % w) continue;
        shape(w);
        const long long most = capacity(w);
        if (most < 1 || ceil_div(P, most) > kNormCluster) continue;
        // Narrow runs, or several blocks to an image, only where the machine holds all of it at once: beyond that the second read comes from the
        // L2 cache and "twice" is faster (32 x 3136 x 256 fp16 in 32 groups 28 us, held 34; 8 x 4096 x 320 17.4 and 22.9).  Within it holding is
        // (32 x 784 x 128 8.0 us, twice 11.5), from sectors of 32 bytes on (8 x 12544 x 64 in runs of 16 bytes 17.7 us, twice 14.6).
        if (w < m && (run(w) < 32 || !one_wave)) continue;
        if (ceil_div(P, most) > 1 && !one_wave) continue;
        p.kind = kNormHeld;
        p.threads = kNormThreads;
        const long long blocks = Nb * (units / w);
        int k = round_up_pow2(ceil_div(P, most));
        // more blocks where the machine has room for them and a thread more than one piece
        while (k < kNormCluster && blocks * k * 2 <= 2 * sms && ceil_div(P, k) > (p.cpt > 1 ? 1 : kNormThreads / p.nch)) k *= 2;
        p.cluster = k;
        for (p.cluster_log = 0; (1 << p.cluster_log) < k; ++p.cluster_log) {}
        p.span = ceil_div(P, k);
        if (p.cpt == 1) {
            // threads for about four pieces each: the passes over them are a chain of latencies.  Where there are blocks for every SM a thread's fixed
            // work counts as well, and 256 do
            while (p.threads < 512 && (blocks * k < sms || ceil_div(p.span, p.threads / p.nch) > 16) && ceil_div(p.span, p.threads / p.nch) > 6) p.threads *= 2;
            while (p.threads > 64 && p.threads / 2 >= p.nch && ceil_div(p.span, p.threads / 2 / p.nch) <= 4) p.threads /= 2;
            p.lanes = p.threads / p.nch;
            p.nv = (int)ceil_div(p.span, p.lanes);
        } else {
            p.lanes = 1;
            p.nv = (int)(p.span * p.cpt);
        }
        return p;
    }
    // nothing to be held: as much of a position as a block's threads take, up to 1 KB, which is read in longer runs
    for (int w = units; w > m; --w)
        if (units % w == 0 && unit_groups * w <= kMaxGroups && (long long)unit_groups * w * cpg * bytes <= 1024 && (long long)unit_groups * w * cpg / p.vec <= kNormThreads) { m = w; break; }
    shape(m);
    p.kind = kNormTwice;
    p.threads = kNormThreads;
    p.lanes = p.cpt > 1 ? 1 : kNormThreads / p.nch;
    // Pieces: as many as make whole waves of the blocks that fit an SM (nine tenths of one at least, where up to four waves allow that), and a few
    // steps each.  Two blocks fit with the statistics' registers, three with those of the second kernel, which cuts the image anew.
    const long long blocks = Nb * (units / m), steps = p.cpt > 1 ? P : ceil_div(P, (long long)p.lanes * 8);
    auto pieces = [&](long long wave, int most) {
        long long k = 1;
        for (long long w = 1; w <= 4; ++w) {
            k = w * wave / blocks;
            if (k * blocks * 10 >= w * wave * 9) break;
        }
        k = k < steps ? k : steps;
        return (int)(k < 1 ? 1 : k < most ? k : most);
    };
    p.cluster = pieces(2ll * sms, kNormSplits);
    p.cluster_log = p.cluster > kNormEntries ? 1 : 0;   // the statistics of two pieces are joined where they are made
    // (1 x 409600 x 128 fp16: 62.3 us, 66.0 with every piece's left to the second kernel, 66.6 with four joined, whose clusters found room on fewer SMs)
    // The positions of a piece are rounded up, so that fewer pieces than planned may hold them all: none is made without a position, but for the second
    // of the last two where those are joined.
    const int joined = 1 << p.cluster_log;
    p.cluster &= ~(joined - 1);
    p.span = ceil_div(P, p.cluster);
    p.cluster = ((int)ceil_div(P, p.span) + joined - 1) & ~(joined - 1);
    p.cuts = pieces(3ll * sms, kNormCuts);
    p.cut_span = ceil_div(P, p.cuts);
    p.cuts = (int)ceil_div(P, p.cut_span);
    return p;
}

// The least dynamic shared memory with which an SM takes no more than `share` blocks that have `own` bytes of static arrays besides, and kSmemBlock of the
// system's.
constexpr int kSmemSM = 228 * 1024, kSmemBlock = 1024;
inline int apart_smem(int share, int own) { return (kSmemSM / (share + 1) / 128 + 1) * 128 - kSmemBlock - own; }

}  // namespace flexiq
