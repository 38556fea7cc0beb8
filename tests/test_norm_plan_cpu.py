"""How a group normalisation is cut up: every value belongs to one thread, and no index leaves its array, for shapes of every kind."""
import os
import subprocess

from paper_2510_02822_b200 import build as fxbuild

SRC = r"""
#include "norm_plan.h"
#include <stdio.h>
#include <random>
#include <vector>
using namespace flexiq;
static unsigned r0 = 0;
static int fail(const char *what, int dt, long long Nb, long long P, int C, int g) { printf("%s: type %d, %lld x %lld x %d, %d groups\n", what, dt, Nb, P, C, g); return 1; }
static int check(int dt, long long Nb, long long P, int C, int groups)
{
    const int full = dt == FLEXIQ_DTYPE_F32 ? 4 : 8, cpg = C / groups;
    const NormPlan p = plan_norm(dt, Nb, P, C, groups, 148);
    auto bad = [&](const char *w) { return fail(w, dt, Nb, P, C, groups); };
    if (p.vec != 1 && (p.vec != full || C % full)) return bad("width");
    if (p.kind == kNormRows) {
        if (P != 1 || p.nch * p.vec != cpg || p.nv * 32 * p.warps < p.nch || (p.nv - 1) * 32 * p.warps >= p.nch || p.nv > 8 || p.nv < 1) return bad("rows");
        if (p.warps != 1 && (p.warps != kRowWarps || p.vec == 1 || p.nv < 3)) return bad("warps of a row");
        return 0;
    }
    if (p.gpb < 1 || groups % p.gpb || p.gpb > kMaxGroups || p.nch * p.vec != p.gpb * cpg) return bad("channel block");
    if (p.vec > 1 && (p.gpb * cpg) % p.vec) return bad("pieces that leave the block");
    if (p.threads > 512 || (p.kind == kNormTwice && p.threads != kNormThreads) || p.threads % 32 || p.threads < 32) return bad("threads");
    if (!p.many && cpg % p.vec) return bad("a piece of two groups summed as one");
    if (p.cpt > 1 && (p.gpb != 1 || p.many || p.threads != kNormThreads || p.lanes != 1 || p.cpt * p.threads < p.nch)) return bad("wide positions");
    if (p.cpt == 1 && (p.lanes < 1 || p.lanes * p.nch > p.threads)) return bad("lanes");
    if (p.cluster < 1 || p.cluster > (p.kind == kNormHeld ? kNormCluster : kNormSplits) || p.span * p.cluster < P || p.span < 1) return bad("pieces of an image");
    if (p.kind == kNormTwice && (p.cuts < 1 || p.cuts > kNormCuts || p.cut_span * p.cuts < P || p.cut_span < 1)) return bad("the second kernel's pieces");
    if (p.kind == kNormTwice && p.cluster >> p.cluster_log > kNormEntries) return bad("statistics left for the second kernel");
    if (p.kind == kNormHeld) {
        if ((p.cluster & (p.cluster - 1)) || p.nv < 1 || p.nv * p.threads * 16 > kNormHold || (p.threads != 64 && p.threads != 128 && p.threads != 256 && p.threads != 512)) return bad("what a block holds");
        std::vector<unsigned char> seen((size_t)p.span * p.nch, 0);
        for (int t = 0; t < p.threads; ++t) {
            int pl, col, k = 0;
            bool live = true;
            if (p.cpt > 1) { pl = 0; col = t; } else { pl = t / p.nch; col = t - pl * p.nch; live = pl < p.lanes; }
            int c = col;
            for (int j = 0; j < p.nv; ++j) {
                if (live && pl < p.span && c < p.nch && seen[(size_t)pl * p.nch + c]++) return bad("twice held");
                if (p.cpt > 1) { c += p.threads; if (++k == p.cpt) { k = 0; c = col; ++pl; } } else pl += p.lanes;
            }
        }
        for (unsigned char s : seen) if (s != 1) return bad("not held");
    }
    auto inverse = [](int d) { return d > 1 ? (unsigned)((0x100000000ull + d - 1) / d) : 0u; };
    for (int d : {p.nch, p.lanes, cpg}) {
        const unsigned inv = inverse(d);
        for (int n = (int)(r0 % 97); n < 65536; n += 61)
            if ((inv ? (int)(((unsigned long long)n * inv) >> 32) : n) != n / d) return bad("quotients by multiplication");
    }
    ++r0;
    if (p.cluster_log < 0 || p.cluster % (1 << p.cluster_log) || (p.kind == kNormHeld && p.cluster != 1 << p.cluster_log)) return bad("clusters");
    // entries: every group's, from the columns that hold a part of it, are those its threads have put
    if (p.many) {
        std::vector<int> has((size_t)p.gpb, 0);
        for (int col = 0; col < p.nch; ++col) {
            int left = cpg - (col * p.vec - col * p.vec / cpg * cpg), w = 0;
            for (int i = 0; i < p.vec; ++i)
                if (--left == 0 || i == p.vec - 1) {
                    if (w >= p.vec) return bad("entries of a thread");
                    const int g = col * p.vec / cpg + w++;
                    if (g >= p.gpb || col < g * cpg / p.vec || col > ((g + 1) * cpg - 1) / p.vec) return bad("an entry of no group");
                    ++has[g];
                    left = cpg;
                }
        }
        for (int g = 0; g < p.gpb; ++g)
            if (has[g] != ((g + 1) * cpg - 1) / p.vec - g * cpg / p.vec + 1) return bad("columns of a group");
    }
    return 0;
}
int main()
{
    std::mt19937_64 r(7);
    auto log_uniform = [&](double hi) { return (long long)__builtin_exp(std::uniform_real_distribution<double>(0, __builtin_log(hi + 0.999))(r)); };
    const int group_counts[] = {1, 2, 3, 4, 5, 8, 16, 32, 32, 64, 128, 300};
    for (int i = 0; i < 40000; ++i) {
        const int groups = group_counts[r() % 12], dt = (int)(r() % 3);
        const long long Nb = log_uniform(30000), P = r() % 4 ? log_uniform(300000) : 1 + r() % 3;
        const int C = groups * (int)log_uniform(9000 / groups + 2);
        if (check(dt, Nb, P, C, groups)) return 1;
    }
    for (int C = 1; C <= 600; ++C)
        for (int g = 1; g <= C; ++g)
            if (C % g == 0)
                for (long long P : {1, 2, 49, 3136, 70000})
                    if (check((C + g) % 3, 1 + C % 5, P, C, g)) return 1;
    return 0;
}
"""


def test_every_value_has_one_thread(tmp_path):
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(SRC)
    include = os.path.join(os.path.dirname(fxbuild.CSRC), os.pardir, "include")
    subprocess.run(["g++", "-O2", "-std=c++17", f"-I{fxbuild.CSRC}", f"-I{include}", str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
