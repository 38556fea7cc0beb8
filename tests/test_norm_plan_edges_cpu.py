"""How a group normalisation is cut up where an image's pieces end with the image, and how its clusters are spread over the SMs."""
import os
import subprocess

from paper_2510_02822_b200 import build as fxbuild

PIECES = r"""
#include "norm_plan.h"
#include <stdio.h>
#include <random>
using namespace flexiq;
static int check(int dt, long long Nb, long long P, int C, int groups, int sms)
{
    const NormPlan p = plan_norm(dt, Nb, P, C, groups, sms);
    if (p.kind != kNormTwice) return 0;
    const int k = 1 << p.cluster_log, entries = p.cluster >> p.cluster_log;
    const bool ok = p.cluster % k == 0 && entries >= 1 && entries <= kNormEntries && p.cuts >= 1 &&
                    (long long)p.cluster * p.span >= P && (long long)p.cuts * p.cut_span >= P &&
                    (long long)(entries - 1) * k * p.span < P &&       // every entry that is joined and written has a position
                    (long long)(p.cluster - k) * p.span < P && (long long)(p.cuts - 1) * p.cut_span < P;
    if (!ok) printf("type %d, %lld x %lld x %d, %d groups, %d SMs: %d pieces of %lld, %d joined; %d of %lld\n", dt, Nb, P, C, groups, sms, p.cluster, p.span, k, p.cuts, p.cut_span);
    return !ok;
}
int main()
{
    int bad = 0;
    const struct { int dt; long long P; int C, groups; } known[] = {
        {1, 6600, 512, 4}, {1, 8712, 512, 32}, {1, 10920, 256, 32}, {1, 9800, 320, 32}, {1, 9604, 320, 32}, {1, 4000, 640, 1}, {0, 6724, 192, 32},
        {0, 10270, 128, 32}, {1, 33282, 128, 32}, {1, 984, 435, 1}, {1, 21316, 256, 32}, {1, 15876, 512, 32}};
    for (auto &k : known) bad += check(k.dt, 1, k.P, k.C, k.groups, 148);
    for (int C : {3, 64, 128, 192, 256, 320, 435, 512, 640, 1280})
        for (int groups : {1, 32})
            if (C % groups == 0)
                for (long long P = 1; P <= 40000; ++P) bad += check((int)(P + C) % 3, 1, P, C, groups, 148);
    std::mt19937_64 r(11);
    auto log_uniform = [&](double hi) { return (long long)__builtin_exp(std::uniform_real_distribution<double>(0, __builtin_log(hi + 0.999))(r)); };
    const int group_counts[] = {1, 2, 3, 4, 5, 8, 16, 32, 64, 300};
    for (int i = 0; i < 400000; ++i) {
        const int groups = group_counts[r() % 10];
        const long long Nb = log_uniform(400), P = log_uniform(3000000);
        bad += check((int)(r() % 3), Nb, P, groups * (int)log_uniform(2000 / groups + 2), groups, r() % 4 ? 148 : 1 + (int)(r() % 200));
    }
    return bad != 0;
}
"""


def run_plan(tmp_path, source):
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(source)
    include = os.path.join(os.path.dirname(fxbuild.CSRC), os.pardir, "include")
    subprocess.run(["g++", "-O2", "-std=c++17", f"-I{fxbuild.CSRC}", f"-I{include}", str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[:2000]


def test_no_piece_without_a_position(tmp_path):
    run_plan(tmp_path, PIECES)


SPREAD = r"""
#include "norm_plan.h"
#include <stdio.h>
using namespace flexiq;
int main()
{
    int bad = 0;
    for (int own = 512; own <= 48 * 1024; own += 512)             // static arrays: up to some 42 KB (512 threads, pieces of several groups)
        for (int share = 1; share <= 2; ++share) {
            const int bytes = apart_smem(share, own), block = bytes + own + 1024;
            if (share * block > 228 * 1024 || (share + 1) * block <= 228 * 1024 || bytes + own > 227 * 1024 || bytes > kSmemSM / 2 || bytes < 0) {
                printf("own %d, %d blocks an SM: %d\n", own, share, bytes);
                ++bad;
            }
        }
    return bad != 0;
}
"""


def test_blocks_apart_but_not_further(tmp_path):
    """So much shared memory that as many blocks as are meant share an SM, no more and no fewer."""
    run_plan(tmp_path, SPREAD)
