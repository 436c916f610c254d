"""How the group norm's launches cut up their maps, built on the host and asked: every column and pixel lies in exactly one workgroup, groups and the checkpoint's blocks
are not cut where a workgroup needs them whole, and threads, LDS and workspace keep their limits."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r'''
#include "group_norm_plan.hpp"
#include <cmath>
#include <cstdio>
#include <random>
using namespace ffi;
typedef long long ll;
#define CHECK(c) do { if (!(c)) { printf("%s: %lld samples, %lld pixels, %lld channels, %lld groups, %d bytes, kept %d, backward %d\n", #c, N, P, C, G, size, kept, back); return 1; } } while (0)
static ll pitch(ll c) { return c <= 512 ? gn_up(c, 16) : gn_up(c, 128); }
int main()
{
    std::mt19937_64 r(1);
    auto any = [&](double most) { return (ll)std::exp(std::uniform_real_distribution<double>(0, std::log(most))(r)); };
    ll whole = 0, split = 0, pieces = 0, few = 0;
    for (int i = 0; i < 100000; ++i) {
        const ll d = i % 2 ? 1ll << r() % 9 : any(i % 3 ? 64 : 65535), G = std::max(1ll, std::min(any(1000), 65535 / d)), C = d * G, P = any(40000), N = any(3000);
        if (C > 65535 || N * P * C > 1ll << 33) continue;
        for (int size : {2, 4})
            for (int back : {0, 1})
                for (int kept : {0, 1}) {
                    if (back && kept) continue;
                    const GnPlan p = gn_plan(N, P, C, G, size, kept, back ? C : pitch(C), back);
                    const ll unit = kept ? 32 : 8, row = gn_up(kept ? pitch(C) : C, unit);
                    const int cells = gn_cells(d, back);
                    CHECK(p.cut.slots >= 1 && p.cut.lanes >= 1 && p.cut.lanes == p.cut.threads / p.cut.slots);
                    CHECK((ll)p.cut.slice * p.cut.slices >= (back ? C : row) && (ll)p.cut.slice * (p.cut.slices - 1) < row);
                    CHECK(p.cut.slice % unit == 0 && p.cut.slots * 8 >= p.cut.slice);
                    if (p.whole) {
                        ++whole;
                        few += p.cut.lanes * (gn_rows(size, back) / 4) >= P;
                        CHECK(p.cut.slices == 1 || p.cut.slice % d == 0);
                        CHECK((ll)p.cut.lanes * gn_rows(size, back) >= P);
                        CHECK(p.cut.threads <= 1024 && gn_lds(p.cut.threads, p.cut.slots, cells, d) <= GN_MOST_LDS);
                    } else {
                        ++split;
                        CHECK(p.cut.threads == GN_SPLIT_THREADS && (ll)p.apply_blocks * p.cut.lanes * GN_APPLY_ROWS >= P);
                        CHECK(p.stat.threads == GN_SPLIT_THREADS && p.stat.lanes >= 1 && p.stat.lanes == GN_SPLIT_THREADS / p.stat.slots);
                        CHECK(gn_lds(GN_SPLIT_THREADS, p.stat.slots, 8, d) <= 65536);
                        if (back) {
                            CHECK(p.blocks >= 1 && p.blocks <= 128);
                        } else if (p.pieces == 1) {
                            CHECK(p.stat.slice % d == 0 && (ll)p.stat.slice * p.stat.slices >= C && (ll)p.blocks * p.stat.lanes * GN_STAT_ROWS >= P);
                        } else {
                            ++pieces;
                            CHECK(p.stat.slice % 8 == 0 && (ll)p.stat.slice * p.pieces >= d && (ll)p.stat.slice * (p.pieces - 1) < d && p.stat.slices == G * p.pieces);
                            CHECK((ll)p.blocks * p.stat.lanes * GN_STAT_ROWS >= P);
                        }
                    }
                }
    }
    printf("%lld %lld %lld %lld", whole, split, pieces, few);
}
'''


def test_every_pixel_and_column_once(tmp_path):
    compiler = shutil.which("g++") or shutil.which("hipcc")
    if compiler is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    subprocess.run([compiler, "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2506_22771_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")], check=True)
    done = subprocess.run([str(tmp_path / "plan")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
    assert all(int(n) > 1000 for n in done.stdout.split()), done.stdout     # (of each kind)
