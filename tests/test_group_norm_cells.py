"""What the group norm's plan counts for a workgroup is what the launched kernel takes: swept on the host over wide rows of few pixels, by the rule of the kernels."""
import os
import shutil
import subprocess

import pytest

import test_group_norm_plan as plan

# Sums of a chunk that are kept apart: a kernel for rows of whole chunks whose halves lie in one group each has two forward, every other kernel eight.
PROGRAM = r'''
#include "group_norm_plan.hpp"
#include <cstdio>
using namespace ffi;
typedef long long ll;
static ll pitch(ll c) { return c <= 512 ? gn_up(c, 16) : gn_up(c, 128); }
int main()
{
    ll ragged = 0, whole = 0, wide = 0;
    auto look = [&](ll N, ll P, ll C, ll G) {
        for (int size : {2, 4})
            for (int back : {0, 1})
                for (int kept : {0, 1}) {
                    if (back && kept) continue;
                    const ll d = C / G;
                    const GnPlan p = gn_plan(N, P, C, G, size, kept, back ? C : pitch(C), back);
                    if (!p.whole) continue;
                    const int cells = !back && C % 8 == 0 && d % 4 == 0 ? 2 : 8;
                    const size_t lds = gn_lds(p.cut.threads, p.cut.slots, cells, d);
                    (C % 8 ? ragged : whole) += 1;
                    wide += cells == 2 && gn_lds(p.cut.threads, p.cut.slots, 8, d) > GN_MOST_LDS;
                    if (lds > GN_MOST_LDS) {
                        printf("%lld samples, %lld pixels, %lld channels, %lld groups, %d bytes, kept %d, backward %d: %zu bytes of LDS\n", N, P, C, G, size, kept, back, lds);
                        return false;
                    }
                }
        return true;
    };
    for (ll N : {1, 8, 300})
        for (ll P : {1, 2, 3, 4, 8, 15, 16, 17, 40}) {
            for (ll C = 4; C <= 65532; C += C < 16 || (C > 5000 && C < 8300) ? 4 : 4 * (1 + C / 64))
                for (ll G : {1, 3, 5, 1501, (int)(C / 4), (int)(C / 12), (int)C})
                    if (G > 0 && C % G == 0 && !look(N, P, C, G)) return 1;
            for (ll C = 5000; C < 8300; C += 7)
                if (!look(N, P, C, 1)) return 1;
        }
    printf("%lld %lld %lld", ragged, whole, wide);
}
'''


def test_a_workgroup_has_the_lds_that_its_kernel_takes(tmp_path):
    compiler = shutil.which("g++") or shutil.which("hipcc")
    if compiler is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "cells.cpp").write_text(PROGRAM)
    subprocess.run([compiler, "-O1", "-std=c++17", "-I" + os.path.join(plan.ROOT, "paper_2506_22771_amd", "csrc"), str(tmp_path / "cells.cpp"), "-o", str(tmp_path / "cells")],
                   check=True)
    done = subprocess.run([str(tmp_path / "cells")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
    assert all(int(n) > 100 for n in done.stdout.split()), done.stdout      # (of rows of both kinds; and some that eight sums a chunk would not let be whole)
