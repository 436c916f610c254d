// Tile and split of the weight gradient from a checkpoint (ckpt_wgrad.hip).  Host code alone, so that it can be built and asked without the kernels.
#pragma once

#include <cstdint>

namespace ffi {

struct WgradPlan {
    int tile, splits;
    int64_t steps, per;
};
static int plan_rows(int terms, int tile) { return terms == 3 && tile > 64 ? 16 : 32; }
// Tile and split of the rows: the pair that takes the least time by what was measured.  Sixteen rows take a workgroup `alone` microseconds where it
// has the compute unit to itself, and `shared` for every workgroup of the unit where there are several, up to `units` of them at once; one round of them has 2 us
// of first loads and last stores, a sum of splits 3 us and its traffic at 5 TB/s.  (2048 rows, 2000 x 2000, fp32: 256x256 in four splits 71 us by this and 74
// measured, 128x128 in two 76 and 81, in one 92 and 94; bf16: 41 and 46, 39 and 44, 39 and 42.)
static WgradPlan wgrad_plan(int64_t rows, int64_t n, int64_t k, int terms)
{
    struct Speed { int tile, units; double alone, shared; };   // per number of terms
    static constexpr Speed speeds[3][3] = {{{256, 1, 0.49, 0.49}, {128, 2, 0.26, 0.165}, {64, 5, 0.10, 0.075}},
                                           {{256, 1, 0.93, 0.93}, {128, 2, 0.45, 0.30}, {64, 4, 0.17, 0.115}},
                                           {{256, 1, 1.45, 1.45}, {128, 2, 0.67, 0.445}, {64, 3, 0.245, 0.175}}};
    static constexpr int splits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256};
    WgradPlan best = {64, 1, 0, 0};
    double least = 0;
    for (const Speed& v : speeds[terms - 1]) {
        const int bm = plan_rows(terms, v.tile);
        const int64_t count = ((n + v.tile - 1) / v.tile) * ((k + v.tile - 1) / v.tile), steps = (rows + bm - 1) / bm;
        for (int s : splits) {
            if (s > 1 && (s > steps || s * n * k > (int64_t(1) << 26))) break;
            const int64_t per = (steps + s - 1) / s, real = per > 0 ? (steps + per - 1) / per : 1;
            const int64_t each = (count * real + 255) / 256, rounds = (each + v.units - 1) / v.units;   // workgroups of a compute unit
            const double alone = (double)rounds * v.alone, shared = (double)each * v.shared;
            const double t = (double)(per * (bm / 16)) * (alone > shared ? alone : shared) + 2.0 * (double)rounds +
                             (real > 1 ? 3.0 + (double)((real + 1) * n * k) * 4e-6 / 5.0 : 0.0);
            if (least == 0 || t < least) {
                least = t;
                best = {v.tile, (int)real, steps, per};
            }
            if (count * s >= 2048) break;   // (every compute unit has its share)
        }
    }
    return best;
}

}  // namespace ffi
