// How the group norm's launches cut up their maps (group_norm.hip).  Host code alone, so that it can be built and asked without the kernels.
//
// A workgroup's threads lie over a slab: `slots` chunks of eight columns wide and `lanes` pixels high, a thread keeping its chunk's columns from pixel to pixel.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace ffi {

constexpr int GN_SPLIT_THREADS = 256;
// Pixels of a thread: that holds its slab in registers, of the statistics' launch, and of the launches that apply what others have summed.  As many as 128 registers hold
// beside the sums.  512 x 32x32 x 128 bf16 forward 62 us with 16 and 72 with 8, backward from codes 111 with 8 and 124 with 16 and 168 registers, three wavefronts a SIMD.
constexpr int gn_rows(int size, bool backward) { return backward ? (size == 4 ? 4 : 8) : (size == 4 ? 8 : 16); }
constexpr int GN_STAT_ROWS = 8, GN_APPLY_ROWS = 4;
constexpr int GN_MOST_GRID = 1 << 20; // workgroups of a launch, one item each: more items are further launches (launch_items).  Those of the joins take item after item
constexpr size_t GN_MOST_LDS = 150 * 1024;

struct GnCut {
    int32_t threads, slots, lanes;   // of a workgroup
    int32_t slice, slices;           // columns of a slice, slices of a row
};
// Sums of a chunk that are kept apart: two where its halves lie in one group each, else eight; of columns always eight.  Of rows of whole chunks, and of any row, whose
// kernel has eight where it ends inside a chunk: what the plan counts and what is launched (by_columns).
static int gn_cells(int64_t d, bool backward) { return !backward && d % 4 == 0 ? 2 : 8; }
static int gn_cells(int64_t channels, int64_t d, bool backward) { return channels % 8 == 0 ? gn_cells(d, backward) : 8; }
// threads that share the sum of a cell over the lanes, at most
static int gn_parts(int threads, int64_t slots, int cells) { return (int)std::max<int64_t>(1, std::min<int64_t>(32, std::min<int64_t>(threads / slots, threads / (slots * cells)))); }
// LDS of a workgroup: sums of two values per cell, of groups, and a row of weights
static size_t gn_lds(int threads, int64_t slots, int cells, int64_t d)
{
    return sizeof(float) * (size_t)(2 * slots * cells * (1 + gn_parts(threads, slots, cells) + threads / slots) + 2 * ((slots * 8 + d - 1) / d + 1) + 8 * slots);
}
struct GnPlan {
    bool whole;          // a workgroup holds whole groups in registers: one launch
    GnCut cut;           // whole: slices of whole groups.  Else those of the launches that apply
    GnCut stat;          // else: slices of the statistics' launch, of whole groups or of pieces of one
    int32_t pieces;      // slices of one group (1: a slice has whole groups)
    int32_t blocks;      // stat: workgroups of a slice over the pixels
    int32_t apply_blocks;
};

constexpr int64_t gn_gcd(int64_t a, int64_t b) { return b == 0 ? a : gn_gcd(b, a % b); }
static int64_t gn_up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

// size: bytes of an element; kept: a checkpoint is written or read, whose blocks of 32 columns lie in one workgroup; span: columns a row has to be covered to
static GnPlan gn_plan(int64_t samples, int64_t pixels, int64_t channels, int64_t groups, int size, bool kept, int64_t span, bool backward)
{
    GnPlan p = {};
    const int64_t d = channels / groups, unit = kept ? 32 : 8, step = d / gn_gcd(d, unit) * unit;
    const int64_t row = gn_up(kept ? span : channels, unit);   // columns of a row with what is behind it
    const int rows = gn_rows(size, backward), cells = gn_cells(channels, d, backward);
    // Slices from the narrowest on: as wide as 128 bytes, then wider while there are workgroups to spare and threads without a pixel, or none that fit.
    // Of the numbers of threads the first that holds lines of 128 bytes (of 64 where no codes are written), or else the widest of any: workgroups that are small run beside others,
    // whose loads, sums and stores overlap, but rows in pieces of 32 bytes are slow (512 x 32x32 x 128 bf16 backward 131 us by 256 threads and 32 bytes, 118 by 512 and 64, 135
    // by 1024 and 128; with codes written 103 in pieces of 128 bytes, 107 in those of 64).
    const int64_t enough = kept ? 128 : 64;
    GnCut best = {};
    for (int threads : {256, 512, 1024}) {
        int64_t most = 0;
        for (int64_t w = std::min(step, row);; w = std::min(w + step, row)) {
            const int64_t slots = (w + 7) / 8;
            if (slots > threads || gn_lds(threads, slots, cells, d) > GN_MOST_LDS) break;
            const int64_t lanes = threads / slots, slices = (row + w - 1) / w;
            if ((pixels + lanes - 1) / lanes > rows) break;
            most = w;
            if (w >= row) break;
            const bool narrow = w * size < 128, idle = pixels * slots < 2 * threads && samples * slices > 1024;
            if (!narrow && !idle) break;
        }
        if (most == 0 || (best.slice > 0 && most <= best.slice)) continue;
        const int32_t slots = (int32_t)((most + 7) / 8);
        best = {threads, slots, threads / slots, (int32_t)most, (int32_t)((row + most - 1) / most)};
        if (most * size >= enough || most >= row) break;
    }
    // Fewer workgroups than compute units: narrower slices, and all the threads there are, for the shortest way through (1 x 32x32 x 128 bf16 9.8 us, by the rule above 13.1).
    // Forward, samples of a chunk for each of 1024 threads at most stay whole, which spares the launch that adds the goodness of slices (1 x 4x4 x 512 bf16 8.1 us, in slices 9.1,
    // 64 x 8x8 x 64 7.3 and 9.3; with 2048 chunks alike, with 4096 10.7 and 9.2).
    const int64_t units = 256;
    if (best.slice > 0 && samples * best.slices < units) {
        int64_t w = !backward && pixels * (row / 8) <= 1024 ? row : std::min(step, row);
        while (w < row && samples * ((row + w - 1) / w) > units) w = std::min(w + step, row);
        const int64_t slots = (w + 7) / 8;
        for (int threads : {1024, 512, 256}) {
            if ((w > best.slice && w < row) || slots > threads || gn_lds(threads, slots, cells, d) > GN_MOST_LDS) continue;
            if (threads > 256 && threads / 2 >= pixels * slots) continue;   // (half of them would do)
            if ((pixels + threads / slots - 1) / (threads / slots) > rows) continue;
            best = {threads, (int32_t)slots, (int32_t)(threads / slots), (int32_t)w, (int32_t)((row + w - 1) / w)};
            break;
        }
    }
    if (best.slice > 0) {
        p.whole = true;
        p.cut = best;
        return p;
    }
    // Statistics by slices of up to 256 columns, of whole groups or of an equal piece of one.
    const int64_t wide = 256;
    int64_t w;
    p.pieces = 1;
    if (d <= wide) {
        w = std::min(wide / d, groups) * d;
        p.stat.slices = (int32_t)((channels + w - 1) / w);
    } else {
        const int64_t pieces = (d + wide - 1) / wide;
        w = gn_up((d + pieces - 1) / pieces, 8);
        p.pieces = (int32_t)((d + w - 1) / w);
        p.stat.slices = (int32_t)(groups * p.pieces);
    }
    p.stat.threads = GN_SPLIT_THREADS;
    p.stat.slice = (int32_t)w;
    p.stat.slots = (int32_t)((w + 7) / 8);
    p.stat.lanes = GN_SPLIT_THREADS / p.stat.slots;
    const int64_t slots = std::min<int64_t>(row / 8, 32);
    p.cut.threads = GN_SPLIT_THREADS;
    p.cut.slots = (int32_t)slots;
    p.cut.lanes = (int32_t)(GN_SPLIT_THREADS / slots);
    p.cut.slice = (int32_t)(slots * 8);
    p.cut.slices = (int32_t)((row + p.cut.slice - 1) / p.cut.slice);
    p.apply_blocks = (int32_t)((pixels + (int64_t)p.cut.lanes * GN_APPLY_ROWS - 1) / ((int64_t)p.cut.lanes * GN_APPLY_ROWS));
    if (!backward) {
        p.blocks = (int32_t)((pixels + (int64_t)p.stat.lanes * GN_STAT_ROWS - 1) / ((int64_t)p.stat.lanes * GN_STAT_ROWS));
    } else {
        // sums of columns, whatever group they are of: the slices that apply, over as many blocks of pixels as keep every compute unit busy
        p.stat = p.cut;
        p.pieces = 1;
        const int64_t most = (pixels + p.cut.lanes - 1) / p.cut.lanes, want = (2048 + samples * p.cut.slices - 1) / (samples * p.cut.slices);
        p.blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(most, want), 128));
    }
    return p;
}

// floats of workspace
static size_t gn_forward_floats(const GnPlan& p, int64_t samples, int64_t groups)
{
    if (p.whole) return (size_t)(samples * p.cut.slices);
    return (size_t)(4 * samples * groups * p.pieces * p.blocks + 4 * samples * groups + samples * p.cut.slices * p.apply_blocks);
}
static size_t gn_backward_floats(const GnPlan& p, int64_t samples, int64_t channels, int64_t groups)
{
    return (size_t)(2 * samples * channels + (p.whole ? 0 : 2 * samples * channels * p.blocks + 2 * samples * groups));
}

}  // namespace ffi
